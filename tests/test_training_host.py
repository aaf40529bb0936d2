"""The host side of the training operators that needs no GPU: what the kernels' sources promise the compiler, when the Python binding
has to be built again."""
import os
import re

import pytest

from paper_2211_00188_b200 import build as builder
from paper_2211_00188_b200 import training

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2211_00188_b200", "csrc")


def kernels(text):
    """(name, parameters, body) of each kernel."""
    text = re.sub(r"//[^\n]*", "", text)
    for part in text.split("__global__")[1:]:
        head = re.search(r"\b(k_\w+)\s*\(", part)
        depth, i = 1, head.end()
        while depth:
            depth += {"(": 1, ")": -1}.get(part[i], 0)
            i += 1
        j = part.index("{", i) + 1
        depth, k = 1, j
        while depth:
            depth += {"{": 1, "}": -1}.get(part[k], 0)
            k += 1
        yield head.group(1), part[head.end():i - 1], part[j:k - 1]


@pytest.mark.parametrize("unit", ["adacgd_train_norm.cu", "adacgd_train_loss.cu"])
def test_dependent_kernels_do_not_promise_that_their_inputs_are_constant(unit):
    """A kernel that may be resident while its predecessor writes cannot take what that writes as const __restrict__: the compiler could
    read it through the non-coherent path, or ahead of the wait."""
    waiting = 0
    for name, parameters, body in kernels(open(os.path.join(CSRC, unit)).read()):
        if "griddepcontrol.wait" in body or "pdl_wait()" in body:
            waiting += 1
            assert not re.search(r"const\s+\w+\s*\*\s*__restrict__", parameters), name
    assert waiting >= (1 if "norm" in unit else 4)


def test_a_binding_of_another_torch_or_interpreter_is_built_again(tmp_path, monkeypatch):
    """The binding uses binary interfaces of both, which its file time says nothing about."""
    builder.build()
    assert not builder.needs_build()
    stamp = tmp_path / "stamp"
    monkeypatch.setattr(builder, "STAMP", str(stamp))
    assert builder.binding_is_stale() and not builder.library_is_stale()       # not known what it was built for
    stamp.write_text(builder.binding_target() + "\n")
    assert not builder.needs_build()
    for other in ("cpython-311-x86_64-linux-gnu, torch " + builder.metadata.version("torch"),
                  builder.binding_target().split(",")[0] + ", torch 2.10.0"):
        stamp.write_text(other + "\n")
        assert builder.binding_is_stale() and builder.needs_build()
        with pytest.raises(ImportError, match="built for"):
            training._load_binding()
