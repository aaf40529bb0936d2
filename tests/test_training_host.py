"""The host side of the training operators that needs no GPU: what the kernels' sources promise the compiler."""
import os
import re

import pytest

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
