"""The kernels of lookup, norm and rotation, and attention, as far as their order can be read off the source: no GPU."""
import os
import re

import pytest

from test_training_host import CSRC, kernels

UNITS = ["adacgd_train_embed.cu", "adacgd_train_rotary.cu", "adacgd_train_attention.cu", "adacgd_train_attention_mma.cu"]
WAIT = re.compile(r"griddepcontrol\.wait|pdl_wait\(\)")


def source(unit):
    return re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, unit)).read())


def returns_before_the_wait(body):
    """The text in front of each `return;` that no wait of its own block, or of one around it, stands before."""
    waited, out = [False], []
    for m in re.finditer(r"[{}]|\breturn\s*;|" + WAIT.pattern, body):
        if m.group() == "{":
            waited.append(waited[-1])
        elif m.group() == "}":
            waited.pop()
        elif m.group().startswith("return"):
            if not waited[-1]:
                out.append(body[max(0, m.start() - 120):m.end()])
        else:
            waited[-1] = True
    return out


def test_the_search_for_returns_finds_one():
    assert returns_before_the_wait("if (x) return; griddepcontrol.wait; if (y) { return; }") == ["if (x) return;"]
    assert not returns_before_the_wait("if (x) { griddepcontrol.wait; return; } for (;;) { } griddepcontrol.wait; return;")


@pytest.mark.parametrize("unit", UNITS)
def test_dependent_kernels_wait_before_each_return(unit):
    """A kernel that may start before its predecessor has ended must not end before it either: the kernels behind it order themselves by its end alone."""
    for name, _, body in kernels(source(unit)):
        if WAIT.search(body):
            assert not returns_before_the_wait(body), name
