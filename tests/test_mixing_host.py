"""The host side of lookup, norm and rotation, and attention that needs no GPU: checks of arguments, what the kernels' sources promise."""
import os
import re

import pytest

import paper_2211_00188_b200 as pkg
from paper_2211_00188_b200 import build as builder
from test_training_host import CSRC, kernels

UNITS = ["adacgd_train_embed.cu", "adacgd_train_rotary.cu", "adacgd_train_attention.cu", "adacgd_train_attention_mma.cu"]


@pytest.fixture(scope="module")
def lib():
    builder.build()
    return pkg.load_training_library()


@pytest.mark.parametrize("name", ["adacgd_embedding", "adacgd_embedding_backward", "adacgd_qk_norm", "adacgd_qk_norm_backward", "adacgd_attention",
                                  "adacgd_attention_backward"])
def test_null_arguments_are_refused(lib, name):
    assert getattr(lib, name)(None, None) == 1
    assert name.encode() in lib.adacgd_train_last_error(None)


@pytest.mark.parametrize("unit", UNITS)
def test_dependent_kernels_do_not_promise_that_their_inputs_are_constant(unit):
    """See the test of the same name of the other training operators."""
    for name, parameters, body in kernels(open(os.path.join(CSRC, unit)).read()):
        if "griddepcontrol.wait" in body:
            assert not re.search(r"const\s+\w+\s*\*\s*__restrict__", parameters), name


def test_waits_are_bounded():
    """Nothing spins on a barrier but the one function that gives up after a time, and no kernel waits on another one's memory."""
    for unit in UNITS + ["adacgd_tcgen05.cuh"]:
        text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, unit)).read())
        assert "while (mbar_try" not in text and "while (!mbar_try" not in text
        if unit != "adacgd_tcgen05.cuh":
            assert "mbar_try" not in text and "try_wait" not in text, unit
    text = open(os.path.join(CSRC, "adacgd_tcgen05.cuh")).read()
    assert re.search(r"clock64\(\) - begin > WAIT_CLOCKS", text)


def test_shared_memory_of_the_tiles_fits():
    """What the layouts of the tensor-core kernels add up to, by the formulas in the source, within the 227 KB a CTA can have."""
    text = open(os.path.join(CSRC, "adacgd_train_attention_mma.cu")).read()
    for dp in (64, 128):
        tile = dp * 256
        totals = {"Fwd": 2 * tile + (5 if dp == 128 else 8) * tile + 256,
                  "Dq": 2 * tile + (5 if dp == 128 else 8) * tile + 4 * 128 * 4 + 256,
                  "Dkv": 2 * tile + (5 if dp == 128 else 8) * tile + 2 * 2 * 128 * 4 + 256}
        assert max(totals.values()) <= 227 * 1024, totals
    for name, stages in (("Fwd", "STAGES = DP == 128 ? 5 : 8"), ("Dq", "KS = DP == 128 ? 3 : 4, VS = DP == 128 ? 2 : 4"), ("Dkv", "STAGES = DP == 128 ? 5 : 8")):
        part = text[text.index(f"struct {name}Layout"):]
        assert stages in part[:600], name

