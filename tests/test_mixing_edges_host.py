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


def layouts():
    """{kernel: (names and byte offsets of its shared memory for heads of up to 64, of up to 128)}: the constants as the source computes them."""
    text = source("adacgd_train_attention_mma.cu")
    out = {}
    for name, kernel in (("FwdLayout", "k_attention_mma"), ("DqLayout", "k_attention_dq_mma"), ("DkvLayout", "k_attention_dkv_mma")):
        body = re.search(r"struct " + name + r" \{(.*?)\};", text, re.S).group(1)
        sizes = []
        for dp in (64, 128):
            at = {"DP": dp, "TILE": 128}
            for line in re.findall(r"static constexpr int ([^;]*);", body):
                for part in line.split(","):
                    left, right = (x.strip() for x in part.split("=", 1))
                    right = re.sub(r"(.+?)\s*\?\s*(.+?)\s*:\s*(.+)", r"(\2) if (\1) else (\3)", right)
                    at[left] = eval(right, {}, at)
            sizes.append(at)
        out[kernel] = sizes
    return out


def test_no_tensor_copy_arrives_where_plain_accesses_came_before():
    """Plain writes to shared memory are not ordered before a copy's writes to the same bytes by a barrier alone.  So the two words in which a CTA
    joins the ends of its mask lie behind the tiles and behind the barriers, inside what the CTA has."""
    text = source("adacgd_train_attention_mma.cu")
    bodies = {name: body for name, _, body in kernels(text)}
    for kernel, sizes in layouts().items():
        scratch = re.findall(r"\btrim\(a, t, ([^;]*?), &", bodies[kernel])
        assert scratch == ["reinterpret_cast<int*>(mma_smem + L::SCRATCH)"], kernel
        for at in sizes:
            stages = at["STAGES"] if "STAGES" in at else at["KS"] + at["VS"]
            tiles = at["RING"] + stages * at["BYTES"]                       # all that copies write
            assert tiles <= at["BARS"] and at["BARS"] + 64 + 16 * stages + 8 <= at["SCRATCH"] and at["SCRATCH"] + 8 <= at["TOTAL"] <= 227 * 1024, kernel


def test_places_among_the_most_tokens_fit_in_32_bits():
    """The numbers that the lookup's gradient and attention form in int, for the most tokens that they take: the end of a window or tile, one step behind the last
    token.  (For 2^31 - 1 tokens each of them would be negative.)"""
    header = open(os.path.join(os.path.dirname(os.path.dirname(CSRC)), "include", "adacgd_train.h")).read()
    most = eval(re.search(r"#define ADACGD_TRAIN_MAX_RUN (\([^)]*\))", header).group(1).replace("ll", ""))
    embed, shared, mma = source("adacgd_train_embed.cu"), source("adacgd_train.cuh"), source("adacgd_train_attention_mma.cu")
    number = lambda text, name: int(re.search(r"\b" + name + r" = (\d+)", text).group(1))  # noqa: E731
    windows = number(shared, "NORM_PARTS")
    assert re.search(r"MAX_WINDOWS = NORM_PARTS;", embed)
    window = -(-most // windows)
    for text, name in ((embed, "SORT_CTA"), (embed, "SUM_CTA"), (mma, "FWD_CTA"), (mma, "BWD_CTA"), (mma, "TILE")):
        assert most + window + 2 * number(text, name) < 2 ** 31
    checks = source("adacgd_train.cu")
    for entry in (r"const char\* check_attention\(.*?\n}", r"adacgd_status adacgd_embedding_backward\(.*?\n}"):
        assert "tokens > ADACGD_TRAIN_MAX_RUN" in re.search(entry, checks, re.S).group()
