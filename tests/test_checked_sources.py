"""Where the checked build looks: every kernel of linear attention, dropout and sampling has index checks,
and every place of the sampling kernel's shared arrays is reached through one.  (Read from the sources, as a
check that is not there cannot fail.)"""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(__file__), "..", "paper_2609_37899_gb300", "csrc")


def _source(name):
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def _body(text, start):
    """The braces' contents from the first { at or after `start`, past the parameters."""
    depth, i = 0, text.index("{", text.index(")", start))
    for j in range(i, len(text)):
        depth += {"{": 1, "}": -1}.get(text[j], 0)
        if depth == 0:
            return text[i:j]
    raise AssertionError("no end")


def _kernels(text):
    return {m.group(1): _body(text, m.end()) for m in
            re.finditer(r"__global__[^;{]*?(\w+_kernel)\(", text)}


@pytest.mark.parametrize("name,kernels,least", [
    ("dropout.cu", {"dropout_groups_kernel", "dropout_kernel"}, 1),
    ("sample.cu", {"sample_kernel"}, 1),
    ("linear_attn.cu", {"plain_kernel", "join_kernel", "step_kernel"}, 1),
    ("linear_attn_tc.cu", {"chunk_kernel", "copies_timeout_kernel"}, 6)])
def test_every_kernel_has_checks(name, kernels, least):
    found = _kernels(_source(name))
    assert set(found) == kernels
    for kernel, body in found.items():
        if kernel != "copies_timeout_kernel":  # a test of its own
            assert body.count("SOMA_CHECK(") >= least, kernel


def test_the_plain_kernels_reads_and_writes():
    body = _kernels(_source("linear_attn.cu"))["plain_kernel"]
    assert body.count("tile.holds(") >= 2 and body.count("within(k0") >= 3
    assert body.count("SOMA_CHECK(") >= 8


@pytest.mark.parametrize("function,check", [
    ("hold", "held_ok"), ("load", "held_ok"), ("fetch", "logits_ok"), ("largest", "slot_ok"),
    ("count", "bin_ok"), ("add", "bin_ok"), ("in_bin", "bin_ok"), ("find", "slot_ok"),
    ("gather", "listed_ok"), ("sort", "listed_ok"), ("listed_key", "listed_ok")])
def test_the_sampling_kernels_places(function, check):
    text = _source("sample.cu")
    row = text[text.index("struct Row {"):]
    m = re.search(r"__device__[^;{]*\b%s\(" % function, row)
    assert check + "(" in _body(row, m.end())
    helper = re.search(r"bool %s\(" % check, row)
    assert "SOMA_CHECK(" in _body(row, helper.end())


def test_no_bound_is_named_that_does_not_exist():
    for name in ("sample.cu", "dropout.cu", "linear_attn.cu", "linear_attn_tc.cu"):
        with open(os.path.join(CSRC, name)) as f:
            text = f.read()
        named = set(re.findall(r"\bk[A-Z]\w+", text))
        code = re.sub(r"//[^\n]*", "", text)
        headers = "".join(open(os.path.join(CSRC, h)).read() for h in os.listdir(CSRC) if h.endswith("h"))
        for word in named:
            assert re.search(r"\b%s\b" % word, code) or re.search(r"\b%s\b" % word, headers), (name, word)
