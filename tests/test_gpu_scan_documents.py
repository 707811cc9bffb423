"""Documents packed into one sequence of the gated linear recurrence do not touch each other,
whatever one of them holds: a step with a reset takes c_{t-1} = 0 and passes no gradient on.

The steps of one document are made NaN in some way; everything outside it has to be what the
formulas give (the 64-bit reference and its tolerances are those of test_gpu_scan), whichever
finite values stand in the document instead."""
import functools

import pytest
import torch

from gpu_common import api
from test_gpu_scan import _case, _near, _reference, _run

pytestmark = pytest.mark.gpu

# (batch, steps, channels, type): tiled and plain kernels, in one piece (300 sequences) and in chunks
# of the steps
SHAPES = [(300, 80, 64, "fp32"), (300, 80, 64, "bf16"), (300, 80, 33, "fp32"), (2, 200, 64, "bf16"),
          (2, 200, 33, "fp32"), (1, 6000, 8, "fp32"), (1, 6000, 8, "bf16"), (1, 6000, 7, "fp32")]


def _poison(s, kind, p, q):
    a, dh = s["a"].clone(), s["dh"].clone()
    if kind == "all":
        a[:, p:q] = float("nan")
    elif kind == "first forget gate":
        a[:, p, 1] = float("nan")
    elif kind == "last forget gate":
        a[:, q - 1, 1] = float("nan")
    elif kind == "gradient":
        dh[:, p:q] = float("nan")
    else:
        a[:, p:q, 2], dh[:, p:q] = float("nan"), float("inf")
    return {**s, "a": a, "dh": dh}


@functools.lru_cache(maxsize=1)
def _documents(B, T, D, dtype, p, q):
    s = _case(B, T, D, dtype, seed=T + p)
    s["resets"] = torch.zeros(B, T, dtype=torch.uint8)
    s["resets"][:, [p, q]] = 1
    return s, _reference(s)


@pytest.mark.parametrize("kind", ["all", "first forget gate", "last forget gate", "gradient",
                                  "input and gradient"])
@pytest.mark.parametrize("p,q", [(13, 21), (16, 24), (41, 43), (30, 67)])
@pytest.mark.parametrize("B,T,D,dtype", SHAPES)
def test_a_document_that_is_not_finite(B, T, D, dtype, p, q, kind):
    s, want = _documents(B, T, D, dtype, p, q)
    assert (api().scan_workspace_bytes(B, T, D) == 0) == (B == 300)
    got = _run(_poison(s, kind, p, q))
    for part in (slice(0, p), slice(q, T)):
        _near(got["h"][:, part], want["h"][:, part], want["he"][:, part], dtype)
        _near(got["da"][:, part], want["da"][:, part], want["dae"][:, part], dtype)
    _near(got["c"], want["c"], want["cle"])
    _near(got["dc0"], want["dc0"], want["dc0e"])


@pytest.mark.parametrize("B,T,D,dtype", SHAPES)
def test_gradient_of_the_last_state_that_is_not_finite(B, T, D, dtype):
    """It ends at the last reset."""
    s = _case(B, T, D, dtype, seed=T)
    s["resets"] = torch.zeros(B, T, dtype=torch.uint8)
    s["resets"][:, 77] = 1
    want = _reference(s)
    s["dcl"] = torch.full_like(s["dcl"], float("nan"))
    got = _run(s)
    _near(got["h"], want["h"], want["he"], dtype)
    _near(got["da"][:, :77], want["da"][:, :77], want["dae"][:, :77], dtype)
    _near(got["dc0"], want["dc0"], want["dc0e"])
