"""A state that is not finite goes on as it is: an infinite one stays infinite with its sign, a NaN
one NaN, up to the next reset, however small the forget gates on the way and however the steps
are cut.  h is then o tanh(+-inf) = +-o, within the 32 u that test_gpu_scan allows."""
import numpy as np
import pytest
import torch

from gpu_common import api
from test_gpu_scan import DT, U, ULP, _case, _near, _reference, _run

pytestmark = pytest.mark.gpu

# tiled and plain kernels, in one piece (300 sequences) and in chunks of the steps
SHAPES = [(300, 80, 64, "fp32"), (300, 80, 64, "bf16"), (300, 80, 33, "fp32"), (2, 200, 64, "fp32"),
          (2, 200, 33, "fp32"), (1, 6000, 8, "fp32"), (1, 6000, 7, "bf16")]


@pytest.mark.parametrize("ragged", ["no", "lengths", "resets"])
@pytest.mark.parametrize("gates", ["ordinary", "closed"])
@pytest.mark.parametrize("B,T,D,dtype", SHAPES)
def test_passes_through(B, T, D, dtype, gates, ragged):
    s = _case(B, T, D, dtype, seed=T + D)
    if gates == "closed":
        s["a"][:, ::3, 1] = -200.0  # exp(-200) is no fp32 number
    n, cut = T, T
    if ragged == "lengths":
        n = T - 5
        s["lengths"] = torch.full((B,), n, dtype=torch.int32)
    if ragged == "resets":
        cut = T // 2 + 3
        s["resets"] = torch.zeros(B, T, dtype=torch.uint8)
        s["resets"][:, cut] = 1
    want = _reference(s)
    inf = float("inf")
    s["c0"][:, 0], s["c0"][:, 1], s["c0"][:, 2] = inf, -inf, float("nan")
    got = _run(s)
    # the other channels, and what comes after the reset, are as they would be without
    for k, e, dt in (("h", "he", dtype), ("c", "cle", "fp32"), ("da", "dae", dtype),
                     ("dc0", "dc0e", "fp32")):
        _near(got[k][..., 3:], want[k][..., 3:], want[e][..., 3:], dt)
    _near(got["h"][:, cut:], want["h"][:, cut:], want["he"][:, cut:], dtype)
    h, o = got["h"].double().cpu().numpy(), 1 / (1 + np.exp(-s["a"][:, :, 3].double().numpy()))
    end = min(n, cut)
    for ch, sign in ((0, 1.0), (1, -1.0)):
        tol = 32 * U * o[:, :end, ch] + ULP[dtype][0] * o[:, :end, ch] + ULP[dtype][1]
        assert (np.abs(h[:, :end, ch] - sign * o[:, :end, ch]) <= tol).all()
    assert np.isnan(h[:, :end, 2]).all()
    c = got["c"].cpu()
    if ragged == "resets":
        _near(c, want["c"], want["cle"])
    else:
        assert (c[:, 0] == inf).all() and (c[:, 1] == -inf).all() and c[:, 2].isnan().all()


@pytest.mark.parametrize("B,T,D,dtype", SHAPES)
def test_large_finite_states_decay(B, T, D, dtype):
    """What lets an infinite state through leaves a finite one as it is: from 1e30 the products of
    forget gates bring the state down to where it would be from anywhere."""
    s = _case(B, T, D, dtype, seed=T + D)
    s["c0"][:, ::2] = 1e30
    want, got = _reference(s), _run(s)
    _near(got["h"], want["h"], want["he"], dtype)
    _near(got["c"], want["c"], want["cle"])


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("D", [64, 33])
def test_one_token(D, dtype):
    s = _case(3, 4, D, dtype, seed=D)
    s["a"][:, 1, 1] = -200.0
    a, c = s["a"].cuda(), s["c0"].cuda()
    c[:, 0], c[:, 1], c[:, 2] = float("inf"), -float("inf"), float("nan")
    h = torch.empty(3, 4, D, dtype=DT[dtype], device="cuda")
    for t in range(4):
        api().scan_step(a[:, t], c, h[:, t])
    assert (c[:, 0] == float("inf")).all() and (c[:, 1] == -float("inf")).all()
    assert c[:, 2].isnan().all() and c[:, 3:].isfinite().all()
    o = 1 / (1 + np.exp(-s["a"][:, :, 3, :2].double().numpy()))
    got = h[:, :, :2].double().cpu().numpy()
    tol = 32 * U * o + ULP[dtype][0] * o + ULP[dtype][1]
    assert (np.abs(got - o * np.array([1.0, -1.0])) <= tol).all()
