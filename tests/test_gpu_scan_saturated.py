"""Gradients of saturated gates, relative to their own size, on the tiled and the plain kernels.

sigmoid'(x) = e / (1 + e)^2 with e = exp(-|x|), of either sign of x: e carries the rounding of its
exponent, |x| log2(e) u in powers of two and as much again for the constant, so 2 |x| u of itself,
and the exponential, two reciprocals or one, and the products some 2^-22 each: (2 |x| + 48) u of
the gradient is allowed.  One step from a given state, so that nothing else enters: with dh = 0 and
dc_last = r, d a_i = r g i (1 - i), d a_f = r c0 f (1 - f), and with dc_last = 0,
d a_o = dh tanh(c) o (1 - o)."""
import numpy as np
import pytest
import torch

from test_gpu_scan import DT, U, ULP, _case, _run

pytestmark = pytest.mark.gpu


def _slope(x):
    e = np.exp(-np.abs(x))
    return e / (1 + e) ** 2


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("D", [64, 128, 33])
def test_relative_to_their_size(D, dtype):
    s = _case(3, 1, D, dtype, seed=D)
    g = torch.Generator().manual_seed(1)
    far = 4 + 12 * torch.rand(3, 1, 4, D, generator=g)
    far[:, :, :, ::2] *= -1
    s["a"] = far.to(DT[dtype])
    s["a"][:, :, 2] = 0.5
    x = s["a"].double().numpy()[:, 0]
    sig = lambda v: 1 / (1 + np.exp(-v))
    c0, r = s["c0"].double().numpy(), s["dcl"].double().numpy()
    dh = s["dh"].clone()

    s["dh"] = torch.zeros_like(dh)
    got = _run(s)["da"].double().cpu().numpy()[:, 0]
    s["dh"], s["dcl"] = dh, torch.zeros_like(s["dcl"])
    got_o = _run(s)["da"].double().cpu().numpy()[:, 0, 3]
    th = np.tanh(sig(x[:, 1]) * c0 + sig(x[:, 0]) * np.tanh(x[:, 2]))
    for have, want, gate in ((got[:, 0], r * np.tanh(x[:, 2]) * _slope(x[:, 0]), 0),
                             (got[:, 1], r * c0 * _slope(x[:, 1]), 1),
                             (got_o, dh.double().numpy()[:, 0] * th * _slope(x[:, 3]), 3)):
        rel, low = ULP[dtype]
        # tanh(c) carries the state's error, 64 u of terms no larger than |c0| + 1
        more = 64 * U * (np.abs(c0) + 1) / np.maximum(np.abs(th), 1e-30) if gate == 3 else 0.0
        tol = np.abs(want) * ((2 * np.abs(x[:, gate]) + 48) * U + rel + more) + low
        assert (np.abs(have - want) <= tol).all(), gate


def test_limits():
    """Gates at and beyond where exp overflows: no NaN, gradients below the least fp32 number."""
    s = _case(1, 1, 64, "fp32", seed=5)
    x = torch.tensor([-float("inf"), -3e38, -200.0, -89.0, -88.0, 88.0, 200.0, float("inf")])
    for k in (0, 1, 3):
        s["a"][0, 0, k] = x.repeat(8)
    got = _run(s)["da"][0, 0].cpu()
    assert got.isfinite().all()
    assert (got[[0, 1, 3]].abs() <= 2.0 ** -120).all()
