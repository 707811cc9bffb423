"""AdamW with stored moments that are not finite: their elements keep parameter and moments, the
others of their tensor are updated, and SOMA_ERR_NONFINITE is recorded.

Tolerances are those of test_gpu_adamw."""
import numpy as np
import pytest
import torch

from gpu_common import api
from test_gpu_adamw import CFG, U, _expected, _opt, _tensors, _value

pytestmark = pytest.mark.gpu

NONFINITE = 6


@np.errstate(invalid="ignore")
def _check_rest(s, before, want, rest, bits, master):
    w, m1, v1, tol, size = want
    got = (s["master"] if master else s["p"])[0].double().cpu().numpy()
    assert (np.abs(got - w) <= tol)[rest].all()
    m, v = (_value(s[k][0], s[k + "s"][0] if bits == 8 else None) for k in ("m", "v"))
    if bits == 32:
        assert (np.abs(m - m1) <= 4 * U * size)[rest].all()
        assert (np.abs(v - v1) <= 4 * U * v1)[rest].all()
        return
    for x, ref, scale in ((m, m1, s["ms"][0]), (v, np.sqrt(v1), s["vs"][0])):
        unit = np.repeat(scale.double().cpu().numpy(), 256)[:len(ref)]
        assert (np.abs(x - ref)
                <= np.maximum(np.abs(ref) / 8, unit * 2.0 ** -9) * 1.00001)[rest].all()


@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("which", ["m", "v", "both"])
@pytest.mark.parametrize("param,master", [("fp32", False), ("bf16", True)])
@pytest.mark.parametrize("bits", [8, 32])
def test_moments(bits, param, master, which, offset):
    s = _tensors((1000,), param, "fp32", bits, master, seed=3, offset=offset)
    hit = torch.tensor([0, 5, 255, 300, 999])
    at = hit.cuda()
    for k in ("m", "v") if which == "both" else (which,):
        if bits == 8:
            s[k][0].view(torch.uint8)[at] = 0x7F  # NaN
        else:
            s[k][0][at] = torch.tensor([float("nan"), float("inf"), float("nan"), float("inf"),
                                        float("nan")], device="cuda")
    rest = np.ones(1000, bool)
    rest[hit.numpy()] = False
    before = {k: s[k][0].clone() for k in ("p", "master", "m", "v")}
    with np.errstate(invalid="ignore"):
        want = _expected(s, 0, bits, master, 4)
    _opt(s, bits, master).step(s["g"], t=4, seed=2, **CFG)
    a = api()
    assert a.get_status() == NONFINITE and a.get_status() == 0
    assert torch.equal(s["p"][0][at], before["p"][at])
    if master:
        assert torch.equal(s["master"][0][at], before["master"][at])
    for k in ("m", "v"):
        now, was = (x[at].double().cpu() for x in (s[k][0], before[k]))
        lost = ~was.isfinite()
        assert torch.equal(now[lost].isnan(), was[lost].isnan())
        if bits == 32:
            assert torch.equal(now.nan_to_num(nan=1e300), was.nan_to_num(nan=1e300))
    _check_rest(s, before, want, rest, bits, master)
    # a second step finds the same elements not finite and no others
    p = s["p"][0].clone()
    _opt(s, bits, master).step(s["g"], t=5, seed=2, **CFG)
    assert a.get_status() == NONFINITE
    assert torch.equal(s["p"][0][at], p[at])
    assert s["p"][0].isfinite().all()


@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("which", ["ms", "vs"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_scales(bad, which, offset):
    """None of the block's 256 elements has moments: the whole block stays as it is, bit for bit."""
    s = _tensors((1000,), "fp32", "bf16", 8, False, seed=4, offset=offset)
    s[which][0][1] = bad
    rest = np.ones(1000, bool)
    rest[256:512] = False
    with np.errstate(invalid="ignore"):
        want = _expected(s, 0, 8, False, 2)
    before = {k: s[k][0].view(torch.uint8).clone() for k in ("p", "m", "v")}
    scales = {k: s[k][0][1].view(torch.int32).item() for k in ("ms", "vs")}
    _opt(s, 8, False).step(s["g"], t=2, seed=2, **CFG)
    assert api().get_status() == NONFINITE
    for k, x in before.items():
        width = x.numel() // 1000
        assert torch.equal(s[k][0].view(torch.uint8)[256 * width:512 * width],
                           x[256 * width:512 * width])
    assert {k: s[k][0][1].view(torch.int32).item() for k in ("ms", "vs")} == scales
    w, m1, v1, tol, size = want
    got = s["p"][0].double().cpu().numpy()
    assert (np.abs(got - w) <= tol)[rest].all()
