"""AdamW over many tensors (soma_adamw_step) against its formulas in 64 bits.

Tolerances, from the rounding of each operation (u = 2^-24, half an ulp of
fp32): a moment is a sum of two products, at most 3 roundings of terms no
larger than |beta m| + |(1-beta) g|, so 4u of that sum; the parameter adds a
quotient of at most 8 roundings to a product of one, so 2u of |p| plus 12u of
the step (and half an ulp of a 16-bit parameter on top).  In 8 bits a value
is one of the two neighbours on the e4m3 grid of its block's scale, whose
distance is at most an eighth of the value or 2^-9 of the scale.
"""
import ctypes

import numpy as np
import pytest
import torch

from gpu_common import api

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
HALF_ULP = {"fp32": 0.0, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}
CFG = dict(lr=3e-3, beta1=0.9, beta2=0.99, eps=1e-6)
DECAY = 0.1


def _tensors(sizes, param, grad, bits, master, seed=0, offset=0):
    """Tensors of the given sizes that start `offset` elements into their allocations."""
    g = torch.Generator().manual_seed(seed)

    def put(x, dtype):
        flat = torch.zeros(x.numel() + offset, dtype=dtype, device="cuda")
        flat[offset:] = x.to(dtype).cuda()
        return flat[offset:]

    s = {k: [] for k in ("p", "g", "m", "v", "ms", "vs", "master")}
    for j, n in enumerate(sizes):
        scale = 10.0 ** -(j % 4)
        w = torch.randn(n, generator=g)
        s["p"].append(put(w, DT[param]))
        s["master"].append(put(w, torch.float32))
        s["g"].append(put(torch.randn(n, generator=g) * scale, DT[grad]))
        m, r = torch.randn(n, generator=g) * scale, (torch.rand(n, generator=g) + 0.1) * scale
        if bits == 32:
            s["m"].append(put(m, torch.float32))
            s["v"].append(put(r * r, torch.float32))
            continue
        for key, x in (("m", m), ("v", r)):
            pad = torch.zeros(-(-n // 256) * 256)
            pad[:n] = x
            top = pad.view(-1, 256).abs().amax(1) / 448
            code = (pad.view(-1, 256) / top[:, None]).view(-1)[:n]
            s[key].append(put(code, torch.float8_e4m3fn))
            s[key + "s"].append(top.cuda())
    return s


def _opt(s, bits, master, decay=DECAY):
    return api().AdamW(s["p"], s["m"], s["v"], s["ms"] if bits == 8 else None,
                       s["vs"] if bits == 8 else None, s["master"] if master else None, decay)


def _value(code, scale):
    x = code.double().cpu().numpy()
    return x if scale is None else x * np.repeat(scale.double().cpu().numpy(), 256)[:x.size]


def _expected(s, k, bits, master, t, scale=1.0):
    """New parameter, moments (root of the second in 8 bits) and the step, in 64 bits."""
    w = (s["master"] if master else s["p"])[k].double().cpu().numpy()
    g = s["g"][k].double().cpu().numpy() * scale
    m = _value(s["m"][k], s["ms"][k] if bits == 8 else None)
    v = _value(s["v"][k], s["vs"][k] if bits == 8 else None)
    v = v * v if bits == 8 else v
    m1 = CFG["beta1"] * m + (1 - CFG["beta1"]) * g
    v1 = CFG["beta2"] * v + (1 - CFG["beta2"]) * g * g
    step = CFG["lr"] * (m1 / (1 - CFG["beta1"] ** t)) / (
        np.sqrt(v1 / (1 - CFG["beta2"] ** t)) + CFG["eps"])
    size = CFG["beta1"] * np.abs(m) + (1 - CFG["beta1"]) * np.abs(g)
    # a step's error also carries the moment's, relative to the moment's terms
    err = np.abs(step) * 12 * U + 4 * U * size * np.abs(CFG["lr"] / (1 - CFG["beta1"] ** t)) / (
        np.sqrt(v1 / (1 - CFG["beta2"] ** t)) + CFG["eps"])
    return w * (1 - CFG["lr"] * DECAY) - step, m1, v1, err + 2 * U * np.abs(w), size


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param,grad,master", [
    ("fp32", "fp32", False), ("fp32", "bf16", False), ("fp32", "fp16", False),
    ("bf16", "bf16", True), ("bf16", "fp32", False), ("fp16", "fp16", True)])
@pytest.mark.parametrize("sizes,offset", [
    ((1,), 0), ((255, 256, 257, 8, 7, 0, 2048, 2049), 0), ((5000, 3, 70001), 1)])
def test_step(param, grad, master, bits, sizes, offset):
    s = _tensors(sizes, param, grad, bits, master, offset=offset)
    want = [_expected(s, k, bits, master, 7, 0.5) for k in range(len(sizes))]
    _opt(s, bits, master).step(s["g"], t=7, seed=11, grad_scale=torch.tensor([0.5], device="cuda"),
                               **CFG)
    assert api().get_status() == 0
    for k, (w, m1, v1, tol, size) in enumerate(want):
        if not sizes[k]:
            continue
        got = (s["master"] if master else s["p"])[k].double().cpu().numpy()
        if not master:
            tol = tol + HALF_ULP[param] * np.abs(w) + (6e-8 if param == "fp16" else 0)
        assert (np.abs(got - w) <= tol).all()
        if master:
            assert torch.equal(s["p"][k], s["master"][k].to(DT[param]))
        m, v = (_value(s[key][k], s[key + "s"][k] if bits == 8 else None) for key in ("m", "v"))
        if bits == 32:
            assert (np.abs(m - m1) <= 4 * U * size).all()
            assert (np.abs(v - v1) <= 4 * U * v1).all()
            continue
        for x, ref, scale in ((m, m1, s["ms"][k]), (v, np.sqrt(v1), s["vs"][k])):
            top = np.abs(np.pad(ref, (0, -len(ref) % 256))).reshape(-1, 256).max(1)
            unit = scale.double().cpu().numpy()
            assert np.allclose(unit, top / 448, rtol=8 * U, atol=0)
            unit = np.repeat(unit, 256)[:len(ref)]
            # neighbours on the grid are an eighth of a value apart at most
            assert (np.abs(x - ref) <= np.maximum(np.abs(ref) / 8, unit * 2.0 ** -9) * 1.00001).all()
        assert (v[v1 > 0] > 0).all()


@pytest.mark.parametrize("bits", [32, 8])
def test_alignment_does_not_change_results(bits):
    sizes = (4097, 256, 300)
    a = _tensors(sizes, "fp32", "bf16", bits, False, seed=3, offset=0)
    b = _tensors(sizes, "fp32", "bf16", bits, False, seed=3, offset=3)
    for s in (a, b):
        for t in (1, 2, 3):
            _opt(s, bits, False).step(s["g"], t=t, seed=5, **CFG)
    for key in ("p", "m", "v", "ms", "vs"):
        for x, y in zip(a[key], b[key]):
            assert torch.equal(x.float(), y.float())


def test_more_tensors_than_one_launch_holds():
    sizes = [1 + (k * 37) % 600 for k in range(800)]
    s = _tensors(sizes, "fp32", "fp32", 32, False, seed=4)
    want = [_expected(s, k, 32, False, 2) for k in range(len(sizes))]
    _opt(s, 32, False).step(s["g"], t=2, **CFG)
    for k, w in enumerate(want):
        assert (np.abs(s["p"][k].double().cpu().numpy() - w[0]) <= w[3]).all()


@pytest.mark.parametrize("bits", [32, 8])
def test_decay_per_tensor_and_empty_lists(bits):
    s = _tensors((300, 300), "fp32", "fp32", bits, False, seed=6)
    for g, m in zip(s["g"], s["m"]):
        g.zero_(), m.view(torch.uint8).zero_()
    before = [p.clone() for p in s["p"]]
    _opt(s, bits, False, [0.0, 0.5]).step(s["g"], t=1, **CFG)
    assert torch.equal(s["p"][0], before[0])
    assert torch.allclose(s["p"][1], before[1] * (1 - CFG["lr"] * 0.5), rtol=2 * U, atol=0)
    api().AdamW([], [], []).step([], t=1, **CFG)


@pytest.mark.parametrize("bits", [32, 8])
def test_nonfinite_gradients_leave_their_elements(bits):
    s = _tensors((1000,), "fp32", "fp32", bits, False, seed=7)
    hit = torch.tensor([0, 5, 255, 256, 999], device="cuda")
    s["g"][0][hit] = torch.tensor([float("nan"), float("inf"), -float("inf"), 3e38, float("nan")],
                                  device="cuda")
    p, m = s["p"][0].clone(), _value(s["m"][0], s["ms"][0] if bits == 8 else None)
    _opt(s, bits, False).step(s["g"], t=3, **CFG)
    a = api()
    assert a.get_status() == 6 and a.get_status() == 0
    assert torch.equal(s["p"][0][hit], p[hit])
    rest = torch.ones(1000, dtype=torch.bool, device="cuda")
    rest[hit] = False
    assert (s["p"][0][rest] != p[rest]).all() and s["p"][0].isfinite().all()
    m2 = _value(s["m"][0], s["ms"][0] if bits == 8 else None)
    at = hit.cpu().numpy()
    assert np.isfinite(m2).all()
    if bits == 32:
        assert (m2[at] == m[at]).all()
    else:
        assert (np.abs(m2[at] - m[at]) <= np.abs(m[at]) / 8 + s["ms"][0].max().item() / 512).all()


def test_nonfinite_scale_skips_the_step():
    s = _tensors((1000,), "fp32", "fp32", 32, False, seed=8)
    p, m = s["p"][0].clone(), s["m"][0].clone()
    for bad in (float("nan"), float("inf")):
        _opt(s, 32, False).step(s["g"], t=1, grad_scale=torch.tensor([bad], device="cuda"), **CFG)
        assert api().get_status() == 6
        assert torch.equal(s["p"][0], p) and torch.equal(s["m"][0], m)


def test_random_rounding_is_unbiased():
    """The mean over many draws of a rounded first moment is the moment: with n draws the
    standard error is at most step / (2 sqrt n); five of them are allowed per element."""
    n, draws = 256, 400
    s = _tensors((n,), "fp32", "fp32", 8, False, seed=9)
    m8, ms = s["m"][0].clone(), s["ms"][0].clone()
    want = _expected(s, 0, 8, False, 1)[1]
    v8, vs, total = s["v"][0].clone(), s["vs"][0].clone(), np.zeros(n)
    for k in range(draws):
        s["m"][0].copy_(m8), s["ms"][0].copy_(ms), s["v"][0].copy_(v8), s["vs"][0].copy_(vs)
        _opt(s, 8, False).step(s["g"], t=1, seed=k, **CFG)
        total += _value(s["m"][0], s["ms"][0])
    step = np.maximum(np.abs(want) / 8, s["ms"][0].item() * 2.0 ** -9)
    assert (np.abs(total / draws - want) <= 5 * step / (2 * np.sqrt(draws))).all()


def test_eight_bit_average_follows_small_changes():
    """A second moment that decays by less than half a grid step per update still decays."""
    p = [torch.zeros(4096, device="cuda")]
    state = api().AdamW.zero_state(p, 8)
    opt = api().AdamW(p, **state)
    g = torch.ones(4096, device="cuda")
    for t in range(1, 11):
        opt.step([g], t=t, lr=0.0, beta2=0.9)
    start = _value(state["exp_avg_sq"][0], state["v_scales"][0]).mean()
    # one element stays at 1 so that the block's scale does; the others see no gradient
    g.zero_()
    g[::256] = 1.0
    for t in range(11, 211):
        opt.step([g], t=t, lr=0.0, beta2=0.99, seed=3)
    end = _value(state["exp_avg_sq"][0], state["v_scales"][0])
    end = end.reshape(-1, 256)[:, 1:].mean()
    assert abs(end / (start * 0.99 ** 100) - 1) < 0.1  # the root decays by sqrt(beta2) per update


def test_runs_on_a_side_stream():
    s = _tensors((100000,), "fp32", "fp32", 32, False, seed=10)
    want = _expected(s, 0, 32, False, 1)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    _opt(s, 32, False).step(s["g"], t=1, stream=st, **CFG)
    st.synchronize()
    assert (np.abs(s["p"][0].double().cpu().numpy() - want[0]) <= want[3]).all()


def test_binding_refuses():
    a = api()
    s = _tensors((256,), "fp32", "fp32", 32, False)
    with pytest.raises(ValueError):
        a.AdamW(s["p"], s["m"], [])
    with pytest.raises(ValueError):
        a.AdamW([s["p"][0].double()], s["m"], s["v"])
    with pytest.raises(ValueError):
        a.AdamW(s["p"], [s["m"][0][:255]], s["v"])
    with pytest.raises(ValueError):
        a.AdamW(s["p"], s["m"], s["v"], weight_decay=[0.1, 0.2])
    opt = _opt(s, 32, False)
    with pytest.raises(ValueError):
        opt.step([s["g"][0][::2]], t=1, lr=1e-3)
    with pytest.raises(ValueError):
        opt.step([], t=1, lr=1e-3)
    with pytest.raises(a.SomaError):
        opt.step(s["g"], t=0, lr=1e-3)
    with pytest.raises(a.SomaError):
        opt.step(s["g"], t=1, lr=float("nan"))
    assert isinstance(ctypes.sizeof(a.soma_adamw_tensor), int)
