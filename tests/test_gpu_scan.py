"""The gated linear recurrence (soma_scan_*) against its formulas in 64 bits.

Tolerances.  u = 2^-24 is half an ulp of fp32.  Every activation, product and
sum is good to a few u of its terms; 32 u of the terms of c_t = f c + i g is
allowed per step and carried on by the recurrence itself,
  e_t = f_t e_{t-1} + 32 u (|f_t c_{t-1}| + |i_t g_t|),
and in the same way for dc, where the error of c enters through tanh'.  The
factors 1 - x and 1 - x^2 lose up to 8 u absolutely.  Results of 16 bits add
half an ulp of their own.
"""
import numpy as np
import pytest
import torch

from gpu_common import api

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
# half an ulp relative to the value, and what underflows
ULP = {"fp32": (U, 2.0 ** -126), "bf16": (2.0 ** -8, 2.0 ** -126), "fp16": (2.0 ** -11, 2.0 ** -25)}


def _case(B, T, D, dtype, seed=0, ragged=False, resets=False, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    s = dict(a=(torch.randn(B, T, 4, D, generator=g) * spread).to(DT[dtype]),
             c0=torch.randn(B, D, generator=g), dh=torch.randn(B, T, D, generator=g).to(DT[dtype]),
             dcl=torch.randn(B, D, generator=g), lengths=None, resets=None, dtype=dtype)
    if ragged:
        n = torch.randint(0, T + 1, (B,), generator=g, dtype=torch.int32)
        n[0] = 0
        n[-1] = T
        s["lengths"] = n
        for b in range(B):
            s["a"][b, n[b]:] = float("nan")
            s["dh"][b, n[b]:] = float("inf")
    if resets:
        s["resets"] = (torch.rand(B, T, generator=g) < 0.2).to(torch.uint8)
    return s


def _reference(s):
    a, dh = s["a"].double().numpy(), s["dh"].double().numpy()
    B, T, _, D = a.shape
    n = np.full(B, T) if s["lengths"] is None else s["lengths"].numpy()
    rs = np.zeros((B, T), bool) if s["resets"] is None else s["resets"].numpy() != 0
    sig = lambda x: 1 / (1 + np.exp(-x))
    c, e = s["c0"].double().numpy(), np.zeros((B, D))
    r = {k: np.zeros((B, T, D)) for k in ("h", "he", "f", "prev", "pe", "th", "ce")}
    for t in range(T):
        on = (t < n)[:, None]
        x = np.where(on[:, None], a[:, t], 0.0)
        i, f, g, o = sig(x[:, 0]), sig(x[:, 1]), np.tanh(x[:, 2]), sig(x[:, 3])
        keep = ~rs[:, t][:, None]
        prev, pe = c * keep, e * keep
        new, ne = f * prev + i * g, f * pe + 32 * U * (np.abs(f * prev) + np.abs(i * g))
        th = np.tanh(new)
        r["prev"][:, t], r["pe"][:, t], r["th"][:, t], r["ce"][:, t] = prev, pe, th, ne
        r["h"][:, t] = np.where(on, o * th, 0)
        r["he"][:, t] = np.where(on, o * (1 - th ** 2) * ne + 32 * U * np.abs(o * th), 0)
        c, e = np.where(on, new, c), np.where(on, ne, e)
    r["c"], r["cle"] = c, e + U * np.abs(c)
    dc, E = s["dcl"].double().numpy(), np.zeros((B, D))
    r["da"], r["dae"] = np.zeros((B, T, 4, D)), np.zeros((B, T, 4, D))
    for t in range(T - 1, -1, -1):
        on = (t < n)[:, None]
        x, y = np.where(on[:, None], a[:, t], 0.0), np.where(on, dh[:, t], 0.0)
        i, f, g, o = sig(x[:, 0]), sig(x[:, 1]), np.tanh(x[:, 2]), sig(x[:, 3])
        th, prev, ce, pe = r["th"][:, t], r["prev"][:, t], r["ce"][:, t], r["pe"][:, t]
        into, A = y * o * (1 - th ** 2), np.abs
        total = dc + into
        Et = E + 32 * U * (A(into) + A(dc)) + A(y * o) * (2 * A(th) * (1 - th ** 2) * ce + 8 * U)
        d = np.stack((total * g * i * (1 - i), total * prev * f * (1 - f),
                      total * i * (1 - g ** 2), y * th * o * (1 - o)), 1)
        de = np.stack((A(g) * i * (1 - i) * Et + 8 * U * A(total * g * i),
                       f * (1 - f) * (A(prev) * Et + A(total) * pe) + 8 * U * A(total * prev * f),
                       i * (1 - g ** 2) * Et + 8 * U * A(total * i),
                       A(y) * o * (1 - o) * (1 - th ** 2) * ce + 8 * U * A(y * th * o)), 1)
        r["da"][:, t] = np.where(on[:, None], d, 0)
        r["dae"][:, t] = np.where(on[:, None], de + 32 * U * A(d), 0)
        keep = ~rs[:, t][:, None]
        dc, E = np.where(on, total * f * keep, dc), np.where(on, (Et * f + 4 * U * A(total * f)) * keep, E)
    r["dc0"], r["dc0e"] = dc, E + U * np.abs(dc)
    return r


def _near(got, want, tol, dtype="fp32"):
    got = got.double().cpu().numpy()
    rel, low = ULP[dtype]
    bad = ~(np.abs(got - want) <= tol + rel * np.abs(want) + low)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:3].tolist(),
                           float(np.nanmax(np.abs(got - want))))


def _cuda(x):
    return None if x is None else x.cuda()


def _run(s, a=None, h=None, dh=None, da=None, stream=None):
    m = api()
    a = s["a"].cuda() if a is None else a
    dh = s["dh"].cuda() if dh is None else dh
    B, T, _, D = a.shape
    h = torch.full((B, T, D), float("nan"), dtype=a.dtype, device="cuda") if h is None else h
    da = torch.full((B, T, 4, D), float("nan"), dtype=a.dtype, device="cuda") if da is None else da
    cl, dc0 = (torch.full((B, D), float("nan"), device="cuda") for _ in range(2))
    marks = m.scan_alloc_checkpoints(B, T, D).fill_(float("nan"))
    kw = dict(lengths=_cuda(s["lengths"]), resets=_cuda(s["resets"]), stream=stream)
    c0, dcl = s["c0"].cuda(), s["dcl"].cuda()
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())
    m.scan_forward(a, h, cl, c0=c0, checkpoints=marks, **kw)
    m.scan_backward(a, marks, dh, da, dc0, dc_last=dcl, **kw)
    torch.cuda.synchronize()
    return dict(h=h, c=cl, da=da, dc0=dc0)


def _check(s, got, r=None):
    r = r or _reference(s)
    _near(got["h"], r["h"], r["he"], s["dtype"])
    _near(got["c"], r["c"], r["cle"])
    _near(got["da"], r["da"], r["dae"], s["dtype"])
    _near(got["dc0"], r["dc0"], r["dc0e"])


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("B,T,D", [
    (1, 1, 1), (3, 1, 70), (2, 2, 33), (1, 7, 64), (2, 15, 65), (5, 16, 2), (1, 17, 129),
    (3, 31, 100), (2, 64, 96), (1, 127, 48), (2, 128, 130), (1, 129, 64), (1, 1000, 66),
    (2, 2049, 40), (40, 40, 480), (1, 6000, 8)])
def test_sizes(B, T, D, dtype):
    s = _case(B, T, D, dtype, seed=B * T + D)
    _check(s, _run(s))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("resets", [False, True])
@pytest.mark.parametrize("B,T,D", [(4, 1, 64), (7, 100, 67), (3, 300, 128), (5, 1025, 32),
                                   (300, 33, 64)])
def test_lengths_and_resets(B, T, D, resets, dtype):
    s = _case(B, T, D, dtype, seed=T, ragged=True, resets=resets)
    _check(s, _run(s))


def test_resets_everywhere_and_at_the_edges():
    s = _case(2, 200, 64, "fp32", seed=1)
    for at in ([0], [199], list(range(200)), [15, 16, 127, 128]):
        s["resets"] = torch.zeros(2, 200, dtype=torch.uint8)
        s["resets"][0, at] = 1
        _check(s, _run(s))


def test_all_sequences_empty():
    s = _case(3, 50, 64, "bf16", seed=2)
    s["lengths"] = torch.tensor([0, -5, 0], dtype=torch.int32)
    s["a"].fill_(float("nan"))
    got = _run(s)
    assert (got["h"] == 0).all() and (got["da"] == 0).all()
    assert torch.equal(got["c"].cpu(), s["c0"]) and torch.equal(got["dc0"].cpu(), s["dcl"])


def test_zero_sizes():
    m = api()
    for B, T, D in ((0, 5, 8), (2, 0, 8), (2, 5, 0)):
        a, h = torch.zeros(B, T, 4, D, device="cuda"), torch.zeros(B, T, D, device="cuda")
        c0, cl = torch.randn(B, D, device="cuda"), torch.zeros(B, D, device="cuda")
        marks = m.scan_alloc_checkpoints(B, T, D)
        m.scan_forward(a, h, cl, c0=c0, checkpoints=marks)
        dc0 = torch.zeros(B, D, device="cuda")
        m.scan_backward(a, marks, h, torch.zeros_like(a), dc0, dc_last=c0)
        assert torch.equal(cl, c0) and torch.equal(dc0, c0)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("D,offset", [(64, 0), (64, 1), (67, 0), (130, 3)])
def test_strides(D, offset, dtype):
    """Time-major, gate-major and sliced tensors give what contiguous ones give, bit for bit
    where the channels a thread owns are the same, and within tolerance always."""
    B, T = 3, 70
    s = _case(B, T, D, dtype, seed=5)
    dt = DT[dtype]

    def put(x, order, lead):
        """x in memory order `order` with `lead` spare elements around its last dimension."""
        y = x.permute(order)
        wide = torch.full((*y.shape[:-1], y.shape[-1] + lead + offset), float("nan"), dtype=dt, device="cuda")
        wide = wide[..., offset:offset + y.shape[-1]]
        wide.copy_(y)
        back = [order.index(k) for k in range(len(order))]
        return wide.permute(back)

    for order, out in (((1, 0, 2, 3), (1, 0, 2)), ((2, 0, 1, 3), (0, 1, 2)), ((0, 2, 1, 3), (1, 0, 2))):
        for lead in (0, 2, 5):
            a = put(s["a"], order, lead)
            nan4, nan3 = torch.full_like(s["a"], float("nan")), torch.full_like(s["dh"], float("nan"))
            got = _run(s, a=a, h=put(nan3, out, lead), dh=put(s["dh"], out, lead),
                       da=put(nan4, order, lead))
            _check(s, got)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("B,D", [(1, 1), (3, 65), (64, 960), (500, 34)])
def test_step_continues_a_forward(B, D, dtype):
    m = api()
    s = _case(B, 5, D, dtype, seed=9)
    r = _reference(s)
    a, c = s["a"].cuda(), s["c0"].cuda()
    h = torch.empty(B, 5, D, dtype=DT[dtype], device="cuda")
    for t in range(5):
        m.scan_step(a[:, t], c, h[:, t])
    _near(h, r["h"], r["he"], dtype)
    _near(c, r["c"], r["cle"])


def test_extreme_gates():
    """Gates far out saturate without NaN, and infinite ones are their limits."""
    s = _case(1, 40, 8, "fp32", seed=3)
    x = torch.tensor([0.0, 1e-30, -1e-4, 20.0, -20.0, 95.0, -95.0, 3e38])
    for t in range(40):
        s["a"][0, t] = torch.stack([x.roll(k * t + k) for k in range(4)])
    _check(s, _run(s))
    s["a"][s["a"] > 90] = float("inf")
    s["a"][s["a"] < -90] = -float("inf")
    _check(s, _run(s))


def test_gradient_against_differences():
    """(L(a + eps w) - L(a - eps w)) / (2 eps) along random directions w, L = <h, dh> + <c_T, dcl>
    in 64 bits by the reference: the error of the central difference is O(eps^2)."""
    s = _case(2, 37, 5, "fp32", seed=4, resets=True)
    got = _run(s)
    eps = 1e-4

    def loss(a, c0):
        r = _reference({**s, "a": a, "c0": c0})
        return (r["h"] * s["dh"].double().numpy()).sum() + (r["c"] * s["dcl"].double().numpy()).sum()

    g = torch.Generator().manual_seed(0)
    for _ in range(4):
        w, w0 = torch.randn(s["a"].shape, generator=g).double(), torch.randn(s["c0"].shape, generator=g).double()
        a, c0 = s["a"].double(), s["c0"].double()
        num = (loss(a + eps * w, c0 + eps * w0) - loss(a - eps * w, c0 - eps * w0)) / (2 * eps)
        ana = (got["da"].double().cpu() * w).sum().item() + (got["dc0"].double().cpu() * w0).sum().item()
        assert abs(num - ana) <= 1e-4 * max(1.0, abs(num))


def test_same_call_gives_the_same_bits_and_streams():
    s = _case(2, 900, 66, "bf16", seed=6, ragged=True, resets=True)
    a, b = _run(s), _run(s, stream=torch.cuda.Stream())
    for k in a:
        assert torch.equal(a[k], b[k])


def test_long_and_far_offsets():
    """Strides that put the last step beyond 2^31 elements."""
    T, D, far = 5, 64, 1 << 29
    s = _case(1, T, D, "bf16", seed=8)
    flat = torch.zeros((T - 1) * far + 4 * D, dtype=torch.bfloat16, device="cuda")
    a = flat.as_strided((1, T, 4, D), (0, far, D, 1))
    a.copy_(s["a"])
    out = torch.zeros((T - 1) * far + 4 * D, dtype=torch.bfloat16, device="cuda")
    _check(s, _run(s, a=a, da=out.as_strided((1, T, 4, D), (0, far, D, 1))))


def test_binding_refuses():
    m = api()
    a, h = torch.zeros(2, 3, 4, 8, device="cuda"), torch.zeros(2, 3, 8, device="cuda")
    with pytest.raises(ValueError):
        m.scan_forward(a, h[:, :2])
    with pytest.raises(ValueError):
        m.scan_forward(a, h.half())
    with pytest.raises(ValueError):
        m.scan_forward(a.double(), h.double())
    with pytest.raises(ValueError):
        m.scan_forward(a[..., ::2], h[..., ::2])
    with pytest.raises(ValueError):
        m.scan_forward(a, h, lengths=torch.zeros(2, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        m.scan_backward(a, torch.zeros(3, device="cuda"), h, torch.zeros_like(a))
    with pytest.raises(ValueError):
        m.scan_step(a[:, 0], torch.zeros(2, 7, device="cuda"), h[:, 0])
