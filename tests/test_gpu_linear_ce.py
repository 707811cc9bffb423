"""Linear cross entropy (soma_linear_ce_*) against its formulas in 64 bits.

Tolerances, u = 2^-24 and hu half an ulp of the 16-bit type (2^-8 bf16, 2^-11
fp16, relative to the value):
 - a logit is a sum of exact products, rounded (or cut) once per four products
   at most: el = 2 u (dim / 4 + 4) sum |h_k e_k|;
 - lse and loss add the rounding of the exponents, 4 u max |l|, of a sum of
   vocab terms, u (64 + 4 sqrt(vocab)), and of the logits;
 - G = g (p - onehot) is off by |g| p times the errors of its exponent, and by
   hu |G| from its rounding; the gradients carry sum |dG| |emb| (or |h|), the
   rounding of their own sums as for a logit, and hu of the result.
"""
import pytest
import torch

from gpu_common import api

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "fp16": torch.float16}
HU = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}
LOW = {"bf16": 2.0 ** -126, "fp16": 2.0 ** -25}
IGNORE = -100


def _case(N, V, d, dtype, seed=0, ignored=0.0, spread=1.5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    emb = (rnd(V, d) * spread / d ** 0.5).to(DT[dtype])
    y = torch.randint(0, V, (N,), generator=g, device="cuda")
    h = (rnd(N, d) + emb[y].float()).to(DT[dtype])
    skip = torch.rand(N, generator=g, device="cuda") < ignored
    y[skip] = IGNORE
    h[skip] = float("nan")
    dloss = (torch.rand(N, generator=g, device="cuda") + 0.1) / max(N, 1)
    dloss[skip] = float("nan")
    return dict(h=h, emb=emb, y=y, dloss=dloss, dtype=dtype)


def _reference(s):
    h, emb, y, hu = s["h"].double(), s["emb"].double(), s["y"], HU[s["dtype"]]
    N, d = h.shape
    V = emb.shape[0]
    keep = (y >= 0) & (y < V)
    h = torch.where(keep[:, None], h, 0.0)
    at = torch.where(keep, y, 0)
    g = torch.where(keep, s["dloss"].double(), 0.0)
    l = h @ emb.T
    el = 2 * U * (d / 4 + 4) * (h.abs() @ emb.abs().T)
    lse = torch.logsumexp(l, 1)
    own = l.gather(1, at[:, None])[:, 0]
    big = l.abs().amax(1)
    elm = el.amax(1)
    e_lse = elm + U * (4 * big + 64 + 4 * V ** 0.5)
    p = torch.exp(l - lse[:, None])
    G = p.clone()
    G[torch.arange(N, device="cuda"), at] -= 1.0
    G *= g[:, None]
    # |g| p (error of the exponent), |g| times the rounding of p - 1, the rounding to 16 bits
    dG = g.abs()[:, None] * (p * (el + e_lse[:, None] + U * (4 * big[:, None] + 8)) + 0.0)
    dG += 4 * U * G.abs() + hu * G.abs() + LOW["bf16"] + 2.0 ** -38 * g.abs().amax()
    dh, demb = G @ emb, G.T @ h
    out = {"loss": (lse - own) * keep, "lse": lse * keep, "dh": dh, "demb": demb}
    tol = {"lse": e_lse * keep, "loss": (e_lse + el.gather(1, at[:, None])[:, 0] + 2 * U * big) * keep,
           "dh": dG @ emb.abs() + 2 * U * (V / 4 + 4) * (G.abs() @ emb.abs()) + hu * dh.abs() + LOW[s["dtype"]],
           "demb": dG.T @ h.abs() + 2 * U * (N / 4 + 4) * (G.abs().T @ h.abs()) + hu * demb.abs() + LOW[s["dtype"]]}
    return out, tol


def _run(s, h=None, emb=None, dh=None, demb=None, stream=None):
    m = api()
    h, emb = s["h"] if h is None else h, s["emb"] if emb is None else emb
    N, d = h.shape
    V = emb.shape[0]
    nan = lambda *shape: torch.full(shape, float("nan"), dtype=h.dtype, device="cuda")
    dh, demb = nan(N, d) if dh is None else dh, nan(V, d) if demb is None else demb
    loss, lse = (torch.full((N,), float("nan"), device="cuda") for _ in range(2))
    ws = m.linear_ce_alloc_workspace(N, V, d, h.dtype, True, h.stride(0) if N > 1 else None,
                                     emb.stride(0) if V > 1 else None).fill_(0xFF)
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())
    m.linear_ce_forward(h, emb, s["y"], loss, lse, ws, ignore_index=IGNORE, stream=stream)
    m.linear_ce_backward(h, emb, s["y"], lse, s["dloss"], dh, demb, ws, ignore_index=IGNORE,
                         stream=stream)
    torch.cuda.synchronize()
    return {"loss": loss, "lse": lse, "dh": dh, "demb": demb}


def _check(s, got):
    want, tol = _reference(s)
    for k, w in want.items():
        off = (got[k].double() - w).abs()
        bad = ~(off <= tol[k])
        assert not bad.any(), (k, int(bad.sum()), bad.nonzero()[:3].tolist(),
                               float(off.nan_to_num(9e9).max()))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("N,V,d", [
    (1, 1, 1), (1, 300, 8), (5, 7, 3), (64, 256, 32), (130, 257, 64), (128, 256, 64),
    (200, 1000, 72), (257, 513, 100), (33, 5000, 136), (300, 70, 65), (1, 40001, 64),
    (700, 300, 200), (2000, 256, 960), (129, 2049, 321), (3, 100, 1400), (1500, 1500, 24)])
def test_sizes(N, V, d, dtype):
    s = _case(N, V, d, dtype, seed=N + V + d)
    _check(s, _run(s))
    assert api().get_status() == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("N,V,d,ignored", [(300, 500, 64, 0.3), (400, 257, 130, 0.9), (140, 64, 40, 1.1)])
def test_ignored_rows(N, V, d, ignored, dtype):
    """Ignored rows hold NaN in h and dloss; with 1.1 every row is ignored."""
    s = _case(N, V, d, dtype, seed=2, ignored=ignored)
    got = _run(s)
    _check(s, got)
    skip = s["y"] == IGNORE
    assert (got["loss"][skip] == 0).all() and (got["dh"][skip] == 0).all()
    assert api().get_status() == 0


def test_no_rows():
    s = _case(0, 300, 40, "bf16")
    got = _run(s)
    assert (got["demb"] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("d,pad", [(64, 8), (64, 3), (67, 0), (67, 6), (40, 1)])
def test_strides(d, pad, dtype):
    """Rows further apart than they are long; the gaps hold NaN and stay untouched."""
    s = _case(150, 600, d, dtype, seed=3)

    def wide(x):
        y = torch.full((x.shape[0], x.shape[1] + pad), float("nan"), dtype=x.dtype, device="cuda")
        y[:, :x.shape[1]] = x
        return y

    h, emb = wide(s["h"]), wide(s["emb"])
    dh, demb = wide(torch.zeros_like(s["h"])), wide(torch.zeros_like(s["emb"]))
    got = _run(s, h=h[:, :d], emb=emb[:, :d], dh=dh[:, :d], demb=demb[:, :d])
    _check(s, got)
    if pad:
        assert dh[:, d:].isnan().all() and demb[:, d:].isnan().all()


def test_gradients_at_unaligned_outputs():
    s = _case(90, 300, 64, "bf16", seed=4)
    flat = [torch.full((n * 64 + 1,), float("nan"), dtype=torch.bfloat16, device="cuda") for n in (90, 300)]
    got = _run(s, dh=flat[0][1:].view(90, 64), demb=flat[1][1:].view(300, 64))
    _check(s, got)
    assert flat[0][0].isnan() and flat[1][0].isnan()


@pytest.mark.parametrize("N,V,d", [(20000, 8000, 16), (70001, 2500, 24)])
def test_several_pieces_of_the_vocabulary(N, V, d):
    s = _case(N, V, d, "bf16", seed=5, ignored=0.1)
    _check(s, _run(s))


def test_targets_outside_the_vocabulary():
    s = _case(50, 100, 32, "bf16", seed=6)
    s["y"][3], s["y"][7], s["y"][9] = 100, -1, 1 << 40
    got = _run(s)
    m = api()
    assert m.get_status() == 6
    bad = torch.tensor([3, 7, 9], device="cuda")
    assert got["loss"][bad].isnan().all() and got["loss"].isnan().sum() == 3
    assert (got["dh"][bad] == 0).all()
    want, tol = _reference(s)
    for k in ("dh", "demb"):
        assert ((got[k].double() - want[k]).abs() <= tol[k]).all()


def test_a_state_that_is_not_finite_is_reported():
    s = _case(200, 300, 32, "bf16", seed=7)
    s["h"][150, 5] = float("inf")
    m = api()
    loss, lse = torch.zeros(200, device="cuda"), torch.zeros(200, device="cuda")
    ws = m.linear_ce_alloc_workspace(200, 300, 32, torch.bfloat16)
    m.linear_ce_forward(s["h"], s["emb"], s["y"], loss, lse, ws)
    assert m.get_status() == 6
    assert loss[150].isnan() and loss.isnan().sum() == 1


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_large_logits(dtype):
    """Logits of several hundred, where exp overflows without the running maximum."""
    s = _case(200, 700, 64, dtype, seed=8, spread=40.0)
    _check(s, _run(s))


def test_upstream_gradients_of_very_different_size():
    s = _case(300, 400, 48, "fp16", seed=9)
    s["dloss"] *= 10.0 ** (-3 * torch.rand(300, device="cuda"))
    s["dloss"][::7] = 0.0
    s["dloss"] *= 4096.0
    got = _run(s)
    _check(s, got)
    assert (got["dh"][::7] == 0).all()


def test_gradient_against_differences():
    """(L(x + eps w) - L(x - eps w)) / (2 eps) of L = <loss, dloss>, by the reference in 64 bits.
    The gradients are rounded to 16 bits, so the directional derivative is off by no more than
    the tolerances of its terms."""
    s = _case(60, 90, 24, "bf16", seed=10)
    got = _run(s)
    _, tol = _reference(s)

    def loss(h, emb):
        l = h @ emb.T
        own = l.gather(1, s["y"][:, None])[:, 0]
        return ((torch.logsumexp(l, 1) - own) * s["dloss"].double()).sum()

    g = torch.Generator(device="cuda").manual_seed(0)
    eps = 1e-4
    for _ in range(4):
        w = [torch.randn(s[k].shape, generator=g, device="cuda").double() for k in ("h", "emb")]
        h, emb = s["h"].double(), s["emb"].double()
        num = (loss(h + eps * w[0], emb + eps * w[1]) - loss(h - eps * w[0], emb - eps * w[1])) / (2 * eps)
        ana = (got["dh"].double() * w[0]).sum() + (got["demb"].double() * w[1]).sum()
        allowed = (tol["dh"] * w[0].abs()).sum() + (tol["demb"] * w[1].abs()).sum() + 1e-6
        assert (num - ana).abs() <= allowed


def test_same_bits_every_time_and_on_a_side_stream():
    s = _case(300, 3001, 200, "bf16", seed=11, ignored=0.1)
    a, b = _run(s), _run(s, stream=torch.cuda.Stream())
    for k in a:
        assert torch.equal(a[k], b[k])


def test_binding_refuses():
    m = api()
    s = _case(20, 30, 16, "bf16")
    loss, lse = torch.zeros(20, device="cuda"), torch.zeros(20, device="cuda")
    ws = m.linear_ce_alloc_workspace(20, 30, 16, torch.bfloat16)
    f = m.linear_ce_forward
    for bad in (lambda: f(s["h"], s["emb"].half(), s["y"], loss, lse, ws),
                lambda: f(s["h"], s["emb"][:, :8], s["y"], loss, lse, ws),
                lambda: f(s["h"], s["emb"], s["y"].int(), loss, lse, ws),
                lambda: f(s["h"], s["emb"], s["y"][:10], loss, lse, ws),
                lambda: m.linear_ce_alloc_workspace(20, 30, 16, torch.float32)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(m.SomaError):
        f(s["h"], s["emb"], s["y"], loss, lse, ws[:16])
    with pytest.raises(m.SomaError):
        f(s["h"].float(), s["emb"].float(), s["y"], loss, lse, ws)
