"""Sampling (soma_sample) against its definition in 64 bits: tokens are equal, log probabilities are
good to fp32 (2^-23 of themselves and 2^-36 absolutely, for sums of weights good to a few 2^-40)."""
import numpy as np
import pytest
import torch

from gpu_common import api

pytestmark = pytest.mark.gpu

DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def _column(x, R, dtype=np.float32):
    return np.asarray(x.cpu() if torch.is_tensor(x) else np.full(R, x), dtype=dtype)


def _reference(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    l = logits.double().cpu().numpy()
    R, V = l.shape
    T, P, M = (_column(x, R).astype(np.float64) for x in (temperature, top_p, min_p))
    K, u = _column(top_k, R, np.int64), u.double().cpu().numpy()
    token, chance = np.full(R, -1), np.full(R, np.nan)
    for r in range(R):
        if np.isnan(l[r]).any() or np.isposinf(l[r]).any() or np.isneginf(l[r]).all():
            continue
        top = l[r].max()
        if T[r] < 2.0 ** -100:
            token[r], chance[r] = l[r].argmax(), 0.0
            continue
        x = (l[r] - top) / min(T[r], 2.0 ** 100)
        w = np.rint(2.0 ** 40 * np.exp(x)).astype(np.int64)
        order = np.argsort(-l[r], kind="stable")
        s = w[order]
        if K[r] > 0:
            s[K[r]:] = 0
        if P[r] < 1:
            want = max(1, int(np.ceil(P[r] * float(s.sum()))))
            s[1:][np.cumsum(s)[:-1] >= want] = 0
        s[s < min(M[r], 1.0) * 2.0 ** 40] = 0
        w[order] = s
        run = np.cumsum(w)
        at = min(int(u[r] * float(run[-1])), int(run[-1]) - 1)
        token[r] = np.searchsorted(run, at, side="right")
        chance[r] = x[token[r]] - np.log(float(run[-1]) * 2.0 ** -40)
    return token, chance


def _run(logits, u, **kw):
    R = logits.shape[0]
    token = torch.full((R,), -7, dtype=torch.int64, device="cuda")
    chance = torch.full((R,), 7.0, device="cuda")
    api().sample(logits, u, token, logprob=chance, **kw)
    return token.cpu().numpy(), chance.double().cpu().numpy()


def _check(logits, u, status=0, **kw):
    token, chance = _run(logits, u, **kw)
    want, p = _reference(logits, u, **kw)
    assert (token == want).all(), np.flatnonzero(token != want)[:5]
    assert (np.isnan(p) == np.isnan(chance)).all()
    fine = ~np.isnan(p)
    assert (np.abs(chance - p)[fine] <= 2.0 ** -23 * np.abs(p[fine]) + 2.0 ** -36).all()
    assert api().get_status() == status


def _logits(R, V, dtype, seed=0, spread=2.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    l = torch.randn(R, V, generator=g, device="cuda") * spread
    l[:, ::97] += torch.rand(R, -(-V // 97), generator=g, device="cuda") * 8
    return l.to(DT[dtype]), torch.rand(R, generator=g, device="cuda")


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("R,V", [(1, 1), (4, 2), (300, 7), (64, 256), (50, 1000), (9, 2049), (20, 5003),
                                 (3, 50021), (2, 131072), (1, 200001)])
def test_temperature(R, V, dtype):
    l, u = _logits(R, V, dtype, seed=V)
    for t in (1.0, 0.3, 5.0):
        _check(l, u, temperature=t)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("R,V", [(40, 50), (64, 256), (30, 3000), (7, 40001), (2, 131072)])
def test_cuts(R, V, dtype):
    l, u = _logits(R, V, dtype, seed=V + 1)
    for kw in (dict(top_k=1), dict(top_k=5), dict(top_k=V // 2), dict(top_k=V), dict(top_k=V + 9),
               dict(top_p=0.0), dict(top_p=0.01), dict(top_p=0.5), dict(top_p=0.9), dict(top_p=0.9999),
               dict(min_p=0.02), dict(min_p=1.0), dict(min_p=2.0), dict(top_k=40, top_p=0.8),
               dict(top_k=30, top_p=0.95, min_p=0.05, temperature=0.6), dict(top_p=0.7, temperature=3.0),
               dict(top_k=1000, top_p=0.999, temperature=2.0)):
        _check(l, u, **kw)


@pytest.mark.parametrize("V", [10, 300, 9000])
def test_ties(V):
    """Equal logits rank by index, on both sides of a cut; the whole row may be one value."""
    g = torch.Generator(device="cuda").manual_seed(V)
    few = torch.randint(0, 3, (60, V), generator=g, device="cuda").float()
    one, u = torch.full((60, V), -3.5, device="cuda"), torch.rand(60, generator=g, device="cuda")
    for l in (few, one, few.bfloat16(), one.half()):
        for kw in (dict(), dict(top_k=3), dict(top_k=V // 2 + 1), dict(top_p=0.37), dict(min_p=0.5),
                   dict(top_k=V // 2 + 1, top_p=0.63), dict(top_k=7, top_p=0.2, temperature=0.5)):
            _check(l, u, **kw)


def test_zeros_of_both_signs_are_equal():
    l = torch.zeros(64, 40, device="cuda")
    l[:, ::2] = -0.0
    u = (torch.arange(64, device="cuda") + 0.5) / 64
    for kw in (dict(), dict(top_k=5), dict(top_p=0.31), dict(temperature=0.0)):
        _check(l, u, **kw)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("V", [33, 7000, 60000])
def test_masks(V, dtype):
    """-infinity and the type's lowest value: never chosen while something else is left."""
    l, u = _logits(12, V, dtype, seed=V)
    l[0::3, V // 3:] = float("-inf")
    l[1::3, : V - 1] = torch.finfo(DT[dtype]).min
    l[2::3, 1:] = float("-inf")
    for kw in (dict(), dict(top_k=4), dict(top_p=0.9), dict(top_k=V // 2, top_p=0.99, min_p=0.001)):
        _check(l, u, **kw)
    l[:] = torch.finfo(DT[dtype]).min
    _check(l, u)
    l[5] = float("-inf")
    _check(l, u, top_p=0.5)


def test_rows_without_an_answer():
    l, u = _logits(6, 500, "fp32")
    l[1, 7], l[2, 499], l[3] = float("nan"), float("inf"), float("-inf")
    _check(l, u, status=6, top_k=9)
    one = torch.ones(6, device="cuda")
    for name in ("temperature", "top_p", "min_p"):
        l, u = _logits(6, 500, "fp32")
        x = one.clone()
        x[4] = float("nan")
        token, chance = _run(l, u, **{name: x})
        assert token[4] == -1 and np.isnan(chance[4]) and (np.delete(token, 4) >= 0).all()
        assert api().get_status() == 6
    for bad in (-0.25, 1.0, 7.0, float("nan")):
        u[2] = bad
        token, _ = _run(l, u)
        assert token[2] == -1 and (np.delete(token, 2) >= 0).all() and api().get_status() == 6


def test_temperatures_of_zero_and_far_ones():
    l, u = _logits(8, 3000, "fp32", seed=5)
    l[:, 100] = l[:, 200] = 50.0
    for t in (0.0, 1e-35, 1e-20, 1e-6, 1e6, 1e30, 1e38, float("inf")):
        _check(l, u, temperature=t)
        _check(l, u, temperature=t, top_k=50, top_p=0.5)


@pytest.mark.parametrize("R,V", [(33, 257), (9, 33000)])
def test_settings_of_each_row(R, V):
    l, u = _logits(R, V, "bf16", seed=R)
    g = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda: torch.rand(R, generator=g, device="cuda")
    t, k = rand() * 2, torch.randint(-2, 60, (R,), generator=g, device="cuda", dtype=torch.int32)
    t[0], k[1] = 0.0, 2 ** 31 - 1
    _check(l, u, temperature=t, top_k=k, top_p=rand() * 1.3, min_p=rand() * 0.1)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("offset,stride", [(0, 1003), (1, 1001), (3, 1008), (0, 1000), (7, 5000)])
def test_rows_of_any_alignment(offset, stride, dtype):
    l, u = _logits(20, 1000, dtype, seed=8)
    flat = torch.full((offset + 20 * stride,), float("nan"), dtype=DT[dtype], device="cuda")
    rows = flat[offset:].view(20, stride)[:, :1000]
    rows.copy_(l)
    _check(rows, u, top_k=77, top_p=0.9)
    _check(rows, u)


def test_the_ends_of_u():
    l, _ = _logits(4, 400, "fp32")
    l[:, :3] = float("-inf")
    u = torch.tensor([0.0, 2.0 ** -24, 1 - 2.0 ** -24, 0.5], device="cuda")
    _check(l, u)
    token, _ = _run(l, u)
    assert token[0] == 3 and token[2] == 399


def test_frequencies():
    """10^5 draws from one row of five tokens: each share within 6 sigma."""
    p = torch.tensor([0.4, 0.05, 0.3, 0.05, 0.2], device="cuda")
    l = p.log().expand(100000, 5).contiguous()
    token, _ = _run(l, torch.rand(100000, device="cuda"))
    share = np.bincount(token, minlength=5) / 1e5
    q = p.cpu().numpy()
    assert (np.abs(share - q) <= 6 * np.sqrt(q * (1 - q) / 1e5)).all()


def test_repeated_calls_and_another_stream():
    l, u = _logits(5, 70000, "bf16", seed=3)
    kw = dict(top_k=0, top_p=0.8, temperature=1.3)
    a = _run(l, u, **kw)
    b = _run(l, u, **kw)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    token, chance = torch.empty(5, dtype=torch.int64, device="cuda"), torch.empty(5, device="cuda")
    api().sample(l, u, token, logprob=chance, stream=side, **kw)
    side.synchronize()
    assert (a[0] == b[0]).all() and (a[1] == b[1]).all()
    assert (token.cpu().numpy() == a[0]).all()
    api().sample(l[:0], u[:0], token[:0])


def test_without_logprob_in_a_graph():
    l, u = _logits(6, 9000, "fp32", seed=4)
    token = torch.empty(6, dtype=torch.int64, device="cuda")
    api().sample(l, u, token, top_p=0.6)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        api().sample(l, u, token, top_p=0.6)
    for seed in (5, 6):
        l2, u2 = _logits(6, 9000, "fp32", seed=seed)
        l.copy_(l2), u.copy_(u2)
        graph.replay()
        torch.cuda.synchronize()
        assert (token.cpu().numpy() == _reference(l2, u2, top_p=0.6)[0]).all()
