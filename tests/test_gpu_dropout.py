"""Dropout from the counter-based generator (soma_dropout) against its definition.

The mask is exact.  A kept value is x / (1 - p') + residual in fp32: one rounding of the factor, of the
product and of the sum (each u = 2^-24 of its term), then half an ulp of the type."""
import numpy as np
import pytest
import torch

import philox_ref
from gpu_common import api

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
ULP = {"fp32": (U, 2.0 ** -126), "bf16": (2.0 ** -8, 2.0 ** -126), "fp16": (2.0 ** -11, 2.0 ** -25)}


def _bits(count, seed, call):
    """16 bits per element, from the generator's definition."""
    n = -(-count // 8)
    c = [np.arange(n, dtype=np.uint64), np.full(n, call & 0xFFFFFFFF, np.uint64),
         np.full(n, call >> 32, np.uint64), np.full(n, 0x80000003, np.uint64)]
    k, low = [seed & 0xFFFFFFFF, seed >> 32], np.uint64(0xFFFFFFFF)
    for _ in range(10):
        a, b = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & low,
             (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    w = np.stack(c, 1)
    return np.stack((w & np.uint64(0xFFFF), w >> np.uint64(16)), 2).reshape(-1)[:count]


def _check(x, y, p, seed, call, residual=None, dtype="fp32"):
    drop = round(p * 65536)
    keep = torch.from_numpy(_bits(x.numel(), seed, call) >= drop).cuda().view(x.shape)
    v = torch.where(keep, x.double() * (65536 / max(65536 - drop, 1)), 0.0)
    r = torch.zeros_like(v) if residual is None else residual.double()
    half, tiny = ULP[dtype]
    tol = 2 * U * v.abs() + U * (v + r).abs() + half * (v + r).abs() * (dtype != "fp32") + tiny
    assert ((y.double() - (v + r)).abs() <= tol).all()
    if residual is None:
        assert torch.equal(y != 0, keep & (y != 0)) and (y[~keep] == 0).all()
    else:
        assert torch.equal(y[~keep], residual[~keep])


def test_the_reference_is_the_generator():
    if not philox_ref.available():
        pytest.skip("torch's header is not installed")
    words = philox_ref.blocks(0x123456789ABCDEF, [[3, 7, 2, 0x80000003]])[0].astype(np.uint64)
    bits = _bits(32, 0x123456789ABCDEF, 7 + (2 << 32))[24:32]
    assert (np.stack((words & np.uint64(0xFFFF), words >> np.uint64(16)), 1).reshape(-1) == bits).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 7), (3, 8), (5, 31), (64, 33), (7, 256), (100, 681),
                                       (33, 1376), (1, 5000), (5000, 1), (700, 3)])
@pytest.mark.parametrize("residual", [False, True])
def test_values(rows, cols, dtype, residual):
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    x, r = (torch.randn(rows, cols, generator=g, device="cuda").to(DT[dtype]) for _ in range(2))
    y = torch.full_like(x, float("nan"))
    api().dropout(x, y, 0.3, seed=11, offset=5, residual=r if residual else None)
    _check(x, y, 0.3, 11, 5, r if residual else None, dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("cols,xs,ys,rs", [(40, 48, 40, 56), (40, 41, 40, 40), (33, 40, 33, 64), (8, 16, 24, 8),
                                           (64, 64, 65, 64)])
def test_strides(cols, xs, ys, rs, dtype):
    """The mask goes by the element's place, whatever the strides; what lies between rows stays."""
    make = lambda s: torch.randn(50, s, device="cuda").to(DT[dtype])
    x, r, wide = make(xs)[:, :cols], make(rs)[:, :cols], torch.full((50, ys), 3.0, dtype=DT[dtype], device="cuda")
    api().dropout(x, wide[:, :cols], 0.5, seed=1, offset=2, residual=r)
    _check(x, wide[:, :cols], 0.5, 1, 2, r, dtype)
    assert (wide[:, cols:] == 3.0).all()


def test_alignment_does_not_change_the_mask():
    flat = torch.randn(4097, device="cuda").bfloat16()
    a, b = torch.empty(4096, device="cuda").bfloat16(), torch.empty(4097, device="cuda").bfloat16()
    x = flat[1:].clone()
    api().dropout(x, a, 0.4, seed=3)
    api().dropout(flat[1:], b[1:], 0.4, seed=3)
    assert torch.equal(a, b[1:])


@pytest.mark.parametrize("p", [0.0, 1.0, 1e-6, 0.999999, 0.5])
def test_ends_of_the_range(p):
    x, r = torch.randn(40, 64, device="cuda"), torch.randn(40, 64, device="cuda")
    y = torch.empty_like(x)
    api().dropout(x, y, p, seed=9, offset=1, residual=r)
    _check(x, y, p, 9, 1, r)
    if round(p * 65536) == 65536:
        assert torch.equal(y, r)
    if round(p * 65536) == 0:
        assert torch.equal(y, x + r)


def test_what_is_dropped_may_be_anything():
    x = torch.full((64, 64), float("nan"), device="cuda")
    x[::2] = float("inf")
    keep = torch.from_numpy(_bits(4096, 4, 0) >= 32768).cuda().view(64, 64)
    y = torch.empty_like(x)
    api().dropout(x, y, 0.5, seed=4)
    assert (y[~keep] == 0).all() and not y[keep].isfinite().any()


def test_in_place_and_the_gradient():
    """y may be x; the gradient of x is the same call on dy: <dy, y> = <dx, x> for every x."""
    x, dy = (torch.randn(301, 77, device="cuda") for _ in range(2))
    y, dx, same = torch.empty_like(x), torch.empty_like(x), x.clone()
    api().dropout(x, y, 0.2, seed=5, offset=9)
    api().dropout(dy, dx, 0.2, seed=5, offset=9)
    api().dropout(same, same, 0.2, seed=5, offset=9)
    assert torch.equal(same, y)
    a, b = (dy.double() * y.double()).sum(), (dx.double() * x.double()).sum()
    assert abs(a - b) <= 4 * U * (dy.double() * y.double()).abs().sum()


def test_calls_differ_and_the_counter_advances_them():
    x, counter = torch.ones(100, 100, device="cuda"), torch.tensor([2 ** 33 + 7], device="cuda")
    a, b, c = (torch.empty_like(x) for _ in range(3))
    api().dropout(x, a, 0.5, seed=1, offset=0)
    api().dropout(x, b, 0.5, seed=1, offset=1)
    api().dropout(x, c, 0.5, seed=2, offset=0)
    for u, v in ((a, b), (a, c), (b, c)):  # independent masks agree in half of 10^4 places, +- 6 sigma
        assert abs((u == v).sum().item() - 5000) <= 300
    api().dropout(x, a, 0.5, seed=1, offset=2 ** 33 + 10)
    api().dropout(x, b, 0.5, seed=1, offset=3, counter=counter)
    assert torch.equal(a, b)
    _check(x, a, 0.5, 1, 2 ** 33 + 10)


def test_share_of_kept_elements():
    x = torch.ones(1000, 1000, device="cuda")
    y = torch.empty_like(x)
    for p in (0.1, 0.35):
        api().dropout(x, y, p, seed=77)
        assert abs((y == 0).double().mean().item() - round(p * 65536) / 65536) <= 6 * (p * (1 - p)) ** 0.5 / 1000


def test_other_dimensions():
    x = torch.randn(3, 5, 24, device="cuda")
    y, z = torch.empty_like(x), torch.empty(15, 24, device="cuda")
    api().dropout(x, y, 0.5, seed=1)
    api().dropout(x.view(15, 24), z, 0.5, seed=1)
    assert torch.equal(y.view(15, 24), z)
    e = torch.empty(0, 5, device="cuda")
    api().dropout(e, e, 0.5, seed=1)
    e = torch.empty(5, 0, device="cuda")
    api().dropout(e, e, 0.5, seed=1)


def test_a_replayed_graph_gets_other_masks_from_its_counter():
    x, counter = torch.ones(64, 64, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    y = torch.empty_like(x)
    api().dropout(x, y, 0.5, seed=3, counter=counter)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        api().dropout(x, y, 0.5, seed=3, counter=counter)
        counter += 1
    got = []
    for k in range(3):
        graph.replay()
        torch.cuda.synchronize()
        _check(x, y, 0.5, 3, k)
        got.append(y.clone())
    assert not torch.equal(got[0], got[1]) and not torch.equal(got[1], got[2])
