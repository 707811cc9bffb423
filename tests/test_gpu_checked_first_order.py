"""The checked build on the first-order operators: on sizes that reach each of their kernels no
index check fails, no canary gap changes, and the results are the default build's."""
import numpy as np
import pytest
import torch

from gpu_common import api
from test_gpu_checked import CANARY, GUARD_WORDS, _default_path, checked_path, using  # noqa: F401

pytestmark = pytest.mark.gpu


def _ce(N, V, d, dtype, pad=0, offset=0, ignored=0.1):
    def run(a):
        g = torch.Generator(device="cuda").manual_seed(N + V + d)
        rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")

        def put(x):
            wide = torch.zeros(x.shape[0], x.shape[1] + pad, dtype=dtype, device="cuda")
            wide[:, :x.shape[1]] = x
            return wide[:, :x.shape[1]]

        def out(n):
            flat = torch.full((n * (d + pad) + offset,), float("nan"), dtype=dtype, device="cuda")
            return flat[offset:].view(n, d + pad)[:, :d]

        emb = put(rnd(V, d) * 1.5 / d ** 0.5)
        y = torch.randint(0, V, (N,), generator=g, device="cuda")
        h = put(rnd(N, d) + emb[y].float())
        skip = torch.rand(N, generator=g, device="cuda") < ignored
        y[skip] = -100
        h[skip] = float("nan")
        dloss = torch.rand(N, generator=g, device="cuda") / N
        loss, lse = (torch.full((N,), float("nan"), device="cuda") for _ in range(2))
        dh, demb = out(N), out(V)
        ws = a.linear_ce_alloc_workspace(N, V, d, dtype, True, d + pad, d + pad)
        a.linear_ce_forward(h, emb, y, loss, lse, ws)
        a.linear_ce_backward(h, emb, y, lse, dloss, dh, demb, ws)
        return dict(loss=loss, lse=lse, dh=dh, demb=demb), ws
    return run


def _scan(B, T, D, dtype, ragged=False):
    def run(a):
        g = torch.Generator(device="cuda").manual_seed(B + T + D)
        rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
        gates, dh = rnd(B, T, 4, D).to(dtype), rnd(B, T, D).to(dtype)
        kw = {}
        if ragged:
            kw["lengths"] = torch.randint(0, T + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
            kw["resets"] = (torch.rand(B, T, generator=g, device="cuda") < 0.1).to(torch.uint8)
        h, da = torch.full_like(dh, float("nan")), torch.full_like(gates, float("nan"))
        c0, dcl = rnd(B, D), rnd(B, D)
        cl, dc0 = torch.empty_like(c0), torch.empty_like(c0)
        marks = a.scan_alloc_checkpoints(B, T, D)
        ws = torch.zeros(max(1, a.scan_workspace_bytes(B, T, D)), dtype=torch.uint8, device="cuda")
        a.scan_forward(gates, h, cl, c0=c0, checkpoints=marks, workspace=ws, **kw)
        a.scan_backward(gates, marks, dh, da, dc0, dc_last=dcl, workspace=ws, **kw)
        a.scan_step(gates[:, 0], c0, dh[:, 0])
        return dict(h=h, c_last=cl, dgates=da, dc0=dc0, c=c0, h1=dh[:, 0]), ws
    return run


def _adamw(sizes, param, bits, master, offset):
    def run(a):
        g = torch.Generator(device="cuda").manual_seed(len(sizes))

        def put(n, dtype):
            flat = torch.zeros(n + offset, dtype=dtype, device="cuda")
            flat[offset:] = torch.randn(n, generator=g, device="cuda").to(dtype)
            return flat[offset:]

        w = [put(n, torch.float32) for n in sizes]
        p = [x.to(param) for x in w]
        opt = a.AdamW(p, **a.AdamW.zero_state(p, bits), masters=w if master else None,
                      weight_decay=0.1)
        for t in (1, 2):
            opt.step([put(n, param) for n in sizes], t=t, lr=1e-2, seed=3)
        out = {f"p{k}": x for k, x in enumerate(p)}
        out.update({f"m{k}": x.float() for k, x in enumerate(opt.tensors[1])})
        return out, None
    return run


BF, FP, F32 = torch.bfloat16, torch.float16, torch.float32
CASES = {
    "ce one tile": _ce(64, 256, 32, BF),
    "ce few rows": _ce(55, 3001, 65, BF),
    "ce one row": _ce(1, 40001, 64, FP, ignored=0.0),
    "ce byte head": _ce(2000, 256, 960, FP),
    "ce odd": _ce(300, 513, 129, BF, pad=2, offset=1),
    "ce copies": _ce(2100, 700, 72, FP),
    "ce pieces": _ce(20000, 8000, 16, BF),
    "scan tiled": _scan(3, 100, 64, BF),
    "scan tiled ragged": _scan(5, 100, 130, F32, ragged=True),
    "scan tiled chunks": _scan(1, 6000, 8, BF),
    "scan plain": _scan(3, 70, 33, FP),
    "scan plain ragged chunks": _scan(2, 3000, 33, F32, ragged=True),
    "scan one step": _scan(7, 1, 64, F32),
    "adamw 32": _adamw((1, 255, 2049, 70001), F32, 32, False, 0),
    "adamw 8 masters": _adamw((7, 256, 2049, 5000), BF, 8, True, 1),
    "adamw many": _adamw([1 + (k * 37) % 600 for k in range(500)], FP, 8, False, 0),
}


@pytest.mark.parametrize("name", list(CASES))
def test_no_check_fails_and_results_agree(checked_path, name):  # noqa: F811
    run = CASES[name]
    with using(_default_path()) as a:
        want, _ = run(a)
        assert a.get_status() == 0
    with using(checked_path) as a:
        assert a.lib().soma_checked_build() == 1
        got, ws = run(a)
        status = a.get_status()
        line = a.lib().soma_debug_check_line(None)
        assert (status, line) == (0, 0), (a.STATUS_NAMES.get(status, status), line)
    for k in want:
        assert torch.equal(got[k].isnan(), want[k].isnan())
        # the same operations in the same order: at most a contraction here and there differs
        x, y = (v[k].float().nan_to_num().cpu().numpy() for v in (got, want))
        rtol = 1e-5 if want[k].dtype == F32 else 2.0 ** -7
        np.testing.assert_allclose(x, y, rtol=rtol, atol=1e-6, err_msg=k)


@pytest.mark.parametrize("name", ["ce byte head", "ce pieces", "scan tiled chunks",
                                  "scan plain ragged chunks"])
def test_canary_gaps_are_intact(checked_path, name):  # noqa: F811
    with using(checked_path) as a:
        _, ws = CASES[name](a)
        assert a.get_status() == 0
    words = ws[:ws.numel() // 4 * 4].view(torch.int32).cpu().numpy().view(np.uint32)
    hit = words == np.uint32(CANARY)
    gaps = hit[:words.size // GUARD_WORDS * GUARD_WORDS].reshape(-1, GUARD_WORDS).all(axis=1)
    assert gaps.sum() >= (2 if name.startswith("scan") else 4)
    assert gaps[0] and gaps[-1]
