"""The checked build on linear attention, dropout and sampling: on sizes that reach each of their kernels
no index check fails, no canary gap changes, and the results are the default build's."""
import pytest
import torch

from test_gpu_checked import _default_path, checked_path, using  # noqa: F401

pytestmark = pytest.mark.gpu


def _attn(B, T, H, dk, dv, dtype, ragged=False):
    def run(a):
        g = torch.Generator(device="cuda").manual_seed(B + T + dk)
        rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
        q, k = (rnd(B, T, H, dk).to(dtype) for _ in range(2))
        v, do = (rnd(B, T, H, dv).to(dtype) for _ in range(2))
        s0, dsl, decay = rnd(B, H, dk, dv), rnd(B, H, dk, dv), -torch.rand(H, generator=g, device="cuda")
        kw = dict(s0=s0, scale=dk ** -0.5)
        if ragged:
            kw["lengths"] = torch.randint(0, T + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
            kw["resets"] = (torch.rand(B, T, generator=g, device="cuda") < 0.1).to(torch.uint8)
        o, sl = torch.full_like(v, float("nan")), torch.empty_like(s0)
        dq, dkk, dvv, ds0 = (torch.full_like(x, float("nan")) for x in (q, k, v, s0))
        ws = torch.zeros(max(1, a.linear_attn_workspace_bytes(B, T, H, dk, dv, dtype)), dtype=torch.uint8,
                         device="cuda")
        a.linear_attn_forward(q, k, v, decay, o, s_last=sl, workspace=ws, **kw)
        a.linear_attn_backward(q, k, v, decay, do, dq, dkk, dvv, ds_last=dsl, ds0=ds0, workspace=ws, **kw)
        o1 = torch.empty(B, H, dv, dtype=dtype, device="cuda")
        a.linear_attn_step(q[:, 0], k[:, 0], v[:, 0], decay, s0, o1)
        return dict(o=o, s_last=sl, dq=dq, dk=dkk, dv=dvv, ds0=ds0, s=s0, o1=o1)
    return run


def _dropout(rows, cols, dtype, pad=0):
    def run(a):
        g = torch.Generator(device="cuda").manual_seed(rows)
        x, r = (torch.randn(rows, cols + pad, generator=g, device="cuda").to(dtype)[:, :cols] for _ in range(2))
        y = torch.empty(rows, cols, dtype=dtype, device="cuda")
        a.dropout(x, y, 0.3, seed=1, offset=2, residual=r)
        return dict(y=y)
    return run


def _sample(R, V, dtype, **kw):
    def run(a):
        g = torch.Generator(device="cuda").manual_seed(V)
        l, u = (torch.randn(R, V, generator=g, device="cuda") * 3).to(dtype), torch.rand(R, generator=g, device="cuda")
        token, lp = torch.empty(R, dtype=torch.int64, device="cuda"), torch.empty(R, device="cuda")
        a.sample(l, u, token, logprob=lp, **kw)
        return dict(token=token, logprob=lp)
    return run


CASES = {
    "attn_fp32": _attn(2, 150, 2, 33, 20, torch.float32, ragged=True),
    "attn_fp32_cut": _attn(1, 2000, 1, 16, 16, torch.float32),
    "attn_64": _attn(2, 300, 2, 64, 40, torch.bfloat16, ragged=True),
    "attn_64_cut": _attn(1, 5000, 1, 64, 64, torch.float16),
    "attn_128": _attn(2, 300, 2, 128, 72, torch.float16, ragged=True),
    "attn_128_cut": _attn(1, 5000, 1, 96, 128, torch.bfloat16, ragged=True),
    "attn_short": _attn(3, 7, 2, 48, 128, torch.bfloat16),
    "dropout": _dropout(30, 64, torch.bfloat16),
    "dropout_odd": _dropout(30, 61, torch.float16, pad=3),
    "sample": _sample(20, 300, torch.float32, top_k=20, top_p=0.9),
    "sample_wide": _sample(3, 70001, torch.bfloat16, top_p=0.9),
    "sample_widest": _sample(2, 200001, torch.float32, top_k=5000, top_p=0.95, min_p=0.001),
}


@pytest.mark.parametrize("name", list(CASES))
def test_no_check_fails_and_results_agree(checked_path, name):  # noqa: F811
    with using(_default_path()) as a:
        want = CASES[name](a)
        assert a.get_status() == 0
    with using(checked_path) as a:
        assert a.lib().soma_checked_build() == 1
        got = CASES[name](a)
        status, line = a.get_status(), a.lib().soma_debug_check_line(None)
        assert (status, line) == (0, 0), (a.STATUS_NAMES.get(status, status), line)
    for k in want:
        # the same operations in the same order: at most a contraction here and there differs
        x, y = (v[k].double() for v in (got, want))
        rtol = {torch.float32: 1e-5, torch.int64: 0.0}.get(want[k].dtype, 2.0 ** -7)
        assert ((x - y).abs() <= rtol * y.abs() + (1e-5 if rtol else 0.0)).all(), k
