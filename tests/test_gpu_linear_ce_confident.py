"""Gradients of rows that are nearly certain of their target.

There the entry of G at the target is p - 1 = -(sum of the other probabilities), a small difference
of numbers near 1, and whatever its exponent l_y - lse is off by enters it in full.  Errors of
random sign are allowed; one that goes the same way in all rows is not.  For a row,
  E = u (4 |l| + 6 sqrt(d) s)
bounds what random roundings do to the exponent: lse is rounded to fp32 and so are the exponent
and what it is made of, and the logit is a sum of d products by multiply-adds with partial sums of
about s = |l| / 4 at most.  So the mean over N rows of the error of the entry, which is read off
dh along the target's row of emb, is allowed 5 E / sqrt(N), the roundings of the constants log2 e
and ln 2, u |l| together, and a hundredth of the entry (what G's and dh's own 16 bits make of
it)."""
import pytest
import torch

from gpu_common import api
from test_gpu_linear_ce import DT, U

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("N,V,d", [(512, 30000, 960), (512, 30000, 4096), (300, 30001, 1055),
                                   (100, 30000, 2048)])
def test_no_bias(N, V, d, dtype):
    m = api()
    g = torch.Generator(device="cuda").manual_seed(d + N)
    emb = (torch.randn(V, d, generator=g, device="cuda") / d ** 0.5).to(DT[dtype])
    y = torch.randint(0, V, (N,), generator=g, device="cuda")
    own = emb[y].double()
    # logits of 20 to 25 at the target, others of mean 0: losses of 1e-6 to 1e-4
    want_l = 20 + 5 * torch.rand(N, generator=g, device="cuda")
    h = (want_l[:, None] * own / (own * own).sum(1, keepdim=True)).to(DT[dtype])
    loss, lse = torch.empty(N, device="cuda"), torch.empty(N, device="cuda")
    dloss = torch.full((N,), 0.25, device="cuda")
    dh, demb = torch.empty_like(h), torch.empty_like(emb)
    ws = m.linear_ce_alloc_workspace(N, V, d, DT[dtype])
    m.linear_ce_forward(h, emb, y, loss, lse, ws)
    m.linear_ce_backward(h, emb, y, lse, dloss, dh, demb, ws)
    assert m.get_status() == 0

    l = h.double() @ emb.double().T
    rows = torch.arange(N, device="cuda")
    at = l[rows, y]
    exact_lse = torch.logsumexp(l, 1)
    G = torch.exp(l - exact_lse[:, None])
    G[rows, y] = 0.0
    rest = G.sum(1)
    assert (rest > 3e-7).all() and (rest < 5e-4).all()  # 30000 exp(-25) = 4e-7
    G[rows, y] = -rest
    ref = 0.25 * (G @ emb.double())
    off = ((dh.double() - ref) * own).sum(1) / (own * own).sum(1) / 0.25
    big = at.max().item()
    E = U * (4 * big + 6 * d ** 0.5 * big / 4)
    allowed = 5 * E / N ** 0.5 + U * big + 0.01 * rest.mean().item()
    assert abs(off.mean().item()) <= allowed, (off.mean().item(), allowed, rest.mean().item())
    # and the loss itself, as the forward call has it
    assert abs((loss.double() - (exact_lse - at)).mean().item()) <= 5 * E / N ** 0.5 + U * big
