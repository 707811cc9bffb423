"""The first-order operators captured in a CUDA graph: a replay gives what a call gives, bit for
bit, also with inputs that changed after the capture."""
import pytest
import torch

from gpu_common import api

pytestmark = pytest.mark.gpu


def _replayed(run, change, outputs):
    """outputs() of `run` called after `change`, and of its graph replayed after it."""
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    change()
    graph.replay()
    torch.cuda.synchronize()
    replay = [x.clone() for x in outputs()]
    for x in outputs():
        x.zero_()
    run()
    torch.cuda.synchronize()
    for a, b in zip(replay, outputs()):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
        assert (b.float() != 0).any()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("N,V,d", [(60, 900, 64), (500, 300, 72), (300, 2000, 67)])
def test_linear_ce(N, V, d, dtype):
    m = api()
    h, emb = torch.randn(N, d, device="cuda").to(dtype), torch.randn(V, d, device="cuda").to(dtype)
    y = torch.randint(0, V, (N,), device="cuda")
    loss, lse, dloss = (torch.full((N,), 0.01, device="cuda") for _ in range(3))
    dh, demb = torch.empty_like(h), torch.empty_like(emb)
    ws = m.linear_ce_alloc_workspace(N, V, d, dtype)

    def run():
        m.linear_ce_forward(h, emb, y, loss, lse, ws)
        m.linear_ce_backward(h, emb, y, lse, dloss, dh, demb, ws)

    def change():
        h.normal_()
        y.random_(0, V)
        dloss.uniform_(0.001, 0.002)

    _replayed(run, change, lambda: [loss, lse, dh, demb])
    assert m.get_status() == 0


@pytest.mark.parametrize("B,T,D,dtype", [(2, 4000, 64, torch.bfloat16), (3, 50, 33, torch.float32),
                                         (40, 64, 256, torch.float16)])
def test_scan(B, T, D, dtype):
    m = api()
    a, dh = torch.randn(B, T, 4, D, device="cuda").to(dtype), torch.randn(B, T, D, device="cuda").to(dtype)
    h, da, marks = torch.empty_like(dh), torch.empty_like(a), m.scan_alloc_checkpoints(B, T, D)
    c, h1 = torch.zeros(B, D, device="cuda"), torch.empty(B, D, device="cuda", dtype=dtype)
    ws = torch.empty(max(1, m.scan_workspace_bytes(B, T, D)), dtype=torch.uint8, device="cuda")

    def run():
        m.scan_forward(a, h, c_last=c, checkpoints=marks, workspace=ws)
        m.scan_backward(a, marks, dh, da, workspace=ws)
        m.scan_step(a[:, 0], c, h1)

    _replayed(run, lambda: (a.normal_(), dh.normal_()), lambda: [h, da, c, h1])
    assert m.get_status() == 0


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw(bits):
    m = api()
    p = [torch.randn(n, device="cuda") for n in (1000, 7, 3001)]
    g = [torch.randn_like(x) for x in p]
    state = m.AdamW.zero_state(p, bits)
    opt = m.AdamW(p, **state, weight_decay=0.1)
    everything = p + [x for k in state.values() for x in k]

    def run():
        for x in everything:
            x.view(torch.uint8).zero_()
        opt.step(g, t=3, lr=1e-2, seed=5)

    _replayed(run, lambda: [x.normal_() for x in g], lambda: [p[0], p[2]] + [s[0] for s in state.values()])
    assert m.get_status() == 0
