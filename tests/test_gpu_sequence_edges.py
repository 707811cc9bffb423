"""Linear attention, dropout and sampling where their callers differ from the plain case: strides that do
not nest, offsets past 32 bits, graphs that share a workspace, several streams at once."""
import pytest
import torch

from gpu_common import api
from test_gpu_dropout import _check as check_dropout
from test_gpu_linear_attn import DT, _case, _check, _run
from test_gpu_sample import _logits, _reference as sample_reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("width", [16, 24, 32, 48, 96, 128])
@pytest.mark.parametrize("gap", [8, 24])
def test_rows_whose_strides_do_not_nest(width, gap, dtype):
    """Heads side by side and a gap after each step that is no multiple of a head: as one row of all heads
    where widths are multiples of 16, by the other kernels where not."""
    B, T, H = 2, 200, 3
    s = _case(B, T, H, width, width, dtype, seed=width + gap)
    t = {}
    for n in ("q", "k", "v", "do"):
        wide = torch.full((B, T, H * width + gap), float("nan"), dtype=DT[dtype], device="cuda")
        t[n] = wide.as_strided((B, T, H, width), (T * (H * width + gap), H * width + gap, width, 1))
        t[n].copy_(s[n])
    m = api()
    out = {n: torch.full((B, T, H, width), float("nan"), dtype=DT[dtype], device="cuda")
           for n in ("o", "dq", "dk", "dv")}
    m.linear_attn_forward(t["q"], t["k"], t["v"], s["g"], out["o"], s0=s["s0"], scale=s["scale"])
    m.linear_attn_backward(t["q"], t["k"], t["v"], s["g"], t["do"], out["dq"], out["dk"], out["dv"],
                           s0=s["s0"], ds_last=s["dsl"], scale=s["scale"])
    _check(s, out, ("o", "dq", "dk", "dv"))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_attention_with_offsets_past_32_bits(dtype):
    """The second sequence starts 2^31 elements further on."""
    s = _case(2, 150, 2, 32, 32, dtype, seed=1)
    far = (1 << 31) + 64
    t = {}
    for n in ("q", "k", "v", "do"):
        flat = torch.empty(far + 150 * 64, dtype=DT[dtype], device="cuda")
        t[n] = flat.as_strided((2, 150, 2, 32), (far, 64, 32, 1))
        t[n].copy_(s[n])
    flat = torch.empty(far + 150 * 64, dtype=DT[dtype], device="cuda")
    o = flat.as_strided((2, 150, 2, 32), (far, 64, 32, 1))
    api().linear_attn_forward(t["q"], t["k"], t["v"], s["g"], o, s0=s["s0"], scale=s["scale"])
    _check(s, {"o": o}, ("o",))


def test_dropout_and_sampling_with_offsets_past_32_bits():
    far = (1 << 30) + 8
    flat = torch.zeros(3 * far, dtype=torch.bfloat16, device="cuda")
    for cols in (40, 33):
        x = flat.as_strided((3, cols), (far, 1))
        x.normal_()
        y = torch.empty(3, cols, dtype=torch.bfloat16, device="cuda")
        api().dropout(x, y, 0.3, seed=2)
        check_dropout(x, y, 0.3, 2, 0, dtype="bf16")
    l, u = _logits(3, 5000, "bf16", seed=3)
    rows = flat.as_strided((3, 5000), (far, 1))
    rows.copy_(l)
    token = torch.empty(3, dtype=torch.int64, device="cuda")
    api().sample(rows, u, token, top_p=0.9)
    assert (token.cpu().numpy() == sample_reference(l, u, top_p=0.9)[0]).all()


def test_two_graphs_on_one_workspace():
    """Replayed in turn, each gives what the calls give."""
    m = api()
    a, b = _case(1, 4000, 1, 64, 64, "bf16", seed=1), _case(1, 3000, 1, 64, 64, "bf16", seed=2)
    ws = m.linear_attn_alloc_workspace(1, 4000, 1, 64, 64, torch.bfloat16)
    assert ws.numel() >= m.linear_attn_workspace_bytes(1, 3000, 1, 64, 64, torch.bfloat16) > 0
    want, graphs, outs = [], [], []
    for s in (a, b):
        want.append(_run(s))
        outs.append({n: torch.empty_like(x) for n, x in want[-1].items()})
    for s, o in zip((a, b), outs):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            m.linear_attn_forward(s["q"], s["k"], s["v"], s["g"], o["o"], s_last=o["s_last"], s0=s["s0"],
                                  scale=s["scale"], workspace=ws)
            m.linear_attn_backward(s["q"], s["k"], s["v"], s["g"], s["do"], o["dq"], o["dk"], o["dv"],
                                   ds_last=s["dsl"], ds0=o["ds0"], s0=s["s0"], scale=s["scale"],
                                   workspace=ws)
        graphs.append(graph)
    for _ in range(2):
        for graph in graphs:
            graph.replay()
    torch.cuda.synchronize()
    for w, o in zip(want, outs):
        for n in w:
            assert torch.equal(w[n], o[n]), n


def test_calls_on_several_streams_at_once():
    m = api()
    cases = [_case(1, 3000, 2, 64, 64, "bf16", seed=k) for k in range(4)]
    want = [_run(s) for s in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    l, u = _logits(30, 20000, "fp32", seed=4)
    tokens = [torch.empty(30, dtype=torch.int64, device="cuda") for _ in cases]
    torch.cuda.synchronize()
    got = []
    for k, (s, st) in enumerate(zip(cases, streams)):
        with torch.cuda.stream(st):
            got.append(_run(s))
            m.sample(l, u, tokens[k], top_k=1000, top_p=0.9)
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        for n in w:
            assert torch.equal(w[n], g[n]), n
    assert all(torch.equal(t, tokens[0]) for t in tokens)
    assert m.get_status() == 0


def test_a_batch_of_padding_alone():
    """Every sequence is empty: states pass through, results are zeros, nothing is read."""
    for dtype in ("fp32", "bf16", "fp16"):
        s = _case(3, 140, 2, 32, 48, dtype, seed=2)
        s["lengths"] = torch.zeros(3, dtype=torch.int32, device="cuda")
        for n in ("q", "k", "v", "do"):
            s[n].fill_(float("nan"))
        out = _run(s)
        assert torch.equal(out["s_last"], s["s0"]) and torch.equal(out["ds0"], s["dsl"])
        assert all(not out[n].any() for n in ("o", "dq", "dk", "dv"))


def test_documents_of_one_step():
    """Every step starts one: each sees itself alone, and no state gets in or out."""
    for dtype in ("fp32", "bf16", "fp16"):
        s = _case(2, 200, 2, 32, 32, dtype, seed=6)
        s["resets"] = torch.ones(2, 200, dtype=torch.uint8, device="cuda")
        out = _run(s)
        _check(s, out)
        assert not out["ds0"].any()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("B,T", [(3, 300), (1, 3000), (2, 17), (2, 16), (2, 15)])
def test_mild_and_strong_decays_of_one_call(B, T, dtype):
    """Decays that the fp32 kernels put off to the end of 16 steps, and such that they do not, next to
    one another: exp(-1/2) is the last of the first kind."""
    decay = [0.0, -1e-3, -0.4999, -0.5, -0.50001, -3.0, -90.0]
    s = _case(B, T, len(decay), 33, 21, dtype, seed=B + T, ragged=B > 1, resets=True, decay=decay)
    _check(s, _run(s))


def test_large_values_in_32_bits():
    """Products of 1e34, with the strongest decay that is put off."""
    s = _case(2, 200, 2, 32, 32, "fp32", seed=9, decay=-0.5)
    s["v"] *= 1e33
    s["do"] *= 1e-3
    s["s0"] *= 1e33
    _check(s, _run(s))
