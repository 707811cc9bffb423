"""The attention expert (first_order.AttentionExpert): linear attention, dropout, the cross entropy and
the draws as they are used together, against the same model in 64 bits with torch's autograd.

Tolerance: every quantity between the operators is rounded to bf16 (half an ulp 2^-8), in a chain of at
most ten roundings from the parameters to a gradient (x, a, the products, the decayed v and the state
inside the attention, h, y, G, dy, da and the gradient itself).  Errors of independent roundings add up in
square; the norm of a gradient's error is allowed 10 * 2^-8 of the gradient's norm."""
import numpy as np
import pytest
import torch

from gpu_common import api

pytestmark = pytest.mark.gpu

TOL = 10 * 2.0 ** -8


def _expert(*args, **kw):
    from paper_2609_37899_gb300.first_order import AttentionExpert
    return AttentionExpert(*args, **kw)


def _attention(e, a, resets=None, lengths=None):
    """h [B, T, dim] of projections [B, T, 3 * dim] in 64 bits, step by step."""
    B, T = a.shape[:2]
    q, k, v = a.view(B, T, 3, e.heads, e.width).unbind(2)
    S = torch.zeros(B, e.heads, e.width, e.width, dtype=torch.float64, device="cuda")
    lam, hs = torch.exp(e.log_decay.double())[None, :, None, None], []
    for t in range(T):
        if resets is not None:
            S = S * (resets[:, t] == 0)[:, None, None, None]
        S = lam * S + k[:, t, :, :, None] * v[:, t, :, None]
        hs.append(e.scale * (q[:, t, :, :, None] * S).sum(2).reshape(B, -1))
    h = torch.stack(hs, 1)
    if lengths is not None:
        h = h * (torch.arange(T, device="cuda")[None] < lengths[:, None])[..., None]
    return h


def _reference(e, tokens, keep, resets=None, lengths=None):
    emb, w = (p.double().detach().requires_grad_() for p in (e.emb, e.w))
    x = emb[tokens[:, :-1]]
    y = x + keep.double() * _attention(e, x @ w.T, resets, lengths)
    loss = torch.nn.functional.cross_entropy((y @ emb.T).view(-1, e.vocab),
                                             tokens[:, 1:].reshape(-1), reduction="none")
    loss = loss.view(e.batch, e.steps)
    if lengths is not None:
        loss = loss * (torch.arange(e.steps, device="cuda")[None] < lengths[:, None])
    return loss, emb, w


@pytest.mark.parametrize("vocab,dim,heads,batch,steps,ragged,p", [
    (256, 64, 2, 4, 50, False, 0.0), (1000, 96, 3, 3, 130, True, 0.25), (256, 128, 1, 1, 700, True, 0.1),
    (256, 256, 2, 2, 300, False, 0.3)])
def test_gradients_of_the_whole_step(vocab, dim, heads, batch, steps, ragged, p):
    e = _expert(vocab, dim, batch, steps, seed=vocab + steps, heads=heads, dropout=p)
    g = torch.Generator(device="cuda").manual_seed(1)
    tokens = torch.randint(0, vocab, (batch, steps + 1), generator=g, device="cuda")
    resets = lengths = None
    if ragged:
        resets = (torch.rand(batch, steps, generator=g, device="cuda") < 0.05).to(torch.uint8)
        lengths = torch.randint(1, steps + 1, (batch,), generator=g, device="cuda", dtype=torch.int32)
    e.t = 3  # another update's mask than the first
    keep = torch.ones(batch, steps, dim, device="cuda")
    api().dropout(keep, keep, p, e.seed, offset=3)
    loss, emb, w = _reference(e, tokens, keep, resets, lengths)
    dloss = torch.rand(batch * steps, generator=g, device="cuda") / (batch * steps)
    (loss.view(-1) * dloss.double()).sum().backward()
    got = e.forward(tokens, resets, lengths)
    demb, dw = e.backward(dloss)
    assert api().get_status() == 0
    assert (got.double() - loss.view(-1)).norm() <= TOL * loss.norm()
    for name, x, ref in (("demb", demb, emb.grad), ("dw", dw, w.grad)):
        err = ((x.double() - ref).norm() / ref.norm()).item()
        assert err <= TOL, (name, err)


def test_dropout_of_the_scan_expert():
    """The scan's expert drops the same way: with everything dropped it is its embedding alone."""
    from paper_2609_37899_gb300.first_order import ScanExpert
    e = ScanExpert(256, 64, 2, 30, seed=4, dropout=1.0)
    tokens = torch.randint(0, 256, (2, 31), device="cuda")
    e.forward(tokens)
    assert torch.equal(e.y, e.emb[tokens[:, :-1]].view(-1, 64))
    e.backward(torch.ones(60, device="cuda"))
    assert not e.dw.any()


@pytest.mark.parametrize("dropout", [0.0, 0.2])
def test_training_steps_run(dropout):
    e = _expert(256, 128, 8, 64, heads=2, dropout=dropout)
    before = [p.clone() for p in (e.emb, e.w)]
    for k in range(3):
        tokens = torch.randint(0, 256, (8, 65), device="cuda")
        assert e.train_step(tokens, 1e-3).isfinite()
    assert e.t == 3 and api().get_status() == 0
    assert all(not torch.equal(a, b) for a, b in zip(before, (e.emb, e.w)))


def _logits(e, tokens):
    x = e.emb[tokens]
    B, P = tokens.shape
    h, _ = e._read((x.reshape(B * P, e.dim) @ e.w.T).view(B, P, -1))
    return ((x[:, -1] + h) @ e.emb.T)


def test_generation_follows_the_prompt_form():
    """Token by token, the likeliest tokens are those that one pass over prompt and answer gives, wherever
    its best logit leads by more than the bf16 noise of the logits."""
    e = _expert(256, 64, 2, 40, seed=3, heads=2)
    prompt = torch.randint(0, 256, (2, 150), device="cuda")
    out = e.generate(prompt, 12)
    full, clear = torch.cat((prompt, out), 1), 0
    for k in range(12):
        logits = _logits(e, full[:, :150 + k]).float()
        best = logits.topk(2, dim=1)
        lead = best.values[:, 0] - best.values[:, 1] > 2.0 ** -6 * logits.abs().amax()
        assert (best.indices[:, 0] == out[:, k])[lead].all()
        clear += lead.sum().item()
    assert clear


@pytest.mark.parametrize("kind", ["scan", "attention"])
def test_drawn_tokens(kind):
    """With u near 0 the first of what remains, with top_k = 1 the likeliest; the same u, the same tokens."""
    from paper_2609_37899_gb300.first_order import ScanExpert
    e = ScanExpert(256, 64, 3, 20, seed=5) if kind == "scan" else _expert(256, 64, 3, 20, seed=5, heads=4)
    prompt = torch.randint(0, 256, (3, 20), device="cuda")
    u = torch.rand(9, 3, device="cuda")
    greedy = e.generate(prompt, 9)
    assert torch.equal(e.generate(prompt, 9, u, top_k=1), greedy)
    assert torch.equal(e.generate(prompt, 9, u, temperature=0.0), greedy)
    a = e.generate(prompt, 9, u, temperature=1.5, top_p=0.9)
    assert torch.equal(a, e.generate(prompt, 9, u, temperature=1.5, top_p=0.9))
    assert (a >= 0).all() and (a < 256).all() and not torch.equal(a, greedy)
    first = torch.empty(3, dtype=torch.int64, device="cuda")
    x = e.emb[prompt]
    h, _ = e._read((x.reshape(60, 64) @ e.w.T).view(3, 20, -1))
    api().sample((x[:, -1] + h) @ e.emb.T, u[0], first, temperature=1.5, top_p=0.9)
    assert torch.equal(a[:, 0], first)


def test_a_step_in_a_graph():
    """Forward and backward of one update captured: a replay on other tokens is what the calls give."""
    e = _expert(256, 64, 2, 200, seed=6, heads=2, dropout=0.2)
    tokens = torch.randint(0, 256, (2, 201), device="cuda")
    dloss = torch.full((400,), 1 / 400, device="cuda")
    e.forward(tokens), e.backward(dloss)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        e.forward(tokens), e.backward(dloss)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        e.forward(tokens), e.backward(dloss)
    tokens.copy_(torch.randint(0, 256, (2, 201), device="cuda"))
    graph.replay()
    torch.cuda.synchronize()
    got = [x.clone() for x in (e.loss, e.dw, e.y, e.dh)]
    e.forward(tokens), e.backward(dloss)
    for a, b in zip(got, (e.loss, e.dw, e.y, e.dh)):
        assert torch.equal(a, b)


def test_traced():
    m = api()
    e = _expert(256, 64, 2, 60, seed=6, heads=2, dropout=0.2)
    tokens = torch.randint(0, 256, (2, 61), device="cuda")
    m.trace_enable(True)
    try:
        m.trace_read_sequence(reset=True), m.trace_read_first_order(reset=True)
        e.train_step(tokens, 1e-3)
        e.generate(tokens, 2, torch.rand(2, 2, device="cuda"))
        got = m.trace_read_sequence(reset=True)
        # two calls of the step, the prompt and two tokens; two masks; two draws
        assert {k: n for k, (_, n) in got.items()} == {"linear_attn": 5, "dropout": 2, "sample": 2}
        assert all(ms > 0 for ms, _ in got.values())
        assert {k: n for k, (_, n) in m.trace_read_first_order(reset=True).items()} == \
            {"linear_ce": 2, "scan": 0, "adamw": 1}
        assert all(n == 0 for _, n in m.trace_read_sequence(reset=True).values())
    finally:
        m.trace_enable(False)
        m.trace_read_sequence(reset=True), m.trace_read_first_order(reset=True)
