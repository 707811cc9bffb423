"""The first-order training step (first_order.ScanExpert): the operators as they are used
together, against the same model in 64 bits with torch's autograd.

Tolerance: every quantity between the operators is rounded to bf16 (half an ulp 2^-8), in a chain
of at most eight roundings from the parameters to a gradient (x, gates, h, y, G, dy, dgates and the
gradient itself).  Errors of independent roundings add up in square; the norm of a gradient's error
is allowed 8 * 2^-8 of the gradient's norm."""
import numpy as np
import pytest
import torch

from gpu_common import api
from paper_2609_37899_gb300 import inputs

pytestmark = pytest.mark.gpu


def _reference(e, tokens, resets=None, lengths=None):
    emb, w = (p.double().detach().requires_grad_() for p in (e.emb, e.w))
    x = emb[tokens[:, :-1]]
    a = (x @ w.T).view(e.batch, e.steps, 4, e.dim)
    c, hs = torch.zeros(e.batch, e.dim, dtype=torch.float64, device="cuda"), []
    for t in range(e.steps):
        i, f, o = (torch.sigmoid(a[:, t, k]) for k in (0, 1, 3))
        prev = c if resets is None else c * (resets[:, t] == 0)[:, None]
        c = f * prev + i * torch.tanh(a[:, t, 2])
        hs.append(o * torch.tanh(c))
    y = x + torch.stack(hs, 1)
    loss = torch.nn.functional.cross_entropy((y @ emb.T).view(-1, e.vocab),
                                             tokens[:, 1:].reshape(-1), reduction="none")
    loss = loss.view(e.batch, e.steps)
    if lengths is not None:
        loss = loss * (torch.arange(e.steps, device="cuda")[None] < lengths[:, None])
    return loss, emb, w


@pytest.mark.parametrize("vocab,dim,batch,steps,ragged", [
    (256, 64, 4, 50, False), (1000, 96, 3, 130, True), (256, 128, 1, 700, True)])
def test_gradients_of_the_whole_step(vocab, dim, batch, steps, ragged):
    from paper_2609_37899_gb300.first_order import ScanExpert
    e = ScanExpert(vocab, dim, batch, steps, seed=vocab + steps)
    g = torch.Generator(device="cuda").manual_seed(1)
    tokens = torch.randint(0, vocab, (batch, steps + 1), generator=g, device="cuda")
    resets = lengths = None
    if ragged:
        resets = (torch.rand(batch, steps, generator=g, device="cuda") < 0.05).to(torch.uint8)
        lengths = torch.randint(1, steps + 1, (batch,), generator=g, device="cuda",
                                dtype=torch.int32)
    loss, emb, w = _reference(e, tokens, resets, lengths)
    dloss = torch.rand(batch * steps, generator=g, device="cuda") / (batch * steps)
    (loss.view(-1) * dloss.double()).sum().backward()
    got = e.forward(tokens, resets, lengths)
    demb, dw = e.backward(dloss)
    assert api().get_status() == 0
    assert (got.double() - loss.view(-1)).norm() <= 8 * 2.0 ** -8 * loss.norm()
    for name, x, ref in (("demb", demb, emb.grad), ("dw", dw, w.grad)):
        err = ((x.double() - ref).norm() / ref.norm()).item()
        assert err <= 8 * 2.0 ** -8, (name, err)


@pytest.mark.parametrize("bits", [8, 32])
def test_training_learns_the_chain(bits):
    """An order-1 Markov chain of entropy about 4.0 nats/byte (Zipf 1.1 rows): from about
    ln 256 = 5.5 the loss comes near the entropy rate of the chain."""
    from paper_2609_37899_gb300.first_order import ScanExpert
    e = ScanExpert(256, 256, 32, 128, bits=bits)
    losses = []
    for k in range(150):
        batch = inputs.expert_batch(1, 32, 128, order=1, seed=0, step=k)[0]
        losses.append(e.train_step(torch.from_numpy(batch.astype(np.int64)).cuda(), 4e-3))
    losses = torch.stack(losses).cpu().numpy()
    assert api().get_status() == 0
    assert losses[0] > 5.2 and losses[-10:].mean() < 4.6


def test_generation_follows_the_scan():
    """Token by token, the likeliest tokens are those that one scan over prompt and answer gives,
    wherever its best logit leads by more than the bf16 noise of the logits."""
    from paper_2609_37899_gb300.first_order import ScanExpert
    e = ScanExpert(256, 64, 2, 40, seed=3)
    prompt = torch.randint(0, 256, (2, 25), device="cuda")
    out = e.generate(prompt, 12)
    full = torch.cat((prompt, out), 1)
    x = e.emb[full]
    gates = (x.reshape(-1, 64) @ e.w.T).view(2, 37, 4, 64)
    h = torch.empty(2, 37, 64, dtype=e.emb.dtype, device="cuda")
    api().scan_forward(gates, h)
    logits = ((x + h).view(-1, 64) @ e.emb.T).view(2, 37, 256).float()
    best = logits[:, 24:36].topk(2, dim=2)
    clear = best.values[..., 0] - best.values[..., 1] > 2.0 ** -6 * logits.abs().amax()
    assert clear.any()
    assert (best.indices[..., 0] == out)[clear].all()
