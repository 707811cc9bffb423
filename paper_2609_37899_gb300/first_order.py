"""A recurrent expert trained by gradients, on the first-order operators.

    python -m paper_2609_37899_gb300.first_order [--dim 512] [--steps 200] [--bits 8]

The zero-order step has a first-order counterpart in the paper: BPTT controls
and, in the seed run, the decoder-path rule for the tied head (Eq. delta,
dE = (1/BT) sum (p - onehot) h^T).  This module is one training step of that
kind for an expert whose LSTM gates depend on the input alone, so that the
whole sequence is one scan:

    x_t = emb[token_t];  a_t = W x_t;  h = scan(a);  y_t = x_t + h_t;
    logits = y_t emb^T (tied);  loss = mean cross entropy of token_{t+1}

The recurrence, the cross entropy and the optimizer run in the library's
kernels (``api.scan_*``, ``api.linear_ce_*``, ``api.AdamW``); the projection
W x and its two gradients are plain matrix products of torch.  Parameters are
bf16 with fp32 masters, moments are fp32 or 8 bits.
"""
from __future__ import annotations

import argparse

import torch

from . import api, inputs


class ScanExpert:
    """One expert: parameters, masters, moments and the buffers of a training
    step of `batch` sequences of `steps` tokens."""

    def __init__(self, vocab: int, dim: int, batch: int, steps: int, seed: int = 0, bits: int = 8,
                 dtype: torch.dtype = torch.bfloat16, weight_decay: float = 0.01,
                 device: str = "cuda"):
        self.vocab, self.dim, self.batch, self.steps = vocab, dim, batch, steps
        g = torch.Generator(device=device).manual_seed(seed)
        emb = torch.randn(vocab, dim, generator=g, device=device) * dim ** -0.5
        w = torch.randn(4 * dim, dim, generator=g, device=device) * dim ** -0.5
        self.masters = [emb, w]
        self.emb, self.w = (p.to(dtype) for p in self.masters)
        params = [self.emb, self.w]
        self.opt = api.AdamW(params, **api.AdamW.zero_state(params, bits), masters=self.masters,
                             weight_decay=weight_decay)
        self.t, self.seed = 0, seed
        n = batch * steps

        def new(*shape, like=dtype):
            return torch.empty(*shape, dtype=like, device=device)

        self.h = new(batch, steps, dim)
        self.c_last = new(batch, dim, like=torch.float32)
        self.loss, self.lse = new(n, like=torch.float32), new(n, like=torch.float32)
        self.marks = api.scan_alloc_checkpoints(batch, steps, dim, device)
        self.dgates, self.dy = new(batch, steps, 4, dim), new(n, dim)
        self.demb, self.dw = new(vocab, dim), new(4 * dim, dim)
        self.scan_ws = torch.empty(max(1, api.scan_workspace_bytes(batch, steps, dim)),
                                   dtype=torch.uint8, device=device)
        self.ce_ws = api.linear_ce_alloc_workspace(n, vocab, dim, dtype, device=device)

    def forward(self, tokens: torch.Tensor, resets: torch.Tensor | None = None,
                lengths: torch.Tensor | None = None) -> torch.Tensor:
        """Loss [batch * steps] of tokens [batch, steps + 1]; targets past a
        sequence's end count as ignored."""
        B, T, d = self.batch, self.steps, self.dim
        self.resets, self.lengths = resets, lengths
        self.inputs = tokens[:, :-1]
        self.targets = tokens[:, 1:].reshape(-1)
        if lengths is not None:
            past = torch.arange(T, device=tokens.device)[None] >= lengths[:, None]
            self.targets = torch.where(past.reshape(-1), -100, self.targets)
        self.x = self.emb[self.inputs]
        self.gates = (self.x.reshape(-1, d) @ self.w.T).view(B, T, 4, d)
        api.scan_forward(self.gates, self.h, self.c_last, lengths=lengths, resets=resets,
                         checkpoints=self.marks, workspace=self.scan_ws)
        self.y = (self.x + self.h).view(-1, d)
        api.linear_ce_forward(self.y, self.emb, self.targets, self.loss, self.lse, self.ce_ws)
        return self.loss

    def backward(self, dloss: torch.Tensor):
        """Gradients of sum(loss * dloss) into demb and dw."""
        d = self.dim
        api.linear_ce_backward(self.y, self.emb, self.targets, self.lse, dloss, self.dy, self.demb,
                               self.ce_ws)
        api.scan_backward(self.gates, self.marks, self.dy.view(self.batch, self.steps, d),
                          self.dgates, lengths=self.lengths, resets=self.resets,
                          workspace=self.scan_ws)
        da = self.dgates.view(-1, 4 * d)
        torch.mm(da.T, self.x.reshape(-1, d), out=self.dw)
        dx = torch.addmm(self.dy, da, self.w)
        # the embedding's rows add up in fp32: a frequent token has many
        into = self.demb.float().index_add_(0, self.inputs.reshape(-1), dx.float())
        self.demb.copy_(into)
        return self.demb, self.dw

    def train_step(self, tokens: torch.Tensor, lr: float, resets=None, lengths=None):
        """One AdamW step on the mean loss; returns it (on the device)."""
        loss = self.forward(tokens, resets, lengths)
        counted = (self.targets != -100).to(torch.float32)
        total = counted.sum().clamp(min=1)
        self.backward(counted / total)
        self.t += 1
        self.opt.step([self.demb, self.dw], t=self.t, lr=lr, seed=self.seed)
        return loss.sum() / total

    @torch.no_grad()
    def generate(self, prompt: torch.Tensor, n: int) -> torch.Tensor:
        """The n likeliest next tokens, one after another, of prompts [B, P]:
        one scan over the prompt, then one token at a time."""
        B, P = prompt.shape
        d, dt = self.dim, self.emb.dtype
        x = self.emb[prompt]
        gates = (x.reshape(-1, d) @ self.w.T).view(B, P, 4, d)
        h = torch.empty(B, P, d, dtype=dt, device=prompt.device)
        c = torch.empty(B, d, dtype=torch.float32, device=prompt.device)
        api.scan_forward(gates, h, c)
        y, out, step_h = x[:, -1] + h[:, -1], [], torch.empty(B, d, dtype=dt, device=prompt.device)
        for _ in range(n):
            out.append((y @ self.emb.T).argmax(1))
            x = self.emb[out[-1]]
            api.scan_step((x @ self.w.T).view(B, 4, d), c, step_h)
            y = x + step_h
        return torch.stack(out, 1)


def main():
    ap = argparse.ArgumentParser(description="train a recurrent expert by gradients")
    ap.add_argument("--dim", type=int, default=512)
    ap.add_argument("--batch", type=int, default=32)
    ap.add_argument("--length", type=int, default=256)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--lr", type=float, default=2e-3)
    ap.add_argument("--bits", type=int, default=8, choices=(8, 32))
    a = ap.parse_args()
    expert = ScanExpert(256, a.dim, a.batch, a.length, bits=a.bits)
    for k in range(a.steps):
        batch = inputs.expert_batch(1, a.batch, a.length, order=1, seed=0, step=k)[0]
        tokens = torch.from_numpy(batch.astype("int64")).cuda()
        loss = expert.train_step(tokens, a.lr)
        if k % 20 == 0 or k == a.steps - 1:
            print(f"step {k}: {loss.item():.4f} nats/byte", flush=True)
    if api.get_status() != 0:
        raise SystemExit("a loss or a gradient was not finite")


if __name__ == "__main__":
    main()
