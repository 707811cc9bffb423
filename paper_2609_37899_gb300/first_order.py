"""A recurrent expert trained by gradients, on the first-order operators.

    python -m paper_2609_37899_gb300.first_order [--dim 512] [--steps 200] [--bits 8]
        [--mixer scan|attention] [--dropout 0.1] [--generate 64]

The zero-order step has a first-order counterpart in the paper: BPTT controls
and, in the seed run, the decoder-path rule for the tied head (Eq. delta,
dE = (1/BT) sum (p - onehot) h^T).  This module is one training step of that
kind for an expert whose LSTM gates depend on the input alone, so that the
whole sequence is one scan:

    x_t = emb[token_t];  a_t = W x_t;  h = scan(a);  y_t = x_t + h_t;
    logits = y_t emb^T (tied);  loss = mean cross entropy of token_{t+1}

``AttentionExpert`` has linear attention with a decay for each head in the
scan's place (a matrix for a state instead of a vector):

    q_t, k_t, v_t = W x_t;  h = attention(q, k, v);  y_t = x_t + h_t

In training, h may pass through dropout before it is added.  ``generate`` reads
a prompt at once and goes on token by token, with the likeliest tokens or with
such that are drawn from given random numbers.

The mixers, dropout, the cross entropy, the optimizer and the draws run in the
library's kernels (``api.scan_*``, ``api.linear_attn_*``, ``api.dropout``,
``api.linear_ce_*``, ``api.AdamW``, ``api.sample``); the projection W x and its
two gradients are plain matrix products of torch.  Parameters are bf16 with fp32
masters, moments are fp32 or 8 bits.
"""
from __future__ import annotations

import argparse

import torch

from . import api, inputs


class ScanExpert:
    """One expert: parameters, masters, moments and the buffers of a training
    step of `batch` sequences of `steps` tokens.  dropout: the share of h's
    elements that a training step drops."""

    projections = 4  # rows of W for each channel: the gates i, f, g, o

    def __init__(self, vocab: int, dim: int, batch: int, steps: int, seed: int = 0, bits: int = 8,
                 dtype: torch.dtype = torch.bfloat16, weight_decay: float = 0.01,
                 device: str = "cuda", dropout: float = 0.0):
        self.vocab, self.dim, self.batch, self.steps = vocab, dim, batch, steps
        self.dropout = dropout
        g = torch.Generator(device=device).manual_seed(seed)
        emb = torch.randn(vocab, dim, generator=g, device=device) * dim ** -0.5
        w = torch.randn(self.projections * dim, dim, generator=g, device=device) * dim ** -0.5
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
        self.loss, self.lse = new(n, like=torch.float32), new(n, like=torch.float32)
        self.da, self.dy = new(n, self.projections * dim), new(n, dim)
        self.dh = None  # the gradient before dropout, from the first step that drops on
        self.demb, self.dw = new(vocab, dim), new(self.projections * dim, dim)
        self.ce_ws = api.linear_ce_alloc_workspace(n, vocab, dim, dtype, device=device)
        self._mixer_buffers(new, device)

    def _mixer_buffers(self, new, device):
        B, T, d = self.batch, self.steps, self.dim
        self.c_last = new(B, d, like=torch.float32)
        self.dgates = self.da.view(B, T, 4, d)
        self.marks = api.scan_alloc_checkpoints(B, T, d, device)
        self.scan_ws = torch.empty(max(1, api.scan_workspace_bytes(B, T, d)), dtype=torch.uint8,
                                   device=device)

    def _mix(self, a, lengths, resets):
        """h of the projections a [B * T, projections * dim]."""
        self.gates = a.view(self.batch, self.steps, 4, self.dim)
        api.scan_forward(self.gates, self.h, self.c_last, lengths=lengths, resets=resets,
                         checkpoints=self.marks, workspace=self.scan_ws)

    def _mix_backward(self, dh):
        """The gradient of the projections into da."""
        api.scan_backward(self.gates, self.marks, dh.view(self.batch, self.steps, self.dim),
                          self.dgates, lengths=self.lengths, resets=self.resets,
                          workspace=self.scan_ws)

    def forward(self, tokens: torch.Tensor, resets: torch.Tensor | None = None,
                lengths: torch.Tensor | None = None) -> torch.Tensor:
        """Loss [batch * steps] of tokens [batch, steps + 1]; targets past a
        sequence's end count as ignored.  The dropout's mask is that of update t."""
        T, d = self.steps, self.dim
        self.resets, self.lengths = resets, lengths
        self.inputs = tokens[:, :-1]
        self.targets = tokens[:, 1:].reshape(-1)
        if lengths is not None:
            past = torch.arange(T, device=tokens.device)[None] >= lengths[:, None]
            self.targets = torch.where(past.reshape(-1), -100, self.targets)
        self.x = self.emb[self.inputs].contiguous()
        self._mix(self.x.reshape(-1, d) @ self.w.T, lengths, resets)
        if self.dropout:
            y = torch.empty_like(self.h)
            api.dropout(self.h, y, self.dropout, self.seed, offset=self.t, residual=self.x)
        else:
            y = self.x + self.h
        self.y = y.view(-1, d)
        api.linear_ce_forward(self.y, self.emb, self.targets, self.loss, self.lse, self.ce_ws)
        return self.loss

    def backward(self, dloss: torch.Tensor):
        """Gradients of sum(loss * dloss) into demb and dw."""
        api.linear_ce_backward(self.y, self.emb, self.targets, self.lse, dloss, self.dy, self.demb,
                               self.ce_ws)
        dh = self.dy
        if self.dropout:
            if self.dh is None:
                self.dh = torch.empty_like(self.dy)
            dh = self.dh
            api.dropout(self.dy, dh, self.dropout, self.seed, offset=self.t)
        self._mix_backward(dh)
        torch.mm(self.da.T, self.x.reshape(-1, self.dim), out=self.dw)
        dx = torch.addmm(self.dy, self.da, self.w)
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

    def _read(self, a):
        """Last h [B, dim] of a prompt's projections [B, P, projections * dim], and the state."""
        B, P, d = a.shape[0], a.shape[1], self.dim
        h = torch.empty(B, P, d, dtype=a.dtype, device=a.device)
        c = torch.empty(B, d, dtype=torch.float32, device=a.device)
        api.scan_forward(a.view(B, P, 4, d), h, c)
        return h[:, -1], c

    def _step(self, a, state, h):
        api.scan_step(a.view(-1, 4, self.dim), state, h)

    @torch.no_grad()
    def generate(self, prompt: torch.Tensor, n: int, u: torch.Tensor | None = None,
                 temperature=1.0, top_k=0, top_p=1.0, min_p=0.0) -> torch.Tensor:
        """n next tokens, one after another, of prompts [B, P]: one pass over the prompt, then
        one token at a time.  The likeliest ones, or, with uniform numbers u fp32 [n, B], tokens
        drawn as api.sample does it."""
        B, P = prompt.shape
        x = self.emb[prompt]
        h, state = self._read((x.reshape(B * P, self.dim) @ self.w.T).view(B, P, -1))
        y, out = x[:, -1] + h, []
        step_h = torch.empty(B, self.dim, dtype=self.emb.dtype, device=prompt.device)
        for k in range(n):
            logits = y @ self.emb.T
            if u is None:
                out.append(logits.argmax(1))
            else:
                out.append(torch.empty(B, dtype=torch.int64, device=prompt.device))
                api.sample(logits, u[k], out[-1], temperature=temperature, top_k=top_k,
                           top_p=top_p, min_p=min_p)
            x = self.emb[out[-1]]
            self._step(x @ self.w.T, state, step_h)
            y = x + step_h
        return torch.stack(out, 1)


class AttentionExpert(ScanExpert):
    """The same with linear attention of `heads` heads.  Decays are given: head j
    of H keeps 1 - 2^-(1 + 6 (j + 1) / H) of its state per step, so that some heads see a
    few steps and some about a hundred."""

    projections = 3  # q, k, v

    def __init__(self, *args, heads: int = 8, **kw):
        self.heads = heads
        super().__init__(*args, **kw)

    def _mixer_buffers(self, new, device):
        B, T, H = self.batch, self.steps, self.heads
        if self.dim % H:
            raise ValueError(f"dim {self.dim} is no multiple of {H} heads")
        self.width = self.dim // H
        self.scale = self.width ** -0.5
        j = torch.arange(1, H + 1, device=device, dtype=torch.float64)
        self.log_decay = torch.log1p(-torch.exp2(-1 - 6 * j / H)).float()
        self.attn_ws = api.linear_attn_alloc_workspace(B, T, H, self.width, self.width,
                                                       self.emb.dtype, device=device)

    def _heads(self, a, B, T):
        """q, k and v [B, T, heads, width] of projections, as views."""
        return a.view(B, T, 3, self.heads, self.width).unbind(2)

    def _mix(self, a, lengths, resets):
        B, T, H = self.batch, self.steps, self.heads
        self.qkv = self._heads(a, B, T)
        api.linear_attn_forward(*self.qkv, self.log_decay, self.h.view(B, T, H, self.width),
                                lengths=lengths, resets=resets, scale=self.scale,
                                workspace=self.attn_ws)

    def _mix_backward(self, dh):
        B, T, H = self.batch, self.steps, self.heads
        api.linear_attn_backward(*self.qkv, self.log_decay, dh.view(B, T, H, self.width),
                                 *self._heads(self.da, B, T), lengths=self.lengths,
                                 resets=self.resets, scale=self.scale, workspace=self.attn_ws)

    def _read(self, a):
        B, P, H, w = a.shape[0], a.shape[1], self.heads, self.width
        h = torch.empty(B, P, H, w, dtype=a.dtype, device=a.device)
        s = torch.empty(B, H, w, w, dtype=torch.float32, device=a.device)
        api.linear_attn_forward(*self._heads(a, B, P), self.log_decay, h, s_last=s,
                                scale=self.scale)
        return h[:, -1].reshape(B, -1), s

    def _step(self, a, state, h):
        B, H = a.shape[0], self.heads
        q, k, v = a.view(B, 3, H, self.width).unbind(1)
        api.linear_attn_step(q, k, v, self.log_decay, state, h.view(B, H, self.width),
                             scale=self.scale)


def main():
    ap = argparse.ArgumentParser(description="train a recurrent expert by gradients")
    ap.add_argument("--dim", type=int, default=512)
    ap.add_argument("--batch", type=int, default=32)
    ap.add_argument("--length", type=int, default=256)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--lr", type=float, default=2e-3)
    ap.add_argument("--bits", type=int, default=8, choices=(8, 32))
    ap.add_argument("--mixer", default="scan", choices=("scan", "attention"))
    ap.add_argument("--heads", type=int, default=8, help="of the attention")
    ap.add_argument("--dropout", type=float, default=0.0)
    ap.add_argument("--generate", type=int, default=0, help="bytes to draw at the end")
    ap.add_argument("--temperature", type=float, default=0.8)
    ap.add_argument("--top-p", type=float, default=0.95)
    a = ap.parse_args()
    more = {} if a.mixer == "scan" else {"heads": a.heads}
    expert = (ScanExpert if a.mixer == "scan" else AttentionExpert)(
        256, a.dim, a.batch, a.length, bits=a.bits, dropout=a.dropout, **more)
    for k in range(a.steps):
        batch = inputs.expert_batch(1, a.batch, a.length, order=1, seed=0, step=k)[0]
        tokens = torch.from_numpy(batch.astype("int64")).cuda()
        loss = expert.train_step(tokens, a.lr)
        if k % 20 == 0 or k == a.steps - 1:
            print(f"step {k}: {loss.item():.4f} nats/byte", flush=True)
    if a.generate:
        u = torch.rand(a.generate, 1, device="cuda",
                       generator=torch.Generator(device="cuda").manual_seed(0))
        drawn = expert.generate(tokens[:1, :a.length], a.generate, u, a.temperature, top_p=a.top_p)
        print("drawn:", drawn[0].tolist())
    if api.get_status() != 0:
        raise SystemExit("a loss or a gradient was not finite")


if __name__ == "__main__":
    main()
