"""Cases of linear attention with a decay per head, dropout and sampling.

`run` computes them in plain torch operations where `own` is false, and through the framework's entry points where it
is true.  `exact` computes the same from the definitions in 64 bits.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
WIDTH = {"bf16": 2, "fp16": 2, "fp32": 4}


# ------------------------------------------------------------------ cases --

def listed():
    return [
        # one token of each of 64 running requests: the states are read and written once
        {"name": "attn_step_64", "op": "attn", "mode": "step", "batch": 64, "steps": 1, "heads": 15, "dk": 64, "dv": 64, "dtype": "bf16", "ragged": False},
        # reading one long prompt: few heads, so the time axis has to be split; the state is kept for the answer
        {"name": "attn_prompt_long", "op": "attn", "mode": "forward", "batch": 1, "steps": 32768, "heads": 8, "dk": 128, "dv": 128, "dtype": "bf16", "ragged": False},
        # documents of different lengths packed with resets, values wider than keys, half precision
        {"name": "attn_train_ragged", "op": "attn", "mode": "train", "batch": 13, "steps": 1000, "heads": 5, "dk": 72, "dv": 96, "dtype": "fp16", "ragged": True},
        # 32 bits, odd widths and length
        {"name": "attn_train_fp32", "op": "attn", "mode": "train", "batch": 4, "steps": 777, "heads": 7, "dk": 33, "dv": 65, "dtype": "fp32", "ragged": False},
        # the training step of a wide layer
        {"name": "attn_train_large", "op": "attn", "mode": "train", "batch": 16, "steps": 4096, "heads": 8, "dk": 128, "dv": 128, "dtype": "bf16", "ragged": False},
        # the branch of 64 tokens: latency counts
        {"name": "dropout_small", "op": "dropout", "rows": 64, "cols": 960, "pad": 0, "p": 0.1, "residual": False, "dtype": "fp32"},
        # odd width in padded rows, half precision
        {"name": "dropout_odd", "op": "dropout", "rows": 3001, "cols": 681, "pad": 7, "p": 0.25, "residual": True, "dtype": "fp16"},
        # the branch of a large training batch, added to the residual stream
        {"name": "dropout_large", "op": "dropout", "rows": 65536, "cols": 1376, "pad": 0, "p": 0.1, "residual": True, "dtype": "bf16"},
        # one running request with a large vocabulary: latency counts
        {"name": "sample_1", "op": "sample", "rows": 1, "vocab": 131072, "top_k": 50, "top_p": 0.9, "min_p": 0.0, "masked": 0.0, "each": False, "dtype": "bf16"},
        # bytes for many requests, by temperature alone
        {"name": "sample_byte", "op": "sample", "rows": 512, "vocab": 256, "top_k": 0, "top_p": 1.0, "min_p": 0.0, "masked": 0.0, "each": False, "dtype": "fp32"},
        # 64 requests with settings of their own, an odd vocabulary, a grammar that masks a third of it
        {"name": "sample_64", "op": "sample", "rows": 64, "vocab": 50021, "top_k": 200, "top_p": 0.95, "min_p": 0.01, "masked": 0.33, "each": True, "dtype": "bf16"},
        # many requests with a large vocabulary in 32 bits, by top-p alone
        {"name": "sample_256", "op": "sample", "rows": 256, "vocab": 131072, "top_k": 0, "top_p": 0.9, "min_p": 0.0, "masked": 0.0, "each": False, "dtype": "fp32"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attn", "attn", "dropout", "sample"])
    if op == "attn":
        mode = rng.choice(["step", "forward", "train", "train"])
        wide = [16, 24, 32, 40, 64, 64, 80, 96, 128, 128]
        dk, dv = (rng.choice(wide) if rng.random() < 0.85 else rng.randrange(3, 128) for _ in range(2))
        while True:
            batch, heads, steps = _log(rng, 1, 64), _log(rng, 1, 24), 1 if mode == "step" else _log(rng, 1, 32768)
            if batch * heads * steps * (dk + dv) <= 6e7:
                break
        return {"op": "attn", "mode": mode, "batch": batch, "steps": steps, "heads": heads, "dk": dk, "dv": dv,
                "dtype": rng.choice(["bf16", "bf16", "fp16", "fp32"]), "ragged": mode != "step" and rng.random() < 0.4}
    if op == "dropout":
        while True:
            rows, cols = _log(rng, 1, 65536), _log(rng, 16, 4096)
            if rows * cols <= 9e7:
                break
        return {"op": "dropout", "rows": rows, "cols": cols, "pad": rng.choice([0, 0, 5, 8]), "p": round(rng.uniform(0.0, 0.6), 3),
                "residual": rng.random() < 0.6, "dtype": rng.choice(["bf16", "bf16", "fp16", "fp32"])}
    while True:
        rows, vocab = _log(rng, 1, 512), _log(rng, 100, 262144)
        if rows * vocab <= 3e7:
            break
    return {"op": "sample", "rows": rows, "vocab": vocab, "top_k": rng.choice([0, 0, 1, 20, 1000]),
            "top_p": rng.choice([1.0, round(rng.uniform(0.05, 0.999), 3)]), "min_p": rng.choice([0.0, 0.0, 0.02]),
            "masked": rng.choice([0.0, 0.0, 0.5]), "each": rng.random() < 0.3, "dtype": rng.choice(["bf16", "fp16", "fp32"])}


# ----------------------------------------------------------------- inputs --

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 2654435761 % (1 << 62))
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _rand(g, *shape):
    return torch.rand(*shape, generator=g, device="cuda")


def prepare(case, seed):
    g, dt = _gen(seed), DTYPES[case["dtype"]]
    s = {"case": case}
    if case["op"] == "attn":
        B, T, H, dk, dv = (case[k] for k in ("batch", "steps", "heads", "dk", "dv"))
        s.update(q=_randn(g, B, T, H, dk).to(dt), k=_randn(g, B, T, H, dk).to(dt), v=_randn(g, B, T, H, dv).to(dt))
        # from heads that keep a thousand steps to such that keep two
        s.update(g=-torch.exp(_rand(g, H) * 6.2 - 6.9), scale=dk ** -0.5, s0=_randn(g, B, H, dk, dv), lengths=None, resets=None)
        if case["ragged"]:
            s["lengths"] = torch.randint(0, T + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
            s["lengths"][0] = T
            s["resets"] = (_rand(g, B, T) < 0.01).to(torch.uint8)
            past = torch.arange(T, device="cuda")[None] >= s["lengths"][:, None]
            for name in "qkv":  # padding holds whatever was there
                s[name][past] = float("nan")
        if case["mode"] == "step":
            s["s"] = s["s0"].clone()
        if case["mode"] == "train":
            s.update(do=_randn(g, B, T, H, dv).to(dt), ds_last=_randn(g, B, H, dk, dv))
    elif case["op"] == "dropout":
        rows, cols, pad = case["rows"], case["cols"], case["pad"]

        def matrix():
            return _randn(g, rows, cols + pad).to(dt)[:, :cols]

        s.update(x=matrix(), dy=matrix(), residual=matrix() if case["residual"] else None, p=case["p"],
                 seed=seed & (2 ** 64 - 1), offset=5 + (seed & 0xFFFF) * 3)
    else:
        R, V = case["rows"], case["vocab"]
        # a few tokens lead, as a trained model's do
        logits = _randn(g, R, V) * 2.0
        lead = ((torch.arange(12, device="cuda") + _rand(g, R, 12) * 0.999) * (V / 12)).long()
        logits.scatter_add_(1, lead, _rand(g, R, 12) * 10.0)
        logits = logits.to(dt)
        if case["masked"]:
            out = _rand(g, R, V) < case["masked"]
            half = torch.arange(R, device="cuda")[:, None] % 2 == 0  # minus infinity in one row, the type's lowest value in the next
            logits[out & half] = float("-inf")
            logits[out & ~half] = torch.finfo(dt).min
        s.update(logits=logits, u=_rand(g, R))
        if case["each"]:  # requests with settings of their own
            s.update(temperature=0.5 + _rand(g, R), top_p=(1.0 - _rand(g, R) * 2.0 * (1.0 - case["top_p"])).clamp(min=0.01), min_p=_rand(g, R) * 2.0 * case["min_p"],
                     top_k=torch.randint(0, 2 * case["top_k"] + 1, (R,), generator=g, device="cuda", dtype=torch.int32))
        else:
            s.update(temperature=0.8, top_k=case["top_k"], top_p=case["top_p"], min_p=case["min_p"])
    return s


def work(case):
    w = WIDTH[case["dtype"]]
    if case["op"] == "attn":
        rows = case["batch"] * case["heads"]
        n, dk, dv = rows * case["steps"], case["dk"], case["dv"]
        state = 4 * rows * dk * dv
        nbytes, flops = n * (2 * dk + 2 * dv) * w + 2 * state, 4 * n * dk * dv
        if case["mode"] == "train":  # q, k, v and do in, dq, dk and dv out; both states' gradients
            nbytes, flops = nbytes + n * (4 * dk + 3 * dv) * w + 3 * state, flops + 10 * n * dk * dv
        return {"bytes": nbytes, "flops": flops}
    if case["op"] == "dropout":
        n = case["rows"] * case["cols"]
        return {"bytes": n * w * (5 if case["residual"] else 4), "flops": 4 * n}
    return {"bytes": case["rows"] * (case["vocab"] * w + 16), "flops": 10 * case["rows"] * case["vocab"]}


# ------------------------------------------------------------- plain forms --

CHUNK = 128


def _attend(x, y, z, g, age, doc, state, doc0, age_end, doc_end):
    """sum over earlier j of the same document of exp(g (age_i - age_j)) <x_i, y_j> z_j, and what `state` (of age 0 and
    document doc0) adds; with the state at age_end."""
    outs, at, cur, g = [], torch.zeros_like(age_end), doc0, g.double()[None, :, None]
    for t in range(0, x.shape[1], CHUNK):
        xc, yc, zc = (a[:, t:t + CHUNK].transpose(1, 2) for a in (x, y, z))
        a, d = age[:, t:t + CHUNK], doc[:, t:t + CHUNK]
        keep = (d[:, :, None] == d[:, None, :]) & torch.ones(a.shape[1], a.shape[1], dtype=torch.bool, device="cuda").tril()
        decay = torch.exp(g[..., None] * (a[:, :, None] - a[:, None, :]).clamp(min=0)[:, None])
        decay = torch.where(keep[:, None], decay, 0.0).float()
        seen = torch.where((d == cur[:, None])[:, None], torch.exp(g * (a - at[:, None])[:, None]), 0.0).float()
        outs.append((((xc @ yc.transpose(2, 3)) * decay) @ zc + seen[..., None] * (xc @ state)).transpose(1, 2))
        end, last = a[:, -1], d[:, -1]
        left = torch.where((d == last[:, None])[:, None], torch.exp(g * (end[:, None] - a)[:, None]), 0.0).float()
        carry = torch.where((cur == last)[:, None], torch.exp(g[..., 0] * (end - at)[:, None]), 0.0).float()
        state = carry[..., None, None] * state + yc.transpose(2, 3) @ (left[..., None] * zc)
        at, cur = end, last
    carry = torch.where((cur == doc_end)[:, None], torch.exp(g[..., 0] * (age_end - at)[:, None]), 0.0).float()
    return torch.cat(outs, 1), carry[..., None, None] * state


def _plain_attn(s):
    case, dt, g, scale = s["case"], s["q"].dtype, s["g"], s["scale"]
    q, k, v = (s[n].float() for n in "qkv")
    B, T = q.shape[:2]
    if case["mode"] == "step":
        s["s"].copy_(torch.exp(g)[None, :, None, None] * s["s"] + k[:, 0, :, :, None] * v[:, 0, :, None, :])
        return {"o": (scale * (q[:, 0, :, :, None] * s["s"]).sum(2)).to(dt), "s": s["s"]}
    live = torch.ones(B, T, dtype=torch.bool, device="cuda")
    if s["lengths"] is not None:
        live = torch.arange(T, device="cuda")[None] < s["lengths"][:, None]
        q, k, v = (torch.where(live[:, :, None, None], a, 0.0) for a in (q, k, v))
    age = live.double().cumsum(1)
    doc = torch.zeros(B, T, device="cuda") if s["resets"] is None else ((s["resets"] != 0) & live).float().cumsum(1)
    end, first, last = age[:, -1], torch.zeros_like(doc[:, 0]), doc[:, -1]
    o, state = _attend(q, k, v, g, age, doc, s["s0"], first, end, last)
    o = (scale * o).to(dt)
    if case["mode"] == "forward":
        return {"o": o, "s_last": state}
    do = torch.where(live[:, :, None, None], s["do"].float(), 0.0)
    dq, _ = _attend(do, v, k, g, age, doc, s["s0"].transpose(2, 3), first, end, last)
    # backwards in time: the last step is of age 0, as the state's gradient after it is
    back, there = (end[:, None] - age).flip(1), doc.flip(1)
    dk, _ = _attend(v.flip(1), do.flip(1), scale * q.flip(1), g, back, there, s["ds_last"].transpose(2, 3), last, end, first)
    dv, ds0 = _attend(k.flip(1), scale * q.flip(1), do.flip(1), g, back, there, s["ds_last"], last, end, first)
    grads = [torch.where(live[:, :, None, None], a, 0.0).to(dt) for a in (scale * dq, dk.flip(1), dv.flip(1))]
    return {"o": o, "s_last": state, "dq": grads[0], "dk": grads[1], "dv": grads[2], "ds0": ds0}


def _philox(words, key):
    """Ten rounds of Philox4x32 on counters held as int64 tensors of 32-bit values."""
    a, b, c, d = words
    for r in range(10):
        p, q = a * 0xD2511F53, c * 0xCD9E8D57
        k0, k1 = (key[0] + r * 0x9E3779B9) & 0xFFFFFFFF, (key[1] + r * 0xBB67AE85) & 0xFFFFFFFF
        a, b, c, d = ((q >> 32) & 0xFFFFFFFF) ^ b ^ k0, q & 0xFFFFFFFF, ((p >> 32) & 0xFFFFFFFF) ^ d ^ k1, p & 0xFFFFFFFF
    return a, b, c, d


def _plain_dropout(s):
    x, dy, dt = s["x"].float(), s["dy"].float(), s["x"].dtype
    # element e takes half e % 2 of word e / 2 % 4 of the block whose counter is (e / 8, offset, 0x80000003)
    q, drop = torch.arange(-(-x.numel() // 8), device="cuda"), round(s["p"] * 65536)
    one = torch.ones_like(q)
    words = _philox((q, one * (s["offset"] & 0xFFFFFFFF), one * (s["offset"] >> 32), one * 0x80000003), (s["seed"] & 0xFFFFFFFF, s["seed"] >> 32))
    words = torch.stack(words, 1)
    bits = torch.stack((words & 0xFFFF, words >> 16), 2).view(-1)[:x.numel()].view(x.shape)
    scale = 65536 / (65536 - drop)
    y, dx = (torch.where(bits >= drop, a * scale, 0.0) for a in (x, dy))
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return {"y": y.to(dt), "dx": dx.to(dt)}


def _column(x, R):
    return (x if torch.is_tensor(x) else torch.full((R,), x, device="cuda")).double()[:, None]


def _plain_sample(s):
    l = s["logits"].double()
    R, V = l.shape
    x = (l - l.amax(1, keepdim=True)) / _column(s["temperature"], R).float().double()
    w = (torch.exp(x) * 2.0 ** 40).round().long()  # whole numbers, so that no order of addition matters
    order = l.sort(dim=1, descending=True, stable=True)[1]  # equal logits in the order of their indexes
    ws = w.gather(1, order)
    top_k = _column(s["top_k"], R).long()
    rank = torch.arange(V, device="cuda")[None]
    ws = torch.where((rank < top_k) | (top_k <= 0), ws, 0)
    total, top_p = ws.sum(1, keepdim=True), _column(s["top_p"], R).float().double()
    before = ws.cumsum(1) - ws
    ws = torch.where((before < top_p * total.double()) | (top_p >= 1) | (rank == 0), ws, 0)
    ws = torch.where(ws.double() >= _column(s["min_p"], R).float().double().clamp(max=1) * 2.0 ** 40, ws, 0)
    w = torch.zeros_like(w).scatter_(1, order, ws)
    total = w.sum(1, keepdim=True)
    at = torch.minimum((s["u"].double()[:, None] * total.double()).floor().long(), total - 1)
    token = (w.cumsum(1) <= at).sum(1)
    chance = x.gather(1, token[:, None]) - torch.log(total.double() * 2.0 ** -40)
    return {"token": token, "logprob": chance[:, 0].float()}


# ----------------------------------------------------- the framework's own --

def _own_attn(s):
    from paper_2609_37899_gb300 import api
    case, q, k, v, g = s["case"], s["q"], s["k"], s["v"], s["g"]
    if "o_out" not in s:  # the buffers a program keeps
        s["o_out"], s["s_out"] = torch.empty_like(v), torch.empty_like(s["s0"])
        if case["mode"] == "train":
            s["dq_out"], s["dk_out"], s["dv_out"], s["ds0_out"] = (torch.empty_like(a) for a in (q, k, v, s["s0"]))
        if case["mode"] != "step":
            s["ws"] = api.linear_attn_alloc_workspace(*q.shape[:3], case["dk"], case["dv"], q.dtype, backward=case["mode"] == "train")
    if case["mode"] == "step":
        api.linear_attn_step(q[:, 0], k[:, 0], v[:, 0], g, s["s"], s["o_out"][:, 0], scale=s["scale"])
        return {"o": s["o_out"][:, 0], "s": s["s"]}
    more = dict(s0=s["s0"], lengths=s["lengths"], resets=s["resets"], scale=s["scale"], workspace=s["ws"])
    api.linear_attn_forward(q, k, v, g, s["o_out"], s_last=s["s_out"], **more)
    if case["mode"] == "forward":
        return {"o": s["o_out"], "s_last": s["s_out"]}
    api.linear_attn_backward(q, k, v, g, s["do"], s["dq_out"], s["dk_out"], s["dv_out"], ds_last=s["ds_last"], ds0=s["ds0_out"], **more)
    return {"o": s["o_out"], "s_last": s["s_out"], "dq": s["dq_out"], "dk": s["dk_out"], "dv": s["dv_out"], "ds0": s["ds0_out"]}


def _own_dropout(s):
    from paper_2609_37899_gb300 import api
    if "y_out" not in s:
        s["y_out"], s["dx_out"] = (torch.empty(s["x"].shape, dtype=s["x"].dtype, device="cuda") for _ in range(2))
    api.dropout(s["x"], s["y_out"], s["p"], seed=s["seed"], offset=s["offset"], residual=s["residual"])
    api.dropout(s["dy"], s["dx_out"], s["p"], seed=s["seed"], offset=s["offset"])
    return {"y": s["y_out"], "dx": s["dx_out"]}


def _own_sample(s):
    from paper_2609_37899_gb300 import api
    if "token" not in s:
        s["token"] = torch.empty(s["u"].shape, dtype=torch.int64, device="cuda")
        s["logprob"] = torch.empty_like(s["u"])
    api.sample(s["logits"], s["u"], s["token"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"], logprob=s["logprob"])
    return {"token": s["token"], "logprob": s["logprob"]}


def run(state):
    op = state["case"]["op"]
    if own:
        return {"attn": _own_attn, "dropout": _own_dropout, "sample": _own_sample}[op](state)
    return {"attn": _plain_attn, "dropout": _plain_dropout, "sample": _plain_sample}[op](state)


# ---------------------------------------------------------------- 64 bits --

def _exact_attn(s):
    """Step by step: S = decay S + k v^T, o = S^T q, dq = S do; then from the end R = dS + q do^T, dk = R v, dv = R^T k."""
    case, scale = s["case"], s["scale"]
    q, k, v = (s[n].double() for n in "qkv")
    B, T, H, _ = q.shape
    decay = torch.exp(s["g"].double())[None, :, None, None]
    if case["mode"] == "step":
        S = decay * s["s"].double() + torch.einsum("bhk,bhv->bhkv", k[:, 0], v[:, 0])
        return {"o": scale * torch.einsum("bhkv,bhk->bhv", S, q[:, 0]), "s": S}
    train, ragged = case["mode"] == "train", s["lengths"] is not None
    do = s["do"].double() if train else None
    S, o, dq = s["s0"].double(), torch.zeros_like(v), torch.zeros_like(q)
    fresh = None if s["resets"] is None else (s["resets"] != 0).t()[:, :, None, None, None]
    for t in range(T):
        kept = S if fresh is None else torch.where(fresh[t], 0.0, S)
        new = torch.addcmul(decay * kept, k[:, t, :, :, None], v[:, t, :, None, :])
        a = scale * torch.matmul(q[:, t, :, None], new)[:, :, 0]
        b = scale * torch.matmul(new, do[:, t, :, :, None])[..., 0] if train else None
        if ragged:
            on = (t < s["lengths"])[:, None, None]
            new, a = torch.where(on[..., None], new, S), torch.where(on, a, 0.0)
            b = torch.where(on, b, 0.0) if train else None
        S, o[:, t] = new, a
        if train:
            dq[:, t] = b
    if not train:
        return {"o": o, "s_last": S}
    R, dk, dv = s["ds_last"].double(), torch.zeros_like(k), torch.zeros_like(v)
    for t in range(T - 1, -1, -1):
        new = torch.addcmul(R, scale * q[:, t, :, :, None], do[:, t, :, None, :])
        a, b = torch.matmul(new, v[:, t, :, :, None])[..., 0], torch.matmul(k[:, t, :, None], new)[:, :, 0]
        back = decay * new if fresh is None else torch.where(fresh[t], 0.0, decay * new)
        if ragged:
            on = (t < s["lengths"])[:, None, None]
            a, b, back = torch.where(on, a, 0.0), torch.where(on, b, 0.0), torch.where(on[..., None], back, R)
        dk[:, t], dv[:, t], R = a, b, back
    return {"o": o, "s_last": S, "dq": dq, "dk": dk, "dv": dv, "ds0": R}


def _exact_dropout(s):
    """Philox4x32-10 on the host, then the definition."""
    n, mask = s["x"].numel(), np.uint64(0xFFFFFFFF)
    bits = np.empty(-(-n // 8) * 8, np.uint16)
    for at in range(0, len(bits) // 8, 1 << 20):
        c0 = np.arange(at, min(at + (1 << 20), len(bits) // 8), dtype=np.uint64)
        c1, c2, c3 = (np.full_like(c0, w) for w in (s["offset"] & 0xFFFFFFFF, s["offset"] >> 32, 0x80000003))
        k0, k1 = s["seed"] & 0xFFFFFFFF, s["seed"] >> 32
        for _ in range(10):
            lo, hi = np.uint64(0xD2511F53) * c0, np.uint64(0xCD9E8D57) * c2
            c0, c1, c2, c3 = (hi >> np.uint64(32)) ^ c1 ^ np.uint64(k0), hi & mask, (lo >> np.uint64(32)) ^ c3 ^ np.uint64(k1), lo & mask
            k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
        block = np.stack((c0, c1, c2, c3), 1).astype(np.uint32)
        bits[8 * at:8 * at + 8 * len(c0)] = np.stack((block & 0xFFFF, block >> 16), 2).reshape(-1)
    drop = round(s["p"] * 65536)
    gain = torch.from_numpy(bits[:n] >= drop).cuda().view(s["x"].shape).double() * (65536 / (65536 - drop))
    y = s["x"].double() * gain
    return {"y": y if s["residual"] is None else y + s["residual"].double(), "dx": s["dy"].double() * gain}


def _exact_sample(s):
    """Request by request, in probabilities."""
    R, out = s["logits"].shape[0], {"token": [], "logprob": []}

    def setting(name, r):
        x = s[name]
        return x[r].item() if torch.is_tensor(x) else float(np.float32(x))

    for r in range(R):
        l = s["logits"][r].double()
        p, order = torch.softmax(l / setting("temperature", r), 0).sort(descending=True, stable=True)
        if setting("top_k", r) > 0:
            p[int(setting("top_k", r)):] = 0.0
        if setting("top_p", r) < 1:
            more = p.cumsum(0) - p >= setting("top_p", r) * p.sum()
            more[0] = False
            p[more] = 0.0
        p[p < min(setting("min_p", r), 1.0) * p[0]] = 0.0
        kept = torch.zeros_like(p).scatter_(0, order, p)
        total = kept.cumsum(0)
        token = torch.searchsorted(total, s["u"][r].double() * total[-1], right=True)
        out["token"].append(token)
        out["logprob"].append(torch.log(kept[token] / total[-1]))
    return {k: torch.stack(v) for k, v in out.items()}


def exact(case, seed):
    if case["op"] == "attn" and case["steps"] * (2 if case["mode"] == "train" else 1) * (2 if case["ragged"] else 1) > 50000:
        return None
    s = prepare(case, seed)
    return {"attn": _exact_attn, "dropout": _exact_dropout, "sample": _exact_sample}[case["op"]](s)
