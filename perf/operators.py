"""Cases of the first-order training operators: linear cross entropy, the gated linear recurrence and AdamW.

`run` computes them in plain torch operations where `own` is false, and through the framework's entry points where it
is true.  `exact` computes the same from the definitions in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
WIDTH = {"bf16": 2, "fp16": 2, "fp32": 4}
E4M3 = torch.float8_e4m3fn
IGNORE = -100
LR, BETA1, BETA2, EPS, DECAY = 1e-3, 0.9, 0.999, 1e-8, 0.01


# ------------------------------------------------------------------ cases --

def listed():
    return [
        # scoring a handful of continuations with a subword vocabulary: the head's weights are read once, little else counts
        {"name": "ce_score_64", "op": "ce", "train": False, "rows": 64, "vocab": 32768, "dim": 960, "dtype": "bf16", "ignored": 0.0},
        # scoring long documents in a batch, the head of the widest expert, odd row count
        {"name": "ce_score_long", "op": "ce", "train": False, "rows": 16385, "vocab": 32768, "dim": 1376, "dtype": "bf16", "ignored": 0.02},
        # the byte head of the framework's experts (256 logits) at its benchmark's 32 x 256 targets, in half precision
        {"name": "ce_train_byte", "op": "ce", "train": True, "rows": 8192, "vocab": 256, "dim": 960, "dtype": "fp16", "ignored": 0.0},
        # a padded batch: odd rows, vocabulary and width that are no multiples of any tile, one row in twelve without a target
        {"name": "ce_train_ragged", "op": "ce", "train": True, "rows": 3001, "vocab": 50021, "dim": 680, "dtype": "bf16", "ignored": 0.08},
        # the training step of a large vocabulary
        {"name": "ce_train_large", "op": "ce", "train": True, "rows": 8192, "vocab": 131072, "dim": 1024, "dtype": "bf16", "ignored": 0.0},
        # one token of each of 64 running requests
        {"name": "scan_step_64", "op": "scan", "mode": "step", "batch": 64, "steps": 1, "dim": 960, "dtype": "bf16", "ragged": False},
        # reading one long prompt: few channels, so the time axis has to be split
        {"name": "scan_prompt_long", "op": "scan", "mode": "forward", "batch": 1, "steps": 32768, "dim": 960, "dtype": "bf16", "ragged": False},
        # a batch of documents of different lengths, packed with resets, odd width, in 32 bits
        {"name": "scan_train_ragged", "op": "scan", "mode": "train", "batch": 13, "steps": 1000, "dim": 481, "dtype": "fp32", "ragged": True},
        # the training step of a wide recurrent layer
        {"name": "scan_train_large", "op": "scan", "mode": "train", "batch": 32, "steps": 2048, "dim": 1376, "dtype": "bf16", "ragged": False},
        # the smallest expert of the framework (49,664 parameters, six tensors): latency counts
        {"name": "adamw_tiny", "op": "adamw", "params": 49664, "tensors": 6, "param": "fp32", "grad": "fp32", "master": False, "bits": 32},
        # 32-bit parameters and moments, bf16 gradients, many tensors
        {"name": "adamw_32_large", "op": "adamw", "params": 200000003, "tensors": 300, "param": "fp32", "grad": "bf16", "master": False, "bits": 32},
        # bf16 parameters with 32-bit masters and 8-bit moments
        {"name": "adamw_8_large", "op": "adamw", "params": 150000001, "tensors": 120, "param": "bf16", "grad": "bf16", "master": True, "bits": 8},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["ce", "ce", "scan", "scan", "adamw"])
    if op == "ce":
        while True:
            rows, vocab, dim = _log(rng, 1, 16385), _log(rng, 256, 131072), _log(rng, 32, 1376)
            if rows * vocab * dim <= 5e11:
                break
        return {"op": "ce", "train": rng.random() < 0.65, "rows": rows, "vocab": vocab, "dim": dim,
                "dtype": rng.choice(["bf16", "bf16", "fp16"]), "ignored": rng.choice([0.0, 0.05, 0.3])}
    if op == "scan":
        mode = rng.choice(["step", "forward", "train", "train"])
        while True:
            batch, dim = _log(rng, 1, 256), _log(rng, 32, 2048)
            steps = 1 if mode == "step" else _log(rng, 1, 65536)
            if batch * dim * steps <= 80e6:
                break
        return {"op": "scan", "mode": mode, "batch": batch, "steps": steps, "dim": dim,
                "dtype": rng.choice(["bf16", "bf16", "fp16", "fp32"]), "ragged": mode != "step" and rng.random() < 0.4}
    param = rng.choice(["fp32", "bf16", "fp16"])
    return {"op": "adamw", "params": _log(rng, 1000, 100000000), "tensors": _log(rng, 1, 400), "param": param,
            "grad": rng.choice(["fp32", "bf16", "fp16"]), "master": param != "fp32", "bits": rng.choice([8, 32])}


# ----------------------------------------------------------------- inputs --

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 2654435761 % (1 << 62))
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _sizes(case):
    """Tensor sizes of an AdamW case: a few large ones and many small ones, of the case's total."""
    k = min(case["tensors"], case["params"])
    w = [1.0 / (1 + (7 * i) % k) ** 0.7 for i in range(k)]
    n = [max(1, int(x / sum(w) * case["params"])) for x in w]
    n[0] += case["params"] - sum(n)
    return n


def prepare(case, seed):
    g = _gen(seed)
    s = {"case": case, "t": 10}
    if case["op"] == "ce":
        N, V, d, dt = case["rows"], case["vocab"], case["dim"], DTYPES[case["dtype"]]
        emb = (_randn(g, V, d) * (1.5 / math.sqrt(d))).to(dt)
        # targets drawn towards the front of the vocabulary, as frequent tokens are; the state leans to its target
        y = (torch.rand(N, generator=g, device="cuda") ** 3 * V).long().clamp_(max=V - 1)
        h = (_randn(g, N, d) + 3.0 * emb[y].float()).to(dt)
        skip = torch.rand(N, generator=g, device="cuda") < case["ignored"]
        y[skip] = IGNORE
        h[skip] = float("nan")  # padding holds whatever was there
        scale = 1024.0 if case["dtype"] == "fp16" else 1.0  # half-precision training scales its loss
        s.update(h=h, emb=emb, y=y, dloss=torch.full((N,), scale / N, device="cuda") * (y != IGNORE))
    elif case["op"] == "scan":
        B, T, D, dt = case["batch"], case["steps"], case["dim"], DTYPES[case["dtype"]]
        shift = torch.tensor([0.0, 2.0, 0.0, 0.5], device="cuda").view(4, 1)  # forget gates lean to keeping
        s.update(gates=torch.empty(B, T, 4, D, dtype=dt, device="cuda"), c0=_randn(g, B, D) * 0.5, lengths=None, resets=None)
        step = max(1, (1 << 24) // (B * 4 * D))
        for t in range(0, T, step):
            n = min(step, T - t)
            s["gates"][:, t:t + n] = (_randn(g, B, n, 4, D) * 1.5 + shift).to(dt)
        if case["ragged"]:
            s["lengths"] = torch.randint(0, T + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
            s["lengths"][0] = T
            s["resets"] = (torch.rand(B, T, generator=g, device="cuda") < 0.01).to(torch.uint8)
            past = torch.arange(T, device="cuda")[None] >= s["lengths"][:, None]
            s["gates"][past] = float("nan")
        if case["mode"] == "step":
            s["c"] = s["c0"].clone()
        if case["mode"] == "train":
            s["dh"] = (_randn(g, B, T, D) * 0.1).to(dt)
            s["dc_last"] = _randn(g, B, D) * 0.1
    else:
        sizes = _sizes(case)
        at, total = [], 0
        for n in sizes:  # every tensor starts at a multiple of 256 in one allocation
            at.append(total)
            total += -(-n // 256) * 256
        live = torch.zeros(total, dtype=torch.bool, device="cuda")
        size = torch.zeros(total // 256, device="cuda")
        for i, (a, n) in enumerate(zip(at, sizes)):
            live[a:a + n] = True
            size[a // 256:(a + n + 255) // 256] = 10.0 ** (-2 - i % 3)  # gradients differ from tensor to tensor
        size = size.repeat_interleave(256)
        master = _randn(g, total).mul_(0.05).mul_(live)
        scale = 1024.0 if case["grad"] == "fp16" else 1.0
        grad = _randn(g, total).mul_(size).mul_(live)
        m = _randn(g, total).mul_(size).mul_(0.2 * live)
        r = _randn(g, total).abs_().add_(0.3).mul_(size).mul_(live)
        s.update(sizes=sizes, at=at, live=live, seed=seed & 0xFFFFFFFF, grad=(grad * scale).to(DTYPES[case["grad"]]),
                 scale=torch.tensor([1.0 / scale], device="cuda"))
        s["p"] = master.to(DTYPES[case["param"]])
        s["master"] = master if case["master"] else None
        if case["bits"] == 32:
            s.update(m=m, v=r * r, ms=None, vs=None)
        else:
            for name, x in (("m", m), ("v", r)):
                top = x.view(-1, 256).abs().amax(1) / 448
                s[name] = (x.view(-1, 256) / top.clamp(min=1e-30)[:, None]).view(-1).to(E4M3)
                s[name + "s"] = top
    return s


def work(case):
    if case["op"] == "ce":
        N, V, d, w = case["rows"], case["vocab"], case["dim"], WIDTH[case["dtype"]]
        nbytes, flops = (N + V) * d * w + 16 * N, 2 * N * V * d
        if case["train"]:  # the logits are computed again, then two more products
            nbytes, flops = nbytes + (N + V) * d * w + 4 * N, flops + 6 * N * V * d
        return {"bytes": nbytes, "flops": flops}
    if case["op"] == "scan":
        n, w, rows = case["batch"] * case["steps"] * case["dim"], WIDTH[case["dtype"]], case["batch"] * case["dim"]
        if case["mode"] == "train":  # gates and dh in, h and dgates out
            return {"bytes": n * 10 * w + rows * 16, "flops": n * 60}
        return {"bytes": n * 5 * w + rows * 8, "flops": n * 25}
    state = 8 if case["bits"] == 32 else 2 + 8 / 256
    p = 4 if case["master"] else WIDTH[case["param"]]
    per = WIDTH[case["grad"]] + 2 * state + 2 * p + (WIDTH[case["param"]] if case["master"] else 0)
    return {"bytes": per * case["params"], "flops": 15 * case["params"]}


# ------------------------------------------------------------- plain forms --

def _plain_ce(s):
    y, h, emb = s["y"], s["h"].float(), s["emb"].float()
    keep = y != IGNORE
    h = torch.where(keep[:, None], h, torch.zeros_like(h))
    at = y.clamp(min=0)[:, None]
    logits = h @ emb.T
    top = logits.amax(1, keepdim=True)
    own_logit = logits.gather(1, at)[:, 0]
    p = (logits - top).exp_()
    total = p.sum(1, keepdim=True)
    lse = (top + total.log())[:, 0]
    loss = (lse - own_logit) * keep
    lse = lse * keep
    if not s["case"]["train"]:
        return {"loss": loss, "lse": lse}
    p.div_(total).scatter_add_(1, at, -torch.ones_like(total))
    p.mul_((s["dloss"] * keep)[:, None])
    dt = s["h"].dtype
    return {"loss": loss, "lse": lse, "dh": (p @ emb).to(dt), "demb": (p.T @ h).to(dt)}


def _scan(f, u):
    """c_t = f_t c_{t-1} + u_t along dim 1 from c = 0: pairs of steps first, then the scan of half the length."""
    T = f.shape[1]
    if T == 1:
        return u
    if T % 2:
        c = _scan(f[:, :-1], u[:, :-1])
        return torch.cat((c, f[:, -1:] * c[:, -1:] + u[:, -1:]), 1)
    f0, f1, u0, u1 = f[:, 0::2], f[:, 1::2], u[:, 0::2], u[:, 1::2]
    odd = _scan(f0 * f1, f1 * u0 + u1)
    even = torch.cat((u0[:, :1], u0[:, 1:] + f0[:, 1:] * odd[:, :-1]), 1)
    return torch.stack((even, odd), 2).flatten(1, 2)


def _plain_scan(s):
    case, a, dt = s["case"], s["gates"].float(), s["gates"].dtype
    B, T, _, D = a.shape
    c0 = s["c"] if case["mode"] == "step" else s["c0"]
    live = torch.ones(B, T, 1, dtype=torch.bool, device=a.device)
    if s["lengths"] is not None:
        live = torch.arange(T, device=a.device)[None, :, None] < s["lengths"][:, None, None]
        a = torch.where(live[..., None], a, torch.zeros_like(a))
    i, f, o, g = a[:, :, 0].sigmoid(), a[:, :, 1].sigmoid(), a[:, :, 3].sigmoid(), a[:, :, 2].tanh()
    carry = f if s["resets"] is None else f * (s["resets"][:, :, None] == 0)
    carry = torch.where(live, carry, torch.ones_like(carry))  # steps past the end keep the state
    u = torch.where(live, i * g, torch.zeros_like(i))
    c = _scan(carry, torch.cat((u[:, :1] + carry[:, :1] * c0[:, None], u[:, 1:]), 1))
    th = c.tanh()
    h = torch.where(live, o * th, torch.zeros_like(th)).to(dt)
    last = c[:, -1].clone()
    if case["mode"] == "step":
        s["c"].copy_(last)
        return {"h": h[:, 0], "c": s["c"]}
    if case["mode"] == "forward":
        return {"h": h, "c_last": last}
    dh = torch.where(live, s["dh"].float(), torch.zeros_like(th))
    into = dh * o * (1 - th * th)
    into = torch.cat((into[:, :-1], into[:, -1:] + s["dc_last"][:, None]), 1).flip(1)
    back = torch.cat((torch.ones_like(carry[:, :1]), carry[:, 1:].flip(1)), 1)
    dc = _scan(back, into).flip(1)
    prev = torch.cat((c0[:, None], c[:, :-1]), 1)
    if s["resets"] is not None:
        prev = prev * (s["resets"][:, :, None] == 0)
    da = torch.stack((dc * g * i * (1 - i), dc * prev * f * (1 - f), dc * i * (1 - g * g), dh * th * o * (1 - o)), 2)
    da = torch.where(live[..., None], da, torch.zeros_like(da)).to(dt)
    return {"h": h, "c_last": last, "dgates": da, "dc0": carry[:, 0] * dc[:, 0]}


def _philox(words, key):
    """Ten rounds of Philox4x32 on counters held as int64 tensors of 32-bit values."""
    a, b, c, d = words
    for r in range(10):
        p, q = a * 0xD2511F53, c * 0xCD9E8D57
        k0, k1 = (key[0] + r * 0x9E3779B9) & 0xFFFFFFFF, (key[1] + r * 0xBB67AE85) & 0xFFFFFFFF
        a, b, c, d = ((q >> 32) & 0xFFFFFFFF) ^ b ^ k0, q & 0xFFFFFFFF, ((p >> 32) & 0xFFFFFFFF) ^ d ^ k1, p & 0xFFFFFFFF
    return a, b, c, d


def _draws(s, n):
    """16 random bits for every parameter: element j of the group of eight q takes half j % 2 of word j / 2 of the
    block whose counter is (q, tensor, update, 0x80000002)."""
    at = torch.tensor(s["at"], device="cuda")
    q = torch.arange(n // 8, device="cuda")
    tensor = torch.bucketize(q * 8, at, right=True) - 1
    q = q - at[tensor] // 8
    words = torch.stack(_philox((q, tensor, torch.full_like(q, s["t"]), torch.full_like(q, 0x80000002)), (s["seed"], 0)), 1)
    return torch.stack((words & 0xFFFF, words >> 16), 2).view(-1)


def _round8(x, bits, floor):
    """x in blocks of 256 as e4m3 values and a scale, rounded at random by 16 bits each; `floor` keeps what is above
    zero from becoming zero."""
    top = x.view(-1, 256).abs().amax(1, keepdim=True)
    full = torch.full_like(top, 448.0)
    some = top > 2.0 ** -100
    inv = torch.where(some, full / top, torch.zeros_like(top))
    y = (x.view(-1, 256).abs() * inv).clamp(max=448.0).view(-1)
    low = torch.where(y < 2.0 ** -6, torch.full_like(y, 2.0 ** -6), torch.zeros_like(y))
    z = (((y + low).view(torch.int32) + (bits.to(torch.int32) << 4)) & -(1 << 20)).view(torch.float32) - low
    if floor:
        z = torch.where(y > 0, z.clamp(min=2.0 ** -9), z)
    return torch.where(x < 0, -z, z).to(E4M3), torch.where(some, top / full, torch.zeros_like(top))[:, 0]


def _plain_adamw(s):
    s["t"] += 1
    t, eight = s["t"], s["case"]["bits"] == 8
    w = (s["p"] if s["master"] is None else s["master"]).float()
    g = s["grad"].float() * s["scale"]
    m, v = s["m"].float(), s["v"].float()
    if eight:
        m, r = (m.view(-1, 256) * s["ms"][:, None]).view(-1), (v.view(-1, 256) * s["vs"][:, None]).view(-1)
        v = r * r
    m1 = m * BETA1 + g * (1 - BETA1)
    v1 = v * BETA2 + (g * g) * (1 - BETA2)
    r1 = v1.sqrt()
    w1 = w * (1 - LR * DECAY) - (m1 / (r1 * (1 / math.sqrt(1 - BETA2 ** t)) + EPS)) * (LR / (1 - BETA1 ** t))
    fine = m1.isfinite() & v1.isfinite() & s["live"]
    w1 = torch.where(fine, w1, w)
    if s["master"] is not None:
        s["master"].copy_(w1)
    s["p"].copy_(w1)
    if eight:
        bits = _draws(s, m.numel())
        s["m"], s["ms"] = _round8(torch.where(fine, m1, m), bits, False)
        s["v"], s["vs"] = _round8(torch.where(fine, r1, r), bits, True)
    else:
        s["m"].copy_(torch.where(fine, m1, m))
        s["v"].copy_(torch.where(fine, v1, v))
    return {k: s[k] for k in ("p", "master", "m", "v", "ms", "vs")}


# ----------------------------------------------------- the framework's own --

def _own_ce(s):
    from paper_2609_37899_gb300 import api
    h, emb = s["h"], s["emb"]
    if "loss" not in s:  # the buffers a program keeps
        s["loss"], s["lse"] = (torch.empty(h.shape[0], device="cuda") for _ in range(2))
        s["ws"] = api.linear_ce_alloc_workspace(h.shape[0], emb.shape[0], h.shape[1], h.dtype, s["case"]["train"])
        if s["case"]["train"]:
            s["dh_out"], s["demb_out"] = torch.empty_like(h), torch.empty_like(emb)
    api.linear_ce_forward(h, emb, s["y"], s["loss"], s["lse"], s["ws"], ignore_index=IGNORE)
    if not s["case"]["train"]:
        return {"loss": s["loss"], "lse": s["lse"]}
    api.linear_ce_backward(h, emb, s["y"], s["lse"], s["dloss"], s["dh_out"], s["demb_out"], s["ws"], ignore_index=IGNORE)
    return {"loss": s["loss"], "lse": s["lse"], "dh": s["dh_out"], "demb": s["demb_out"]}


def _own_scan(s):
    from paper_2609_37899_gb300 import api
    a, mode = s["gates"], s["case"]["mode"]
    B, T, _, D = a.shape
    if "h_out" not in s:  # the buffers a program keeps
        s["h_out"] = torch.empty(B, T, D, dtype=a.dtype, device="cuda")
        if mode != "step":
            s["c_last"] = torch.empty(B, D, device="cuda")
        if mode == "train":
            s["marks"] = api.scan_alloc_checkpoints(B, T, D)
            s["dgates_out"], s["dc0_out"] = torch.empty_like(a), torch.empty(B, D, device="cuda")
    if mode == "step":
        api.scan_step(a[:, 0], s["c"], s["h_out"][:, 0])
        return {"h": s["h_out"][:, 0], "c": s["c"]}
    api.scan_forward(a, s["h_out"], s["c_last"], c0=s["c0"], lengths=s["lengths"], resets=s["resets"], checkpoints=s.get("marks"))
    if mode == "forward":
        return {"h": s["h_out"], "c_last": s["c_last"]}
    api.scan_backward(a, s["marks"], s["dh"], s["dgates_out"], s["dc0_out"], dc_last=s["dc_last"], lengths=s["lengths"], resets=s["resets"])
    return {"h": s["h_out"], "c_last": s["c_last"], "dgates": s["dgates_out"], "dc0": s["dc0_out"]}


def _views(s, name, block=1):
    flat = s[name]
    return None if flat is None else [flat[a // block:a // block + -(-n // block)] for a, n in zip(s["at"], s["sizes"])]


def _own_adamw(s):
    from paper_2609_37899_gb300 import api
    if "opt" not in s:  # the handle a program keeps
        s["opt"] = api.AdamW(_views(s, "p"), _views(s, "m"), _views(s, "v"), m_scales=_views(s, "ms", 256), v_scales=_views(s, "vs", 256),
                             masters=_views(s, "master"), weight_decay=DECAY)
        s["grads"] = _views(s, "grad")
    s["t"] += 1
    s["opt"].step(s["grads"], t=s["t"], lr=LR, beta1=BETA1, beta2=BETA2, eps=EPS, seed=s["seed"], grad_scale=s["scale"])
    return {k: s[k] for k in ("p", "master", "m", "v", "ms", "vs")}


def run(state):
    op = state["case"]["op"]
    if own:
        return {"ce": _own_ce, "scan": _own_scan, "adamw": _own_adamw}[op](state)
    return {"ce": _plain_ce, "scan": _plain_scan, "adamw": _plain_adamw}[op](state)


# ---------------------------------------------------------------- 64 bits --

def _exact_ce(s):
    h, emb, y = s["h"], s["emb"].double(), s["y"]
    N, out = h.shape[0], {"loss": [], "lse": [], "dh": []}
    demb = torch.zeros_like(emb)
    for a in range(0, N, 1024):
        keep = y[a:a + 1024] != IGNORE
        x = torch.nan_to_num(h[a:a + 1024].double(), nan=0.0)
        logits = x @ emb.T
        lse = torch.logsumexp(logits, 1)
        at = torch.where(keep, y[a:a + 1024], 0)
        rows = torch.arange(len(at), device="cuda")
        out["loss"].append(torch.where(keep, lse - logits[rows, at], 0.0))
        out["lse"].append(torch.where(keep, lse, 0.0))
        if s["case"]["train"]:
            p = torch.exp(logits - lse[:, None])
            p[rows, at] -= 1.0
            p *= torch.where(keep, s["dloss"][a:a + 1024].double(), 0.0)[:, None]
            out["dh"].append(p @ emb)
            demb += p.T @ x
    got = {k: torch.cat(v) for k, v in out.items() if v}
    return {**got, "demb": demb} if s["case"]["train"] else got


def _exact_scan(s):
    case, a = s["case"], s["gates"]
    B, T, _, D = a.shape
    c = s["c0"].double()
    hs, cs, ends = torch.zeros(B, T, D, dtype=torch.float64, device="cuda"), [], s["lengths"]
    for t in range(T):
        x = a[:, t].double()
        cs.append(c)
        new = c if s["resets"] is None else c * (s["resets"][:, t] == 0)[:, None]
        new = torch.sigmoid(x[:, 1]) * new + torch.sigmoid(x[:, 0]) * torch.tanh(x[:, 2])
        h = torch.sigmoid(x[:, 3]) * torch.tanh(new)
        if ends is not None:
            on = (t < ends)[:, None]
            new, h = torch.where(on, new, c), torch.where(on, h, 0.0)
        c, hs[:, t] = new, h
    if case["mode"] == "step":
        return {"h": hs[:, 0], "c": c}
    if case["mode"] == "forward":
        return {"h": hs, "c_last": c}
    last, dc = c, s["dc_last"].double()
    da = torch.zeros(B, T, 4, D, dtype=torch.float64, device="cuda")
    for t in range(T - 1, -1, -1):
        x, dh = a[:, t].double(), s["dh"][:, t].double()
        i, f, g, o = torch.sigmoid(x[:, 0]), torch.sigmoid(x[:, 1]), torch.tanh(x[:, 2]), torch.sigmoid(x[:, 3])
        prev = cs[t] if s["resets"] is None else cs[t] * (s["resets"][:, t] == 0)[:, None]
        th = torch.tanh(f * prev + i * g)
        total = dc + dh * o * (1 - th ** 2)
        d = torch.stack((total * g * i * (1 - i), total * prev * f * (1 - f), total * i * (1 - g ** 2), dh * th * o * (1 - o)), 1)
        back = total * f if s["resets"] is None else total * f * (s["resets"][:, t] == 0)[:, None]
        if ends is not None:
            on = (t < ends)[:, None]
            d, back = torch.where(on[:, None], d, 0.0), torch.where(on, back, dc)
        da[:, t], dc = d, back
    return {"h": hs, "c_last": last, "dgates": da, "dc0": dc}


def _exact_round8(x, bits, floor):
    """The e4m3 grid in 64 bits: a step of 2^(e-3) in [2^e, 2^(e+1)), of 2^-9 below 2^-6."""
    x = x.view(-1, 256)
    scale = x.abs().amax(1, keepdim=True) / 448
    y = torch.where(scale > 0, x.abs() / scale.clamp(min=1e-300), 0.0).view(-1)
    step = torch.exp2(torch.floor(torch.log2(y.clamp(min=2.0 ** -6))).clamp(max=8) - 3)
    z = (torch.floor(y / step + bits.double() / 65536) * step).clamp(max=448)
    if floor:
        z = torch.where((y > 0) & (z == 0), 2.0 ** -9, z)
    return torch.sign(x.view(-1)) * z, scale[:, 0]


def _exact_adamw(s):
    t = s["t"] = s["t"] + 1
    w = (s["p"] if s["master"] is None else s["master"]).double()
    g = s["grad"].double() * s["scale"].double()
    m, v = s["m"].double(), s["v"].double()
    if s["ms"] is not None:
        m = m * s["ms"].double().repeat_interleave(256)
        v = (v * s["vs"].double().repeat_interleave(256)) ** 2
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * g ** 2
    new = w - LR * DECAY * w - LR * (m / (1 - BETA1 ** t)) / ((v / (1 - BETA2 ** t)).sqrt() + EPS)
    new = torch.where(s["live"], new, w)
    out = {"p": new, "master": None if s["master"] is None else new, "m": m, "v": v, "ms": None, "vs": None}
    if s["ms"] is not None:
        bits = _draws(s, m.numel())
        out["m"], out["ms"] = _exact_round8(m, bits, False)
        out["v"], out["vs"] = _exact_round8(v.sqrt(), bits, True)
    return out


def exact(case, seed):
    if case["op"] == "ce" and case["rows"] * case["vocab"] * case["dim"] * (6 if case["train"] else 2) > 1.2e13:
        return None
    s = prepare(case, seed)
    return {"ce": _exact_ce, "scan": _exact_scan, "adamw": _exact_adamw}[case["op"]](s)
