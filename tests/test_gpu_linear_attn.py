"""Linear attention with a decay per head (soma_linear_attn_*) against its formulas in 64 bits.

Tolerances.  Let u = 2^-24 and h be half an ulp of the type relative to a value (fp32: u, bf16: 2^-8,
fp16: 2^-11).  With E the same sums over absolute values (|q|, |k|, |v|, |S|), every result
  out = scale (sum l^(i-j) <x_i, y_j> z_j + ... S)
is off by at most
  (dk + dv + T + 64) u E      fp32 products and sums: one u for every product and addition, and a few
                              for the powers of the decay; tensor cores cut off instead of rounding
  3 h E                       16 bits on the tensor cores: the products <x, y>, and for earlier chunks
                              the decayed z and the state, are each rounded once (h), the two products
                              of such roundings well below the third h
  h |out| + tiny              16 bits: the rounding of the result, and what underflows
and a state in memory by 2 h^2 E in place of 3 h E (both halves of the decayed z are kept), and in fp16
2^-24 of the largest term where that is more.
Those are worst cases of single values.  Over many values of independent roundings the errors add up in
square: each of the three is h / sqrt(3) rms of terms whose squares add up to those of the result for
random signs, so 2 h of the norm is allowed for the norm of the error (and 1e-5 in fp32).
"""
import numpy as np
import pytest
import torch

from gpu_common import api

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
HALF = {"fp32": U, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}
TINY = {"fp32": 2.0 ** -120, "bf16": 2.0 ** -120, "fp16": 2.0 ** -24}


def _case(B, T, H, dk, dv, dtype, seed=0, ragged=False, resets=False, decay=None):
    g = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g)
    s = dict(q=rnd(B, T, H, dk), k=rnd(B, T, H, dk), v=rnd(B, T, H, dv), do=rnd(B, T, H, dv))
    s = {n: x.to(DT[dtype]) for n, x in s.items()}
    s.update(g=-torch.exp(torch.rand(H, generator=g) * 6.5 - 6.5) if decay is None
             else torch.tensor(decay, dtype=torch.float32).expand(H).clone(),
             s0=rnd(B, H, dk, dv), dsl=rnd(B, H, dk, dv), scale=dk ** -0.5, lengths=None, resets=None,
             dtype=dtype)
    if ragged:
        n = torch.randint(0, T + 1, (B,), generator=g, dtype=torch.int32)
        n[0], n[-1] = 0, T
        s["lengths"] = n
        for b in range(B):
            for name in ("q", "k", "v", "do"):
                s[name][b, n[b]:] = float("nan")
    if resets:
        s["resets"] = (torch.rand(B, T, generator=g) < 0.07).to(torch.uint8)
        if T:
            s["resets"][0, 0] = 1
    return {k: v.cuda() if torch.is_tensor(v) else v for k, v in s.items()}


def _reference(s, absolute=False):
    """Outputs and gradients step by step in 64 bits; of the absolute values: the envelope E."""
    live = torch.ones(s["q"].shape[:2], dtype=torch.bool, device="cuda")
    B, T, H, dk = s["q"].shape
    if s["lengths"] is not None:
        live = torch.arange(T, device="cuda")[None] < s["lengths"][:, None]
    put = lambda x: torch.where(live[:, :, None, None], x.double(), 0.0)
    q, k, v, do = (put(s[n]) for n in ("q", "k", "v", "do"))
    S, R = s["s0"].double(), s["dsl"].double()
    if absolute:
        q, k, v, do, S, R = (x.abs() for x in (q, k, v, do, S, R))
    lam = torch.exp(s["g"].double())[None, :, None, None]
    rs = torch.zeros(B, T, device="cuda") if s["resets"] is None else s["resets"]
    o, dq, dkk, dv = (torch.zeros_like(x) for x in (v, q, k, v))
    for t in range(T):
        on = live[:, t, None, None, None]
        kept = torch.where((rs[:, t] != 0)[:, None, None, None], 0.0, lam * S)
        S = torch.where(on, kept + k[:, t, :, :, None] * v[:, t, :, None], S)
        o[:, t] = torch.where(on[..., 0], (q[:, t, :, :, None] * S).sum(2) * s["scale"], 0.0)
        dq[:, t] = torch.where(on[..., 0], (S * do[:, t, :, None]).sum(3) * s["scale"], 0.0)
    for t in range(T - 1, -1, -1):
        on = live[:, t, None, None, None]
        new = R + s["scale"] * q[:, t, :, :, None] * do[:, t, :, None]
        dkk[:, t] = torch.where(on[..., 0], (new * v[:, t, :, None]).sum(3), 0.0)
        dv[:, t] = torch.where(on[..., 0], (k[:, t, :, :, None] * new).sum(2), 0.0)
        back = torch.where((rs[:, t] != 0)[:, None, None, None], 0.0, lam * new)
        R = torch.where(on, back, R)
    return dict(o=o, s_last=S, dq=dq, dk=dkk, dv=dv, ds0=R)


def _run(s, tensors=None, **kw):
    m, out = api(), {}
    t = tensors or s
    nan = lambda x: torch.full_like(x, float("nan"))
    out["o"], out["s_last"] = nan(t["v"]), nan(s["s0"])
    out["dq"], out["dk"], out["dv"], out["ds0"] = nan(t["q"]), nan(t["k"]), nan(t["v"]), nan(s["s0"])
    more = dict(s0=s["s0"], lengths=s["lengths"], resets=s["resets"], scale=s["scale"], **kw)
    m.linear_attn_forward(t["q"], t["k"], t["v"], s["g"], out["o"], s_last=out["s_last"], **more)
    m.linear_attn_backward(t["q"], t["k"], t["v"], s["g"], t["do"], out["dq"], out["dk"], out["dv"],
                           ds_last=s["dsl"], ds0=out["ds0"], **more)
    return out


def _check(s, out, names=("o", "s_last", "dq", "dk", "dv", "ds0")):
    ref, env = _reference(s), _reference(s, absolute=True)
    B, T, H, dk = s["q"].shape
    h, rounds = HALF[s["dtype"]], (dk + s["v"].shape[3] + T + 64) * U
    for n in names:
        state = n in ("s_last", "ds0")
        err = (out[n].double() - ref[n]).abs()
        if s["dtype"] == "fp32":
            tol = rounds * env[n] + 2 * U * ref[n].abs() + 2.0 ** -120
        elif state:
            tol = (rounds + 2 * h * h + 2.0 ** -24) * env[n] + 2.0 ** -24
        else:
            tol = (rounds + 3 * h) * env[n] + h * ref[n].abs() + TINY[s["dtype"]]
        assert out[n].isfinite().all(), n
        assert (err <= tol).all(), (n, (err - tol).max().item(), (err / tol).max().item())
        if ref[n].numel() > 500 and not state:
            bound = 1e-5 if s["dtype"] == "fp32" else 2 * h
            assert err.norm() <= bound * ref[n].norm(), (n, (err.norm() / ref[n].norm()).item())


SHAPES = [(1, 1, 1, 1, 1), (2, 5, 3, 16, 16), (2, 127, 2, 64, 64), (1, 128, 2, 128, 128),
          (2, 129, 1, 128, 64), (3, 300, 2, 40, 72), (2, 257, 2, 33, 65), (1, 1000, 1, 8, 120),
          (1, 400, 3, 96, 128)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_forward_and_backward(shape, dtype):
    s = _case(*shape, dtype, seed=sum(shape))
    out = _run(s)
    _check(s, out)
    assert api().get_status() == 0


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("shape", [(4, 200, 2, 64, 64), (5, 130, 2, 24, 40), (3, 513, 1, 128, 128),
                                   (3, 260, 3, 37, 21)])
@pytest.mark.parametrize("ragged,resets", [(True, False), (False, True), (True, True)])
def test_lengths_and_resets(shape, dtype, ragged, resets):
    s = _case(*shape, dtype, seed=sum(shape) + 1, ragged=ragged, resets=resets)
    _check(s, _run(s))
    assert api().get_status() == 0


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("decay", [0.0, -1e-4, -0.7, -20.0, -200.0, float("-inf")])
def test_decays(decay, dtype):
    """No decay at all, and such that nothing (in the end: exactly nothing) is kept."""
    s = _case(2, 300, 2, 32, 48, dtype, seed=3, decay=decay)
    _check(s, _run(s))
    assert api().get_status() == 0


@pytest.mark.parametrize("bad", [0.5, float("nan"), float("inf")])
def test_a_decay_above_one_is_reported(bad):
    s = _case(2, 150, 2, 32, 32, "bf16", seed=4)
    s["g"][1] = bad
    out = _run(s)
    assert api().get_status() == 6
    ref = _reference({**s, "g": s["g"].clone().fill_(s["g"][0].item())})
    assert out["o"][:, :, 1].isnan().all() and out["dq"][:, :, 1].isnan().all()
    err = (out["o"][:, :, 0].double() - ref["o"][:, :, 0]).norm()
    assert err <= 2 * HALF["bf16"] * ref["o"][:, :, 0].norm()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("B,T,H,dk,dv", [(1, 4100, 1, 64, 64), (2, 3000, 1, 128, 96), (1, 9000, 2, 16, 32)])
@pytest.mark.parametrize("ragged", [False, True])
def test_long_sequences_of_few_heads(B, T, H, dk, dv, dtype, ragged):
    """The time axis is cut here, and joined again."""
    s = _case(B, T, H, dk, dv, dtype, seed=T, ragged=ragged and B > 1, resets=ragged,
              decay=None if ragged else -0.002)
    _check(s, _run(s))


def test_gradients_against_differences():
    """<gradient, d> against (L(x + e d) - L(x - e d)) / 2e of the kernel's own forward call in fp32,
    L = <o, do> + <s_last, dsl>.  L is linear in q, k and v apart, so the differences have no error of
    their own but the roundings: 2 (dk + dv + T + 64) u E / 2e with e = 1 and E the envelope's sum."""
    m, s = api(), _case(2, 140, 2, 24, 40, "fp32", seed=9, resets=True)
    out, env = _run(s), _reference(s, absolute=True)
    size = (env["o"] * s["do"].double().abs()).sum() + (env["s_last"] * s["dsl"].double().abs()).sum()
    tol = 8 * (24 + 40 + 140 + 64) * U * size.item()

    def value(**new):
        t = {**s, **new}
        o, sl = torch.empty_like(t["v"]), torch.empty_like(s["s0"])
        m.linear_attn_forward(t["q"], t["k"], t["v"], s["g"], o, s_last=sl, s0=t["s0"],
                              resets=s["resets"], scale=s["scale"])
        return (o.double() * s["do"].double()).sum() + (sl.double() * s["dsl"].double()).sum()

    for name, grad in (("q", "dq"), ("k", "dk"), ("v", "dv"), ("s0", "ds0")):
        d = torch.randn_like(s[name])
        diff = (value(**{name: s[name] + d}) - value(**{name: s[name] - d})) / 2
        assert abs((out[grad].double() * d.double()).sum() - diff) <= tol, name


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_gradients_against_autograd(dtype):
    s = _case(2, 70, 2, 16, 24, dtype, seed=12)
    q, k, v, s0 = (s[n].double().requires_grad_() for n in ("q", "k", "v", "s0"))
    S, lam, os_ = s0, torch.exp(s["g"].double())[None, :, None, None], []
    for t in range(70):
        S = lam * S + k[:, t, :, :, None] * v[:, t, :, None]
        os_.append(s["scale"] * (q[:, t, :, :, None] * S).sum(2))
    ((torch.stack(os_, 1) * s["do"].double()).sum() + (S * s["dsl"].double()).sum()).backward()
    ref = _reference(s)
    for n, x in (("dq", q), ("dk", k), ("dv", v), ("ds0", s0)):
        assert (x.grad - ref[n]).norm() <= 1e-12 * ref[n].norm(), n
    _check(s, _run(s))


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("layout", ["heads_first", "one_buffer", "odd_rows", "odd_start", "shared"])
def test_layouts(layout, dtype):
    """Strides, alignments and orders other than the dense one give the same results."""
    B, T, H, dk, dv = 2, 200, 4, 32, 32
    s = _case(B, T, H, dk, dv, dtype, seed=21)
    t = {}
    if layout == "heads_first":
        t = {n: s[n].permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) for n in ("q", "k", "v", "do")}
    elif layout == "one_buffer":
        wide = torch.cat([s[n] for n in ("q", "k", "v", "do")], 3).contiguous()
        t = {n: wide[..., 32 * i:32 * i + 32] for i, n in enumerate(("q", "k", "v", "do"))}
    elif layout == "odd_rows":
        for n in ("q", "k", "v", "do"):
            wide = torch.full((B, T, H, 37), float("nan"), dtype=DT[dtype], device="cuda")
            wide[..., :32] = s[n]
            t[n] = wide[..., :32]
    elif layout == "odd_start":
        for n in ("q", "k", "v", "do"):
            flat = torch.full((s[n].numel() + 1,), float("nan"), dtype=DT[dtype], device="cuda")
            flat[1:] = s[n].reshape(-1)
            t[n] = flat[1:].view_as(s[n])
    else:  # all heads read the same k and v; the gradients are each head's
        for n in ("k", "v"):
            s[n] = s[n][:, :, :1].expand(B, T, H, 32)
        t = {"q": s["q"], "k": s["k"], "v": s["v"], "do": s["do"]}
    m = api()
    out = {n: torch.full((B, T, H, 32), float("nan"), dtype=DT[dtype], device="cuda")
           for n in ("o", "dq", "dk", "dv")}
    out["s_last"], out["ds0"] = (torch.full_like(s["s0"], float("nan")) for _ in range(2))
    m.linear_attn_forward(t["q"], t["k"], t["v"], s["g"], out["o"], s_last=out["s_last"], s0=s["s0"],
                          scale=s["scale"])
    m.linear_attn_backward(t["q"], t["k"], t["v"], s["g"], t["do"], out["dq"], out["dk"], out["dv"],
                           s0=s["s0"], ds_last=s["dsl"], ds0=out["ds0"], scale=s["scale"])
    _check(s, out)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_outputs_of_other_strides_leave_the_rest(dtype):
    s = _case(2, 150, 3, 40, 24, dtype, seed=5, ragged=True)
    m = api()
    wide = torch.full((2, 3, 150, 31), 7.0, dtype=DT[dtype], device="cuda")
    o = wide.permute(0, 2, 1, 3)[..., :24]
    m.linear_attn_forward(s["q"], s["k"], s["v"], s["g"], o, s0=s["s0"], lengths=s["lengths"],
                          scale=s["scale"])
    _check(s, {"o": o}, ("o",))
    assert (wide[..., 24:] == 7.0).all()


def test_without_states():
    """No state on either side: the same as zeros, and none is written."""
    for dtype in ("fp32", "bf16"):
        s = _case(2, 170, 2, 64, 32, dtype, seed=6)
        s["s0"].zero_(), s["dsl"].zero_()
        m, out = api(), {n: torch.empty_like(s[r]) for n, r in (("o", "v"), ("dq", "q"), ("dk", "k"), ("dv", "v"))}
        m.linear_attn_forward(s["q"], s["k"], s["v"], s["g"], out["o"], scale=s["scale"])
        m.linear_attn_backward(s["q"], s["k"], s["v"], s["g"], s["do"], out["dq"], out["dk"], out["dv"],
                               scale=s["scale"])
        _check(s, out, ("o", "dq", "dk", "dv"))


@pytest.mark.parametrize("shape", [(0, 5, 2, 8, 8), (2, 0, 2, 8, 8), (2, 5, 0, 8, 8)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_empty(shape, dtype):
    s = _case(*shape, dtype)
    out = _run(s)
    if shape[1] == 0:
        assert torch.equal(out["s_last"], s["s0"]) and torch.equal(out["ds0"], s["dsl"])
    assert api().get_status() == 0


def test_what_is_not_finite_in_padding_is_not_read():
    for dtype in ("fp32", "bf16", "fp16"):
        s = _case(3, 140, 2, 32, 32, dtype, seed=8, ragged=True)
        a = _run(s)
        for b in range(3):
            for n in ("q", "k", "v", "do"):
                s[n][b, s["lengths"][b]:] = float("inf")
        b = _run(s)
        for n in a:
            assert torch.equal(a[n], b[n]) and a[n].isfinite().all(), n


@pytest.mark.parametrize("size", [1e-6, 3e4])
def test_half_precision_keeps_its_range(size):
    """Gradients far below 1, and values near the largest: states and products beyond what fp16 holds
    are scaled, so that only the results have to fit."""
    s = _case(2, 260, 2, 32, 32, "fp16", seed=31, decay=-0.01)
    if size < 1:
        s["do"] = (s["do"].float() * size * 1000).half()
        s["dsl"] *= size * 1000
    else:
        s["v"] = (s["v"].float().clamp(-1, 1) * size).half()
        s["k"] = (s["k"].float() * 0.02).half()
        s["q"] = (s["q"].float() * 0.02).half()
        s["s0"] *= size
        s["dsl"] *= 1e-3
        s["do"] = (s["do"].float() * 1e-4).half()
    _check(s, _run(s))


def test_repeated_calls_agree_bit_for_bit():
    for shape in ((2, 700, 2, 64, 64), (1, 5000, 1, 128, 128)):
        s = _case(*shape, "bf16", seed=2)
        a, b = _run(s), _run(s)
        for n in a:
            assert torch.equal(a[n], b[n]), n


def test_another_stream_and_no_workspace():
    s = _case(1, 4000, 1, 64, 64, "bf16", seed=7)
    want, m = _run(s), api()
    side = torch.cuda.Stream()
    o = torch.empty_like(s["v"])
    side.wait_stream(torch.cuda.current_stream())
    m.linear_attn_forward(s["q"], s["k"], s["v"], s["g"], o, s0=s["s0"], scale=s["scale"], stream=side)
    side.synchronize()
    assert torch.equal(o, want["o"])


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("B,H,dk,dv", [(1, 1, 1, 1), (3, 2, 64, 64), (2, 5, 128, 128), (4, 3, 33, 65),
                                       (70, 3, 40, 24), (2, 2, 128, 3), (2, 1, 2, 127)])
def test_step(B, H, dk, dv, dtype):
    """Token by token: o and the state follow the recurrence (fp32 but for o's rounding)."""
    s = _case(B, 4, H, dk, dv, dtype, seed=B + dk)
    m, state, outs = api(), s["s0"].clone(), []
    for t in range(4):
        o = torch.full((B, H, dv), float("nan"), dtype=DT[dtype], device="cuda")
        m.linear_attn_step(s["q"][:, t], s["k"][:, t], s["v"][:, t], s["g"], state, o, scale=s["scale"])
        outs.append(o)
    ref, env = _reference(s), _reference(s, absolute=True)
    got = {"o": torch.stack(outs, 1), "s_last": state}
    rounds = (dk + dv + 68) * U
    for n in got:
        h = HALF[dtype] if n == "o" else 0.0
        tol = rounds * env[n] + h * ref[n].abs() + TINY[dtype]
        assert ((got[n].double() - ref[n]).abs() <= tol).all(), n


def test_step_with_a_misaligned_state():
    s = _case(2, 1, 3, 32, 32, "bf16", seed=1)
    flat = torch.zeros(s["s0"].numel() + 1, device="cuda")
    state = flat[1:].view_as(s["s0"])
    state.copy_(s["s0"])
    o = torch.empty(2, 3, 32, dtype=torch.bfloat16, device="cuda")
    api().linear_attn_step(s["q"][:, 0], s["k"][:, 0], s["v"][:, 0], s["g"], state, o, scale=s["scale"])
    ref, env = _reference(s), _reference(s, absolute=True)
    assert ((o[:, None].double() - ref["o"]).abs() <= 200 * U * env["o"] + 2.0 ** -8 * ref["o"].abs()).all()
    assert ((state.double() - ref["s_last"]).abs() <= 8 * U * env["s_last"]).all()


def test_a_prompt_and_its_tokens_join():
    """The state that a prompt leaves goes on token by token."""
    s = _case(2, 150, 2, 32, 64, "bf16", seed=14)
    m, state = api(), torch.empty_like(s["s0"])
    o = torch.empty(2, 140, 2, 64, dtype=torch.bfloat16, device="cuda")
    cut = {n: s[n][:, :140] for n in ("q", "k", "v")}
    m.linear_attn_forward(cut["q"], cut["k"], cut["v"], s["g"], o, s_last=state, s0=s["s0"], scale=s["scale"])
    parts = [o]
    for t in range(140, 150):
        o1 = torch.empty(2, 2, 64, dtype=torch.bfloat16, device="cuda")
        m.linear_attn_step(s["q"][:, t], s["k"][:, t], s["v"][:, t], s["g"], state, o1, scale=s["scale"])
        parts.append(o1[:, None])
    _check(s, {"o": torch.cat(parts, 1), "s_last": state}, ("o", "s_last"))
