"""Host-side checks of linear attention, dropout and sampling: no launch is made."""
import ctypes

import pytest
import torch

FAKE = ctypes.c_void_p(0x10000)  # never dereferenced: validation fails first
ODD = ctypes.c_void_p(0x10001)
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def soma():
    from paper_2609_37899_gb300 import build
    build.build()
    from paper_2609_37899_gb300 import api
    return api


def test_structures_have_the_sizes_of_the_abi(soma):
    for name, size in (("soma_attn_dims", 32), ("soma_attn_strides", 24), ("soma_sample_config", 48),
                       ("soma_sequence_times", 48)):
        assert ctypes.sizeof(getattr(soma, name)) == size


def test_linear_attn_refusals(soma):
    L, D, S = soma.lib(), soma.soma_attn_dims, soma.soma_attn_strides
    ok, s = D(2, 3, 4, 8, 16), S(192, 64, 16)

    def fwd(q=FAKE, st=s, dtype=1, d=ok, decay=FAKE, scale=1.0, s0=None, lengths=None, o=FAKE, s_last=None):
        return L.soma_linear_attn_forward(q, st, FAKE, s, FAKE, s, dtype, d, decay, scale, s0, lengths,
                                          None, o, s, s_last, None, 0, None)

    def bwd(d=ok, do=FAKE, dq=FAKE, dv=FAKE, s0=None, dsl=None, ds0=None, dtype=1, scale=1.0):
        return L.soma_linear_attn_backward(FAKE, s, FAKE, s, FAKE, s, dtype, d, FAKE, scale, s0, None,
                                           None, do, s, dsl, dq, s, FAKE, s, dv, s, ds0, None, 0, None)

    def step(q=FAKE, d=ok, state=FAKE, dtype=1, scale=1.0):
        return L.soma_linear_attn_step(q, s, FAKE, s, FAKE, s, dtype, d, FAKE, scale, state, FAKE, s, None)

    for bad in (D(-1, 3, 4, 8, 16), D(2, -1, 4, 8, 16), D(2, 3, -4, 8, 16), D(2, 3, 4, 0, 16),
                D(2, 3, 4, 8, 0), D(2, 3, 4, 129, 16), D(2, 3, 4, 8, 129), D(1 << 31, 3, 1, 8, 16),
                D(2, 1 << 31, 4, 8, 16), D(2, 3, (1 << 16) + 1, 8, 16), D(1 << 20, 3, 1 << 10, 8, 16)):
        assert fwd(d=bad) == 2 and bwd(d=bad) == 2 and step(d=bad) == 2
        assert L.soma_linear_attn_workspace_bytes(bad, 1, 0) == -1
    assert L.soma_linear_attn_workspace_bytes(ok, 3, 0) == -1
    assert L.soma_linear_attn_workspace_bytes(ok, 1, 2) == -1
    assert L.soma_linear_attn_workspace_bytes(ok, 1, 1) >= 0
    for f in (fwd, bwd, step):
        assert f(dtype=3) == 1 and f(scale=INF) == 1 and f(scale=NAN) == 1
    assert fwd(q=None) == 1 and fwd(o=None) == 1 and fwd(decay=None) == 1
    assert fwd(q=ODD) == 1 and fwd(o=ODD) == 1 and fwd(decay=ODD) == 1 and fwd(s0=ODD) == 1
    assert fwd(lengths=ODD) == 1 and fwd(s_last=ODD) == 1 and fwd(st=S(192, -64, 16)) == 1
    assert bwd(do=None) == 1 and bwd(dq=None) == 1 and bwd(dv=ODD) == 1 and bwd(ds0=ODD) == 1
    assert step(q=None) == 1 and step(state=None) == 1 and step(state=ODD) == 1 and step(q=ODD) == 1
    # outputs whose rows would lie on one another
    for st in (S(192, 64, 0), S(192, 0, 16), S(0, 64, 16), S(192, 64, 15)):
        assert L.soma_linear_attn_forward(FAKE, s, FAKE, s, FAKE, s, 1, ok, FAKE, 1.0, None, None, None,
                                          FAKE, st, None, None, 0, None) == 1
        if st.t:
            assert L.soma_linear_attn_step(FAKE, s, FAKE, s, FAKE, s, 1, ok, FAKE, 1.0, FAKE, FAKE, st,
                                           None) == 1
    states = 2 * 4 * 8 * 16
    for off in (0, 4, 4 * (states - 1), -4 * (states - 1)):
        a, b = ctypes.c_void_p(0x20000), ctypes.c_void_p(0x20000 + off)
        assert fwd(s0=a, s_last=b) == 1 and bwd(s0=a, ds0=b) == 1 and bwd(dsl=a, ds0=b) == 1
    # few heads and many steps: a workspace
    long, need = D(1, 1 << 16, 1, 64, 64), [L.soma_linear_attn_workspace_bytes(D(1, 1 << 16, 1, 64, 64), 1, k) for k in (0, 1)]
    assert 0 < need[0] < need[1]
    far = S(1 << 22, 64, 64)
    for ws, n in ((None, need[0]), (ODD, need[0]), (FAKE, need[0] - 1)):
        assert L.soma_linear_attn_forward(FAKE, far, FAKE, far, FAKE, far, 1, long, FAKE, 1.0, None, None,
                                          None, FAKE, far, None, ws, n, None) == 3
    assert L.soma_linear_attn_backward(FAKE, far, FAKE, far, FAKE, far, 1, long, FAKE, 1.0, None, None, None,
                                       FAKE, far, None, FAKE, far, FAKE, far, FAKE, far, None, FAKE,
                                       need[1] - 1, None) == 3
    # nothing to do is fine without pointers
    none = D(0, 3, 4, 8, 16)
    assert fwd(q=None, o=None, decay=None, d=none) == 0 and step(q=None, state=None, d=none) == 0
    assert bwd(do=None, dq=None, dv=None, d=D(2, 3, 0, 8, 16)) == 0


def test_dropout_refusals(soma):
    f = soma.lib().soma_dropout

    def call(x=FAKE, xs=8, r=None, rs=8, y=FAKE, ys=8, dtype=1, rows=4, cols=8, p=0.5, counter=None):
        return f(x, xs, r, rs, y, ys, dtype, rows, cols, p, 0, 0, counter, None)

    for bad in (dict(rows=-1), dict(cols=-1), dict(rows=1 << 32, cols=8, xs=8)):
        assert call(**bad) == 2
    for bad in (dict(dtype=3), dict(p=-0.1), dict(p=1.1), dict(p=NAN), dict(xs=7), dict(ys=7),
                dict(r=FAKE, rs=7), dict(x=ODD), dict(y=ODD), dict(r=ODD), dict(counter=ctypes.c_void_p(0x10004)),
                dict(x=None), dict(y=None)):
        assert call(**bad) == 1, bad
    assert call(rows=0, x=None, y=None) == 0 and call(cols=0, x=None, y=None) == 0


def test_sample_refusals(soma):
    f, C = soma.lib().soma_sample, soma.soma_sample_config

    def call(logits=FAKE, stride=10, dtype=0, rows=2, vocab=10, u=FAKE, tokens=FAKE, lp=None, **kw):
        cfg = C(**{**dict(temperature=1.0, top_p=1.0, min_p=0.0, top_k=0), **kw})
        return f(logits, stride, dtype, rows, vocab, cfg, u, tokens, lp, None)

    for bad in (dict(rows=-1), dict(rows=(1 << 24) + 1), dict(vocab=0), dict(vocab=(1 << 20) + 1)):
        assert call(**bad) == 2
    for bad in (dict(dtype=3), dict(stride=9), dict(logits=ODD), dict(u=ODD), dict(tokens=ctypes.c_void_p(0x10004)),
                dict(lp=ODD), dict(temperature=-1.0), dict(temperature=NAN), dict(top_p=NAN), dict(min_p=NAN),
                dict(temperatures=0x10001), dict(top_ps=0x10001), dict(min_ps=0x10001), dict(top_ks=0x10001),
                dict(logits=None), dict(u=None), dict(tokens=None)):
        assert call(**bad) == 1, bad
    assert call(rows=0, logits=None, u=None, tokens=None) == 0


def test_the_binding_refuses_what_it_can_see(soma):
    """Shapes, dtypes and places, before the library is asked."""
    q, g = torch.zeros(2, 3, 4, 8), torch.zeros(4)
    with pytest.raises(ValueError, match=r"q and v"):
        soma.linear_attn_forward(q[0], q, q, g, q)
    with pytest.raises(ValueError, match="unsupported dtype"):
        soma.linear_attn_forward(q.double(), q, q, g, q)
    with pytest.raises(ValueError, match="logits"):
        soma.sample(torch.zeros(4), torch.zeros(4), torch.zeros(4))
    with pytest.raises(ValueError, match="unsupported dtype"):
        soma.dropout(q.double(), q.double(), 0.5, 0)
    with pytest.raises(ValueError, match="one dimension"):
        soma.dropout(torch.tensor(1.0), torch.tensor(1.0), 0.5, 0)
    with pytest.raises(ValueError, match="workspace"):
        soma.linear_attn_alloc_workspace(1, 1, 1, 200, 8, torch.bfloat16)


def test_the_binding_refuses_another_device(soma, monkeypatch):
    class There:
        is_cuda = True

        def get_device(self):
            return 1

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ValueError, match="current device is cuda:0"):
        soma._here(q=There())
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    soma._here(q=There(), s0=None)
