"""Host-side checks of the first-order entry points: no launch is made."""
import ctypes

import pytest

FAKE = ctypes.c_void_p(0x10000)  # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def soma():
    from paper_2609_37899_gb300 import build
    build.build()
    from paper_2609_37899_gb300 import api
    return api


def _row(soma, **kw):
    at = {k: 0x10000 for k in ("param", "grad", "m", "v")}
    return (soma.soma_adamw_tensor * 1)(soma.soma_adamw_tensor(**{**at, "count": 10, **kw}))


def test_adamw_refusals(soma):
    f = soma.lib().soma_adamw_step

    def cfg(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, t=1, param=0, grad=0, bits=32):
        return soma.soma_adamw_config(lr, beta1, beta2, eps, 0, t, param, grad, bits)

    bad_cfg = [cfg(lr=float("inf")), cfg(beta1=1.0), cfg(beta1=-0.1), cfg(beta2=float("nan")),
               cfg(eps=0.0), cfg(eps=1e-60), cfg(eps=float("inf")), cfg(t=0), cfg(param=3),
               cfg(grad=-1), cfg(bits=16)]
    for c in bad_cfg:
        assert f(_row(soma), 1, c, None, None) == 1
    bad_row = [dict(param=None), dict(grad=None), dict(m=None), dict(v=None), dict(count=-1),
               dict(count=(1 << 40) + 1), dict(weight_decay=-1.0), dict(param=0x10002),
               dict(weight_decay=float("nan")), dict(m_scale=0x10000), dict(master=0x10000),
               dict(v=0x10001)]
    for r in bad_row:
        assert f(_row(soma, **r), 1, cfg(), None, None) == 1
    assert f(_row(soma), 1, cfg(bits=8), None, None) == 1  # 8 bits without scales
    assert f(_row(soma), -1, cfg(), None, None) == 1
    assert f(None, 1, cfg(), None, None) == 1
    assert f(_row(soma), 1, cfg(), ctypes.c_void_p(0x10002), None) == 1
    rows = (soma.soma_adamw_tensor * 2)(_row(soma, master=0x10000)[0], _row(soma)[0])
    assert f(rows, 2, cfg(param=1), None, None) == 1  # a master for one of two tensors


def test_scan_refusals(soma):
    L, dims, st = soma.lib(), soma.soma_scan_dims, soma.soma_scan_strides
    ok, s, odd = dims(2, 3, 8), st(96, 32, 8), ctypes.c_void_p(0x10001)

    def fwd(gates=FAKE, gs=s, dtype=0, d=ok, c0=None, lengths=None, h=FAKE, ws=None, n=0):
        return L.soma_scan_forward(gates, gs, dtype, d, c0, lengths, None, h, s, None, None, ws, n,
                                   None)

    def bwd(marks=FAKE, d=ok, dgates=FAKE, ws=None, n=0):
        return L.soma_scan_backward(FAKE, s, 0, d, marks, None, None, FAKE, s, None, dgates, s,
                                    None, ws, n, None)

    assert L.soma_scan_checkpoint_count(ok) == 8 * 2
    assert L.soma_scan_checkpoint_count(dims(2, 17, 8)) == 8 * 2 * 3
    assert L.soma_scan_workspace_bytes(ok) == 0
    for bad in (dims(-1, 3, 8), dims(2, -3, 8), dims(2, 3, -8), dims(1 << 31, 3, 8),
                dims(2, 1 << 31, 8), dims(2, 3, (1 << 24) + 1), dims(1 << 30, 1, 1 << 20)):
        assert L.soma_scan_checkpoint_count(bad) == -1
        assert L.soma_scan_workspace_bytes(bad) == -1
        assert fwd(d=bad) == 2 and bwd(d=bad) == 2
    assert L.soma_scan_step(FAKE, s, 0, -1, 8, FAKE, FAKE, s, None) == 2
    assert fwd(dtype=3) == 1
    assert fwd(gs=st(-96, 32, 8)) == 1
    assert fwd(gates=None) == 1
    assert fwd(h=None) == 1
    assert fwd(gates=odd, dtype=1) == 1
    assert fwd(c0=odd) == 1
    assert fwd(lengths=odd) == 1
    assert bwd(marks=None) == 1
    assert bwd(dgates=None) == 1
    assert L.soma_scan_step(FAKE, s, 0, 2, 8, None, FAKE, s, None) == 1
    assert L.soma_scan_step(FAKE, s, 7, 2, 8, FAKE, FAKE, s, None) == 1
    # nothing to do is fine without pointers
    assert fwd(gates=None, d=dims(0, 3, 8), h=None) == 0
    # few channels, many steps: a workspace
    long = dims(1, 1 << 16, 64)
    need = L.soma_scan_workspace_bytes(long)
    assert need > 0
    assert fwd(d=long) == 3 and bwd(d=long) == 3
    assert fwd(d=long, ws=odd, n=need) == 3 and bwd(d=long, ws=FAKE, n=7) == 3


def test_linear_ce_refusals(soma):
    L, D = soma.lib(), soma.soma_linear_ce_dims
    ok, odd = D(20, 30, 16, 16, 16, 1), ctypes.c_void_p(0x10008)
    big = 1 << 40
    fw, bw = L.soma_linear_ce_workspace_bytes(ok, 0), L.soma_linear_ce_workspace_bytes(ok, 1)
    assert fw > 0 and bw > 0
    for bad in (D(-1, 30, 16, 16, 16, 1), D(20, 0, 16, 16, 16, 1), D(20, 30, 0, 16, 16, 1),
                D(20, 30, 16, 15, 16, 1), D(20, 30, 16, 16, 15, 1), D(20, 30, 16, 16, 16, 0),
                D(20, 30, 16, 16, 16, 3), D((1 << 30) + 1, 30, 16, 16, 16, 1),
                D(20, (1 << 30) + 1, 16, 16, 16, 1), D(20, 30, 65537, 65537, 65537, 1)):
        assert L.soma_linear_ce_workspace_bytes(bad, 0) == 0
        assert L.soma_linear_ce_workspace_bytes(bad, 1) == 0
        assert L.soma_linear_ce_forward(FAKE, FAKE, bad, FAKE, -1, FAKE, FAKE, FAKE, big, None) == 2
        assert L.soma_linear_ce_backward(FAKE, FAKE, bad, FAKE, -1, FAKE, FAKE, FAKE, 16, FAKE, 16,
                                         FAKE, big, None) == 2
    for k in range(5):  # h, emb, targets, loss, lse missing
        p = [None if j == k else FAKE for j in range(5)]
        assert L.soma_linear_ce_forward(p[0], p[1], ok, p[2], -1, p[3], p[4], FAKE, big, None) == 1
    assert L.soma_linear_ce_forward(odd, FAKE, ok, FAKE, -1, FAKE, FAKE, FAKE, big, None) == 1
    assert L.soma_linear_ce_forward(FAKE, odd, ok, FAKE, -1, FAKE, FAKE, FAKE, big, None) == 1
    assert L.soma_linear_ce_forward(FAKE, FAKE, ok, FAKE, -1, FAKE, FAKE, None, big, None) == 3
    assert L.soma_linear_ce_forward(FAKE, FAKE, ok, FAKE, -1, FAKE, FAKE, FAKE, fw - 1, None) == 3
    assert L.soma_linear_ce_forward(None, FAKE, D(0, 30, 16, 16, 16, 1), None, -1, None, None, None,
                                    0, None) == 0
    for k in range(7):  # h, emb, targets, lse, dloss, dh, demb missing
        p = [None if j == k else FAKE for j in range(7)]
        assert L.soma_linear_ce_backward(p[0], p[1], ok, p[2], -1, p[3], p[4], p[5], 16, p[6], 16,
                                         FAKE, big, None) == 1
    assert L.soma_linear_ce_backward(FAKE, FAKE, ok, FAKE, -1, FAKE, FAKE, FAKE, 15, FAKE, 16, FAKE,
                                     big, None) == 1
    assert L.soma_linear_ce_backward(FAKE, FAKE, ok, FAKE, -1, FAKE, FAKE, FAKE, 16, FAKE, 15, FAKE,
                                     big, None) == 1
    assert L.soma_linear_ce_backward(FAKE, FAKE, ok, FAKE, -1, FAKE, FAKE, FAKE, 16, FAKE, 16, FAKE,
                                     bw - 1, None) == 3
