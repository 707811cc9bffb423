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
    assert L.soma_scan_checkpoint_count(ok) == 16
    assert L.soma_scan_checkpoint_count(dims(2, 17, 8)) == 32
    for bad in (dims(-1, 3, 8), dims(2, -3, 8), dims(2, 3, -8), dims(1 << 31, 3, 8),
                dims(2, 1 << 31, 8), dims(2, 3, (1 << 24) + 1), dims(1 << 30, 1, 1 << 20)):
        assert L.soma_scan_checkpoint_count(bad) == -1
        assert L.soma_scan_forward(FAKE, s, 0, bad, None, None, None, FAKE, s, None, None, None) == 2
        assert L.soma_scan_backward(FAKE, s, 0, bad, FAKE, None, None, FAKE, s, None, FAKE, s, None,
                                    None) == 2
    assert L.soma_scan_step(FAKE, s, 0, -1, 8, FAKE, FAKE, s, None) == 2
    assert L.soma_scan_forward(FAKE, s, 3, ok, None, None, None, FAKE, s, None, None, None) == 1
    assert L.soma_scan_forward(FAKE, st(-96, 32, 8), 0, ok, None, None, None, FAKE, s, None, None,
                               None) == 1
    assert L.soma_scan_forward(None, s, 0, ok, None, None, None, FAKE, s, None, None, None) == 1
    assert L.soma_scan_forward(FAKE, s, 0, ok, None, None, None, None, s, None, None, None) == 1
    assert L.soma_scan_forward(odd, s, 1, ok, None, None, None, FAKE, s, None, None, None) == 1
    assert L.soma_scan_forward(FAKE, s, 0, ok, odd, None, None, FAKE, s, None, None, None) == 1
    assert L.soma_scan_forward(FAKE, s, 0, ok, None, odd, None, FAKE, s, None, None, None) == 1
    assert L.soma_scan_backward(FAKE, s, 0, ok, None, None, None, FAKE, s, None, FAKE, s, None,
                                None) == 1
    assert L.soma_scan_backward(FAKE, s, 0, ok, FAKE, None, None, FAKE, s, None, None, s, None,
                                None) == 1
    assert L.soma_scan_step(FAKE, s, 0, 2, 8, None, FAKE, s, None) == 1
    assert L.soma_scan_step(FAKE, s, 7, 2, 8, FAKE, FAKE, s, None) == 1
    # nothing to do is fine without pointers
    assert L.soma_scan_forward(None, s, 0, dims(0, 3, 8), None, None, None, None, s, None, None,
                               None) == 0


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
