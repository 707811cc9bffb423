"""Host-side limits of the first-order entry points: no launch is made."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def soma():
    from paper_2609_37899_gb300 import build
    build.build()
    from paper_2609_37899_gb300 import api
    return api


@pytest.mark.parametrize("eps", [1e-39, 1e-40, 1.4e-45, 1.17e-38])
def test_eight_bit_eps_is_a_normal_number(soma, eps):
    row = (soma.soma_adamw_tensor * 1)(soma.soma_adamw_tensor(
        **{k: 0x10000 for k in ("param", "grad", "m", "v", "m_scale", "v_scale")}, count=10))
    cfg = soma.soma_adamw_config(1e-3, 0.9, 0.999, eps, 0, 1, 0, 0, 8)
    assert soma.lib().soma_adamw_step(row, 1, cfg, None, None) == 1


def test_structures_have_the_sizes_of_the_abi(soma):
    """Seven pointers, a 64-bit count and a double; four doubles, a 64-bit seed, four 32-bit
    words; and so on."""
    for name, size in (("soma_adamw_tensor", 72), ("soma_adamw_config", 56),
                       ("soma_scan_dims", 24), ("soma_scan_strides", 24),
                       ("soma_linear_ce_dims", 48)):
        assert ctypes.sizeof(getattr(soma, name)) == size


def test_states_of_the_recurrence_must_not_overlap(soma):
    """c_last in the place of c0 (or of a part of it) would hold what the sizes make of it: some are cut
    into chunks that still read c0 when the last one is done.  The same of dc0 and dc_last."""
    L, st = soma.lib(), soma.soma_scan_strides(96, 32, 8)
    fake, at = ctypes.c_void_p(0x10000), lambda n: ctypes.c_void_p(0x20000 + 4 * n)
    for dims, far in (((2, 3, 8), 16), ((1, 1 << 16, 64), 64)):
        d = soma.soma_scan_dims(*dims)
        for off in (0, 1, far - 1, 1 - far):
            assert L.soma_scan_forward(fake, st, 0, d, at(0), None, None, fake, st, at(off), None,
                                       fake, 1 << 40, None) == 1
            assert L.soma_scan_backward(fake, st, 0, d, fake, None, None, fake, st, at(0), fake, st,
                                        at(off), fake, 1 << 40, None) == 1
