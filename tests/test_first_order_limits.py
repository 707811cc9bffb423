"""Host-side limits of the first-order entry points: no launch is made."""
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
