"""Very small eps and moments that are zero (the rows of an embedding that were never used): the
step is 0 / eps = 0, never NaN.  The 8-bit form refuses an eps below fp32's normal numbers."""
import pytest
import torch

from gpu_common import api

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits,eps", [(32, 1e-40), (32, 1e-38), (8, 1.2e-38), (8, 1e-30)])
def test_zero_moments(bits, eps):
    a = api()
    p = [torch.randn(700, device="cuda")]
    was = p[0].clone()
    opt = a.AdamW(p, **a.AdamW.zero_state(p, bits))
    opt.step([torch.zeros(700, device="cuda")], t=1, lr=1e-2, eps=eps)
    assert a.get_status() == 0
    assert torch.equal(p[0], was)


def test_eight_bits_refuse_subnormal_eps():
    a = api()
    p = [torch.randn(700, device="cuda")]
    opt = a.AdamW(p, **a.AdamW.zero_state(p, 8))
    for eps in (1e-39, 1e-40, 1e-44):
        with pytest.raises(a.SomaError):
            opt.step([torch.zeros(700, device="cuda")], t=1, lr=1e-2, eps=eps)
