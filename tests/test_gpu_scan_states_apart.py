"""States that touch but do not overlap are accepted: neighbours in one allocation."""
import pytest
import torch

from gpu_common import api
from test_gpu_scan import _case, _near, _reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,T,D", [(3, 40, 64), (1, 6000, 8)])
def test_neighbours(B, T, D):
    m = api()
    s = _case(B, T, D, "fp32", seed=T)
    want = _reference(s)
    both, back = torch.empty(2, B, D, device="cuda"), torch.empty(2, B, D, device="cuda")
    both[0], back[1] = s["c0"], s["dcl"]
    a, h = s["a"].cuda(), torch.empty(B, T, D, device="cuda")
    marks, da = m.scan_alloc_checkpoints(B, T, D), torch.empty(B, T, 4, D, device="cuda")
    m.scan_forward(a, h, both[1], c0=both[0], checkpoints=marks)
    m.scan_backward(a, marks, s["dh"].cuda(), da, back[0], dc_last=back[1])
    _near(both[1], want["c"], want["cle"])
    _near(back[0], want["dc0"], want["dc0e"])
    with pytest.raises(m.SomaError):
        m.scan_forward(a, h, both[0], c0=both[0], checkpoints=marks)
    with pytest.raises(m.SomaError):
        m.scan_backward(a, marks, s["dh"].cuda(), da, back[1], dc_last=back[1])
