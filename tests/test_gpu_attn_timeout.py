"""A wait of linear attention's tensor-core kernels that runs out: the status says so, every copy that was
under way has landed before the kernel leaves its shared memory, no further one is made, and the context
stays usable.

Which phase of a place's barrier its last copy completes is index arithmetic: the last test restates it on
the CPU, copy by copy."""
import pytest
import torch

from gpu_common import api
from test_gpu_linear_attn import _case, _check, _run

SOMA_ERR_TIMEOUT = 5


@pytest.mark.gpu
def test_copies_land_and_the_context_survives():
    a = api()
    assert a.get_status() == 0
    src = torch.randn(5, 256, device="cuda")
    out = a.debug_attn_timeout(src, 2000)
    assert a.get_status() == SOMA_ERR_TIMEOUT and a.get_status() == 0
    assert torch.equal(out[:1024].view(4, 256), src[[0, 4, 2, 3]])
    assert out[1024:].tolist() == [1, 3, 1]  # the copy after the timeout was refused
    for dtype in ("bf16", "fp16"):
        for shape in ((2, 100, 2, 64, 64), (2, 300, 1, 128, 128)):
            s = _case(*shape, dtype)
            _check(s, _run(s))
    assert a.get_status() == 0


@pytest.mark.gpu
def test_refusals():
    a = api()
    src = torch.randn(1281, device="cuda")
    for bad in (lambda: a.debug_attn_timeout(src[1:], 2000),
                lambda: a.debug_attn_timeout(src[:1280], 0),
                lambda: a.debug_attn_timeout(src[:1280], (1 << 22) + 1)):
        with pytest.raises(a.SomaError):
            bad()


def test_the_phase_of_the_last_copy():
    """Wherever the loader breaks off, waiting for the parity of each place's last phase returns when that
    phase is over and not before; one copy at most is under way in a place, as it is copied into again only
    after the products have waited for the copy before."""
    for whole in range(20):          # chunks copied whole
        for part in range(3):        # and of the next one nothing, x, or x and y
            counts = {"x": whole + (part > 0), "y": whole + (part > 1), "z": whole}
            phases = {"x": counts["x"], "z": counts["z"]}
            for place in range(2):   # y's places take chunks in turn
                phases[f"y{place}"] = len([k for k in range(counts["y"]) if k % 2 == place])
                assert phases[f"y{place}"] == (counts["y"] + 1 - place) // 2
            for n in phases.values():
                if n:
                    landed, under_way, parity = n, n - 1, (n - 1) & 1
                    # a wait for a parity is over when the phase under way has the other one
                    assert (landed & 1) != parity and (under_way & 1) == parity
