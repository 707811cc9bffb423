"""A wait of the recurrence's kernels that runs out: the status says so, the copy that was under way
has landed before the kernel leaves its shared memory, and the context stays usable.

Which phase of a stage's barrier its last copy completes is index arithmetic: the second test
restates it on the CPU, fill by fill."""
import pytest
import torch

from gpu_common import api
from test_gpu_scan import _case, _check, _run

SOMA_ERR_TIMEOUT = 5


@pytest.mark.gpu
def test_copies_land_and_the_context_survives():
    a = api()
    assert a.get_status() == 0
    src = torch.randn(1024, device="cuda")
    out = a.debug_scan_timeout(src, 2000)
    assert a.get_status() == SOMA_ERR_TIMEOUT and a.get_status() == 0
    assert torch.equal(out[:1024], src)
    assert out[1024] == 1  # the fill after the timeout was refused
    s = _case(2, 100, 64, "bf16")
    _check(s, _run(s))
    assert a.get_status() == 0


@pytest.mark.gpu
def test_refusals():
    a = api()
    src = torch.randn(1025, device="cuda")
    for bad in (lambda: a.debug_scan_timeout(src[1:], 2000),
                lambda: a.debug_scan_timeout(src[:1024], 0),
                lambda: a.debug_scan_timeout(src[:1024], (1 << 22) + 1)):
        with pytest.raises(a.SomaError):
            bad()


def test_the_phase_of_the_last_copy():
    """fills go round the ring from stage 0: stage i has had (fills + depth - 1 - i) // depth of
    them, and waiting for the parity of its last phase returns at once where the phase is over and
    never where another, still incomplete one has the other parity."""
    for depth in (2, 3, 4):
        for fills in range(40):
            had = [0] * depth
            for k in range(fills):
                had[k % depth] += 1
            for i in range(depth):
                n = (fills + depth - 1 - i) // depth
                assert n == had[i]
                if n:
                    landed, under_way = n, n - 1  # phases completed
                    parity = (n - 1) & 1
                    # a wait for a parity is over when the phase under way has the other one
                    assert (landed & 1) != parity and (under_way & 1) == parity
