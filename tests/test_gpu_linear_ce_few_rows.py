"""Linear cross entropy with few rows, where the roundings of G do not average out in demb.

A row of demb is then a few entries of G times a few states, often a single one.  demb has to be
about as good as its rounding to 16 bits: its error's norm may exceed the rounding's own by a
twentieth (G's two halves leave 2^-16 of it in bf16, 2^-22 in fp16), plus 1e-5 of demb (G's
entries in fp32: exponents of logits up to about 16, 16 roundings of 2^-24 each, and sums)."""
import pytest
import torch

from gpu_common import api
from test_gpu_linear_ce import _case, _check, _reference, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("N,V,d,ignored", [
    (1, 500, 64, 0.0), (3, 4000, 72, 0.0), (15, 3000, 100, 0.0), (55, 2000, 65, 0.2),
    (128, 5000, 128, 0.1), (127, 257, 40, 0.0)])
def test_rounding_of_demb(N, V, d, ignored, dtype):
    s = _case(N, V, d, dtype, seed=N + d, ignored=ignored)
    # one gradient for all rows: what its entries at the targets are off by goes one way
    s["dloss"] = torch.where(s["dloss"].isnan(), s["dloss"], torch.full_like(s["dloss"], 1 / 3))
    got = _run(s)
    _check(s, got)
    want = _reference(s)[0]["demb"]
    rounding = (want.to(got["demb"].dtype).double() - want).norm().item()
    off = (got["demb"].double() - want).norm().item()
    assert off <= 1.05 * rounding + 1e-5 * want.norm().item()
    assert api().get_status() == 0


def test_several_pieces():
    """So large a vocabulary that both halves of G take several pieces."""
    s = _case(100, 700001, 24, "bf16", seed=4, ignored=0.1)
    _check(s, _run(s))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("N,V,d", [(200, 20000, 64), (625, 30000, 72), (1000, 20000, 65)])
def test_one_gradient_for_all_rows(N, V, d, dtype):
    """With one dloss for all rows, G's entries at the targets are just below a power of two and
    off by at most half of what rounding can cost, evenly: hu / 2 / sqrt(3) = 0.29 hu.  demb's own
    rounding is off by hu / sqrt(3) times 0.72, the mean over the values' mantissas: 0.42 hu.
    Together 1.22 times the latter (for entries all off by the same up to hu: 2.6); 1.4 is allowed."""
    s = _case(N, V, d, dtype, seed=N, spread=0.5)
    s["dloss"] = torch.full_like(s["dloss"], 1 / 3)
    got = _run(s)
    _check(s, got)
    want = _reference(s)[0]["demb"]
    rounding = (want.to(got["demb"].dtype).double() - want).norm().item()
    off = (got["demb"].double() - want).norm().item()
    assert off <= 1.4 * rounding + 1e-5 * want.norm().item()
