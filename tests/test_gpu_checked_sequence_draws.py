"""The checked build on linear attention, dropout and sampling over drawn sizes, lengths, strides and
settings: no index check fails, and the results are the default build's.

Both builds do the same operations in the same order; at most a contraction here and there differs.  So whole
numbers are equal, 16-bit results a rounding apart (2^-7 relative), and fp32 ones the fp32 errors of their sums
of up to 128 + 128 + 6000 + 64 terms apart, each 2^-24 of the largest value's size."""
import random

import pytest
import torch

from test_gpu_checked import _default_path, checked_path, using  # noqa: F401
from test_gpu_checked_sequence import _attn, _dropout, _sample

pytestmark = pytest.mark.gpu
SUMS = (128 + 128 + 6000 + 64) * 2.0 ** -24
TYPES = (torch.float32, torch.bfloat16, torch.float16)


def _draw(op, seed):
    rng = random.Random(seed)
    dtype = rng.choice(TYPES)
    log = lambda lo, hi: int(lo * (hi / lo) ** rng.random())
    if op == "attn":
        widths = [rng.choice((1, 7, 8, 24, 33, 64, 65, 72, 100, 120, 128)) for _ in range(2)]
        return _attn(log(1, 5), log(1, 6000), rng.randint(1, 4), *widths, dtype, ragged=rng.random() < 0.6)
    if op == "dropout":
        return _dropout(log(1, 3000), log(1, 900), dtype, pad=rng.choice((0, 0, 1, 8)))
    kw = {}
    if rng.random() < 0.6:
        kw["top_k"] = log(1, 9000)
    if rng.random() < 0.6:
        kw["top_p"] = rng.choice((0.1, 0.9, 0.999, 1.0))
    if rng.random() < 0.3:
        kw["min_p"] = 0.01
    kw["temperature"] = rng.choice((0.0, 0.3, 1.0, 3.0, 30.0))
    return _sample(log(1, 20), log(1, 300000), dtype, **kw)


@pytest.mark.parametrize("seed", range(14))
@pytest.mark.parametrize("op", ["attn", "dropout", "sample"])
def test_no_check_fails_and_results_agree(checked_path, op, seed):  # noqa: F811
    run = _draw(op, seed)
    with using(_default_path()) as a:
        want = run(a)
        assert a.get_status() == 0
    with using(checked_path) as a:
        got = run(a)
        status, line = a.get_status(), a.lib().soma_debug_check_line(None)
        assert (status, line) == (0, 0), (a.STATUS_NAMES.get(status, status), line)
    for k in want:
        x, y = (v[k].double() for v in (got, want))
        size = y.abs().amax() if y.numel() else 0.0
        rtol = {torch.float32: 0.0, torch.int64: 0.0}.get(want[k].dtype, 2.0 ** -7)
        atol = 0.0 if want[k].dtype == torch.int64 else SUMS * size
        assert ((x - y).abs() <= rtol * y.abs() + atol).all(), k
