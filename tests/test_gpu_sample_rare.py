"""Sampling's contract at its ends: tokens of the least weights.

The log probability is that of the logit, (l - max) / T - log(W 2^-40), good to fp32 (2^-23 of itself, and
2^-36 for what a sum of weights may be off), not the logarithm of the whole-number weight, which for a weight
of 1 may be off by log 2."""
import numpy as np
import pytest
import torch

from gpu_common import api

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("depth", [27.5, 28.0, 28.25, 26.875, 26.5])
@pytest.mark.parametrize("V", [40, 5000])
def test_the_log_probability_of_a_rare_token(depth, V, dtype):
    l = torch.full((1, V), float("-inf"), dtype=dtype, device="cuda")
    l[0, 3], l[0, V - 1] = -depth, 0.0
    x = float(l[0, 3])
    weight = np.rint(2.0 ** 40 * np.exp(x))
    assert 1 <= weight <= 4
    u = torch.zeros(1, device="cuda")
    token, lp = torch.empty(1, dtype=torch.int64, device="cuda"), torch.empty(1, device="cuda")
    api().sample(l, u, token, logprob=lp)
    assert token.item() == 3  # the first of any weight
    want = x - np.log1p(weight * 2.0 ** -40)
    assert abs(lp.item() - want) <= 2.0 ** -23 * abs(want) + 2.0 ** -36
    assert api().get_status() == 0


def test_a_weight_of_none_is_never_chosen():
    l = torch.full((1, 40), float("-inf"), device="cuda")
    l[0, 3], l[0, 39] = -28.5, 0.0
    token, lp = torch.empty(1, dtype=torch.int64, device="cuda"), torch.empty(1, device="cuda")
    api().sample(l, torch.zeros(1, device="cuda"), token, logprob=lp)
    assert token.item() == 39 and lp.item() == 0.0
