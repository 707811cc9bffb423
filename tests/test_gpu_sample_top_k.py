"""Sampling with a top_k that is no number of 32 bits."""
import pytest
import torch

from gpu_common import api

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("k", [2 ** 31, 2 ** 32 + 1, 2 ** 40, -2 ** 31 - 1, -2 ** 32 + 1, 2 ** 31 - 1])
def test_a_top_k_past_32_bits(k):
    """More than the vocabulary, or less than one, is all of it."""
    g = torch.Generator(device="cuda").manual_seed(1)
    l = torch.randn(50, 300, generator=g, device="cuda")
    u = torch.rand(50, generator=g, device="cuda")
    a, b = (torch.empty(50, dtype=torch.int64, device="cuda") for _ in range(2))
    api().sample(l, u, a)
    api().sample(l, u, b, top_k=k)
    assert torch.equal(a, b)
