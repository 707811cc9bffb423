"""Host logic of the attention expert: no GPU."""
import pytest
import torch


def test_heads_have_to_divide_the_width():
    from paper_2609_37899_gb300 import first_order
    e = first_order.AttentionExpert.__new__(first_order.AttentionExpert)
    e.batch, e.steps, e.dim, e.heads = 2, 3, 10, 4
    with pytest.raises(ValueError, match="no multiple"):
        e._mixer_buffers(None, "cpu")


def test_projections_are_split_into_heads():
    from paper_2609_37899_gb300 import first_order
    e = first_order.AttentionExpert.__new__(first_order.AttentionExpert)
    e.heads, e.width = 2, 3
    a = torch.arange(2 * 4 * 18.0).view(8, 18)
    q, k, v = e._heads(a, 2, 4)
    assert q.shape == (2, 4, 2, 3) and q.data_ptr() == a.data_ptr()
    assert torch.equal(k[1, 2, 1], a[6, 9:12]) and torch.equal(v[0, 0, 0], a[0, 12:15])
