"""What an expert keeps: a forward call's y stays when the next one has run, x and the gates' gradient
have the sequences' shape, and without dropout there is no buffer for it."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _expert(kind, **kw):
    from paper_2609_37899_gb300 import first_order
    if kind == "scan":
        return first_order.ScanExpert(256, 64, 2, 30, seed=4, **kw)
    return first_order.AttentionExpert(256, 64, 2, 30, seed=4, heads=2, **kw)


@pytest.mark.parametrize("dropout", [0.0, 0.25])
@pytest.mark.parametrize("kind", ["scan", "attention"])
def test_outputs_of_two_forward_calls(kind, dropout):
    e = _expert(kind, dropout=dropout)
    g = torch.Generator(device="cuda").manual_seed(2)
    tokens = torch.randint(0, 256, (2, 2, 31), generator=g, device="cuda")
    e.forward(tokens[0])
    first, kept = e.y, e.y.clone()
    e.forward(tokens[1])
    assert torch.equal(first, kept) and not torch.equal(e.y, kept)
    assert e.x.shape == (2, 30, 64) and e.y.shape == (60, 64)
    assert torch.equal(e.x, e.emb[tokens[1][:, :-1]])


def test_the_scan_experts_gradients_of_its_gates():
    e = _expert("scan")
    tokens = torch.randint(0, 256, (2, 31), device="cuda")
    e.forward(tokens)
    e.backward(torch.ones(60, device="cuda"))
    assert e.dgates.shape == (2, 30, 4, 64) and e.dgates.any()
    dw = e.dgates.view(-1, 256).T @ e.x.reshape(-1, 64)
    assert torch.equal(dw, e.dw)


@pytest.mark.parametrize("kind", ["scan", "attention"])
def test_memory_without_dropout(kind):
    """A step without dropout holds no gradient of the dropped branch; one that is given dropout later does."""
    def bytes_of(e):
        return sum(x.numel() * x.element_size() for x in vars(e).values() if torch.is_tensor(x))

    e = _expert(kind)
    tokens = torch.randint(0, 256, (2, 31), device="cuda")
    e.forward(tokens)
    e.backward(torch.ones(60, device="cuda"))
    assert not hasattr(e, "dh") or e.dh is None
    before = bytes_of(e)
    e.dropout = 0.5
    e.forward(tokens)
    e.backward(torch.ones(60, device="cuda"))
    assert bytes_of(e) == before + 60 * 64 * 2
    e.dropout = 0.0
    e.forward(tokens)
    e.backward(torch.ones(60, device="cuda"))
    assert torch.isfinite(e.demb.float()).all()


@pytest.mark.parametrize("dropout", [0.0, 0.25])
def test_tokens_of_any_layout(dropout):
    g = torch.Generator(device="cuda").manual_seed(3)
    across = torch.randint(0, 256, (31, 2), generator=g, device="cuda").T
    losses = []
    for tokens in (across, across.contiguous()):
        e = _expert("scan", dropout=dropout)
        losses.append(e.forward(tokens).clone())
        e.backward(torch.ones(60, device="cuda"))
    assert torch.equal(*losses)
