"""A trace tells the first-order operators from the zero-order step, and from one another."""
import pytest
import torch

from gpu_common import api, run_step
from paper_2609_37899_gb300 import inputs

pytestmark = pytest.mark.gpu


def _first_order():
    m = api()
    h, emb = torch.randn(40, 64, device="cuda").bfloat16(), torch.randn(90, 64, device="cuda").bfloat16()
    y, dl = torch.randint(0, 90, (40,), device="cuda"), torch.ones(40, device="cuda")
    loss, lse = torch.empty(40, device="cuda"), torch.empty(40, device="cuda")
    ws = m.linear_ce_alloc_workspace(40, 90, 64, torch.bfloat16)
    m.linear_ce_forward(h, emb, y, loss, lse, ws)
    m.linear_ce_backward(h, emb, y, lse, dl, torch.empty_like(h), torch.empty_like(emb), ws)
    a, out = torch.randn(2, 9, 4, 64, device="cuda"), torch.empty(2, 9, 64, device="cuda")
    marks = m.scan_alloc_checkpoints(2, 9, 64)
    m.scan_forward(a, out, checkpoints=marks)
    m.scan_backward(a, marks, out, torch.empty_like(a))
    m.scan_step(a[:, 0], torch.zeros(2, 64, device="cuda"), out[:, 0])
    p = [torch.randn(100, device="cuda") for _ in range(400)]
    m.AdamW(p, **m.AdamW.zero_state(p)).step([torch.ones_like(x) for x in p], t=1, lr=1e-3)


def test_classes():
    m = api()
    c = inputs.CONFIGS["tiny"]

    def spsa():
        run_step(inputs.config_params("tiny"), inputs.config_batch("tiny"), c["E"], c["H"],
                 c["n_pert"], c["eps"], c["lr"], 0, 0)

    m.trace_enable(True)
    try:
        m.trace_read(reset=True), m.trace_read_first_order(reset=True)
        _first_order()
        assert all(n == 0 for _, n in m.trace_read(reset=True).values())
        first = m.trace_read_first_order(reset=True)
        # two calls, three calls, and two launches for 400 tensors
        assert {k: n for k, (_, n) in first.items()} == {"linear_ce": 2, "scan": 3, "adamw": 2}
        assert all(ms > 0 for ms, _ in first.values())
        spsa()
        assert all(n == 0 for _, n in m.trace_read_first_order(reset=True).values())
        alone = {k: n for k, (_, n) in m.trace_read(reset=True).items()}
        _first_order()
        spsa()
        assert {k: n for k, (_, n) in m.trace_read(reset=True).items()} == alone
        # reading one set leaves the other's records
        assert m.trace_read_first_order(reset=False)["scan"][1] == 3
        assert m.trace_read_first_order(reset=True)["scan"][1] == 3
        assert m.trace_read_first_order(reset=True)["scan"][1] == 0
    finally:
        m.trace_enable(False)
        m.trace_read(reset=True), m.trace_read_first_order(reset=True)
