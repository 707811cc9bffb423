"""The workspace of linear attention's calls: one that is made for a batch serves every smaller one, which
may be cut into more segments and need more."""
import random

import pytest
import torch


@pytest.fixture(scope="module")
def soma():
    from paper_2609_37899_gb300 import build
    build.build()
    from paper_2609_37899_gb300 import api
    return api


def _own(soma, batch, steps, heads, dk, dv, dtype, backward):
    return soma.lib().soma_linear_attn_workspace_bytes(soma.soma_attn_dims(batch, steps, heads, dk, dv),
                                                       soma.DTYPES[dtype], int(backward))


SIZES = [(16, 4096, 8, 128, 128, torch.bfloat16), (300, 32768, 1, 64, 64, torch.float16),
         (200, 2048, 8, 128, 128, torch.float32), (40, 777, 7, 33, 65, torch.float32),
         (1, 32768, 8, 128, 128, torch.bfloat16), (70, 5000, 3, 40, 72, torch.bfloat16)]


@pytest.mark.parametrize("batch,steps,heads,dk,dv,dtype", SIZES)
def test_it_serves_every_smaller_batch(soma, batch, steps, heads, dk, dv, dtype):
    n = soma.linear_attn_workspace_bytes(batch, steps, heads, dk, dv, dtype)
    own = [_own(soma, b, steps, heads, dk, dv, dtype, k) for b in range(batch + 1) for k in (0, 1)]
    assert n == max(own)  # and no larger than it has to be
    forward = soma.linear_attn_workspace_bytes(batch, steps, heads, dk, dv, dtype, backward=False)
    assert forward == max(own[::2])
    assert soma.linear_attn_alloc_workspace(batch, steps, heads, dk, dv, dtype, device="cpu").numel() == n


def test_many_sequences_are_not_cut(soma):
    """What it rests on: from three rounds of CTAs on (the widest 152, two for narrow ones, up to 20 in
    fp32) a call needs none."""
    rng = random.Random(3)
    for _ in range(300):
        dk, dv, heads = rng.randint(1, 128), rng.randint(1, 128), rng.choice((1, 2, 7, 16))
        dtype = rng.choice((torch.float32, torch.bfloat16, torch.float16))
        steps = int(2 ** rng.uniform(0, 24))
        batch = 3 * 152 * 20 // heads + rng.randint(1, 50000)
        for k in (0, 1):
            assert _own(soma, batch, steps, heads, dk, dv, dtype, k) == 0


def test_larger_batches_ask_for_no_less(soma):
    rng = random.Random(4)
    for _ in range(30):
        dk, dv = rng.randint(1, 16) * 8, rng.randint(1, 16) * 8
        steps, heads = rng.randint(1, 9000), rng.randint(1, 9)
        sizes = [soma.linear_attn_workspace_bytes(b, steps, heads, dk, dv, torch.bfloat16)
                 for b in (0, 1, 2, 5, 16, 64, 1000)]
        assert sizes[0] == 0 and sizes == sorted(sizes)


def test_invalid_sizes(soma):
    f, D = soma.lib().soma_linear_attn_workspace_bytes_upto, soma.soma_attn_dims
    assert f(D(1, 1, 1, 129, 8), 1, 0) == -1 and f(D(1, 1, 1, 8, 8), 3, 0) == -1
    assert f(D(1, 1, 1, 8, 8), 1, 2) == -1 and f(D(0, 5, 0, 8, 8), 1, 1) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_one_workspace_for_all_batches(dtype):
    from gpu_common import api
    from test_gpu_linear_attn import DT, _case, _check, _run
    a = api()
    ws = a.linear_attn_alloc_workspace(40, 3000, 8, 128, 128, DT[dtype])
    for batch in (40, 12, 2, 1):
        s = _case(batch, 3000, 8, 128, 128, dtype, seed=batch, decay=-0.05)
        out = _run(s, workspace=ws)
        if batch == 1:
            _check(s, out)
        assert all(x.isfinite().all() for x in out.values())
    assert a.get_status() == 0
