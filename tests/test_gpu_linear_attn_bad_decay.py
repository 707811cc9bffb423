"""A head whose log decay is above 0 or NaN (soma_linear_attn_*): everything that its steps reach is NaN,
whether a decay enters that place or not, in each of the kernels; other heads are as they were."""
import pytest
import torch

from gpu_common import api
from test_gpu_linear_attn import HALF, _case, _reference, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("shape", [(3, 150, 2, 32, 32), (2, 300, 2, 128, 72), (3, 70, 2, 33, 20),
                                   (2, 1, 2, 16, 16), (2, 6000, 2, 16, 16)])
@pytest.mark.parametrize("ragged,resets", [(False, False), (True, False), (False, True), (True, True)])
@pytest.mark.parametrize("bad", [0.5, float("nan")])
def test_all_that_its_steps_reach_is_nan(shape, dtype, ragged, resets, bad):
    B, T = shape[:2]
    s = _case(*shape, dtype, seed=sum(shape), ragged=ragged, resets=resets, decay=-0.1)
    s["g"][1] = bad
    out = _run(s)
    assert api().get_status() == 6
    for b in range(B):
        n = T if s["lengths"] is None else int(s["lengths"][b])
        for name in ("o", "dq", "dk", "dv"):
            assert out[name][b, :n, 1].isnan().all(), (name, b)
            assert (out[name][b, n:, 1] == 0).all(), (name, b)
        if n == 0:
            assert torch.equal(out["s_last"][b, 1], s["s0"][b, 1])
            assert torch.equal(out["ds0"][b, 1], s["dsl"][b, 1])
            continue
        assert out["s_last"][b, 1].isnan().all(), b
        if s["resets"] is not None and s["resets"][b, 0]:
            assert (out["ds0"][b, 1] == 0).all()  # no step sees s0
        else:
            assert out["ds0"][b, 1].isnan().all(), b
    if T > 1000:
        return
    ref = _reference({**s, "g": torch.full_like(s["g"], -0.1)})
    bound = 1e-5 if dtype == "fp32" else 2 * HALF[dtype]
    for name in ("o", "dq", "dk", "dv"):
        err = (out[name][:, :, 0].double() - ref[name][:, :, 0]).norm()
        assert err <= bound * ref[name][:, :, 0].norm(), name


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_one_token(dtype):
    s = _case(3, 1, 2, 32, 48, dtype, seed=2, decay=-0.1)
    s["g"][1] = float("nan")
    state, o = s["s0"].clone(), torch.zeros(3, 2, 48, dtype=s["v"].dtype, device="cuda")
    api().linear_attn_step(s["q"][:, 0], s["k"][:, 0], s["v"][:, 0], s["g"], state, o, scale=s["scale"])
    assert api().get_status() == 6
    assert o[:, 1].isnan().all() and state[:, 1].isnan().all()
    assert o[:, 0].isfinite().all() and state[:, 0].isfinite().all()


def test_a_decay_of_none_or_all_is_not_one():
    for decay in (0.0, -0.0, float("-inf")):
        s = _case(2, 140, 2, 32, 32, "bf16", seed=3, decay=decay)
        assert all(x.isfinite().all() for x in _run(s).values())
    assert api().get_status() == 0
