"""Linear attention where a dimension has one element: the stride along it says nothing, so the call takes
the kernels, and gives the bits, that it has with any other stride."""
import pytest
import torch

from gpu_common import api
from test_gpu_linear_attn import DT, _case, _check

pytestmark = pytest.mark.gpu


def _run(s, tensors, outs):
    m = api()
    kw = dict(s0=s["s0"], scale=s["scale"])
    m.linear_attn_forward(tensors["q"], tensors["k"], tensors["v"], s["g"], outs["o"], **kw)
    m.linear_attn_backward(tensors["q"], tensors["k"], tensors["v"], s["g"], tensors["do"], outs["dq"],
                           outs["dk"], outs["dv"], ds_last=s["dsl"], **kw)
    return outs


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("shape,dim", [((1, 200, 3, 32, 32), 0), ((2, 1, 3, 32, 32), 1), ((2, 200, 1, 32, 32), 2),
                                       ((1, 130, 1, 128, 64), 0)])
@pytest.mark.parametrize("which", ["inputs", "outputs"])
def test_its_stride_is_any(shape, dim, dtype, which):
    s = _case(*shape, dtype, seed=sum(shape) + dim)
    dense = {n: s[n] for n in ("q", "k", "v", "do")}
    new = lambda: {n: torch.full_like(s[r], float("nan")) for n, r in
                   (("o", "v"), ("dq", "q"), ("dk", "k"), ("dv", "v"))}

    def odd(x):  # the same elements, an odd stride along `dim`
        strides = list(x.stride())
        strides[dim] = strides[dim] + 1 if dim == 0 else 4097
        return x.as_strided(x.shape, strides)

    want = _run(s, dense, new())
    _check(s, want, ("o", "dq", "dk", "dv"))
    if which == "inputs":
        got = _run(s, {n: odd(x) for n, x in dense.items()}, new())
    else:
        got = _run(s, dense, {n: odd(x) for n, x in new().items()})
    assert all(x.dtype == DT[dtype] for x in got.values())
    for n in want:
        assert torch.equal(got[n], want[n]), n
    assert api().get_status() == 0
