"""A shape outside the limits is refused as a shape by the calls that pack the stash, whatever the tensors beside it are."""
import pytest

import paper_2604_19241_amd as moe
from paper_2604_19241_amd import binding as b
from test_more_operators_host import I8, I32, U8, gpu


@pytest.mark.parametrize("kw", [dict(I=96), dict(T=-1), dict(k=17), dict(k=9), dict(T=1 << 28, k=4), dict(e_count=9), dict(T=1 << 27, k=16, E=16, I=1 << 30)])
def test_shapes_outside_the_limits(kw):
    call = b._load_call()
    args = dict(T=8, d=64, E=8, k=2, I=64, e_start=0, e_count=8) | kw
    shape = moe.make_shape(**args)
    n = moe.alloc_saved(moe.make_shape(8, 64, 8, 2, 64), "cpu").numel()
    tensors = gpu(I32, args["e_count"] + 1), gpu(U8, n), gpu(I8, 16, 128), gpu(U8, 16, 4)
    for function in (call.saved_pack, call.saved_unpack):
        assert function(b._addressof(shape), *tensors, 0) == b.MOE_ERR_SHAPE, function.__name__
