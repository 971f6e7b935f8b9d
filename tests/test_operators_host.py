"""What the projection with adapters and the balance loss refuse, before anything reaches a device."""
import ctypes

import pytest
import torch

import paper_2604_19241_amd as moe
from paper_2604_19241_amd import binding as b

FAKE = 0x1000


@pytest.fixture(scope="module")
def lib():
    if not b.LIB_PATH.exists():
        from paper_2604_19241_amd import build
        build.build()
    return b.load_library()


def test_struct_sizes():
    assert ctypes.sizeof(b.MoEAdapterShape) == 20 and ctypes.sizeof(b.MoEBalanceShape) == 24 and ctypes.sizeof(b.MoEBalanceStatsC) == 40


GOOD = dict(T=600, K=64, N=128, rank=16, adapters=4)


def adapter_calls(lib, s, **kw):
    """Return codes of plan, forward and backward."""
    a = dict(ids=FAKE, plan=FAKE, pbytes=1 << 30, x=FAKE, ldx=s.K, w=FAKE, a=FAKE, b=FAKE, scale=None, y=FAKE, f32=0, h=FAKE, ws=FAKE, nbytes=1 << 40,
             dy=FAKE, lddy=s.N, dx=FAKE, da=FAKE, db=FAKE)
    a.update(kw)
    r = ctypes.byref(s)
    return {
        "plan": lambda: lib.moe_adapter_plan(r, a["ids"], a["plan"], a["pbytes"], None),
        "forward": lambda: lib.moe_adapter_forward(r, a["x"], a["ldx"], a["w"], a["a"], a["b"], a["scale"], a["ids"], a["plan"], a["y"], a["f32"], a["h"],
                                                   a["ws"], a["nbytes"], None),
        "backward": lambda: lib.moe_adapter_backward(r, a["dy"], a["lddy"], a["x"], a["ldx"], a["w"], a["a"], a["b"], a["scale"], a["ids"], a["plan"],
                                                     a["h"], a["dx"], a["da"], a["db"], a["ws"], a["nbytes"], None)}


@pytest.mark.parametrize("kw", [dict(T=-1), dict(T=(1 << 26) + 1), dict(K=0), dict(K=60), dict(K=(1 << 16) + 8), dict(N=4), dict(N=129), dict(rank=0), dict(rank=12),
                                dict(rank=136), dict(adapters=0), dict(adapters=1025), dict(T=1 << 26, K=8192)])
def test_adapter_shapes_outside_the_limits(lib, kw):
    s = moe.make_adapter_shape(**(GOOD | kw))
    assert lib.moe_adapter_workspace_bytes(ctypes.byref(s), None, None) == b.MOE_ERR_SHAPE
    for call in adapter_calls(lib, s).values():
        assert call() == b.MOE_ERR_SHAPE


def test_adapter_arguments(lib):
    s = moe.make_adapter_shape(**GOOD)
    assert lib.moe_adapter_workspace_bytes(None, None, None) == b.MOE_ERR_ARG
    need, plan = b._adapter_bytes(s)
    assert need > 0 and plan >= 4 * 600 and plan % 4 == 0
    for kw in (dict(ids=None), dict(plan=None), dict(ids=0x1002), dict(plan=0x1004)):
        for call in adapter_calls(lib, s, **kw).values():
            assert call() == b.MOE_ERR_ARG, kw
    assert adapter_calls(lib, s, pbytes=plan - 1)["plan"]() == b.MOE_ERR_WORKSPACE
    both = (dict(x=None), dict(x=0x1008), dict(ldx=56), dict(ldx=68), dict(ldx=1 << 60), dict(ldx=-64), dict(w=None), dict(a=None), dict(b=None), dict(ws=None),
            dict(w=0x1008), dict(a=0x1008), dict(b=0x1008), dict(scale=0x1002), dict(ws=0x1080), dict(h=0x1008))
    for kw in both + (dict(y=None), dict(y=0x1008), dict(f32=2)):
        assert adapter_calls(lib, s, **kw)["forward"]() == b.MOE_ERR_ARG, kw
    for kw in both + (dict(dy=None), dict(lddy=120), dict(dx=None), dict(da=None), dict(db=None), dict(h=None), dict(dx=0x1008), dict(da=0x1008), dict(db=0x1008)):
        assert adapter_calls(lib, s, **kw)["backward"]() == b.MOE_ERR_ARG, kw
    for name in ("forward", "backward"):
        assert adapter_calls(lib, s, nbytes=need - 1)[name]() == b.MOE_ERR_WORKSPACE


def test_few_tokens_need_no_plan(lib):
    s = moe.make_adapter_shape(T=512, K=64, N=128, rank=16, adapters=4)
    assert b._adapter_bytes(s)[1] == 0
    assert adapter_calls(lib, s, ids=None, plan=None)["plan"]() == b.MOE_OK   # nothing to do
    assert adapter_calls(lib, s, ids=None, plan=None)["forward"]() == b.MOE_ERR_ARG
    wide = moe.make_adapter_shape(T=512, K=7168, N=7168, rank=16, adapters=4)   # may be sorted, need not be
    assert b._adapter_bytes(wide)[1] > 0
    assert adapter_calls(lib, wide, plan=None, nbytes=0)["forward"]() == b.MOE_ERR_WORKSPACE
    assert adapter_calls(lib, moe.make_adapter_shape(T=513, K=64, N=128, rank=16, adapters=4), plan=None, nbytes=0)["forward"]() == b.MOE_ERR_ARG


BAL = dict(T=100, E=16, k=2, seqs=2)


@pytest.mark.parametrize("kw", [dict(T=-1), dict(E=0), dict(E=1025), dict(k=0), dict(k=17, E=64), dict(k=3, E=2), dict(seqs=0), dict(seqs=65537), dict(T=1 << 30)])
def test_balance_shapes_outside_the_limits(lib, kw):
    s = moe.make_balance_shape(**(BAL | kw))
    assert lib.moe_balance_workspace_bytes(ctypes.byref(s), None) == b.MOE_ERR_SHAPE
    st = b.MoEBalanceStatsC(*[FAKE] * 5)
    assert lib.moe_balance_forward(ctypes.byref(s), FAKE, FAKE, FAKE, None, ctypes.byref(st), FAKE, 1 << 40, None) == b.MOE_ERR_SHAPE
    assert lib.moe_balance_backward(ctypes.byref(s), FAKE, FAKE, FAKE, ctypes.byref(st), None, None, FAKE, FAKE, 0, None) == b.MOE_ERR_SHAPE


def test_balance_arguments(lib):
    s = moe.make_balance_shape(**BAL)
    need = moe.moe_balance_workspace_bytes(s)

    def both(logits=FAKE, idx=FAKE, offsets=FAKE, mask=None, stats=(FAKE,) * 5, ws=FAKE, nbytes=need, w=None, dw=None, u=FAKE, d=FAKE, bf16=0):
        st = ctypes.byref(b.MoEBalanceStatsC(*stats)) if stats else None
        return (lib.moe_balance_forward(ctypes.byref(s), logits, idx, offsets, mask, st, ws, nbytes, None),
                lib.moe_balance_backward(ctypes.byref(s), logits, idx, offsets, st, w, dw, u, d, bf16, None))

    for kw in (dict(logits=None), dict(idx=None), dict(offsets=None), dict(stats=None), dict(stats=(FAKE, None, FAKE, FAKE, FAKE)),
               dict(stats=(FAKE, FAKE, None, FAKE, FAKE)), dict(stats=(FAKE, FAKE, FAKE, FAKE, None)), dict(logits=0x1002), dict(idx=0x1001), dict(offsets=0x1002)):
        assert both(**kw) == (b.MOE_ERR_ARG,) * 2, kw
    small = ctypes.byref(s)
    st = ctypes.byref(b.MoEBalanceStatsC(*[FAKE] * 5))
    for ws, n, code in ((None, need, b.MOE_ERR_ARG), (0x1080, need, b.MOE_ERR_ARG), (FAKE, need - 1, b.MOE_ERR_WORKSPACE)):
        assert lib.moe_balance_forward(small, FAKE, FAKE, FAKE, None, st, ws, n, None) == code
    for stats in ((None, FAKE, FAKE, FAKE, FAKE), (FAKE, FAKE, FAKE, None, FAKE)):
        st2 = ctypes.byref(b.MoEBalanceStatsC(*stats))
        assert lib.moe_balance_forward(small, FAKE, FAKE, FAKE, None, st2, FAKE, need, None) == b.MOE_ERR_ARG
    for w, dw, u, d, bf16 in ((FAKE, None, FAKE, FAKE, 0), (None, FAKE, FAKE, FAKE, 0), (None, None, None, FAKE, 0), (None, None, FAKE, None, 0),
                              (None, None, FAKE, FAKE, 2), (None, None, FAKE, 0x1002, 0), (0x1001, FAKE, FAKE, FAKE, 0)):
        assert lib.moe_balance_backward(small, FAKE, FAKE, FAKE, st, w, dw, u, d, bf16, None) == b.MOE_ERR_ARG


def test_the_binding_refuses_other_tensors():
    s = moe.make_adapter_shape(**GOOD)
    with pytest.raises(AssertionError):
        moe.moe_adapter_plan(s, torch.zeros(600, dtype=torch.int32))   # not on the GPU
    with pytest.raises(AssertionError):
        moe.moe_balance_forward(moe.make_balance_shape(4, 8, 2), torch.zeros((4, 8)), torch.zeros((4, 2), dtype=torch.int32))


def test_the_binding_fails_loudly_without_its_extension_module(monkeypatch, tmp_path):
    monkeypatch.setattr(b, "_call", None)
    monkeypatch.setattr(b, "CALL_PATH", tmp_path / "nope.so")
    with pytest.raises(FileNotFoundError):
        moe.moe_adapter_plan(moe.make_adapter_shape(**GOOD), torch.zeros(600, dtype=torch.int32))


def test_the_extension_module_refuses_what_is_no_argument():
    call, s = b._load_call(), moe.make_adapter_shape(**GOOD)
    with pytest.raises(TypeError):
        call.adapter_plan(0)
    with pytest.raises(ValueError):
        call.adapter_plan(0, torch.zeros(600, dtype=torch.int32), 0)
    with pytest.raises(AssertionError):
        call.adapter_plan(b.ctypes.addressof(s), None, 0)
    with pytest.raises(TypeError):
        call.adapter_plan("shape", torch.zeros(600, dtype=torch.int32), 0)


def test_a_plan_that_is_given_is_filled_or_refused(lib):
    """With 257 to 512 tokens some widths read a plan and others do not: none that a wide shape may read stays unwritten without an error."""
    for T in (257, 400, 512):
        narrow, wide = moe.make_adapter_shape(T, 64, 128, 16, 4), moe.make_adapter_shape(T, 1 << 16, 1 << 16, 128, 4)
        assert b._adapter_bytes(narrow)[1] == 0
        need = b._adapter_bytes(wide)[1]
        assert need > 0 and need == b._adapter_bytes(moe.make_adapter_shape(T, 1 << 16, 32768, 8, 4))[1]   # by tokens and adapters alone
        for nbytes in (0, need - 1):
            assert adapter_calls(lib, narrow, pbytes=nbytes)["plan"]() == b.MOE_ERR_WORKSPACE
        assert adapter_calls(lib, narrow, plan=0x1004)["plan"]() == b.MOE_ERR_ARG
        assert adapter_calls(lib, narrow, ids=None)["plan"]() == b.MOE_ERR_ARG
        assert adapter_calls(lib, narrow, plan=None)["plan"]() == b.MOE_OK
        assert adapter_calls(lib, wide, plan=None)["plan"]() == b.MOE_ERR_ARG
        # a call without a plan has room for its own
        ws = b._adapter_bytes(wide)[0]
        assert adapter_calls(lib, wide, plan=None, nbytes=ws - 1)["forward"]() == b.MOE_ERR_WORKSPACE
    most = moe.make_adapter_shape(256, 1 << 16, 1 << 16, 128, 4)   # no width sorts
    assert b._adapter_bytes(most)[1] == 0 and adapter_calls(lib, most, plan=FAKE, pbytes=0)["plan"]() == b.MOE_OK


def test_plans_of_other_numbers_of_tokens_have_other_sizes():
    """By which the binding knows that a table is the batch's own: blocks of the plan get longer from 16384 tokens on, its bytes do not get fewer."""
    for n in (1, 7, 1024):
        last = 0
        for T in [257, 258, 300, 511, 512] + list(range(513, 700)) + list(range(16000, 17000)) + [1 << 20, 1 << 22]:
            need = b._adapter_bytes(moe.make_adapter_shape(T, 1 << 16, 1 << 16, 8, n))[1]
            assert need > last, (T, n)
            last = need


class NoMemory(torch.Tensor):
    """A tensor of a GPU that is not there: sizes, type and device, and a null pointer that the library refuses."""

    @staticmethod
    def __new__(cls, dtype, sizes, device):
        return torch.Tensor._make_wrapper_subclass(cls, sizes, dtype=dtype, device=device)

    @classmethod
    def __torch_dispatch__(cls, func, types, args=(), kwargs=None):
        raise NotImplementedError(func)


def test_tensors_on_several_gpus_are_refused():
    call, bf, f32, i32, u8 = b._load_call(), torch.bfloat16, torch.float32, torch.int32, torch.uint8
    T, K, N, r, n = 40, 64, 72, 8, 3
    s = moe.make_adapter_shape(T, K, N, r, n)
    E, k, S = 16, 2, 2
    bal = moe.make_balance_shape(T, E, k, S)
    stats = {"counts": (i32, (S, E)), "tokens": (i32, (S + 1,)), "lse": (f32, (T,))}
    operands = {"w": (bf, (K, N)), "a": (bf, (n, r, K)), "b": (bf, (n, r, N)), "scale": (f32, (n,)), "ids": (i32, (T,))}
    inputs = {"logits": (f32, (T, E)), "topk_idx": (i32, (T, k)), "seq_offsets": (i32, (S + 1,))}
    calls = (   # shape, the tensors in their order and what stands between them
        (call.adapter_forward, s, {"x": (bf, (T, K))} | operands | {"table": None, "adapters": n, "fp32": False, "h": (f32, (T, r)), "y": (bf, (T, N)), "ws": (u8, (1 << 30,)), "stream": 0}),
        (call.adapter_backward, s, {"dy": (bf, (T, N)), "x": (bf, (T, K))} | operands | {"table": None, "adapters": n, "h": (f32, (T, r)), "dx": (bf, (T, K)), "da": (f32, (n, r, K)),
                                                                                        "db": (f32, (n, r, N)), "ws": (u8, (1 << 30,)), "stream": 0}),
        (call.balance_backward, bal, inputs | stats | {"topk_w": (f32, (T, k)), "dtopk_w": (f32, (T, k)), "dloss": (f32, (1,)), "bf16": False, "out": (f32, (T, E)), "stream": 0}))
    for function, shape, kw in calls:
        def made(other=None):
            return [NoMemory(*v, "cuda:1" if name == other else "cuda:0") if type(v) is tuple else v for name, v in kw.items()]
        assert function(b._addressof(shape), *made()) == b.MOE_ERR_ARG   # as the library says of a null pointer
        for name, v in kw.items():
            if type(v) is tuple:
                with pytest.raises(AssertionError, match="GPU"):
                    function(b._addressof(shape), *made(name))
    # (the balance loss allocates its results before it calls the library)
    for other in ("topk_idx", "seq_offsets", "mask"):
        args = [NoMemory(*v, "cuda:1" if name == other else "cuda:0") for name, v in (inputs | {"mask": (torch.bool, (T,))}).items()]
        with pytest.raises(AssertionError, match="GPU"):
            call.balance_forward(b._addressof(bal), *args, None, 0)
