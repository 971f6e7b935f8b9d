"""What moving tokens, the packed stash and the 4-bit operators refuse, before anything reaches a device."""
import ctypes

import pytest
import torch

import paper_2604_19241_amd as moe
from paper_2604_19241_amd import binding as b
from test_operators_host import NoMemory

FAKE, ODD = 0x1000, 0x1008
BF, F32, I32, U8, I8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8, torch.int8
ARG, SHAPE = b.MOE_ERR_ARG, b.MOE_ERR_SHAPE


@pytest.fixture(scope="module")
def lib():
    if not b.LIB_PATH.exists():
        from paper_2604_19241_amd import build
        build.build()
    return b.load_library()


def move_calls(lib, s, **kw):
    a = dict(x=FAKE, ld=s.d if s else 64, rows=FAKE, row_of=FAKE, w=None, f32=0, tokens=FAKE, o=FAKE, dw=FAKE)
    a.update(kw)
    r = ctypes.byref(s) if s else None
    return {"dispatch_forward": lambda: lib.moe_dispatch_forward(r, a["x"], a["ld"], a["f32"], a["row_of"], a["rows"], None),
            "dispatch_backward": lambda: lib.moe_dispatch_backward(r, a["rows"], a["f32"], a["row_of"], a["tokens"], None),
            "combine_forward": lambda: lib.moe_combine_forward(r, a["rows"], a["f32"], a["row_of"], a["w"], a["tokens"], None),
            "combine_backward": lambda: lib.moe_combine_backward(r, a["x"], a["ld"], a["o"], a["f32"], a["row_of"], a["w"], a["rows"], a["dw"], None)}


@pytest.mark.parametrize("kw", [dict(T=-1), dict(k=0), dict(k=17), dict(T=1 << 28, k=4), dict(d=0), dict(d=12), dict(d=(1 << 20) + 8), dict(rows=-1), dict(T=1 << 19, d=1 << 20)])
def test_shapes_outside_the_limits_of_moving(lib, kw):
    s = moe.make_dispatch_shape(**(dict(T=40, k=4, d=64, rows=160) | kw))
    assert all(call() == SHAPE for call in move_calls(lib, s).values())


def test_arguments_of_moving(lib):
    assert ctypes.sizeof(b.MoEDispatchShape) == 16
    assert moe.make_dispatch_shape(5, 3, 64).rows == 15
    s = moe.make_dispatch_shape(40, 4, 64)
    assert all(call() == ARG for call in move_calls(lib, None).values())
    for kw in (dict(row_of=None), dict(row_of=0x1002), dict(f32=2), dict(f32=-1), dict(rows=None), dict(rows=ODD)):
        assert all(call() == ARG for call in move_calls(lib, s, **kw).values()), kw
    for kw in (dict(x=None), dict(x=ODD), dict(ld=56), dict(ld=68), dict(ld=-64), dict(ld=1 << 60)):
        for name in ("dispatch_forward", "combine_backward"):
            assert move_calls(lib, s, **kw)[name]() == ARG, kw
    for kw in (dict(tokens=None), dict(tokens=ODD)):
        for name in ("dispatch_backward", "combine_forward"):
            assert move_calls(lib, s, **kw)[name]() == ARG, kw
    for kw in (dict(o=None), dict(o=ODD), dict(w=0x1002), dict(dw=0x1002)):
        assert move_calls(lib, s, **kw)["combine_backward"]() == ARG, kw
    assert move_calls(lib, s, w=0x1002)["combine_forward"]() == ARG
    none = moe.make_dispatch_shape(0, 4, 64, 10)
    assert all(call() == b.MOE_OK for call in move_calls(lib, none, x=None, tokens=None, row_of=None).values())   # nothing to do


@pytest.mark.parametrize("kw", [dict(I=96), dict(T=-1), dict(k=17), dict(e_count=0), dict(e_start=7)])
def test_shapes_outside_the_limits_of_the_stash(lib, kw):
    s = moe.make_shape(**(dict(T=8, d=64, E=8, k=2, I=64, e_start=0, e_count=8) | kw))
    r = b.MoERoutingC(*[FAKE] * 6)
    for f in (lib.moe_saved_pack, lib.moe_saved_unpack):
        assert f(ctypes.byref(s), ctypes.byref(r), FAKE, FAKE, FAKE, None) == SHAPE


def test_arguments_of_the_packed_stash(lib):
    s, r = moe.make_shape(8, 64, 8, 2, 64), b.MoERoutingC(*[FAKE] * 6)
    def pack(shape=s, routing=r, saved=FAKE, codes=FAKE, scales=FAKE):  # noqa: E306
        p = [ctypes.byref(v) if v is not None else None for v in (shape, routing)]
        return lib.moe_saved_pack(*p, saved, codes, scales, None), lib.moe_saved_unpack(*p, codes, scales, saved, None)
    for kw in (dict(shape=None), dict(routing=None), dict(routing=b.MoERoutingC(FAKE, FAKE, FAKE, None, FAKE, FAKE)), dict(routing=b.MoERoutingC(FAKE, FAKE, FAKE, 0x1002, FAKE, FAKE)),
               dict(saved=None), dict(codes=None), dict(scales=None), dict(saved=0x1080), dict(codes=ODD), dict(scales=0x1002)):
        assert pack(**kw) == (ARG, ARG), kw
    assert pack(shape=moe.make_shape(0, 64, 8, 2, 64), saved=None, codes=None, scales=None) == (b.MOE_OK,) * 2


@pytest.mark.parametrize("rows,K", [(-1, 64), (1 << 31, 64), (10, 0), (10, 12), (10, (1 << 16) + 8), (1 << 21, 1 << 16)])
def test_shapes_outside_the_limits_of_4_bits(lib, rows, K):
    assert lib.moe_mx_quantize(FAKE, 1 << 17, 0, rows, K, FAKE, FAKE, None) == SHAPE
    assert lib.moe_mx_values(FAKE, FAKE, rows, K, FAKE, 0, None) == SHAPE


def test_arguments_of_4_bits(lib):
    def quantize(x=FAKE, ld=64, f32=0, codes=FAKE, scales=FAKE):
        return lib.moe_mx_quantize(x, ld, f32, 10, 64, codes, scales, None)
    for kw in (dict(x=None), dict(x=ODD), dict(ld=56), dict(ld=68), dict(ld=1 << 60), dict(f32=2), dict(codes=None), dict(codes=ODD), dict(scales=None), dict(scales=ODD)):
        assert quantize(**kw) == ARG, kw
    for args in ((None, FAKE, FAKE, 0), (FAKE, None, FAKE, 0), (FAKE, FAKE, None, 0), (ODD, FAKE, FAKE, 0), (FAKE, ODD, FAKE, 0), (FAKE, FAKE, ODD, 0), (FAKE, FAKE, FAKE, 2)):
        assert lib.moe_mx_values(args[0], args[1], 10, 64, args[2], args[3], None) == ARG, args
    for E, K, N in ((0, 64, 64), (1025, 64, 64), (4, 60, 64), (4, 64, 60), (4, 64, 0), (4, 64, (1 << 16) + 8), (4, (1 << 16) + 8, 64), (1024, 1 << 16, 1 << 16)):
        assert lib.moe_mx_quantize_weights(FAKE, E, K, N, FAKE, FAKE, None) == SHAPE, (E, K, N)
    for args in ((None, FAKE, FAKE), (ODD, FAKE, FAKE), (FAKE, None, FAKE), (FAKE, FAKE, ODD)):
        assert lib.moe_mx_quantize_weights(args[0], 4, 64, 64, *args[1:], None) == ARG
    assert lib.moe_mx_quantize(None, 64, 0, 0, 64, None, None, None) == b.MOE_OK and lib.moe_mx_values(None, None, 0, 64, None, 0, None) == b.MOE_OK


GOOD = dict(rows=100, K=64, N=72, experts=4)


def product_calls(lib, s, **kw):
    a = dict(a=FAKE, sc=FAKE, a_rows=100, perm=None, k=1, w=FAKE, ws=FAKE, u=FAKE, us=FAKE, offsets=FAKE, y=FAKE, f32=0, hc=None, hs=None)
    a.update(kw)
    r = ctypes.byref(s) if s else None
    head = (r, a["a"], a["sc"], a["a_rows"], a["perm"], a["k"], a["w"], a["ws"])
    return {"product": lambda: lib.moe_mx_product(*head, a["offsets"], a["y"], a["f32"], None),
            "gate_up": lambda: lib.moe_mx_gate_up(*head, a["u"], a["us"], a["offsets"], a["y"], a["hc"], a["hs"], None)}


@pytest.mark.parametrize("kw", [dict(rows=-1), dict(rows=1 << 30), dict(K=0), dict(K=60), dict(K=(1 << 16) + 8), dict(N=4), dict(N=73), dict(N=(1 << 16) + 8), dict(experts=0), dict(experts=1025),
                                dict(rows=1 << 21, K=1 << 16), dict(rows=1 << 21, N=1 << 16), dict(experts=1024, K=1 << 16, N=1 << 16)])
def test_shapes_outside_the_limits_of_the_products(lib, kw):
    s = moe.make_mx_shape(**(GOOD | kw))
    assert all(call() == SHAPE for call in product_calls(lib, s, a_rows=1 << 22).values())


def test_arguments_of_the_products(lib):
    assert ctypes.sizeof(b.MoEMXShape) == 16
    s = moe.make_mx_shape(**GOOD)
    assert all(call() == ARG for call in product_calls(lib, None).values())
    for kw in (dict(a=None), dict(a=ODD), dict(sc=None), dict(sc=ODD), dict(w=None), dict(w=ODD), dict(ws=None), dict(ws=ODD), dict(offsets=None), dict(offsets=0x1002), dict(y=None), dict(y=ODD),
               dict(k=0), dict(k=-1), dict(a_rows=99), dict(perm=FAKE, a_rows=0), dict(perm=0x1002)):
        for name, call in product_calls(lib, s, **kw).items():
            assert call() == ARG, (name, kw)
    for kw in (dict(a_rows=-1), dict(a_rows=1 << 31), dict(a_rows=(1 << 29) + 1)):
        assert all(call() == SHAPE for call in product_calls(lib, s, **kw).values()), kw
    assert product_calls(lib, s, f32=2)["product"]() == ARG
    for kw in (dict(u=None), dict(u=ODD), dict(us=None), dict(us=ODD), dict(hc=FAKE, hs=FAKE), dict(y=None, hc=FAKE), dict(y=None, hs=FAKE), dict(y=None, hc=ODD, hs=FAKE), dict(y=None, hc=FAKE, hs=ODD)):
        assert product_calls(lib, s, **kw)["gate_up"]() == ARG, kw
    none = moe.make_mx_shape(**(GOOD | dict(rows=0)))
    assert all(call() == b.MOE_OK for call in product_calls(lib, none, a=None, sc=None, a_rows=0, y=None).values())   # nothing to do
    q = moe.MXTensor(torch.zeros((4, 64), dtype=U8), torch.zeros((4, 4), dtype=U8), 64)
    with pytest.raises(AssertionError):
        moe.moe_mx_product(moe.make_mx_shape(4, 128, 8, 1), q, q, torch.zeros(2, dtype=I32))   # another K


def gpu(dtype, *sizes, device="cuda:0"):
    return NoMemory(dtype, sizes, device)


def calls():
    """Every call of the extension module with tensors that have no memory: the library refuses their null pointers."""
    call = b._load_call()
    T, k, d, rows = 40, 4, 64, 100
    move = moe.make_dispatch_shape(T, k, d, rows)
    layer = moe.make_shape(T, 64, 8, k, 64)
    n = moe.alloc_saved(layer, "cpu").numel()
    packed = {"codes": (I8, (T * k, 128)), "scales": (U8, (T * k, 4))}
    mxs = moe.make_mx_shape(**GOOD)

    def operand(name, *sizes):
        return {name: (U8, (*sizes, 64)), name + "_scales": (U8, (*sizes, 4))}

    mxt = {"codes": (U8, (10, 64)), "scales": (U8, (10, 4))}
    return [
        (call.dispatch_forward, [move], {"x": (BF, (T, d)), "row_of": (I32, (T, k)), "out": (BF, (rows, d)), "stream": 0}),
        (call.combine_forward, [move], {"rows": (F32, (rows, d)), "row_of": (I32, (T, k)), "weights": (F32, (T, k)), "out": (F32, (T, d)), "stream": 0}),
        (call.combine_forward, [move], {"rows": (F32, (rows, d)), "row_of": (I32, (T, k)), "weights": None, "out": (F32, (T, d)), "stream": 0}),
        (call.combine_backward, [move], {"dy": (BF, (T, d)), "o": (BF, (rows, d)), "row_of": (I32, (T, k)), "weights": (F32, (T, k)), "do": (BF, (rows, d)), "dw": (F32, (T, k)),
                                         "want": True, "stream": 0}),
        (call.saved_pack, [layer], {"offsets": (I32, (9,)), "saved": (U8, (n,))} | packed | {"stream": 0}),
        (call.saved_unpack, [layer], {"offsets": (I32, (9,)), "saved": (U8, (n,))} | packed | {"stream": 0}),
        (call.mx_quantize, [], {"x": (BF, (10, 72))} | mxt | {"stream": 0}),
        (call.mx_quantize_weights, [], {"w": (BF, (2, 72, 5 * 8)), "codes": (U8, (2, 40, 64)), "scales": (U8, (2, 40, 4)), "stream": 0}),
        (call.mx_product, [mxs], operand("a", 100) | operand("w", 4, 72) | {"offsets": (I32, (5,)), "perm": (I32, (100,)), "k": 2, "f32": False, "y": (BF, (100, 72)), "stream": 0}),
        (call.mx_gate_up, [mxs], operand("a", 30) | operand("g", 4, 72) | operand("u", 4, 72) | {"offsets": (I32, (5,)), "perm": (I32, (100,)), "k": 2, "q": True,
                                                                                               "h": (U8, (100, 64)), "hs": (U8, (100, 4)), "stream": 0}),
        (call.mx_gate_up, [mxs], operand("a", 100) | operand("g", 4, 72) | operand("u", 4, 72) | {"offsets": (I32, (5,)), "perm": None, "k": 1, "q": False, "h": (BF, (100, 72)),
                                                                                                "none": None, "stream": 0}),
        (call.mx_values, [], mxt | {"K": 72, "f32": False, "out": (BF, (10, 72)), "stream": 0}),
    ]


def made(kw, **other):
    return [gpu(*v[:1], *v[1], device=other.get(n, "cuda:0")) if type(v) is tuple else v for n, v in kw.items()]


def test_tensors_of_other_types_sizes_and_gpus_are_refused():
    for function, shape, kw in calls():
        at = [b._addressof(s) for s in shape]
        assert function(*at, *made(kw)) == ARG, function.__name__   # as the library says of a null pointer
        for name, v in kw.items():
            if type(v) is not tuple:
                continue
            with pytest.raises(AssertionError, match="GPU"):
                function(*at, *made(kw, **{name: "cuda:1"}))
            with pytest.raises(AssertionError, match="GPU"):
                function(*at, *made(kw, **{name: "cpu"}))
            dtype, sizes = v
            for wrong in ((torch.float16, sizes), (dtype, (64,) if name == "saved" else sizes[:-1] + (sizes[-1] - 1,))):
                if name in ("x", "w") and wrong[0] is dtype and not shape:
                    continue   # (the first tensor of a call says its sizes)
                with pytest.raises(AssertionError):
                    function(*at, *made(kw | {name: wrong}))
        with pytest.raises(TypeError):
            function(*at)


def test_what_is_no_row_of_tensors_is_refused():
    call = b._load_call()
    with pytest.raises(AssertionError):
        call.mx_quantize(gpu(BF, 10), None, None, 0)
    with pytest.raises(AssertionError):
        call.mx_quantize_weights(gpu(BF, 10, 64), None, None, 0)
    with pytest.raises(AssertionError):
        call.mx_quantize(torch.zeros((10, 64)).T, None, None, 0)
    for x in (torch.zeros((4, 64)), torch.zeros((4, 64), dtype=BF)):   # not on the GPU
        with pytest.raises(AssertionError):
            moe.moe_mx_quantize(x)
    with pytest.raises(AssertionError):
        moe.moe_mx_values(moe.MXTensor(torch.zeros((4, 64), dtype=U8), torch.zeros((4, 4), dtype=U8), 128))
    with pytest.raises(AssertionError):
        moe.moe_dispatch_forward(moe.make_dispatch_shape(4, 2, 64), torch.zeros((4, 64)), torch.zeros((4, 2), dtype=I32))
    for K in (0, 1 << 17):
        assert call.mx_values(gpu(U8, 10, 64), gpu(U8, 10, 4), K, False, None, 0) == SHAPE
