"""Refusals of the token operators' C ABI, on the CPU: every call here fails
the host's validation, or has no rows, so no HIP call is made."""
import ctypes
import os

import pytest
import torch

from paper_1912_03203_amd import dynconv as dc

OK, ERR_NULL, ERR_SHAPE, ERR_DTYPE, ERR_UNSUPPORTED, ERR_CAPACITY, ERR_ALIGN, ERR_WORKSPACE, \
    ERR_HIP, ERR_ARG = range(10)
FAKE = 0x7F0000000000
FAR = FAKE + (1 << 40)


@pytest.fixture(scope="module")
def lib():
    override = os.environ.get("DYNCONV_TEST_LIB")
    if override:
        return dc.load(override)
    if not os.path.exists(dc.LIB_PATH):
        from paper_1912_03203_amd import build

        build.build()
    return dc.load()


def test_route(lib):
    f, size = lib.dynconv_route, lib.dynconv_route_workspace_bytes

    def call(logits=FAKE, tokens=100, dt=0, experts=64, top_k=8, bias=None, mask=None, flags=0, routes="ok", ws=FAKE,
             nbytes=None, **fields):
        r = dc.RoutesStruct(FAKE, FAKE, FAKE, FAKE, 800)
        for k, v in fields.items():
            setattr(r, k, v)
        nbytes = size(100, 64, 8) if nbytes is None else nbytes
        return f(logits, tokens, dt, experts, top_k, bias, mask, flags, 1.0, ctypes.byref(r) if routes else None, ws,
                 nbytes, None)

    assert call(logits=None) == ERR_NULL
    assert call(routes=None) == ERR_NULL
    for field in ("expert", "weight", "rows", "starts"):
        assert call(**{field: None}) == ERR_NULL
    assert call(dt=3) == ERR_DTYPE
    assert call(tokens=-1) == ERR_SHAPE
    assert call(experts=0) == ERR_SHAPE
    assert call(top_k=0) == ERR_SHAPE
    assert call(top_k=65) == ERR_SHAPE
    assert call(top_k=17) == ERR_UNSUPPORTED
    assert call(experts=1025) == ERR_UNSUPPORTED
    assert call(tokens=1 << 28) == ERR_SHAPE  # 2^31 assignments
    assert call(flags=4) == ERR_ARG
    assert call(capacity=799) == ERR_CAPACITY
    assert call(logits=FAKE + 2) == ERR_ALIGN
    assert call(bias=FAKE + 1) == ERR_ALIGN
    assert call(rows=FAKE + 2) == ERR_ALIGN
    assert call(ws=None) == ERR_WORKSPACE
    assert call(nbytes=size(100, 64, 8) - 1) == ERR_WORKSPACE
    assert size(-1, 64, 8) == 0 and size(4, 64, 17) == 0 and size(4, 0, 1) == 0
    assert size(0, 64, 8) > 0


def linear(c_in=64, c_out=32, w=FAKE, b=None, act=0):
    return dc.LinearStruct(c_in, c_out, w, b, act)


def test_grouped_linear(lib):
    def call(x=FAKE, x_rows=100, y=FAR, y_rows=100, dt=2, l=None, groups=4, starts=FAKE, rows=100, src=None, src_div=1,
             dst=None):
        l = linear() if l is None else l
        return lib.dynconv_grouped_linear(x, x_rows, y, y_rows, dt, ctypes.byref(l), groups, starts, rows, src, src_div,
                                          dst, None)

    assert lib.dynconv_grouped_linear(FAKE, 1, FAR, 1, 2, None, 1, FAKE, 1, None, 1, None, None) == ERR_NULL
    assert call(x=None) == ERR_NULL
    assert call(y=None) == ERR_NULL
    assert call(starts=None) == ERR_NULL
    assert call(l=linear(w=None)) == ERR_NULL
    assert call(dt=-1) == ERR_DTYPE
    for kw in ({"x_rows": -1}, {"y_rows": -1}, {"rows": -1}, {"groups": 0}, {"rows": 1 << 31}):
        assert call(**kw) == ERR_SHAPE
    assert call(l=linear(c_in=0)) == ERR_SHAPE
    assert call(l=linear(c_in=60)) == ERR_UNSUPPORTED
    assert call(l=linear(c_out=65544)) == ERR_UNSUPPORTED
    assert call(groups=1025) == ERR_UNSUPPORTED
    assert call(l=linear(act=5)) == ERR_ARG
    assert call(src=FAKE, src_div=0) == ERR_ARG
    assert call(src_div=2) == ERR_ARG        # a divisor without a list
    assert call(x_rows=99) == ERR_SHAPE      # without src every position reads its own row
    assert call(y_rows=99) == ERR_SHAPE
    assert call(x=FAKE + 8) == ERR_ALIGN
    assert call(l=linear(b=FAKE + 4)) == ERR_ALIGN
    assert call(starts=FAKE + 2) == ERR_ALIGN
    assert call(y=FAKE + 64) == ERR_SHAPE    # overlap
    assert call(x_rows=0, y_rows=0, rows=0, x=None, y=None) == OK  # nothing to do
    # more workgroups than a launch counts: rows are refused, not cut off
    assert call(x_rows=2**31 - 1, y_rows=2**31 - 1, rows=2**31 - 1, y=FAKE + (1 << 60), groups=1,
                l=linear(c_in=8, c_out=65536)) == ERR_UNSUPPORTED


def experts(**over):
    e = dc.ExpertsStruct(64, 32, 64, 8, FAKE, None, FAKE, None, FAKE, None, dc.ACT_SILU)
    for k, v in over.items():
        setattr(e, k, v)
    return e


def test_experts(lib):
    size = lib.dynconv_experts_workspace_bytes

    def up(v):
        return (v + 255) // 256 * 256

    # hidden rows in the storage type, then the experts' outputs in fp32
    need = size(10, ctypes.byref(experts()), 2, 2)
    assert need == up(20 * 32 * 2) + up(20 * 64 * 4)

    def call(x=FAKE, y=FAR, tokens=10, dt=2, e=None, top_k=2, flags=0, ws=FAKE, nbytes=need, routes=True, **fields):
        r = dc.RoutesStruct(FAKE, FAKE, FAKE, FAKE, 20)
        for k, v in fields.items():
            setattr(r, k, v)
        return lib.dynconv_experts_forward(x, y, tokens, dt, ctypes.byref(e or experts()), top_k,
                                           ctypes.byref(r) if routes else None, flags, ws, nbytes, None)

    assert lib.dynconv_experts_forward(FAKE, FAR, 10, 2, None, 2, None, 0, FAKE, need, None) == ERR_NULL
    assert call(x=None) == ERR_NULL
    assert call(routes=False) == ERR_NULL
    for field in ("expert", "weight", "rows", "starts"):
        assert call(**{field: None}) == ERR_NULL
        assert call(**{field: FAKE + 2}) == ERR_ALIGN
    assert call(e=experts(w_project=None)) == ERR_NULL
    assert call(dt=9) == ERR_DTYPE
    assert call(tokens=-1) == ERR_SHAPE
    assert call(e=experts(c_hidden=20)) == ERR_UNSUPPORTED
    assert call(e=experts(experts=4), top_k=5) == ERR_SHAPE
    assert call(e=experts(act=-1)) == ERR_ARG
    assert call(flags=2) == ERR_ARG
    assert call(e=experts(c_out=32), flags=1) == ERR_SHAPE  # nothing to add the layer's input to
    assert call(capacity=19) == ERR_CAPACITY
    assert call(e=experts(w_gate=FAKE + 8)) == ERR_ALIGN
    assert call(ws=FAKE + 8) == ERR_ALIGN
    assert call(y=FAKE + 128) == ERR_SHAPE
    assert call(y=FAKE, e=experts(c_out=32)) == ERR_SHAPE   # in place needs equal widths
    assert call(ws=None) == ERR_WORKSPACE
    assert call(nbytes=need - 1) == ERR_WORKSPACE
    assert call(tokens=0, x=None, y=None) == OK
    assert size(10, ctypes.byref(experts(c_in=4)), 2, 2) == 0


def adapters(**over):
    a = dc.AdaptersStruct(4, 16, FAKE, FAKE, None, None)
    for k, v in over.items():
        setattr(a, k, v)
    return a


def test_adapter_linear(lib):
    size = lib.dynconv_adapter_workspace_bytes
    need = size(100, ctypes.byref(linear()), ctypes.byref(adapters()), 1)
    assert need >= 100 * 16 * 2

    def call(x=FAKE, y=FAR, rows=100, dt=1, l=None, a=None, ids=FAKE, ws=FAKE, nbytes=need):
        return lib.dynconv_adapter_linear(x, y, rows, dt, ctypes.byref(l or linear()), ctypes.byref(a or adapters()), ids,
                                          ws, nbytes, None)

    assert lib.dynconv_adapter_linear(FAKE, FAR, 100, 1, None, None, FAKE, FAKE, need, None) == ERR_NULL
    assert call(x=None) == ERR_NULL
    assert call(ids=None) == ERR_NULL
    assert call(a=adapters(up=None)) == ERR_NULL
    assert call(dt=3) == ERR_DTYPE
    assert call(rows=-1) == ERR_SHAPE
    assert call(l=linear(c_out=0)) == ERR_SHAPE
    assert call(l=linear(c_in=12)) == ERR_UNSUPPORTED
    assert call(l=linear(act=7)) == ERR_ARG
    assert call(a=adapters(adapters=0)) == ERR_SHAPE
    assert call(a=adapters(max_rank=12)) == ERR_UNSUPPORTED
    assert call(a=adapters(max_rank=264)) == ERR_UNSUPPORTED
    assert call(a=adapters(down=FAKE + 8)) == ERR_ALIGN
    assert call(a=adapters(scales=FAKE + 2)) == ERR_ALIGN
    assert call(ids=FAKE + 1) == ERR_ALIGN
    assert call(y=FAKE) == ERR_SHAPE
    assert call(ws=None) == ERR_WORKSPACE
    assert call(nbytes=need - 1) == ERR_WORKSPACE
    assert call(rows=0, x=None, y=None, ids=None) == OK


def test_blocks_keep_their_activations(lib):
    """SiLU and GELU are the token operators': a block still refuses them."""
    b = dc.Block(32, 192, 32, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, dc.ACT_SILU, 2, 0, FAKE, 0.0)
    s = dc.Shape(2, 8, 8, 32)
    assert lib.dynconv_block_forward(FAKE, FAKE, s, 1, ctypes.byref(b), None, FAKE, 1 << 30, None) == ERR_ARG


def test_binding_checks_its_tensors():
    """Types, shapes, layouts and devices are checked before the library is called."""
    x = torch.zeros(6, 16, dtype=torch.float16)
    w = torch.zeros(3, 8, 16, dtype=torch.float16)
    y = torch.zeros(6, 8, dtype=torch.float16)
    starts = torch.zeros(4, dtype=torch.int32)

    def bad(match, *args, **kw):
        with pytest.raises(dc.DynconvError, match=match):
            dc.GroupedLinear(*args, **kw)

    bad("x: an fp32", x.to(torch.float64), y, w, None, starts)
    bad("w: dtype", x, y, w.float(), None, starts)
    bad("x: shape", x[:, :8].contiguous(), y, w, None, starts)
    bad("x: the tensor is not contiguous", x.t().contiguous().t(), y, w, None, starts)
    bad("starts: shape", x, y, w, None, starts[:3])
    bad("starts: dtype", x, y, w, None, starts.long())
    bad("b: shape", x, y, w, torch.zeros(3, 16), starts)
    bad("src and dst", x, y, w, None, starts, src=starts, dst=starts[:2])
    bad("y: on meta", x, y.to("meta"), w, None, starts)
    bad("not on a GPU", x, y, w, None, starts)
    with pytest.raises(dc.DynconvError, match="not on a GPU"):
        dc.Router(torch.zeros(4, 8), 2)
    with pytest.raises(dc.DynconvError, match="mask: dtype"):
        dc.Router(torch.zeros(4, 8), 2, mask=torch.ones(4, dtype=torch.bool))
    with pytest.raises(dc.DynconvError, match="rejected"):
        dc.Router(torch.zeros(4, 8), 9)
    with pytest.raises(dc.DynconvError, match="b_gate without"):
        dc.ExpertWeights(w, torch.zeros(3, 16, 8, dtype=torch.float16), b_gate=torch.zeros(3, 8)).check(x)
    with pytest.raises(dc.DynconvError, match="device tensor"):
        dc.route(torch.zeros(4, 8), 2)
