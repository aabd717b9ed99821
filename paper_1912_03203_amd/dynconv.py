"""Python binding of the C ABI in include/dynconv.h (argument marshalling only).

Every computation happens in the HIP library ``libdynconv.so`` built next to
this file; this module passes device pointers of torch tensors, sizes and the
current HIP stream through ctypes.  There is no fallback: if the library is
missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdynconv.so")

F32, F16, BF16 = 0, 1, 2
ACT_NONE, ACT_RELU, ACT_RELU6 = 0, 1, 2
STACK_DENSE, STACK_UNFUSED, STACK_GSOFTMAX = 1, 2, 4

_TORCH_DTYPE = {F32: torch.float32, F16: torch.float16, BF16: torch.bfloat16}
_CODE = {torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16}
NAME_TO_DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}

EXPORTED = (
    "dynconv_status_str", "dynconv_version", "dynconv_mask", "dynconv_mask_gsoftmax",
    "dynconv_indices_workspace_bytes",
    "dynconv_build_indices", "dynconv_block_workspace_bytes", "dynconv_block_forward",
    "dynconv_stack_workspace_bytes", "dynconv_stack_forward", "dynconv_stack_launch_names",
    "dynconv_stack_forward_profiled", "dynconv_shuffle_stack_workspace_bytes",
    "dynconv_shuffle_stack_forward", "dynconv_shuffle_stack_launch_names",
    "dynconv_shuffle_stack_forward_profiled", "dynconv_network_output_shape",
    "dynconv_network_workspace_bytes", "dynconv_network_forward", "dynconv_network_launch_names",
    "dynconv_network_forward_profiled", "dynconv_stack_noalloc_max_workspace_bytes",
    "dynconv_stack_forward_noalloc", "dynconv_route_workspace_bytes", "dynconv_route",
    "dynconv_grouped_linear", "dynconv_experts_workspace_bytes", "dynconv_experts_forward",
    "dynconv_adapter_workspace_bytes", "dynconv_adapter_linear",
)


class Shape(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int32), ("h", ctypes.c_int32), ("w", ctypes.c_int32),
                ("c", ctypes.c_int32)]


class Block(ctypes.Structure):
    _fields_ = [
        ("c_in", ctypes.c_int32), ("c_hidden", ctypes.c_int32), ("c_out", ctypes.c_int32),
        ("w_expand", ctypes.c_void_p), ("b_expand", ctypes.c_void_p),
        ("w_dw", ctypes.c_void_p), ("b_dw", ctypes.c_void_p),
        ("w_project", ctypes.c_void_p), ("b_project", ctypes.c_void_p),
        ("act_expand", ctypes.c_int32), ("act_dw", ctypes.c_int32), ("act_project", ctypes.c_int32),
        ("w_mask", ctypes.c_void_p), ("b_mask", ctypes.c_float),
    ]


class Layer(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("stride", ctypes.c_int32), ("gated", ctypes.c_int32),
                ("c_in", ctypes.c_int32), ("c_out", ctypes.c_int32), ("w", ctypes.c_void_p),
                ("b", ctypes.c_void_p), ("act", ctypes.c_int32), ("blk", Block)]


LAYER_CONV3X3, LAYER_BLOCK, LAYER_CONV1X1 = 0, 1, 2


class Indices(ctypes.Structure):
    _fields_ = [("active", ctypes.c_void_p), ("dilated", ctypes.c_void_p),
                ("nbr", ctypes.c_void_p), ("counts", ctypes.c_void_p),
                ("capacity", ctypes.c_int64)]


class DynconvError(RuntimeError):
    pass


_lib = None


def load(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load the HIP library; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise DynconvError("libdynconv.so is not built (%s); run __graft_entry__.build()" % path)
    lib = ctypes.CDLL(path)
    vp, sz, i32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32
    lib.dynconv_status_str.argtypes = [ctypes.c_int]
    lib.dynconv_status_str.restype = ctypes.c_char_p
    lib.dynconv_version.argtypes = []
    lib.dynconv_version.restype = ctypes.c_char_p
    lib.dynconv_mask.argtypes = [vp, Shape, ctypes.c_int, vp, ctypes.c_float, vp, vp, vp]
    lib.dynconv_mask.restype = ctypes.c_int
    lib.dynconv_mask_gsoftmax.argtypes = [vp, Shape, ctypes.c_int, vp, ctypes.c_float, vp, vp, vp]
    lib.dynconv_mask_gsoftmax.restype = ctypes.c_int
    lib.dynconv_indices_workspace_bytes.argtypes = [Shape]
    lib.dynconv_indices_workspace_bytes.restype = sz
    lib.dynconv_build_indices.argtypes = [vp, Shape, i32, ctypes.POINTER(Indices), vp, sz, vp]
    lib.dynconv_build_indices.restype = ctypes.c_int
    lib.dynconv_block_workspace_bytes.argtypes = [Shape, ctypes.POINTER(Block), ctypes.c_int]
    lib.dynconv_block_workspace_bytes.restype = sz
    lib.dynconv_block_forward.argtypes = [vp, vp, Shape, ctypes.c_int, ctypes.POINTER(Block),
                                          ctypes.POINTER(Indices), vp, sz, vp]
    lib.dynconv_block_forward.restype = ctypes.c_int
    lib.dynconv_stack_workspace_bytes.argtypes = [Shape, ctypes.POINTER(Block), i32, ctypes.c_int,
                                                  i32]
    lib.dynconv_stack_workspace_bytes.restype = sz
    lib.dynconv_stack_forward.argtypes = [vp, vp, Shape, ctypes.c_int, ctypes.POINTER(Block), i32,
                                          i32, vp, vp, vp, sz, vp]
    lib.dynconv_stack_forward.restype = ctypes.c_int
    lib.dynconv_stack_launch_names.argtypes = [Shape, ctypes.POINTER(Block), i32, ctypes.c_int, i32,
                                               i32, ctypes.POINTER(ctypes.c_char_p), i32]
    lib.dynconv_stack_launch_names.restype = i32
    lib.dynconv_stack_forward_profiled.argtypes = [vp, vp, Shape, ctypes.c_int,
                                                   ctypes.POINTER(Block), i32, i32, vp, vp, vp, sz,
                                                   vp, ctypes.POINTER(ctypes.c_void_p), i32]
    lib.dynconv_stack_forward_profiled.restype = ctypes.c_int
    lib.dynconv_stack_noalloc_max_workspace_bytes.argtypes = []
    lib.dynconv_stack_noalloc_max_workspace_bytes.restype = sz
    lib.dynconv_stack_forward_noalloc.argtypes = [vp, vp, Shape, ctypes.c_int, ctypes.POINTER(Block), i32,
                                                  i32, vp, vp, vp]
    lib.dynconv_stack_forward_noalloc.restype = ctypes.c_int
    lib.dynconv_shuffle_stack_workspace_bytes.argtypes = [Shape, ctypes.POINTER(Block), i32,
                                                          ctypes.c_int, i32]
    lib.dynconv_shuffle_stack_workspace_bytes.restype = sz
    lib.dynconv_shuffle_stack_forward.argtypes = [vp, vp, Shape, ctypes.c_int, ctypes.POINTER(Block),
                                                  i32, i32, vp, vp, vp, sz, vp]
    lib.dynconv_shuffle_stack_forward.restype = ctypes.c_int
    lib.dynconv_shuffle_stack_launch_names.argtypes = [Shape, ctypes.POINTER(Block), i32, ctypes.c_int,
                                                       i32, ctypes.POINTER(ctypes.c_char_p), i32]
    lib.dynconv_shuffle_stack_launch_names.restype = i32
    lib.dynconv_shuffle_stack_forward_profiled.argtypes = [vp, vp, Shape, ctypes.c_int,
                                                           ctypes.POINTER(Block), i32, i32, vp, vp, vp,
                                                           sz, vp, ctypes.POINTER(ctypes.c_void_p), i32]
    lib.dynconv_shuffle_stack_forward_profiled.restype = ctypes.c_int
    lib.dynconv_network_output_shape.argtypes = [Shape, ctypes.POINTER(Layer), i32, ctypes.POINTER(Shape)]
    lib.dynconv_network_output_shape.restype = ctypes.c_int
    lib.dynconv_network_workspace_bytes.argtypes = [Shape, ctypes.POINTER(Layer), i32, ctypes.c_int, i32]
    lib.dynconv_network_workspace_bytes.restype = sz
    lib.dynconv_network_forward.argtypes = [vp, vp, Shape, ctypes.c_int, ctypes.POINTER(Layer), i32, i32, vp,
                                            vp, vp, sz, vp]
    lib.dynconv_network_forward.restype = ctypes.c_int
    lib.dynconv_network_launch_names.argtypes = [Shape, ctypes.POINTER(Layer), i32, ctypes.c_int, i32, i32,
                                                 ctypes.POINTER(ctypes.c_char_p), i32]
    lib.dynconv_network_launch_names.restype = i32
    lib.dynconv_network_forward_profiled.argtypes = [vp, vp, Shape, ctypes.c_int, ctypes.POINTER(Layer), i32,
                                                     i32, vp, vp, vp, sz, vp, ctypes.POINTER(ctypes.c_void_p),
                                                     i32]
    lib.dynconv_network_forward_profiled.restype = ctypes.c_int
    _declare_tokens(lib)
    _lib = lib
    return lib


def status_str(code: int) -> str:
    return load().dynconv_status_str(code).decode()


def _check(code: int, what: str):
    if code != 0:
        raise DynconvError("%s failed: %s (status %d)" % (what, status_str(code), code))


def _stream(stream=None):
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def dtype_code(dtype) -> int:
    return _CODE[dtype]


def shape_of(x: torch.Tensor) -> Shape:
    n, h, w, c = x.shape
    return Shape(n, h, w, c)


# ------------------------------------------------------------------ weights
@dataclass
class BlockWeights:
    """Device copies of one block's folded weights plus the C struct that
    points at them (the tensors must outlive every call that uses it)."""

    w_expand: torch.Tensor
    b_expand: torch.Tensor
    w_dw: torch.Tensor
    b_dw: torch.Tensor
    w_project: torch.Tensor
    b_project: torch.Tensor
    w_mask: torch.Tensor
    b_mask: float
    acts: tuple = (ACT_RELU6, ACT_RELU6, ACT_NONE)

    @classmethod
    def from_arrays(cls, wts: dict, dtype, device="cuda", b_mask=0.0, acts=None):
        def dev(a, dt):
            return torch.as_tensor(a).to(device=device, dtype=dt).contiguous()

        return cls(dev(wts["w1"], dtype), dev(wts["b1"], torch.float32),
                   dev(wts["w2"], dtype).reshape(-1, 9).contiguous(), dev(wts["b2"], torch.float32),
                   dev(wts["w3"], dtype), dev(wts["b3"], torch.float32),
                   dev(wts["w_m"], torch.float32), float(b_mask),
                   tuple(acts) if acts is not None else tuple(wts.get("acts", (2, 2, 0))))

    def struct(self) -> Block:
        E, C = self.w_expand.shape
        Co = self.w_project.shape[0]
        return Block(C, E, Co, self.w_expand.data_ptr(), self.b_expand.data_ptr(),
                     self.w_dw.data_ptr(), self.b_dw.data_ptr(), self.w_project.data_ptr(),
                     self.b_project.data_ptr(), self.acts[0], self.acts[1], self.acts[2],
                     self.w_mask.data_ptr(), float(self.b_mask))


@dataclass
class IndexBuffers:
    active: torch.Tensor
    dilated: torch.Tensor
    nbr: torch.Tensor
    counts: torch.Tensor

    @classmethod
    def alloc(cls, npos: int, device="cuda"):
        z = dict(device=device, dtype=torch.int32)
        return cls(torch.empty(max(npos, 1), **z), torch.empty(max(npos, 1), **z),
                   torch.empty(max(npos, 1) * 9, **z), torch.zeros(2, **z))

    def struct(self) -> Indices:
        return Indices(self.active.data_ptr(), self.dilated.data_ptr(), self.nbr.data_ptr(),
                       self.counts.data_ptr(), self.active.numel())


# ------------------------------------------------------------------ calls
def mask(x: torch.Tensor, w_mask: torch.Tensor, b_mask: float, out=None, logits=None, stream=None,
         gsoftmax=False):
    """Hard mask of one block (uint8 [N*H*W]); optional fp32 logits.  With
    gsoftmax the G-Softmax decision (dynconv_mask_gsoftmax) is taken."""
    lib = load()
    n, h, w, _ = x.shape
    if out is None:
        out = torch.empty(n * h * w, dtype=torch.uint8, device=x.device)
    fn = lib.dynconv_mask_gsoftmax if gsoftmax else lib.dynconv_mask
    _check(fn(_ptr(x), shape_of(x), dtype_code(x.dtype), _ptr(w_mask), ctypes.c_float(b_mask), _ptr(out),
              _ptr(logits), _stream(stream)), "dynconv_mask")
    return out


def indices_workspace_bytes(shape: Shape) -> int:
    return load().dynconv_indices_workspace_bytes(shape)


def build_indices(mask_t: torch.Tensor, shape: Shape, dilate: int, idx: IndexBuffers,
                  ws: torch.Tensor, stream=None):
    lib = load()
    s = idx.struct()
    _check(lib.dynconv_build_indices(_ptr(mask_t), shape, int(dilate), ctypes.byref(s), _ptr(ws),
                                     ws.numel() * ws.element_size(), _stream(stream)),
           "dynconv_build_indices")


def block_workspace_bytes(shape: Shape, blk: BlockWeights, dtype) -> int:
    s = blk.struct()
    return load().dynconv_block_workspace_bytes(shape, ctypes.byref(s), dtype_code(dtype))


def block_forward(x: torch.Tensor, y: torch.Tensor, blk: BlockWeights, idx, ws: torch.Tensor,
                  stream=None):
    lib = load()
    s = blk.struct()
    ids = idx.struct() if idx is not None else None
    _check(lib.dynconv_block_forward(_ptr(x), _ptr(y), shape_of(x), dtype_code(x.dtype),
                                     ctypes.byref(s), ctypes.byref(ids) if ids is not None else None,
                                     _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)),
           "dynconv_block_forward")
    return y


def round_up(v: int, m: int) -> int:
    return (v + m - 1) // m * m


def padded_branch_arrays(wts: dict) -> dict:
    """A ShuffleNetV2 branch's weights (cb channels, hidden E) zero-padded to
    the channel counts the library takes: cp = round_up(cb, 8) inputs and
    outputs, round_up(E, 16) hidden channels.  Padded hidden channels have
    zero weights and biases (their activations are 0 for NONE, RELU, RELU6),
    padded outputs are discarded by the unit, padded inputs are zero."""
    import numpy as np

    E, cb = np.asarray(wts["w1"]).shape
    cp, ep = round_up(cb, 8), round_up(E, 16)

    def pad(a, shape):
        a = np.asarray(a, np.float32)
        out = np.zeros(shape, np.float32)
        out[tuple(slice(0, n) for n in a.shape)] = a
        return out

    out = dict(wts)
    out.update(w1=pad(wts["w1"], (ep, cp)), b1=pad(wts["b1"], (ep,)), w2=pad(wts["w2"], (ep, 9)),
               b2=pad(wts["b2"], (ep,)), w3=pad(wts["w3"], (cp, ep)), b3=pad(wts["b3"], (cp,)),
               w_m=pad(wts["w_m"], (cp,)))
    return out


def _blocks_array(blocks):
    arr = (Block * len(blocks))()
    for i, b in enumerate(blocks):
        arr[i] = b.struct()
    return arr


def stack_workspace_bytes(shape: Shape, blocks, dtype, flags=0) -> int:
    arr = _blocks_array(blocks)
    return load().dynconv_stack_workspace_bytes(shape, arr, len(blocks), dtype_code(dtype), flags)


class Stack:
    """A prepared stack call y = blocks(x): the block array and pointers are
    marshalled once, so repeated launches (a timed loop, a graph capture) cost
    a single ctypes call.  y may be x (in place)."""

    def __init__(self, x: torch.Tensor, y: torch.Tensor, blocks, flags=0, masks=None, counts=None,
                 ws=None):
        self.lib = load()
        self.x, self.y = x, y
        self.blocks = list(blocks)
        self.arr = _blocks_array(self.blocks)
        self.shape = shape_of(x)
        self.dtype = dtype_code(x.dtype)
        self.flags = int(flags)
        need = self.lib.dynconv_stack_workspace_bytes(self.shape, self.arr, len(self.blocks),
                                                      self.dtype, self.flags)
        if need == 0:
            raise DynconvError("dynconv_stack_workspace_bytes rejected the stack")
        if ws is None:
            ws = torch.empty(need, dtype=torch.uint8, device=x.device)
        self.ws = ws
        self.masks = masks
        self.counts = counts

    def launch_names(self):
        lib = self.lib
        args = (self.shape, self.arr, len(self.blocks), self.dtype, self.flags,
                1 if self.x.data_ptr() == self.y.data_ptr() else 0)
        total = lib.dynconv_stack_launch_names(*args, None, 0)
        if total < 0:
            raise DynconvError("dynconv_stack_launch_names rejected the stack")
        names = (ctypes.c_char_p * total)()
        lib.dynconv_stack_launch_names(*args, names, total)
        return [n.decode() for n in names]

    def _args(self, stream):
        return (_ptr(self.x), _ptr(self.y), self.shape, self.dtype, self.arr, len(self.blocks),
                self.flags, _ptr(self.masks), _ptr(self.counts), _ptr(self.ws),
                self.ws.numel() * self.ws.element_size(), _stream(stream))

    def __call__(self, stream=None):
        _check(self.lib.dynconv_stack_forward(*self._args(stream)), "dynconv_stack_forward")
        return self.y

    def profiled(self, events, stream=None):
        """Same call, with launch i timed by the raw HIP events
        (events[2i], events[2i+1]); len(events) >= 2 * number of launches."""
        arr = (ctypes.c_void_p * len(events))(*events)
        _check(self.lib.dynconv_stack_forward_profiled(*self._args(stream), arr, len(events)),
               "dynconv_stack_forward_profiled")
        return self.y


def stack_forward(x: torch.Tensor, y: torch.Tensor, blocks, flags=0, masks=None, counts=None,
                  ws=None, stream=None):
    return Stack(x, y, blocks, flags, masks, counts, ws)(stream)


def stack_noalloc_max_workspace_bytes() -> int:
    return int(load().dynconv_stack_noalloc_max_workspace_bytes())


def stack_forward_noalloc(x: torch.Tensor, y: torch.Tensor, blocks, flags=0, masks=None, counts=None,
                          stream=None):
    """dynconv_stack_forward_noalloc: the stack call on the library's static
    per-device scratch array instead of a caller workspace."""
    lib = load()
    arr = _blocks_array(blocks)
    _check(lib.dynconv_stack_forward_noalloc(_ptr(x), _ptr(y), shape_of(x), dtype_code(x.dtype), arr,
                                             len(blocks), int(flags), _ptr(masks), _ptr(counts),
                                             _stream(stream)),
           "dynconv_stack_forward_noalloc")
    return y


class ShuffleStack:
    """A prepared ShuffleNetV2 unit stack y = units(x) (dynconv_shuffle_stack_forward);
    `branches` are BlockWeights on the padded channel counts (padded_branch_arrays).
    x and y must not overlap."""

    def __init__(self, x: torch.Tensor, y: torch.Tensor, branches, flags=0, masks=None, counts=None,
                 ws=None):
        self.lib = load()
        self.x, self.y = x, y
        self.branches = list(branches)
        self.arr = _blocks_array(self.branches)
        self.shape = shape_of(x)
        self.dtype = dtype_code(x.dtype)
        self.flags = int(flags)
        need = self.lib.dynconv_shuffle_stack_workspace_bytes(self.shape, self.arr, len(self.branches),
                                                              self.dtype, self.flags)
        if need == 0:
            raise DynconvError("dynconv_shuffle_stack_workspace_bytes rejected the units")
        if ws is None:
            ws = torch.empty(need, dtype=torch.uint8, device=x.device)
        self.ws = ws
        self.masks = masks
        self.counts = counts

    def launch_names(self):
        lib = self.lib
        args = (self.shape, self.arr, len(self.branches), self.dtype, self.flags)
        total = lib.dynconv_shuffle_stack_launch_names(*args, None, 0)
        if total < 0:
            raise DynconvError("dynconv_shuffle_stack_launch_names rejected the units")
        names = (ctypes.c_char_p * total)()
        lib.dynconv_shuffle_stack_launch_names(*args, names, total)
        return [n.decode() for n in names]

    def _args(self, stream):
        return (_ptr(self.x), _ptr(self.y), self.shape, self.dtype, self.arr, len(self.branches),
                self.flags, _ptr(self.masks), _ptr(self.counts), _ptr(self.ws),
                self.ws.numel() * self.ws.element_size(), _stream(stream))

    def __call__(self, stream=None):
        _check(self.lib.dynconv_shuffle_stack_forward(*self._args(stream)), "dynconv_shuffle_stack_forward")
        return self.y

    def profiled(self, events, stream=None):
        arr = (ctypes.c_void_p * len(events))(*events)
        _check(self.lib.dynconv_shuffle_stack_forward_profiled(*self._args(stream), arr, len(events)),
               "dynconv_shuffle_stack_forward_profiled")
        return self.y


class NetworkWeights:
    """Device copies of a layer list (dicts as paper_1912_03203_amd.inputs
    builds them) and the C layer array pointing at them; gated blocks get
    their mask biases from `biases` (one per gated block, in order)."""

    def __init__(self, layers, dtype, biases=None, device="cuda"):
        self.keep = []
        self.arr = (Layer * len(layers))()
        gi = 0

        def dev(a, dt):
            t = torch.as_tensor(a).to(device=device, dtype=dt).contiguous()
            self.keep.append(t)
            return t

        for i, L in enumerate(layers):
            if L["kind"] in ("conv3x3", "conv1x1"):
                w = dev(L["w"], dtype)
                b = dev(L["b"], torch.float32)
                kind = LAYER_CONV3X3 if L["kind"] == "conv3x3" else LAYER_CONV1X1
                self.arr[i] = Layer(kind, int(L.get("stride", 1)), 0, int(w.shape[1]), int(w.shape[0]),
                                    w.data_ptr(), b.data_ptr(), int(L["act"]), Block())
                continue
            acts = L.get("acts", (ACT_RELU6, ACT_RELU6, ACT_NONE))
            w2 = dev(L["w2"], dtype).reshape(-1, 9).contiguous()
            self.keep.append(w2)
            b2 = dev(L["b2"], torch.float32)
            w3 = dev(L["w3"], dtype)
            b3 = dev(L["b3"], torch.float32)
            E = int(w2.shape[0])
            c_out = int(w3.shape[0])
            if L.get("w1") is not None:
                w1 = dev(L["w1"], dtype)
                b1 = dev(L["b1"], torch.float32)
                c_in, w1p, b1p = int(w1.shape[1]), w1.data_ptr(), b1.data_ptr()
            else:
                c_in, w1p, b1p = E, None, None
            gated = 1 if L.get("gated") else 0
            wm_p, bm = None, 0.0
            if gated:
                wm = dev(L["w_m"], torch.float32)
                wm_p = wm.data_ptr()
                bm = float(biases[gi]) if biases is not None else 0.0
                gi += 1
            blk = Block(c_in, E, c_out, w1p, b1p, w2.data_ptr(), b2.data_ptr(), w3.data_ptr(), b3.data_ptr(),
                        int(acts[0]), int(acts[1]), int(acts[2]), wm_p, bm)
            self.arr[i] = Layer(LAYER_BLOCK, int(L["stride"]), gated, c_in, c_out, None, None, 0, blk)
        self.n = len(layers)
        self.ngated = gi if biases is not None else sum(1 for L in layers if L.get("gated"))

    def set_bias(self, gated_index, value):
        gi = 0
        for i in range(self.n):
            if self.arr[i].gated:
                if gi == gated_index:
                    self.arr[i].blk.b_mask = float(value)
                    return
                gi += 1
        raise IndexError(gated_index)


def network_output_shape(shape: Shape, net: NetworkWeights) -> Shape:
    out = Shape()
    _check(load().dynconv_network_output_shape(shape, net.arr, net.n, ctypes.byref(out)),
           "dynconv_network_output_shape")
    return out


class Network:
    """A prepared whole-network call y = layers(x) (dynconv_network_forward).
    x and y must not overlap; y has the shape network_output_shape gives."""

    def __init__(self, x: torch.Tensor, y: torch.Tensor, net: NetworkWeights, flags=0, masks=None, counts=None,
                 ws=None):
        self.lib = load()
        self.x, self.y, self.net = x, y, net
        self.shape = shape_of(x)
        self.dtype = dtype_code(x.dtype)
        self.flags = int(flags)
        need = self.lib.dynconv_network_workspace_bytes(self.shape, net.arr, net.n, self.dtype, self.flags)
        if need == 0:
            raise DynconvError("dynconv_network_workspace_bytes rejected the network")
        self.ws = torch.empty(need, dtype=torch.uint8, device=x.device) if ws is None else ws
        self.masks = masks
        self.counts = counts

    def launch_names(self):
        args = (self.shape, self.net.arr, self.net.n, self.dtype, self.flags, 1 if self.counts is not None else 0)
        total = self.lib.dynconv_network_launch_names(*args, None, 0)
        if total < 0:
            raise DynconvError("dynconv_network_launch_names rejected the network")
        names = (ctypes.c_char_p * total)()
        self.lib.dynconv_network_launch_names(*args, names, total)
        return [n.decode() for n in names]

    def _args(self, stream):
        return (_ptr(self.x), _ptr(self.y), self.shape, self.dtype, self.net.arr, self.net.n, self.flags,
                _ptr(self.masks), _ptr(self.counts), _ptr(self.ws), self.ws.numel() * self.ws.element_size(),
                _stream(stream))

    def __call__(self, stream=None):
        _check(self.lib.dynconv_network_forward(*self._args(stream)), "dynconv_network_forward")
        return self.y

    def profiled(self, events, stream=None):
        arr = (ctypes.c_void_p * len(events))(*events)
        _check(self.lib.dynconv_network_forward_profiled(*self._args(stream), arr, len(events)),
               "dynconv_network_forward_profiled")
        return self.y


# ---------------------------------------------------------- token operators
ACT_SILU, ACT_GELU = 3, 4
ROUTE_SIGMOID, ROUTE_RENORMALIZE, ROUTE_SCORE_BIAS = 1, 2, 8
EXPERTS_RESIDUAL = 1


class RoutesStruct(ctypes.Structure):
    _fields_ = [("expert", ctypes.c_void_p), ("weight", ctypes.c_void_p), ("rows", ctypes.c_void_p),
                ("starts", ctypes.c_void_p), ("capacity", ctypes.c_int64)]


class LinearStruct(ctypes.Structure):
    _fields_ = [("c_in", ctypes.c_int32), ("c_out", ctypes.c_int32), ("w", ctypes.c_void_p), ("b", ctypes.c_void_p),
                ("act", ctypes.c_int32)]


class ExpertsStruct(ctypes.Structure):
    _fields_ = [("c_in", ctypes.c_int32), ("c_hidden", ctypes.c_int32), ("c_out", ctypes.c_int32),
                ("experts", ctypes.c_int32), ("w_expand", ctypes.c_void_p), ("b_expand", ctypes.c_void_p),
                ("w_gate", ctypes.c_void_p), ("b_gate", ctypes.c_void_p), ("w_project", ctypes.c_void_p),
                ("b_project", ctypes.c_void_p), ("act", ctypes.c_int32)]


class AdaptersStruct(ctypes.Structure):
    _fields_ = [("adapters", ctypes.c_int32), ("max_rank", ctypes.c_int32), ("down", ctypes.c_void_p),
                ("up", ctypes.c_void_p), ("ranks", ctypes.c_void_p), ("scales", ctypes.c_void_p)]


def _declare_tokens(lib):
    vp, sz, i32, i64, ci = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32, ctypes.c_int64, ctypes.c_int
    p = ctypes.POINTER
    for name, res, args in (
            ("dynconv_route_workspace_bytes", sz, [i64, i32, i32]),
            ("dynconv_route", ci, [vp, i64, ci, i32, i32, vp, vp, i32, ctypes.c_float, p(RoutesStruct), vp, sz, vp]),
            ("dynconv_grouped_linear", ci, [vp, i64, vp, i64, ci, p(LinearStruct), i32, vp, i64, vp, i32, vp, vp]),
            ("dynconv_experts_workspace_bytes", sz, [i64, p(ExpertsStruct), ci, i32]),
            ("dynconv_experts_forward", ci, [vp, vp, i64, ci, p(ExpertsStruct), i32, p(RoutesStruct), i32, vp, sz, vp]),
            ("dynconv_adapter_workspace_bytes", sz, [i64, p(LinearStruct), p(AdaptersStruct), ci]),
            ("dynconv_adapter_linear", ci, [vp, vp, i64, ci, p(LinearStruct), p(AdaptersStruct), vp, vp, sz, vp])):
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = res, args


def _need(t, name, dtype, shape, like):
    """t is a dense tensor of this dtype and shape (None: any size) on like's device."""
    if not isinstance(t, torch.Tensor):
        raise DynconvError("%s: a tensor is needed" % name)
    if t.dtype != dtype:
        raise DynconvError("%s: dtype %s, not %s" % (name, dtype, t.dtype))
    if t.dim() != len(shape) or any(w is not None and n != w for n, w in zip(t.shape, shape)):
        raise DynconvError("%s: shape %s, not %s" % (name, tuple(shape), tuple(t.shape)))
    if not t.is_contiguous():
        raise DynconvError("%s: the tensor is not contiguous" % name)
    if t.device != like.device:
        raise DynconvError("%s: on %s, not on %s" % (name, t.device, like.device))


def _storage(x, name):
    if not isinstance(x, torch.Tensor) or x.dtype not in _CODE:
        raise DynconvError("%s: an fp32, fp16 or bf16 tensor is needed" % name)


def _int32(v, name):
    """v as it reaches the library: ctypes would cut a larger number to 32 bits."""
    try:
        n = int(v)
    except (TypeError, ValueError, OverflowError):
        n = None
    if n is None or n != v:
        raise DynconvError("%s: a whole number is needed, not %r" % (name, v))
    if not -2**31 <= n < 2**31:
        raise DynconvError("%s: %d does not fit in 32 bits" % (name, n))
    return n


class _Prepared:
    """A call marshalled once: calling it enqueues it on `stream` (default: the
    current stream of the tensors' device).  The object holds its tensors and its
    workspace, so it has to live until its work is done, and calls of one object
    must not overlap in time."""

    def _prepare(self, device, fn, name, args):
        if device.type != "cuda":
            raise DynconvError("%s: the tensors are on %s, not on a GPU" % (name, device))
        self._device, self._fn, self._name, self._cargs = device, fn, name, args
        self._index = device.index if device.index is not None else torch.cuda.current_device()

    def __call__(self, stream=None):
        if stream is not None and stream.device.index != self._index:
            raise DynconvError("%s: the stream is on another device" % self._name)
        if torch.cuda.current_device() == self._index:
            return self._enqueue(stream)
        with torch.cuda.device(self._index):
            return self._enqueue(stream)

    def _enqueue(self, stream):
        handle = (stream if stream is not None else torch.cuda.current_stream(self._index)).cuda_stream
        code = self._fn(*self._cargs, handle)
        if code != 0:
            _check(code, self._name)
        return self._result()


def _scratch(nbytes, ws, device, name):
    if nbytes == 0:
        raise DynconvError("%s rejected the arguments" % name)
    if ws is None:
        return torch.empty(nbytes, dtype=torch.uint8, device=device)
    if ws.device != device or not ws.is_contiguous():
        raise DynconvError("ws: a contiguous tensor on %s is needed" % device)
    return ws


def _tensors(d):
    """The tensors of a dataclass as they are now: its fields may be given others."""
    return tuple(t for t in vars(d).values() if isinstance(t, torch.Tensor))


def _raw(t):
    return None if t is None or t.numel() == 0 else t.data_ptr()


@dataclass
class Routes:
    """A router's result (dynconv_routes): expert [T, k] int32, weight [T, k]
    fp32, rows [T * k] int32, starts [experts + 1] int32."""

    expert: torch.Tensor
    weight: torch.Tensor
    rows: torch.Tensor
    starts: torch.Tensor

    @classmethod
    def alloc(cls, tokens: int, experts: int, top_k: int, device="cuda"):
        def new(shape, dtype):
            return torch.empty(shape, dtype=dtype, device=device)

        return cls(new((tokens, top_k), torch.int32), new((tokens, top_k), torch.float32),
                   new((tokens * top_k,), torch.int32), new((experts + 1,), torch.int32))

    def check(self, tokens, experts, top_k, like):
        _need(self.expert, "expert", torch.int32, (tokens, top_k), like)
        _need(self.weight, "weight", torch.float32, (tokens, top_k), like)
        _need(self.rows, "rows", torch.int32, (tokens * top_k,), like)
        _need(self.starts, "starts", torch.int32, (experts + 1,), like)

    def struct(self) -> RoutesStruct:
        return RoutesStruct(_raw(self.expert), _raw(self.weight), _raw(self.rows), _raw(self.starts), self.rows.numel())


class Router(_Prepared):
    """A prepared dynconv_route call: logits [T, experts] -> Routes.  bias is added to
    the logits, or with ROUTE_SCORE_BIAS to the scores (a balancing bias); it decides
    who is chosen and does not count in the weights."""

    def __init__(self, logits, top_k, bias=None, mask=None, flags=0, scale=1.0, routes=None, ws=None):
        lib = load()
        _storage(logits, "logits")
        _need(logits, "logits", logits.dtype, (None, None), logits)
        tokens, experts = logits.shape
        top_k, flags = _int32(top_k, "top_k"), _int32(flags, "flags")
        if bias is not None:
            _need(bias, "bias", torch.float32, (experts,), logits)
        if mask is not None:
            _need(mask, "mask", torch.uint8, (tokens,), logits)
        nbytes = lib.dynconv_route_workspace_bytes(tokens, experts, top_k)
        self.ws = _scratch(nbytes, ws, logits.device, "dynconv_route_workspace_bytes")
        self.routes = Routes.alloc(tokens, experts, top_k, logits.device) if routes is None else routes
        self.routes.check(tokens, experts, top_k, logits)
        self.keep = (logits, bias, mask) + _tensors(self.routes)
        self.struct = self.routes.struct()
        self._prepare(logits.device, lib.dynconv_route, "dynconv_route",
                      (_raw(logits), tokens, dtype_code(logits.dtype), experts, top_k, _raw(bias), _raw(mask),
                       flags, float(scale), ctypes.byref(self.struct), self.ws.data_ptr(),
                       self.ws.numel() * self.ws.element_size()))

    def _result(self):
        return self.routes


def route(logits, top_k, bias=None, mask=None, flags=0, scale=1.0, stream=None) -> Routes:
    """One dynconv_route call on new buffers of `stream`."""
    return _once(Router, stream, logits, top_k, bias, mask, flags, scale)


def _once(kind, stream, x, *args, **kw):
    """A prepared call made, run and dropped: what it allocates belongs to the stream
    it runs on, and what it was given is not used again before that stream is done."""
    if not isinstance(x, torch.Tensor) or not x.is_cuda:
        raise DynconvError("a device tensor is needed")
    with torch.cuda.device(x.device):
        if stream is None:
            return kind(x, *args, **kw)()
        with torch.cuda.stream(stream):
            call = kind(x, *args, **kw)
            for t in call.keep:
                if t is not None:
                    t.record_stream(stream)
            return call(stream)


class GroupedLinear(_Prepared):
    """A prepared dynconv_grouped_linear call: position p of group g, for
    starts[g] <= p < starts[g + 1], is y[dst[p]] = act(w[g] x[src[p] // src_div] + b[g])
    (without src or dst: row p)."""

    def __init__(self, x, y, w, b, starts, src=None, src_div=1, dst=None, act=ACT_NONE):
        lib = load()
        _storage(x, "x")
        _need(w, "w", x.dtype, (None, None, None), x)
        groups, c_out, c_in = w.shape
        _need(x, "x", x.dtype, (None, c_in), x)
        _need(y, "y", x.dtype, (None, c_out), x)
        _need(starts, "starts", torch.int32, (groups + 1,), x)
        if b is not None:
            _need(b, "b", torch.float32, (groups, c_out), x)
        rows = min(x.shape[0], y.shape[0])
        for name, t in (("src", src), ("dst", dst)):
            if t is not None:
                _need(t, name, torch.int32, (None,), x)
                rows = t.numel()
        if src is not None and dst is not None and src.numel() != dst.numel():
            raise DynconvError("src and dst: %d and %d positions" % (src.numel(), dst.numel()))
        self.y = y
        self.keep = (x, y, w, b, starts, src, dst)
        self.linear = LinearStruct(c_in, c_out, _raw(w), _raw(b), _int32(act, "act"))
        src_div = _int32(src_div, "src_div")
        self._prepare(x.device, lib.dynconv_grouped_linear, "dynconv_grouped_linear",
                      (_raw(x), x.shape[0], _raw(y), y.shape[0], dtype_code(x.dtype), ctypes.byref(self.linear), groups,
                       _raw(starts), rows, _raw(src), src_div, _raw(dst)))

    def _result(self):
        return self.y


def grouped_linear(x, y, w, b, starts, src=None, src_div=1, dst=None, act=ACT_NONE, stream=None):
    return _once(GroupedLinear, stream, x, y, w, b, starts, src, src_div, dst, act)


@dataclass
class ExpertWeights:
    """An expert layer's weights (dynconv_experts): w_expand, w_gate
    [experts, hidden, c_in], w_project [experts, c_out, hidden] in the storage
    dtype; fp32 biases or None."""

    w_expand: torch.Tensor
    w_project: torch.Tensor
    w_gate: torch.Tensor = None
    b_expand: torch.Tensor = None
    b_gate: torch.Tensor = None
    b_project: torch.Tensor = None
    act: int = ACT_SILU

    def check(self, x):
        _need(self.w_expand, "w_expand", x.dtype, (None, None, None), x)
        n, h, c = self.w_expand.shape
        _need(x, "x", x.dtype, (None, c), x)
        _need(self.w_project, "w_project", x.dtype, (n, None, h), x)
        if self.w_gate is not None:
            _need(self.w_gate, "w_gate", x.dtype, (n, h, c), x)
        elif self.b_gate is not None:
            raise DynconvError("b_gate without w_gate")
        for name, width in (("b_expand", h), ("b_gate", h), ("b_project", self.w_project.shape[1])):
            t = getattr(self, name)
            if t is not None:
                _need(t, name, torch.float32, (n, width), x)

    def struct(self) -> ExpertsStruct:
        n, h, c = self.w_expand.shape
        return ExpertsStruct(c, h, self.w_project.shape[1], n, _raw(self.w_expand), _raw(self.b_expand),
                             _raw(self.w_gate), _raw(self.b_gate), _raw(self.w_project), _raw(self.b_project),
                             _int32(self.act, "act"))


class Experts(_Prepared):
    """A prepared dynconv_experts_forward call; y may be x (in place)."""

    def __init__(self, x, y, weights: ExpertWeights, routes: Routes, flags=0, ws=None):
        lib = load()
        _storage(x, "x")
        weights.check(x)
        tokens, experts = x.shape[0], weights.w_expand.shape[0]
        _need(y, "y", x.dtype, (tokens, weights.w_project.shape[1]), x)
        top_k = routes.expert.shape[-1]
        routes.check(tokens, experts, top_k, x)
        flags = _int32(flags, "flags")
        self.struct, self.rstruct = weights.struct(), routes.struct()
        code = dtype_code(x.dtype)
        nbytes = lib.dynconv_experts_workspace_bytes(tokens, ctypes.byref(self.struct), code, top_k)
        self.ws = _scratch(nbytes, ws, x.device, "dynconv_experts_workspace_bytes")
        self.y = y
        self.keep = (x, y) + _tensors(weights) + _tensors(routes)
        self._prepare(x.device, lib.dynconv_experts_forward, "dynconv_experts_forward",
                      (_raw(x), _raw(y), tokens, code, ctypes.byref(self.struct), top_k, ctypes.byref(self.rstruct),
                       flags, self.ws.data_ptr(), self.ws.numel() * self.ws.element_size()))

    def _result(self):
        return self.y


def experts_forward(x, y, weights: ExpertWeights, routes: Routes, flags=0, stream=None):
    return _once(Experts, stream, x, y, weights, routes, flags)


@dataclass
class Adapters:
    """Low-rank adapters (dynconv_adapters): down [n, max_rank, c_in], up
    [n, c_out, max_rank] in the storage dtype, scales fp32 [n] or None, ranks
    int32 [n] or None."""

    down: torch.Tensor
    up: torch.Tensor
    scales: torch.Tensor = None
    ranks: torch.Tensor = None

    def check(self, x, c_out):
        _need(self.down, "down", x.dtype, (None, None, x.shape[1]), x)
        n, rank, _ = self.down.shape
        _need(self.up, "up", x.dtype, (n, c_out, rank), x)
        if self.scales is not None:
            _need(self.scales, "scales", torch.float32, (n,), x)
        if self.ranks is not None:
            _need(self.ranks, "ranks", torch.int32, (n,), x)

    def struct(self) -> AdaptersStruct:
        return AdaptersStruct(self.down.shape[0], self.down.shape[1], _raw(self.down), _raw(self.up), _raw(self.ranks),
                              _raw(self.scales))


class AdapterLinear(_Prepared):
    """A prepared dynconv_adapter_linear call:
    y[r] = act(w x[r] + b + scales[i] * up[i] (down[i] x[r])), i = ids[r]."""

    def __init__(self, x, y, w, b, adapters: Adapters, ids, act=ACT_NONE, ws=None):
        lib = load()
        _storage(x, "x")
        _need(w, "w", x.dtype, (None, None), x)
        c_out, c_in = w.shape
        _need(x, "x", x.dtype, (None, c_in), x)
        rows = x.shape[0]
        _need(y, "y", x.dtype, (rows, c_out), x)
        _need(ids, "ids", torch.int32, (rows,), x)
        if b is not None:
            _need(b, "b", torch.float32, (c_out,), x)
        adapters.check(x, c_out)
        self.linear = LinearStruct(c_in, c_out, _raw(w), _raw(b), _int32(act, "act"))
        self.struct = adapters.struct()
        code = dtype_code(x.dtype)
        nbytes = lib.dynconv_adapter_workspace_bytes(rows, ctypes.byref(self.linear), ctypes.byref(self.struct), code)
        self.ws = _scratch(nbytes, ws, x.device, "dynconv_adapter_workspace_bytes")
        self.y = y
        self.keep = (x, y, w, b, ids) + _tensors(adapters)
        self._prepare(x.device, lib.dynconv_adapter_linear, "dynconv_adapter_linear",
                      (_raw(x), _raw(y), rows, code, ctypes.byref(self.linear), ctypes.byref(self.struct), _raw(ids),
                       self.ws.data_ptr(), self.ws.numel() * self.ws.element_size()))

    def _result(self):
        return self.y


def adapter_linear(x, y, w, b, adapters: Adapters, ids, act=ACT_NONE, stream=None):
    return _once(AdapterLinear, stream, x, y, w, b, adapters, ids, act)
