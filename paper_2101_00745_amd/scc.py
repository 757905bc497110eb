"""Thin Python binding of the SCC C ABI (include/scc.h): argument marshalling only, the everyday calls in native code
(csrc/binding/scc_binding.cpp), all others here through ctypes.

Every step of the computation runs in the HIP kernels of libscc_hip.so.  PyTorch supplies
device memory (``torch.empty``), raw pointers (``data_ptr``) and the current HIP stream,
nothing else.  There is no CPU path: if the library is missing or a tensor is not on the
GPU the call raises.
"""
import ctypes
import functools
import math
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libscc_hip.so")

SCC_F32, SCC_BF16 = 0, 1
SCC_ERR_SHAPE, SCC_ERR_LAUNCH, SCC_ERR_OPTION = -2, -6, -8
SYMBOLS = ("scc_window_params", "scc_forward", "scc_forward_workspace_bytes", "scc_forward_ws", "scc_backward_input",
           "scc_backward_input_workspace_bytes", "scc_backward_input_ws",
           "scc_backward_weight_workspace_bytes", "scc_backward_weight", "scc_backward_weight_static",
           "scc_backward_workspace_bytes", "scc_backward", "scc_forward_path", "scc_backward_weight_path", "scc_backward_path",
           "scc_depthwise3x3_out", "scc_depthwise3x3_forward", "scc_depthwise3x3_backward_workspace_bytes",
           "scc_depthwise3x3_backward", "scc_dw_forward_workspace_bytes", "scc_dw_forward_fusable", "scc_dw_forward",
           "scc_dw_forward_scratch", "scc_dw_forward_path", "scc_dw_forward_scratch_path",
           "scc_dw_backward_workspace_bytes", "scc_dw_backward", "scc_dw_backward_as_workspace_bytes", "scc_dw_backward_as",
           "scc_gated_forward_workspace_bytes", "scc_gated_forward_path", "scc_gated_forward", "scc_gated_backward_workspace_bytes",
           "scc_gated_backward", "scc_orthogonal_workspace_bytes", "scc_orthogonalise", "scc_orthogonal_step",
           "scc_norm_forward", "scc_norm_quantised", "scc_norm_backward_workspace_bytes", "scc_norm_backward",
           "scc_vocabulary_loss_workspace_bytes", "scc_vocabulary_loss", "scc_vocabulary_gradients_workspace_bytes",
           "scc_vocabulary_gradients", "scc_adamw_step", "scc_status_string")
ACTIVATIONS = {"silu": 0, "gelu": 1}    # scc_activation of include/scc.h
REDUCTIONS = {"none": 0, "sum": 1, "mean": 2}    # scc_reduction of include/scc.h
STATE_BLOCK = 256                       # elements of a scale of AdamW's states in 8 bits
MOST_ADAMW = 1 << 34                    # elements of a weight that scc_adamw_step takes
STATIC_SCRATCH_BYTES = 32 << 20    # SCC_STATIC_SCRATCH_BYTES of include/scc.h

_lib = None
_native = None      # the module of the plain calls


class _OrthogonalOptions(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_float), ("momentum", ctypes.c_float), ("weight_decay", ctypes.c_float), ("nesterov", ctypes.c_int),
                ("steps", ctypes.c_int), ("a", ctypes.c_float), ("b", ctypes.c_float), ("c", ctypes.c_float), ("eps", ctypes.c_float)]


class _AdamwOptions(ctypes.Structure):
    _fields_ = [(name, ctypes.c_double) for name in ("lr", "beta1", "beta2", "eps", "weight_decay")] + [("seed", ctypes.c_uint64)]


class SccError(RuntimeError):
    def __init__(self, status, message):
        super().__init__(message)
        self.status = status


def load():
    """Load libscc_hip.so (built in-tree by ``paper_2101_00745_amd.build``)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError("libscc_hip.so is not built: run `python -m paper_2101_00745_amd.build` "
                          "(or __graft_entry__.build()) first; there is no fallback path")
    lib = ctypes.CDLL(LIB_PATH)
    c_int, c_dbl, c_vp, c_sz = ctypes.c_int, ctypes.c_double, ctypes.c_void_p, ctypes.c_size_t
    ip = ctypes.POINTER(c_int)
    shape = [c_int, c_int, c_int, c_int, c_int, c_int, c_dbl, c_int]  # N Cin Cout H W cg co dtype
    lib.scc_window_params.argtypes = [c_int, c_int, c_int, c_dbl, ip, ip, ip]
    lib.scc_window_params.restype = c_int
    lib.scc_forward.argtypes = [c_vp, c_vp, c_vp] + shape + [c_vp]
    lib.scc_forward.restype = c_int
    lib.scc_backward_input.argtypes = [c_vp, c_vp, c_vp] + shape + [c_vp]
    lib.scc_backward_input.restype = c_int
    for name in ("scc_forward", "scc_backward_input"):
        query, call = getattr(lib, name + "_workspace_bytes"), getattr(lib, name + "_ws")
        query.argtypes, query.restype = shape, c_sz
        call.argtypes, call.restype = [c_vp, c_vp, c_vp] + shape + [c_vp, c_sz, c_vp], c_int
    lib.scc_backward_weight_workspace_bytes.argtypes = shape
    lib.scc_backward_weight_workspace_bytes.restype = c_sz
    lib.scc_backward_weight.argtypes = [c_vp, c_vp, c_vp] + shape + [c_vp, c_sz, c_vp]
    lib.scc_backward_weight.restype = c_int
    lib.scc_backward_workspace_bytes.argtypes = shape
    lib.scc_backward_workspace_bytes.restype = c_sz
    lib.scc_backward.argtypes = [c_vp] * 5 + shape + [c_vp, c_sz, c_vp]
    lib.scc_backward.restype = c_int
    for name in ("scc_forward_path", "scc_backward_weight_path", "scc_backward_path"):
        getattr(lib, name).argtypes, getattr(lib, name).restype = shape + [c_sz], c_int
    lib.scc_backward_weight_static.argtypes = [c_vp, c_vp, c_vp] + shape + [c_vp]
    lib.scc_backward_weight_static.restype = c_int
    lib.scc_depthwise3x3_out.argtypes = [c_int, c_int]
    lib.scc_depthwise3x3_out.restype = c_int
    lib.scc_depthwise3x3_forward.argtypes = [c_vp, c_vp, c_vp] + [c_int] * 6 + [c_vp]
    lib.scc_depthwise3x3_forward.restype = c_int
    lib.scc_depthwise3x3_backward_workspace_bytes.argtypes = [c_int] * 6
    lib.scc_depthwise3x3_backward_workspace_bytes.restype = c_sz
    lib.scc_depthwise3x3_backward.argtypes = [c_vp] * 5 + [c_int] * 6 + [c_vp, c_sz, c_vp]
    lib.scc_depthwise3x3_backward.restype = c_int
    dw_shape = [c_int] * 7 + [c_dbl, c_int]     # N, Cin, Cout, H, W, dw_stride, cg, co, dtype
    lib.scc_dw_forward_workspace_bytes.argtypes = dw_shape
    lib.scc_dw_forward_workspace_bytes.restype = c_sz
    lib.scc_dw_forward_fusable.argtypes = dw_shape
    lib.scc_dw_forward_fusable.restype = c_int
    lib.scc_dw_forward.argtypes = [c_vp] * 4 + dw_shape + [c_vp, c_sz, c_vp]
    lib.scc_dw_forward.restype = c_int
    lib.scc_dw_forward_scratch.argtypes = lib.scc_dw_forward.argtypes
    lib.scc_dw_forward_scratch.restype = c_int
    for query in (lib.scc_dw_forward_path, lib.scc_dw_forward_scratch_path):
        query.argtypes = dw_shape + [c_sz]
        query.restype = c_int
    lib.scc_dw_backward_workspace_bytes.argtypes = dw_shape
    lib.scc_dw_backward_workspace_bytes.restype = c_sz
    lib.scc_dw_backward.argtypes = [c_vp] * 7 + dw_shape + [c_vp, c_sz, c_vp]
    lib.scc_dw_backward.restype = c_int
    lib.scc_dw_backward_as_workspace_bytes.argtypes = dw_shape + [c_int]
    lib.scc_dw_backward_as_workspace_bytes.restype = c_sz
    lib.scc_dw_backward_as.argtypes = [c_vp] * 7 + dw_shape + [c_int, c_vp, c_sz, c_vp]
    lib.scc_dw_backward_as.restype = c_int
    lib.scc_gated_forward_workspace_bytes.argtypes = shape
    lib.scc_gated_forward_workspace_bytes.restype = c_sz
    lib.scc_gated_forward_path.argtypes = shape
    lib.scc_gated_forward_path.restype = c_int
    lib.scc_gated_forward.argtypes = [c_vp] * 3 + shape[:-1] + [c_int, c_int, c_vp, c_sz, c_vp]     # ... co act dtype
    lib.scc_gated_forward.restype = c_int
    lib.scc_gated_backward_workspace_bytes.argtypes = shape + [c_int]
    lib.scc_gated_backward_workspace_bytes.restype = c_sz
    lib.scc_gated_backward.argtypes = [c_vp] * 5 + shape[:-1] + [c_int, c_int, c_int, c_vp, c_sz, c_vp]
    lib.scc_gated_backward.restype = c_int
    vpp = ctypes.POINTER(c_vp)
    lib.scc_orthogonal_workspace_bytes.argtypes = [c_int, ip, ip]
    lib.scc_orthogonal_workspace_bytes.restype = c_sz
    for name, lists in (("scc_orthogonalise", 2), ("scc_orthogonal_step", 3)):
        call = getattr(lib, name)
        call.argtypes = [c_int] + [vpp] * lists + [ip, ip, ctypes.POINTER(_OrthogonalOptions), c_int, c_vp, c_sz, c_vp]
        call.restype = c_int
    c_float, c_ll = ctypes.c_float, ctypes.c_longlong
    maps = [c_int] * 4                  # N C H W
    lib.scc_norm_forward.argtypes = [c_vp] * 5 + maps + [c_float, c_int, c_vp]
    lib.scc_norm_quantised.argtypes = [c_vp] * 6 + maps + [c_float, c_int, c_vp]
    lib.scc_norm_backward_workspace_bytes.argtypes = maps + [c_int]
    lib.scc_norm_backward_workspace_bytes.restype = c_sz
    lib.scc_norm_backward.argtypes = [c_vp] * 7 + maps + [c_float, c_int, c_int, c_vp, c_sz, c_vp]
    lib.scc_vocabulary_loss_workspace_bytes.argtypes = maps + [c_int] * 3
    lib.scc_vocabulary_loss_workspace_bytes.restype = c_sz
    lib.scc_vocabulary_loss.argtypes = [c_vp] * 5 + maps + [c_int, c_ll, c_int, c_int, c_vp, c_sz, c_vp]
    lib.scc_vocabulary_gradients_workspace_bytes.argtypes = maps + [c_int] * 2
    lib.scc_vocabulary_gradients_workspace_bytes.restype = c_sz
    lib.scc_vocabulary_gradients.argtypes = [c_vp] * 7 + maps + [c_int, c_ll, c_int, c_int, c_int, c_vp, c_sz, c_vp]
    lib.scc_adamw_step.argtypes = [c_int] + [vpp] * 6 + [ctypes.POINTER(c_ll), ctypes.POINTER(_AdamwOptions), c_ll, c_vp, c_int, c_vp]
    for name in ("scc_norm_forward", "scc_norm_quantised", "scc_norm_backward", "scc_vocabulary_loss", "scc_vocabulary_gradients", "scc_adamw_step"):
        getattr(lib, name).restype = c_int
    lib.scc_status_string.argtypes = [c_int]
    lib.scc_status_string.restype = ctypes.c_char_p
    _lib = lib
    return lib


class _NoNative:
    """Finds no call plain."""

    @staticmethod
    def forward(*args):
        return None

    backward = dw_forward = dw_backward = dw_block = gated_forward = gated_backward = gated_block = orthogonalise = orthogonal_step = forward
    norm_forward = norm_quantised = norm_block = vocabulary_loss = vocabulary_block = adamw_step = adamw_fits = forward


def _load_native():
    """The plain calls: each answers None where a call is not plain (or fails, if it only reads its arguments), and the general way below
    it then goes on.  Where
    the module is not built, or not for this torch, every call takes that way: the same kernels, some microseconds more of host time."""
    global _native
    load()
    try:
        from . import _binding
        from .build import binding_tag
        if getattr(_binding, "built_for", None) != binding_tag():
            raise ImportError("built for " + getattr(_binding, "built_for", "another one"))
        _native = _binding
    except ImportError as e:
        import warnings
        _native = _NoNative
        warnings.warn("plain calls go through ctypes: the binding's native part is not built for this torch (%s); "
                      "`python -m paper_2101_00745_amd.build` builds it" % e, RuntimeWarning, stacklevel=3)
    return _native


def scc_status_string(status):
    return load().scc_status_string(int(status)).decode()


def _check(status):
    if status != 0:
        raise SccError(status, scc_status_string(status))


def scc_window_params(Cin, Cout, cg, co):
    """(L, stride, period) of Algorithm 1 for this layer; host only."""
    L, s, p = ctypes.c_int(), ctypes.c_int(), ctypes.c_int()
    _check(load().scc_window_params(Cin, Cout, cg, float(co), ctypes.byref(L), ctypes.byref(s), ctypes.byref(p)))
    return L.value, s.value, p.value


_CODES = {torch.float32: SCC_F32, torch.bfloat16: SCC_BF16}


def _dtype_code(t):
    code = _CODES.get(t.dtype)
    if code is None:
        raise TypeError("SCC tensors must be float32 or bfloat16, got %s" % t.dtype)
    return code


def _dev(*tensors):
    for t in tensors:
        if not t.is_cuda:
            raise ValueError("SCC tensors must live on the GPU (there is no CPU path)")
        if not t.is_contiguous():
            raise ValueError("SCC tensors must be dense and contiguous (NCHW)")
    dev = tensors[0].device
    for t in tensors[1:]:
        if t.device != dev:
            raise ValueError("SCC tensors must share one device")
    return dev


def _stream_address(index):
    return torch.cuda.current_stream(index).cuda_stream


# the address alone, without a Stream object around it; a torch that lacks this function still has the other way
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", _stream_address)


def _launch(dev, call, *args):
    """call(*args, current stream of dev) with dev as the current device.  A small layer's pass is bound by the host, so the
    device is switched only where it is another one and no Stream object is made (one 8x8 image, 32 channels, forward and
    scc_backward: 28 us with both, 22 without)."""
    index = dev.index
    if torch.cuda.current_device() == index:
        status = call(*args, _raw_stream(index))
    else:
        with torch.cuda.device(index):
            status = call(*args, _raw_stream(index))
    if status != 0:
        _check(status)


@functools.lru_cache(maxsize=4096)
def _workspace_need(query, *shape):
    """Bytes the library's query function of that name answers; it depends on its integer arguments and co alone."""
    return int(getattr(load(), query)(*shape))


def _moved(*tensors):
    """Tells autograd that tensors of the caller's (None: none given) have other values now, so that a graph which saved one is not run on
    them."""
    tensors = [t for t in tensors if t is not None]
    if tensors:
        torch.autograd.graph.increment_version(tensors)


def _scratch(need, dev, workspace=None):
    """(tensor to keep alive until the call has been enqueued, its address, its size); nothing where nothing is needed."""
    if workspace is None:
        if need == 0:
            return None, None, 0
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    return workspace, workspace.data_ptr(), workspace.numel() * workspace.element_size()


def scc_forward_workspace_bytes(N, Cin, Cout, H, W, cg, co, dtype=torch.float32):
    code = SCC_F32 if dtype == torch.float32 else SCC_BF16
    return int(load().scc_forward_workspace_bytes(N, Cin, Cout, H, W, cg, float(co), code))


def scc_forward(x, w, cg, co, out=None, workspace=None):
    """y = SCC(x; w): x [N,Cin,H,W], w [Cout,Cin//cg] -> y [N,Cout,H,W] (same dtype).  Layers that pack their weights take a
    workspace for it; without one it is allocated, unless `out` is given: such a call allocates nothing and runs the
    kernels that need none."""
    if out is None and workspace is None:
        y = (_native or _load_native()).forward(x, w, cg, co)
        if y is not None:
            return y
    dev = _dev(x, w)
    N, Cin, H, W = x.shape
    Cout = w.shape[0]
    if w.dtype != x.dtype or w.dim() != 2 or (cg >= 1 and Cin % cg == 0 and w.shape[1] != Cin // cg):
        raise ValueError("w must be [Cout, Cin//cg] with the dtype of x")
    y = x.new_empty((N, Cout, H, W)) if out is None else out
    if out is not None:
        _dev(out)
        assert out.shape == (N, Cout, H, W) and out.dtype == x.dtype
    shape = (N, Cin, Cout, H, W, cg, float(co), _dtype_code(x))
    need = _workspace_need("scc_forward_workspace_bytes", *shape) if workspace is None and out is None else 0
    ws, ws_ptr, ws_len = _scratch(need, dev, workspace)
    _launch(dev, load().scc_forward_ws, x.data_ptr(), w.data_ptr(), y.data_ptr(), *shape, ws_ptr, ws_len)
    _moved(out)
    return y


def scc_backward_input_workspace_bytes(N, Cin, Cout, H, W, cg, co, dtype=torch.float32):
    code = SCC_F32 if dtype == torch.float32 else SCC_BF16
    return int(load().scc_backward_input_workspace_bytes(N, Cin, Cout, H, W, cg, float(co), code))


def scc_backward_input(dy, w, Cin, cg, co, out=None, workspace=None):
    """dx from dy [N,Cout,H,W] and w [Cout,Cin//cg] -> dx [N,Cin,H,W].  out, workspace: as for scc_forward."""
    dev = _dev(dy, w)
    N, Cout, H, W = dy.shape
    if w.dtype != dy.dtype or w.dim() != 2 or w.shape[0] != Cout or \
            (cg >= 1 and Cin % cg == 0 and w.shape[1] != Cin // cg):
        raise ValueError("w must be [Cout, Cin//cg] with the dtype of dy")
    dx = dy.new_empty((N, Cin, H, W)) if out is None else out
    if out is not None:
        _dev(out)
        assert out.shape == (N, Cin, H, W) and out.dtype == dy.dtype
    shape = (N, Cin, Cout, H, W, cg, float(co), _dtype_code(dy))
    need = _workspace_need("scc_backward_input_workspace_bytes", *shape) if workspace is None and out is None else 0
    ws, ws_ptr, ws_len = _scratch(need, dev, workspace)
    _launch(dev, load().scc_backward_input_ws, dy.data_ptr(), w.data_ptr(), dx.data_ptr(), *shape, ws_ptr, ws_len)
    _moved(out)
    return dx


def scc_backward_weight_workspace_bytes(N, Cin, Cout, H, W, cg, co, dtype=torch.float32):
    code = SCC_F32 if dtype == torch.float32 else SCC_BF16
    return int(load().scc_backward_weight_workspace_bytes(N, Cin, Cout, H, W, cg, float(co), code))


def scc_backward_weight(x, dy, cg, co, out=None, workspace=None):
    """dw (float32 [Cout, Cin//cg]) from x [N,Cin,H,W] and dy [N,Cout,H,W]."""
    dev = _dev(x, dy)
    N, Cin, H, W = x.shape
    Cout = dy.shape[1]
    if dy.dtype != x.dtype or dy.shape != (N, Cout, H, W):
        raise ValueError("dy must be [N,Cout,H,W] with the dtype of x")
    shape = (N, Cin, Cout, H, W, cg, float(co), _dtype_code(x))
    need = _workspace_need("scc_backward_weight_workspace_bytes", *shape) if workspace is None else 0
    if workspace is None and need > 0:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    L = Cin // cg if cg >= 1 and Cin % cg == 0 else 1
    dw = torch.empty((Cout, L), dtype=torch.float32, device=dev) if out is None else out
    if out is not None:
        _dev(out)
        assert out.shape == (Cout, L) and out.dtype == torch.float32
    ws_ptr = workspace.data_ptr() if workspace is not None else None
    ws_len = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _launch(dev, load().scc_backward_weight, x.data_ptr(), dy.data_ptr(), dw.data_ptr(), *shape, ws_ptr, ws_len)
    _moved(out)
    return dw


def scc_backward_weight_static(x, dy, cg, co, out):
    """scc_backward_weight on the library's own static scratch: the call itself allocates nothing, so the
    caller passes the output tensor ``out`` (float32 [Cout, Cin//cg])."""
    dev = _dev(x, dy, out)
    N, Cin, H, W = x.shape
    Cout = dy.shape[1]
    if dy.dtype != x.dtype or dy.shape != (N, Cout, H, W):
        raise ValueError("dy must be [N,Cout,H,W] with the dtype of x")
    L = Cin // cg if cg >= 1 and Cin % cg == 0 else 1
    if out.shape != (Cout, L) or out.dtype != torch.float32:
        raise ValueError("out must be float32 [Cout, Cin//cg]")
    _launch(dev, load().scc_backward_weight_static, x.data_ptr(), dy.data_ptr(), out.data_ptr(), N, Cin, Cout, H, W, cg,
            float(co), _dtype_code(x))
    _moved(out)
    return out


def scc_backward_workspace_bytes(N, Cin, Cout, H, W, cg, co, dtype=torch.float32):
    code = SCC_F32 if dtype == torch.float32 else SCC_BF16
    return int(load().scc_backward_workspace_bytes(N, Cin, Cout, H, W, cg, float(co), code))


def scc_backward(x, dy, w, cg, co, out_dx=None, out_dw=None, workspace=None):
    """(dx, dw) of one layer in one call: x [N,Cin,H,W], dy [N,Cout,H,W], w [Cout,Cin//cg]."""
    if out_dx is None and out_dw is None and workspace is None:
        both = (_native or _load_native()).backward(x, dy, w, cg, co)
        if both is not None:
            return both
    dev = _dev(x, dy, w)
    N, Cin, H, W = x.shape
    Cout = dy.shape[1]
    if dy.dtype != x.dtype or dy.shape != (N, Cout, H, W):
        raise ValueError("dy must be [N,Cout,H,W] with the dtype of x")
    if w.dtype != x.dtype or w.dim() != 2 or w.shape[0] != Cout or \
            (cg >= 1 and Cin % cg == 0 and w.shape[1] != Cin // cg):
        raise ValueError("w must be [Cout, Cin//cg] with the dtype of x")
    shape = (N, Cin, Cout, H, W, cg, float(co), _dtype_code(x))
    need = _workspace_need("scc_backward_workspace_bytes", *shape) if workspace is None else 0
    if workspace is None and need > 0:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    L = Cin // cg if cg >= 1 and Cin % cg == 0 else 1
    dx = torch.empty_like(x) if out_dx is None else out_dx
    dw = torch.empty((Cout, L), dtype=torch.float32, device=dev) if out_dw is None else out_dw
    for o, shp, dt in ((out_dx, x.shape, x.dtype), (out_dw, (Cout, L), torch.float32)):
        if o is not None:
            _dev(o)
            assert o.shape == shp and o.dtype == dt
    ws_ptr = workspace.data_ptr() if workspace is not None else None
    ws_len = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _launch(dev, load().scc_backward, x.data_ptr(), dy.data_ptr(), w.data_ptr(), dx.data_ptr(), dw.data_ptr(), *shape,
            ws_ptr, ws_len)
    _moved(out_dx, out_dw)
    return dx, dw


def scc_depthwise3x3_out(size, dw_stride):
    """Rows (columns) the depthwise 3x3 stage produces from `size` rows at spatial stride `dw_stride`."""
    r = int(load().scc_depthwise3x3_out(int(size), int(dw_stride)))
    _check(min(r, 0))
    return r


def _out(size, dw_stride):
    """scc_depthwise3x3_out without a call into the library, which only speaks up where there is an error."""
    return (size - 1) // dw_stride + 1 if size > 0 and dw_stride >= 1 else scc_depthwise3x3_out(size, dw_stride)


def scc_depthwise3x3_forward(x, kdw, dw_stride=1, out=None):
    """z = DW3x3(x; kdw): x [N,C,H,W], kdw [C,3,3] -> z [N,C,Ho,Wo] (Eq. 2: centred taps, zero outside the map)."""
    dev = _dev(x, kdw)
    N, C, H, W = x.shape
    if kdw.dtype != x.dtype or tuple(kdw.shape) != (C, 3, 3):
        raise ValueError("kdw must be [C, 3, 3] with the dtype of x")
    dw_stride = int(dw_stride)
    Ho, Wo = _out(H, dw_stride), _out(W, dw_stride)
    z = x.new_empty((N, C, Ho, Wo)) if out is None else out
    if out is not None:
        _dev(out)
        assert out.shape == (N, C, Ho, Wo) and out.dtype == x.dtype
    _launch(dev, load().scc_depthwise3x3_forward, x.data_ptr(), kdw.data_ptr(), z.data_ptr(), N, C, H, W, dw_stride,
            _dtype_code(x))
    _moved(out)
    return z


def scc_depthwise3x3_backward(x, kdw, dz, dw_stride=1, need_dx=True, need_dk=True, out_dx=None, out_dk=None,
                              workspace=None):
    """(dx, dkdw) of the depthwise 3x3 stage: x [N,C,H,W], kdw [C,3,3], dz [N,C,Ho,Wo] -> dx like x, dkdw [C,3,3] float32.
    A gradient that is not needed comes back as None."""
    dev = _dev(x, kdw, dz)
    N, C, H, W = x.shape
    dw_stride = int(dw_stride)
    Ho, Wo = _out(H, dw_stride), _out(W, dw_stride)
    if kdw.dtype != x.dtype or tuple(kdw.shape) != (C, 3, 3):
        raise ValueError("kdw must be [C, 3, 3] with the dtype of x")
    if dz.dtype != x.dtype or tuple(dz.shape) != (N, C, Ho, Wo):
        raise ValueError("dz must be [N, C, Ho, Wo] with the dtype of x")
    if not (need_dx or need_dk):
        return None, None
    code = _dtype_code(x)
    need = _workspace_need("scc_depthwise3x3_backward_workspace_bytes", N, C, H, W, dw_stride, code) if need_dk else 0
    if workspace is None and need > 0:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    dx = (torch.empty_like(x) if out_dx is None else out_dx) if need_dx else None
    dk = (torch.empty((C, 3, 3), dtype=torch.float32, device=dev) if out_dk is None else out_dk) if need_dk else None
    for o, shp, dt in ((out_dx, x.shape, x.dtype), (out_dk, (C, 3, 3), torch.float32)):
        if o is not None:
            _dev(o)
            assert o.shape == shp and o.dtype == dt
    ws_ptr = workspace.data_ptr() if workspace is not None else None
    ws_len = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _launch(dev, load().scc_depthwise3x3_backward, x.data_ptr(), kdw.data_ptr(), dz.data_ptr(),
            dx.data_ptr() if dx is not None else None, dk.data_ptr() if dk is not None else None, N, C, H, W, dw_stride,
            code, ws_ptr, ws_len)
    _moved(out_dx if need_dx else None, out_dk if need_dk else None)
    return dx, dk


def scc_dw_forward_workspace_bytes(N, Cin, Cout, H, W, dw_stride, cg, co, dtype=torch.float32):
    code = SCC_F32 if dtype == torch.float32 else SCC_BF16
    return int(load().scc_dw_forward_workspace_bytes(N, Cin, Cout, H, W, int(dw_stride), cg, float(co), code))


def scc_dw_forward_fusable(N, Cin, Cout, H, W, dw_stride, cg, co, dtype=torch.float32):
    """True when the fused kernel can run the layer (it then also runs without a workspace)."""
    code = SCC_F32 if dtype == torch.float32 else SCC_BF16
    r = int(load().scc_dw_forward_fusable(N, Cin, Cout, H, W, int(dw_stride), cg, float(co), code))
    _check(min(r, 0))
    return r == 1


def scc_dw_forward(x, kdw, w, cg, co, dw_stride=1, out=None, workspace=None, fused=None):
    """y = SCC(DW3x3(x; kdw); w), the forward of a DW + SCC block: x [N,Cin,H,W], kdw [Cin,3,3], w [Cout,Cin//cg]
    -> y [N,Cout,Ho,Wo].  fused=None: the path the library prefers (a workspace is allocated when it asks for
    one); fused=True: no workspace is passed, so a kernel that needs none runs (the fused one, or the one for few columns) or
    the call is refused; fused=False: the two stages through a workspace, also where the library would fuse.  A `workspace`
    that is given holds the depthwise output afterwards wherever the library asks for one."""
    if fused is None and out is None and workspace is None:
        y = (_native or _load_native()).dw_forward(x, kdw, w, cg, co, dw_stride)
        if y is not None:
            return y
    dev = _dev(x, kdw, w)
    N, Cin, H, W = x.shape
    Cout = w.shape[0]
    if kdw.dtype != x.dtype or tuple(kdw.shape) != (Cin, 3, 3):
        raise ValueError("kdw must be [Cin, 3, 3] with the dtype of x")
    if w.dtype != x.dtype or w.dim() != 2 or (cg >= 1 and Cin % cg == 0 and w.shape[1] != Cin // cg):
        raise ValueError("w must be [Cout, Cin//cg] with the dtype of x")
    dw_stride = int(dw_stride)
    Ho, Wo = _out(H, dw_stride), _out(W, dw_stride)
    if fused is False:
        z = scc_depthwise3x3_forward(x, kdw, dw_stride)
        # an out tensor: no packing of the weights, as in the library's own two stages
        return scc_forward(z, w, cg, co, out=x.new_empty((N, Cout, Ho, Wo)) if out is None else out)
    shape = (N, Cin, Cout, H, W, dw_stride, cg, float(co), _dtype_code(x))
    need = _workspace_need("scc_dw_forward_workspace_bytes", *shape)
    call = load().scc_dw_forward
    if fused:
        workspace = None
    elif workspace is None and need > 0:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
        call = load().scc_dw_forward_scratch
    y = x.new_empty((N, Cout, Ho, Wo)) if out is None else out
    if out is not None:
        _dev(out)
        assert out.shape == (N, Cout, Ho, Wo) and out.dtype == x.dtype
    ws_ptr = workspace.data_ptr() if workspace is not None else None
    ws_len = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _launch(dev, call, x.data_ptr(), kdw.data_ptr(), w.data_ptr(), y.data_ptr(), *shape, ws_ptr, ws_len)
    _moved(out)
    return y


def scc_dw_backward(x, kdw, w, dy, cg, co, dw_stride=1):
    """(dx, dkdw, dw), all gradients of a DW + SCC block in one call: x [N,Cin,H,W], kdw [Cin,3,3], w [Cout,Cin//cg],
    dy [N,Cout,Ho,Wo]; dkdw and dw are float32."""
    return _dw_backward(x, kdw, w, dy, cg, co, dw_stride, False)


def _dw_backward(x, kdw, w, dy, cg, co, dw_stride, stored):
    """scc_dw_backward; stored: dkdw and dw in the type of x, rounded from the same sums."""
    grads = (_native or _load_native()).dw_backward(x, kdw, w, dy, cg, co, dw_stride, stored)
    if grads is not None:
        return grads
    dev = _dev(x, kdw, w, dy)
    N, Cin, H, W = x.shape
    Cout = w.shape[0]
    if kdw.dtype != x.dtype or tuple(kdw.shape) != (Cin, 3, 3):
        raise ValueError("kdw must be [Cin, 3, 3] with the dtype of x")
    if w.dtype != x.dtype or w.dim() != 2 or (cg >= 1 and Cin % cg == 0 and w.shape[1] != Cin // cg):
        raise ValueError("w must be [Cout, Cin//cg] with the dtype of x")
    dw_stride = int(dw_stride)
    if dy.dtype != x.dtype or tuple(dy.shape) != (N, Cout, _out(H, dw_stride), _out(W, dw_stride)):
        raise ValueError("dy must be [N, Cout, Ho, Wo] with the dtype of x")
    shape = (N, Cin, Cout, H, W, dw_stride, cg, float(co), _dtype_code(x))
    grad = x.dtype if stored else torch.float32
    shape += (_CODES[grad],)
    ws, ws_ptr, ws_len = _scratch(_workspace_need("scc_dw_backward_as_workspace_bytes", *shape), dev)
    dx = torch.empty_like(x)
    dk = torch.empty((Cin, 3, 3), dtype=grad, device=dev)
    dw = torch.empty(w.shape, dtype=grad, device=dev)
    _launch(dev, load().scc_dw_backward_as, x.data_ptr(), kdw.data_ptr(), w.data_ptr(), dy.data_ptr(), dx.data_ptr(),
            dk.data_ptr(), dw.data_ptr(), *shape, ws_ptr, ws_len)
    return dx, dk, dw


def _activation(act):
    """The library's code of an activation's name; a code stays what it is."""
    code = ACTIVATIONS.get(act, act if act in ACTIVATIONS.values() else None)
    if code is None:
        raise ValueError("act must be one of %s, got %r" % (", ".join(sorted(ACTIVATIONS)), act))
    return code


def _gated_layer(x, w, cg, co):
    """(N, Cin, Cout, H, W, cg, co) of a gated layer."""
    if x.dim() != 4:
        raise ValueError("x must be [N, Cin, H, W]")
    N, Cin, H, W = x.shape
    if w.dtype != x.dtype or w.dim() != 3 or w.shape[0] != 2 or (cg >= 1 and Cin % cg == 0 and w.shape[2] != Cin // cg):
        raise ValueError("w must be [2, Cout, Cin//cg] with the dtype of x")
    return N, Cin, w.shape[1], H, W, cg, float(co)


def scc_gated_forward_workspace_bytes(N, Cin, Cout, H, W, cg, co, dtype=torch.float32):
    code = SCC_F32 if dtype == torch.float32 else SCC_BF16
    return int(load().scc_gated_forward_workspace_bytes(N, Cin, Cout, H, W, cg, float(co), code))


def scc_gated_forward(x, w, cg, co, act="silu", out=None, workspace=None):
    """y = act(SCC(x; w[0])) * SCC(x; w[1]), the layer that a gated feed-forward block opens with: x [N,Cin,H,W], w [2,Cout,Cin//cg]
    -> y [N,Cout,H,W] (same dtype).  A sequence of S tokens is a map of S x 1, single tokens are N maps of 1 x 1.  act: "silu" or
    "gelu" (with erf).  A workspace is allocated where the layer needs one and none is given."""
    code = _activation(act)
    if out is None and workspace is None:
        y = (_native or _load_native()).gated_forward(x, w, cg, co, code)
        if y is not None:
            return y
    dev = _dev(x, w)
    layer = _gated_layer(x, w, cg, co)
    y = x.new_empty((x.shape[0], w.shape[1], x.shape[2], x.shape[3])) if out is None else out
    if out is not None:
        _dev(x, out)
        if out.shape != (x.shape[0], w.shape[1], x.shape[2], x.shape[3]) or out.dtype != x.dtype:
            raise ValueError("out must be [N, Cout, H, W] with the dtype of x")
    dtype = _dtype_code(x)
    ws, ws_ptr, ws_len = _scratch(_workspace_need("scc_gated_forward_workspace_bytes", *layer, dtype), dev, workspace)
    _launch(dev, load().scc_gated_forward, x.data_ptr(), w.data_ptr(), y.data_ptr(), *layer, code, dtype, ws_ptr, ws_len)
    _moved(out)
    return y


def scc_gated_backward(x, w, dy, cg, co, act="silu"):
    """(dx, dw) of scc_gated_forward: dy [N,Cout,H,W] -> dx like x, dw [2,Cout,Cin//cg] float32."""
    return _gated_backward(x, w, dy, cg, co, act, False)


def _gated_backward(x, w, dy, cg, co, act, stored):
    """scc_gated_backward; stored: dw in the type of x, rounded from the same sums."""
    code = _activation(act)
    grads = (_native or _load_native()).gated_backward(x, w, dy, cg, co, code, stored)
    if grads is not None:
        return grads
    dev = _dev(x, w, dy)
    layer = _gated_layer(x, w, cg, co)
    if dy.dtype != x.dtype or tuple(dy.shape) != (x.shape[0], w.shape[1], x.shape[2], x.shape[3]):
        raise ValueError("dy must be [N, Cout, H, W] with the dtype of x")
    dtype = _dtype_code(x)
    grad = x.dtype if stored else torch.float32
    need = _workspace_need("scc_gated_backward_workspace_bytes", *layer, dtype, _CODES[grad])
    ws, ws_ptr, ws_len = _scratch(need, dev)
    dx = torch.empty_like(x)
    dw = torch.empty(w.shape, dtype=grad, device=dev)
    _launch(dev, load().scc_gated_backward, x.data_ptr(), w.data_ptr(), dy.data_ptr(), dx.data_ptr(), dw.data_ptr(), *layer, code, dtype,
            _CODES[grad], ws_ptr, ws_len)
    return dx, dw


# published with the Muon optimiser (K. Jordan and others, 2024); brings singular values between 0.001 and 1 to 0.7 .. 1.2 in five steps
NEWTON_SCHULZ = (3.4445, -4.7750, 2.0315)


def _matrices(*lists):
    """Lists of equally many matrices, one in each list per weight, of one device; the first and second of one dtype."""
    first = lists[0]
    if len(first) == 0 or any(len(l) != len(first) for l in lists):
        raise ValueError("lists of equally many matrices are wanted, at least one")
    dev = _dev(*(t for l in lists for t in l))
    for ts in zip(*lists):
        if any(t.dim() != 2 or t.shape != ts[0].shape for t in ts):
            raise ValueError("a weight, its gradient and its momentum are matrices of the same shape")
        if ts[0].dtype != first[0].dtype or (len(ts) > 1 and ts[1].dtype != first[0].dtype):
            raise ValueError("weights and gradients of one call share their dtype")
    return dev, _dtype_code(first[0])


def _overlap(written, read):
    """Whether memory of one of the written tensors belongs to another tensor of either list as well."""
    spans = sorted((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size(), w) for ts, w in ((written, True), (read, False)) for t in ts)
    end = end_written = 0
    for first, last, w in spans:
        if first < (end if w else end_written):
            return True
        end = max(end, last)
        end_written = max(end_written, last) if w else end_written
    return False


def _orthogonal(dev, name, lists, options, dtype):
    count = len(lists[0])
    pointers = [(ctypes.c_void_p * count)(*[t.data_ptr() for t in l]) for l in lists]
    rows = (ctypes.c_int * count)(*[t.shape[0] for t in lists[0]])
    cols = (ctypes.c_int * count)(*[t.shape[1] for t in lists[0]])
    lib = load()
    ws, ws_ptr, ws_len = _scratch(int(lib.scc_orthogonal_workspace_bytes(count, rows, cols)), dev)
    _launch(dev, getattr(lib, name), count, *pointers, rows, cols, ctypes.byref(options), dtype, ws_ptr, ws_len)


def scc_orthogonalise(matrices, steps=5, coefficients=NEWTON_SCHULZ, eps=1e-7):
    """The matrices with their singular values brought near 1 by `steps` Newton-Schulz steps x <- a x + (b x x^T + c (x x^T)^2) x from
    x / (||x||_F + eps): a list of [rows, cols], float32 or bfloat16 -> a list of the same."""
    out = (_native or _load_native()).orthogonalise(matrices, steps, *coefficients, eps)
    if out is not None:
        return out
    dev, dtype = _matrices(matrices)
    out = [torch.empty_like(t) for t in matrices]
    _orthogonal(dev, "scc_orthogonalise", (matrices, out), _OrthogonalOptions(0, 0, 0, 0, steps, *coefficients, eps), dtype)
    return out


def scc_orthogonal_step(weights, grads, momenta, lr, momentum=0.95, weight_decay=0.0, nesterov=True, steps=5, coefficients=NEWTON_SCHULZ,
                        eps=1e-7):
    """One step of the orthogonalised momentum update on a list of weight matrices, in place:
    m <- momentum m + g, u = g + momentum m (nesterov) or m, w <- (1 - lr weight_decay) w - lr sqrt(max(1, rows/cols)) O(u), O as
    scc_orthogonalise.  weights and grads: float32 or bfloat16, one dtype for all; momenta: float32; no weight or momentum may overlap another tensor
    of the call.  A graph that saved a weight cannot be
    run backward afterwards, as after any change in place."""
    native = _native or _load_native()
    status = native.orthogonal_step(weights, grads, momenta, lr, momentum, weight_decay, nesterov, steps, *coefficients, eps)
    if status is not None:                      # made, if it failed too: once more would move a part of the list twice
        return _check(status)
    dev, dtype = _matrices(weights, grads, momenta)
    if any(m.dtype != torch.float32 for m in momenta):
        raise ValueError("momenta are float32")
    if _overlap((*weights, *momenta), grads):
        raise ValueError("weights and momenta may not share memory with each other or with a gradient")
    options = _OrthogonalOptions(lr, momentum, weight_decay, int(bool(nesterov)), steps, *coefficients, eps)
    try:
        _orthogonal(dev, "scc_orthogonal_step", (weights, grads, momenta), options, dtype)
    except SccError as e:
        if e.status == SCC_ERR_LAUNCH:          # in the middle of a list, perhaps
            _moved(*weights, *momenta)
        raise
    _moved(*weights, *momenta)


def _norm_map(x, w, residual):
    """(device, (N, C, H, W)) of a residual norm's call."""
    dev = _dev(x, w) if residual is None else _dev(x, w, residual)
    if x.dim() != 4:
        raise ValueError("x must be [N, C, H, W]")
    if w.dtype != x.dtype or tuple(w.shape) != (x.shape[1],):
        raise ValueError("w must be [C] with the dtype of x")
    if residual is not None and (residual.dtype != x.dtype or residual.shape != x.shape):
        raise ValueError("residual must have the shape and dtype of x")
    return dev, tuple(x.shape)


def _address(t):
    return None if t is None else t.data_ptr()


def scc_norm_forward(x, w, residual=None, eps=1e-6):
    """(y, h) of the residual norm in front of a feed-forward block: h = x + residual, y = h / sqrt(mean_c h^2 + eps) * w, over the channels of
    [N,C,H,W]; w [C].  Without a residual h is x itself."""
    both = (_native or _load_native()).norm_forward(x, w, residual, eps)
    if both is not None:
        return both
    dev, shape = _norm_map(x, w, residual)
    y = torch.empty_like(x)
    h = None if residual is None else torch.empty_like(x)
    _launch(dev, load().scc_norm_forward, x.data_ptr(), _address(residual), w.data_ptr(), _address(h), y.data_ptr(), *shape, float(eps),
            _dtype_code(x))
    return y, x if h is None else h


def scc_norm_quantised(x, w, residual=None, eps=1e-6):
    """(q, scale, h): the residual norm's y in 8 bits, q (float8_e4m3fn, the shape of x) * scale (float32 [N,H,W], a power of two for each pixel)."""
    out = (_native or _load_native()).norm_quantised(x, w, residual, eps)
    if out is not None:
        return out
    dev, shape = _norm_map(x, w, residual)
    q = torch.empty(shape, dtype=torch.float8_e4m3fn, device=dev)
    scale = torch.empty((shape[0], *shape[2:]), dtype=torch.float32, device=dev)
    h = None if residual is None else torch.empty_like(x)
    _launch(dev, load().scc_norm_quantised, x.data_ptr(), _address(residual), w.data_ptr(), _address(h), q.data_ptr(), scale.data_ptr(), *shape,
            float(eps), _dtype_code(x))
    return q, scale, x if h is None else h


def scc_norm_backward(x, w, dy, residual=None, dh=None, eps=1e-6):
    """(dx, dw) of scc_norm_forward: dx like x, the gradient of x and of the residual, dw [C] float32.  dh: the gradient that reaches h by itself.  In
    float32 the h that the forward returned can stand for x and the residual."""
    return _norm_backward(x, w, dy, residual, dh, eps, False)


def _norm_backward(x, w, dy, residual, dh, eps, stored):
    """scc_norm_backward; stored: dw in the type of x, rounded from the same sums."""
    dev, shape = _norm_map(x, w, residual)
    for t in (dy,) if dh is None else (dy, dh):
        _dev(x, t)
        if t.dtype != x.dtype or t.shape != x.shape:
            raise ValueError("dy and dh must have the shape and dtype of x")
    code = _dtype_code(x)
    ws, ws_ptr, ws_len = _scratch(_workspace_need("scc_norm_backward_workspace_bytes", *shape, code), dev)
    dx = torch.empty_like(x)
    dw = torch.empty(shape[1], dtype=x.dtype if stored else torch.float32, device=dev)
    _launch(dev, load().scc_norm_backward, x.data_ptr(), _address(residual), w.data_ptr(), dy.data_ptr(), _address(dh), dx.data_ptr(), dw.data_ptr(),
            *shape, float(eps), code, _CODES[dw.dtype], ws_ptr, ws_len)
    return dx, dw


def _reduction(reduction):
    """The library's code of a reduction's name."""
    if reduction not in REDUCTIONS:
        raise ValueError("reduction must be one of %s, got %r" % (", ".join(sorted(REDUCTIONS)), reduction))
    return REDUCTIONS[reduction]


def _vocabulary(x, w, target, ignore_index):
    """(device, (N, C, H, W), V, ignore_index) of a vocabulary loss's call."""
    dev = _dev(x, w, target)
    if x.dim() != 4:
        raise ValueError("x must be [N, C, H, W]")
    if w.dtype != x.dtype or w.dim() != 2 or w.shape[1] != x.shape[1]:
        raise ValueError("w must be [V, C] with the dtype of x")
    if target.dtype != torch.int64 or tuple(target.shape) != (x.shape[0], *x.shape[2:]):
        raise ValueError("target must be int64 [N, H, W]")
    return dev, tuple(x.shape), w.shape[0], int(ignore_index)


def scc_vocabulary_loss(x, w, target, reduction="mean", ignore_index=-100):
    """(loss, lse): -log softmax over v of sum_c x[n,c,h,w] w[v,c], at v = target[n,h,w], without the logits in memory; x [N,C,H,W], w [V,C],
    target int64 [N,H,W].  loss: float32, [N,H,W] for "none", else one value; "mean" over the tokens whose target is not ignore_index, 0 if there
    are none.  lse: float32 [N,H,W], for scc_vocabulary_gradients."""
    code = _reduction(reduction)
    both = (_native or _load_native()).vocabulary_loss(x, w, target, code, ignore_index)
    if both is not None:
        return both
    dev, shape, V, ignored = _vocabulary(x, w, target, ignore_index)
    dtype = _dtype_code(x)
    ws, ws_ptr, ws_len = _scratch(_workspace_need("scc_vocabulary_loss_workspace_bytes", *shape, V, code, dtype), dev)
    lse = torch.empty(target.shape, dtype=torch.float32, device=dev)
    loss = torch.empty(target.shape if code == 0 else (), dtype=torch.float32, device=dev)
    _launch(dev, load().scc_vocabulary_loss, x.data_ptr(), w.data_ptr(), target.data_ptr(), loss.data_ptr(), lse.data_ptr(), *shape, V, ignored,
            code, dtype, ws_ptr, ws_len)
    return loss, lse


def scc_vocabulary_gradients(x, w, target, lse, dloss, reduction="mean", ignore_index=-100):
    """(dx, dw) of scc_vocabulary_loss from the lse that it returned: dx like x, dw [V,C] float32; dloss: the loss's gradient, float32 of its shape.  Of bfloat16
    tensors the softmax and dloss x are rounded to 11 bits between the products, so dw's terms are off by 2^-12 each."""
    return _vocabulary_gradients(x, w, target, lse, dloss, _reduction(reduction), ignore_index, False)


def _vocabulary_gradients(x, w, target, lse, dloss, code, ignore_index, stored):
    """scc_vocabulary_gradients; stored: dw in the type of x, rounded from the same sums."""
    dev, shape, V, ignored = _vocabulary(x, w, target, ignore_index)
    _dev(x, lse, dloss)
    if lse.dtype != torch.float32 or lse.shape != target.shape:
        raise ValueError("lse must be float32 [N, H, W]")
    if dloss.dtype != torch.float32 or tuple(dloss.shape) != (tuple(target.shape) if code == 0 else ()):
        raise ValueError("dloss must be float32 with the shape of the loss")
    dtype = _dtype_code(x)
    ws, ws_ptr, ws_len = _scratch(_workspace_need("scc_vocabulary_gradients_workspace_bytes", *shape, V, dtype), dev)
    dx = torch.empty_like(x)
    dw = torch.empty(w.shape, dtype=x.dtype if stored else torch.float32, device=dev)
    _launch(dev, load().scc_vocabulary_gradients, x.data_ptr(), w.data_ptr(), target.data_ptr(), lse.data_ptr(), dloss.data_ptr(), dx.data_ptr(),
            dw.data_ptr(), *shape, V, ignored, code, dtype, _CODES[dw.dtype], ws_ptr, ws_len)
    return dx, dw


def _check_adamw(weights, grads, first, second, first_scales, second_scales):
    """The device and dtype of an AdamW call whose lists fit together."""
    if (first_scales is None) != (second_scales is None):
        raise ValueError("first_scales and second_scales go together")
    lists = [weights, grads, first, second] + ([first_scales, second_scales] if first_scales is not None else [])
    if len(weights) == 0 or any(len(l) != len(weights) for l in lists):
        raise ValueError("lists of equally many tensors are wanted, at least one")
    dev = _dev(*(t for l in lists for t in l))
    state = torch.float32 if first_scales is None else torch.float8_e4m3fn
    for w, g, m, v in zip(weights, grads, first, second):
        if g.shape != w.shape or m.shape != w.shape or v.shape != w.shape:
            raise ValueError("a weight, its gradient and its states have the same shape")
        if w.dtype != weights[0].dtype or g.dtype != w.dtype:
            raise ValueError("weights and gradients of one call share their dtype")
        if m.dtype != state or v.dtype != state:
            raise ValueError("states are float32, or float8_e4m3fn with scales")
    if first_scales is not None:
        for w, ms, vs in zip(weights, first_scales, second_scales):
            if any(s.dtype != torch.float32 or s.numel() != -(-w.numel() // STATE_BLOCK) for s in (ms, vs)):
                raise ValueError("scales are float32, one for each %d elements of a weight" % STATE_BLOCK)
    if _overlap([t for l in (lists[0], *lists[2:]) for t in l], grads):
        raise ValueError("weights and states may not share memory with each other or with a gradient")
    return dev, _dtype_code(weights[0])


def _check_step(step, dev):
    if step.dtype != torch.int64 or step.numel() != 1 or step.device != dev:
        raise ValueError("step must be a number, or an int64 tensor of one element on the weights' device")


def _refuse_adamw(weights, grads, first, second, first_scales, second_scales, lr, step, betas, eps, weight_decay):
    """Raises what scc_adamw_step would refuse these arguments with."""
    if not (_native or _load_native()).adamw_fits(weights, grads, first, second, first_scales, second_scales):
        _check_adamw(weights, grads, first, second, first_scales, second_scales)
    if any(w.numel() > MOST_ADAMW for w in weights):
        _check(SCC_ERR_SHAPE)
    if not (all(math.isfinite(v) for v in (lr, eps, weight_decay)) and eps >= 0 and all(0 <= b < 1 for b in betas)):
        _check(SCC_ERR_OPTION)
    if isinstance(step, torch.Tensor):
        _check_step(step, weights[0].device)


def scc_adamw_step(weights, grads, first, second, lr, step, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.0, first_scales=None,
                   second_scales=None, seed=0):
    """A step of AdamW on a list of weights of any shapes, in place: m <- b1 m + (1 - b1) g, v <- b2 v + (1 - b2) g^2, w <- (1 - lr weight_decay) w -
    lr (m / (1 - b1^step)) / (sqrt(v / (1 - b2^step)) + eps).  weights and grads: float32 or bfloat16, one dtype for all.  States: float32, or with
    first_scales and second_scales (float32, one for each 256 elements of a weight) float8_e4m3fn, m = first * scale, v = (second * scale)^2,
    rounded at random with the stored values' expectation kept: a hash of seed, step and place.  step: from 1; or an int64 tensor of one element on
    the GPU, read when the call runs, for calls that are captured and replayed (lr, betas, eps and weight_decay are read at the capture).  No weight or state may overlap another tensor of the call.  A graph that
    saved a weight cannot be run backward afterwards, as after any change in place."""
    native = _native or _load_native()
    status = native.adamw_step(weights, grads, first, second, first_scales, second_scales, lr, step, betas[0], betas[1], eps, weight_decay, seed)
    if status is not None:                      # made, if it failed too: once more would move a part of the list twice
        return _check(status)
    dev, dtype = _check_adamw(weights, grads, first, second, first_scales, second_scales)
    device_step = None
    if isinstance(step, torch.Tensor):
        _check_step(step, dev)
        device_step, step = step.data_ptr(), 1
    count = len(weights)
    lists = [weights, grads, first, second, first_scales, second_scales]
    pointers = [None if l is None else (ctypes.c_void_p * count)(*[t.data_ptr() for t in l]) for l in lists]
    sizes = (ctypes.c_longlong * count)(*[w.numel() for w in weights])
    options = _AdamwOptions(lr, betas[0], betas[1], eps, weight_decay, int(seed) & (2 ** 64 - 1))
    moved = [t for l in (weights, first, second, first_scales or (), second_scales or ()) for t in l]
    try:
        _launch(dev, load().scc_adamw_step, count, *pointers, sizes, ctypes.byref(options), int(step), device_step, dtype)
    except SccError as e:
        if e.status == SCC_ERR_LAUNCH:          # in the middle of a list, perhaps
            _moved(*moved)
        raise
    _moved(*moved)
