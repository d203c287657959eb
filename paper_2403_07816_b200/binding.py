"""ctypes binding of libbtx.so: same names as the C ABI, argument marshalling only.

Tensors are torch CUDA tensors (torch supplies device memory and streams); every step of the
layer runs inside the library.  There is no CPU fallback: if the library is missing or the
tensors are not on a CUDA device the calls raise.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from operator import index

import torch

BTX_OK = 0
BTX_ERR_INVALID_ARG, BTX_ERR_UNSUPPORTED, BTX_ERR_WORKSPACE, BTX_ERR_ARCH, BTX_ERR_CUDA, BTX_ERR_TIMEOUT = 1, 2, 3, 4, 5, 6
BTX_F32, BTX_BF16 = 0, 1
ROUTE_TOPK, ROUTE_SWITCH, ROUTE_SOFT, ROUTE_SAMPLE1, ROUTE_GIVEN = 0, 1, 2, 3, 4
PARAM_AVERAGE, PARAM_FFN = 0, 1
FFN_STACK, FFN_SPLIT, FFN_BLEND = 0, 1, 2
SCORE_SOFTMAX, SCORE_SIGMOID = 0, 1
GROUP_MAX, GROUP_SUM2 = 0, 1

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libbtx.so")
_lib = None


class BtxError(RuntimeError):
    def __init__(self, status, where):
        self.status = int(status)
        msg = lib().btx_status_string(self.status).decode()
        super().__init__(f"{where}: {msg} (status {self.status})")


class MoeDesc(C.Structure):
    _fields_ = [("T", C.c_int32), ("d_model", C.c_int32), ("d_ff", C.c_int32), ("E", C.c_int32), ("k", C.c_int32),
                ("dtype", C.c_int32), ("routing", C.c_int32), ("lb_alpha", C.c_float),
                ("lb_stopgrad_u", C.c_int32), ("save_for_backward", C.c_int32), ("skip_wgrad", C.c_int32),
                ("gumbel_tau", C.c_float), ("capacity_factor", C.c_float)]


class RoutingOut(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("logits", "topk_idx", "gates", "probs", "counts", "offsets", "perm",
                                           "inv_perm", "u", "p", "lb_loss")]


class MergeItem(C.Structure):
    _fields_ = [("kind", C.c_int32), ("layer", C.c_int32), ("numel", C.c_uint64),
                ("src", C.POINTER(C.c_void_p)), ("dst", C.c_void_p)]


class RouteDesc(C.Structure):
    _fields_ = [("T", C.c_int32), ("E", C.c_int32), ("k", C.c_int32), ("dtype", C.c_int32), ("score", C.c_int32),
                ("n_group", C.c_int32), ("topk_group", C.c_int32), ("group_score", C.c_int32), ("renorm", C.c_int32),
                ("scale", C.c_float)]


class Mx4MoeDesc(C.Structure):
    _fields_ = [("T", C.c_int32), ("d_model", C.c_int32), ("d_ff", C.c_int32), ("E", C.c_int32), ("k", C.c_int32),
                ("dtype", C.c_int32)]


class Fp8MoeDesc(C.Structure):
    _fields_ = Mx4MoeDesc._fields_


class NormDesc(C.Structure):
    _fields_ = [("T", C.c_int32), ("d_model", C.c_int32), ("dtype", C.c_int32), ("eps", C.c_float)]


EXPORTS = ["btx_moe_sizes", "btx_moe_forward", "btx_moe_backward", "btx_moe_step_host",
           "btx_lb_loss_workspace_size", "btx_lb_loss", "btx_lb_loss_noalloc", "btx_merge_workspace_size", "btx_merge", "btx_merge_ffn_workspace_size", "btx_merge_ffn",
           "btx_route", "btx_route_backward",
           "btx_mx4_sizes", "btx_mx4_quantize", "btx_mx4_dequantize", "btx_mx4_matmul_workspace_size", "btx_mx4_matmul",
           "btx_mx4_moe_workspace_size", "btx_mx4_moe_forward",
           "btx_fp8_sizes", "btx_fp8_quantize", "btx_fp8_dequantize", "btx_fp8_matmul_workspace_size", "btx_fp8_matmul",
           "btx_fp8_moe_workspace_size", "btx_fp8_moe_forward",
           "btx_rms_norm", "btx_rms_norm_backward_workspace_size", "btx_rms_norm_backward",
           "btx_device_status", "btx_selftest_wait_expiry", "btx_selftest_separate_launches", "btx_set_stage_events", "btx_status_string", "btx_version"]


def lib():
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2403_07816_b200.build`")
        L = C.CDLL(LIB_PATH)
        vp, i32, f32, sz = C.c_void_p, C.c_int32, C.c_float, C.c_size_t
        L.btx_moe_sizes.argtypes = [C.POINTER(MoeDesc), C.POINTER(sz), C.POINTER(sz)]
        L.btx_moe_forward.argtypes = [C.POINTER(MoeDesc), vp, vp, vp, vp, vp, vp, vp, vp, C.POINTER(RoutingOut), vp, vp,
                                      sz, vp]
        L.btx_moe_backward.argtypes = [C.POINTER(MoeDesc), vp, vp, vp, vp, vp, vp, vp, vp, f32, vp, vp, vp, vp, vp, vp,
                                       vp, vp, i32, vp, sz, vp]
        L.btx_moe_step_host.argtypes = [C.POINTER(MoeDesc)] + [vp] * 15 + [f32] + [vp] * 5 + [i32, vp, vp, sz, vp, vp]
        L.btx_set_stage_events.argtypes = [C.POINTER(vp), i32]
        L.btx_selftest_wait_expiry.argtypes = [vp, sz, vp]
        L.btx_selftest_separate_launches.argtypes = [i32]
        L.btx_lb_loss_workspace_size.argtypes = [C.POINTER(MoeDesc), C.POINTER(sz)]
        L.btx_lb_loss.argtypes = [C.POINTER(MoeDesc), vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.btx_lb_loss_noalloc.argtypes = [C.POINTER(MoeDesc), vp, vp, vp, vp, vp, vp, vp]
        L.btx_merge_workspace_size.argtypes = [i32, C.c_uint64, C.POINTER(sz)]
        L.btx_merge.argtypes = [i32, i32, C.POINTER(MergeItem), C.c_uint64, vp, sz, vp]
        L.btx_merge_ffn_workspace_size.argtypes = [i32, i32, C.POINTER(sz)]
        L.btx_merge_ffn.argtypes = [i32, i32, i32, i32, i32, i32, C.POINTER(vp), C.POINTER(vp), C.POINTER(vp), vp, vp, vp,
                                    vp, sz, vp]
        L.btx_route.argtypes = [C.POINTER(RouteDesc), vp, C.c_int64, vp, vp, vp, vp, vp, vp, vp]
        L.btx_route_backward.argtypes = [C.POINTER(RouteDesc), vp, C.c_int64, vp, vp, vp, C.c_int64, vp]
        i64 = C.c_int64
        L.btx_mx4_sizes.argtypes = [i32, i32, i32, C.POINTER(sz), C.POINTER(sz)]
        L.btx_mx4_quantize.argtypes = [i32, vp, i64, i64, i32, i32, i32, i32, i32, i32, vp, vp, vp]
        L.btx_mx4_dequantize.argtypes = [i32, vp, vp, i32, i32, i32, vp, vp]
        L.btx_mx4_matmul_workspace_size.argtypes = [i32, i32, i32, i32, i32, C.POINTER(sz)]
        L.btx_mx4_matmul.argtypes = [i32, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp, sz, vp]
        L.btx_mx4_moe_workspace_size.argtypes = [C.POINTER(Mx4MoeDesc), C.POINTER(sz)]
        L.btx_mx4_moe_forward.argtypes = [C.POINTER(Mx4MoeDesc), vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.btx_fp8_sizes.argtypes = [i32, i32, i32, C.POINTER(sz), C.POINTER(sz)]
        L.btx_fp8_matmul_workspace_size.argtypes = [i32, i32, i32, i32, i32, C.POINTER(sz)]
        L.btx_fp8_moe_workspace_size.argtypes = [C.POINTER(Fp8MoeDesc), C.POINTER(sz)]
        L.btx_rms_norm_backward_workspace_size.argtypes = [C.POINTER(NormDesc), C.POINTER(sz)]
        # The calls that take a few microseconds on the device hand every argument (addresses, sizes, strides; no floats) over
        # in a register or stack slot of 64 bits, as ctypes does fastest for pointers.
        for name, n in (("btx_fp8_quantize", 16), ("btx_fp8_dequantize", 8), ("btx_fp8_matmul", 14), ("btx_fp8_moe_forward", 13),
                        ("btx_rms_norm", 13), ("btx_rms_norm_backward", 15)):
            getattr(L, name).argtypes = [vp] * n
        L.btx_device_status.argtypes = [vp, vp, C.POINTER(i32)]
        L.btx_status_string.argtypes = [i32]
        L.btx_status_string.restype = C.c_char_p
        L.btx_version.restype = i32
        for name in EXPORTS:
            if name not in ("btx_status_string", "btx_version"):
                getattr(L, name).restype = i32
        _lib = L
    return _lib


def _dtype_code(t) -> int:
    if t == torch.float32:
        return BTX_F32
    if t == torch.bfloat16:
        return BTX_BF16
    raise TypeError(f"unsupported dtype {t}")


def _ptr(t):
    if t is None:
        return None
    if not t.is_cuda:
        raise RuntimeError("btx: tensors must live on a CUDA device (there is no CPU path)")
    if not t.is_contiguous():
        raise RuntimeError("btx: tensors must be contiguous")
    return C.c_void_p(t.data_ptr())


def _stream(device):
    return C.c_void_p(torch.cuda.current_stream(device).cuda_stream)


def _on(device):
    """The library works on the current device (its helper stream, multiprocessor count and static scratch
    are looked up per current device): every call runs with the tensors' device made current."""
    if torch.device(device).type != "cuda":
        raise RuntimeError("btx: tensors must live on a CUDA device (there is no CPU path)")
    return torch.cuda.device(device)


def make_desc(T, d_model, d_ff, E, k, dtype, routing=ROUTE_TOPK, lb_alpha=0.01, lb_stopgrad_u=False,
              save_for_backward=False, skip_wgrad=False, gumbel_tau=0.0, capacity_factor=0.0) -> MoeDesc:
    code = _dtype_code(dtype) if isinstance(dtype, torch.dtype) else int(dtype)
    return MoeDesc(T, d_model, d_ff, E, k, code, routing, lb_alpha, int(lb_stopgrad_u), int(save_for_backward),
                   int(skip_wgrad), float(gumbel_tau), float(capacity_factor))


def btx_moe_sizes(desc: MoeDesc):
    ws, sv = C.c_size_t(0), C.c_size_t(0)
    s = lib().btx_moe_sizes(C.byref(desc), C.byref(ws), C.byref(sv))
    if s != BTX_OK:
        raise BtxError(s, "btx_moe_sizes")
    return ws.value, sv.value


@dataclass
class Routing:
    logits: torch.Tensor
    topk_idx: torch.Tensor
    gates: torch.Tensor
    probs: torch.Tensor
    counts: torch.Tensor
    offsets: torch.Tensor
    perm: torch.Tensor
    inv_perm: torch.Tensor
    u: torch.Tensor
    p: torch.Tensor
    lb_loss: torch.Tensor

    @staticmethod
    def empty(desc: MoeDesc, device):
        k = desc.E if desc.routing == ROUTE_SOFT else desc.k
        T, E, R = desc.T, desc.E, desc.T * k
        f = dict(dtype=torch.float32, device=device)
        i = dict(dtype=torch.int32, device=device)
        return Routing(torch.empty((T, E), **f), torch.empty((T, k), **i), torch.empty((T, k), **f),
                       torch.empty((T, E), **f), torch.empty(E, **i), torch.empty(E + 1, **i), torch.empty(R, **i),
                       torch.empty(R, **i), torch.empty(E, **f), torch.empty(E, **f), torch.empty(1, **f))

    @staticmethod
    def given(desc: MoeDesc, topk_idx, gates):
        """The caller's choice [T,k] int32 and gates [T,k] fp32 for ROUTE_GIVEN, with room for the permutation."""
        dev, R = _device(topk_idx), desc.T * desc.k
        _arg(topk_idx, "topk_idx", (desc.T, desc.k), torch.int32, dev)
        _arg(gates, "gates", (desc.T, desc.k), torch.float32, dev)
        i = dict(dtype=torch.int32, device=topk_idx.device)
        return Routing(None, topk_idx, gates, None, torch.empty(desc.E, **i), torch.empty(desc.E + 1, **i),
                       torch.empty(R, **i), torch.empty(R, **i), None, None, None)

    def as_struct(self) -> RoutingOut:
        return RoutingOut(*[None if t is None else t.data_ptr() for t in (self.logits, self.topk_idx, self.gates, self.probs, self.counts,
                                                   self.offsets, self.perm, self.inv_perm, self.u, self.p,
                                                   self.lb_loss)])


def alloc_buffers(desc: MoeDesc, device):
    """(workspace, saved) byte tensors of the sizes btx_moe_sizes reports."""
    ws, sv = btx_moe_sizes(desc)
    return (torch.empty(ws, dtype=torch.uint8, device=device),
            torch.empty(max(sv, 16), dtype=torch.uint8, device=device))


def btx_moe_forward(desc, x, w_router, router_bias, w1, w3, w2, y, routing, saved, workspace, router_noise=None):
    ro = routing.as_struct() if routing is not None else None
    with _on(x.device):
        s = lib().btx_moe_forward(C.byref(desc), _ptr(x), _ptr(w_router), _ptr(router_bias), _ptr(router_noise),
                                  _ptr(w1), _ptr(w3), _ptr(w2),
                                  _ptr(y), C.byref(ro) if ro is not None else None, _ptr(saved), _ptr(workspace),
                                  workspace.numel(), _stream(x.device))
    if s != BTX_OK:
        raise BtxError(s, "btx_moe_forward")


def btx_moe_backward(desc, x, w_router, router_bias, w1, w3, w2, dy, lb_grad_scale, saved, dx, dw_router, dbias,
                     dw1, dw3, dw2, accumulate, workspace, router_noise=None, dlogits=None):
    """With ROUTE_GIVEN w_router, dw_router and dbias are None and dlogits receives d gates [T,k]."""
    with _on(x.device):
        s = lib().btx_moe_backward(C.byref(desc), _ptr(x), _ptr(w_router), _ptr(router_bias), _ptr(router_noise),
                                   _ptr(w1), _ptr(w3), _ptr(w2),
                                   _ptr(dy), float(lb_grad_scale), _ptr(saved), _ptr(dx), _ptr(dw_router), _ptr(dbias),
                                   _ptr(dlogits), _ptr(dw1), _ptr(dw3), _ptr(dw2), int(accumulate), _ptr(workspace),
                                   workspace.numel(), _stream(x.device))
    if s != BTX_OK:
        raise BtxError(s, "btx_moe_backward")


def btx_moe_step_host(desc, x_host, dy_host, y_host, dx_host, loss_host, x_dev, dy_dev, y_dev, dx_dev, w_router,
                      router_bias, w1, w3, w2, lb_grad_scale, dw_router, dbias, dw1, dw3, dw2, accumulate, saved,
                      workspace, router_noise=None, copy_stream=None):
    """Forward + backward with activations in (pinned) host tensors; see btx.h.  `copy_stream` is an
    optional torch.cuda.Stream on which the dy upload and the y download overlap the compute."""
    for t in (x_host, dy_host, y_host, dx_host, loss_host):
        if t.is_cuda or not t.is_contiguous():
            raise RuntimeError("btx_moe_step_host: host tensors must be contiguous CPU tensors")
    hp = lambda t: C.c_void_p(t.data_ptr())
    with _on(x_dev.device):
        s = lib().btx_moe_step_host(C.byref(desc), hp(x_host), hp(dy_host), hp(y_host), hp(dx_host), hp(loss_host),
                                    _ptr(x_dev), _ptr(dy_dev), _ptr(y_dev), _ptr(dx_dev), _ptr(w_router),
                                    _ptr(router_bias), _ptr(router_noise), _ptr(w1), _ptr(w3), _ptr(w2),
                                    float(lb_grad_scale),
                                    _ptr(dw_router), _ptr(dbias), _ptr(dw1), _ptr(dw3), _ptr(dw2), int(accumulate),
                                    _ptr(saved), _ptr(workspace), workspace.numel(), _stream(x_dev.device),
                                    C.c_void_p(copy_stream.cuda_stream) if copy_stream is not None else None)
    if s != BTX_OK:
        raise BtxError(s, "btx_moe_step_host")


_stage_keepalive = None


def btx_set_stage_events(events):
    """events: list of torch.cuda.Event(enable_timing=True) that have been recorded at least once
    (so that their handles exist), or None to switch the hook off."""
    global _stage_keepalive
    if events is None:
        _stage_keepalive = None
        s = lib().btx_set_stage_events(None, 0)
    else:
        arr = (C.c_void_p * len(events))(*[e.cuda_event for e in events])
        _stage_keepalive = (arr, events)
        s = lib().btx_set_stage_events(arr, len(events))
    if s != BTX_OK:
        raise BtxError(s, "btx_set_stage_events")


def btx_lb_loss_workspace_size(desc):
    sz = C.c_size_t(0)
    s = lib().btx_lb_loss_workspace_size(C.byref(desc), C.byref(sz))
    if s != BTX_OK:
        raise BtxError(s, "btx_lb_loss_workspace_size")
    return sz.value


def btx_lb_loss(desc, logits, loss, u, p, dlogits, workspace, router_bias=None):
    with _on(logits.device):
        s = lib().btx_lb_loss(C.byref(desc), _ptr(logits), _ptr(router_bias), _ptr(loss), _ptr(u), _ptr(p),
                              _ptr(dlogits), _ptr(workspace), workspace.numel(), _stream(logits.device))
    if s != BTX_OK:
        raise BtxError(s, "btx_lb_loss")


def btx_lb_loss_noalloc(desc, logits, loss, u, p, dlogits, router_bias=None):
    """btx_lb_loss on the library's own static scratch: no workspace argument, nothing allocated."""
    with _on(logits.device):
        s = lib().btx_lb_loss_noalloc(C.byref(desc), _ptr(logits), _ptr(router_bias), _ptr(loss), _ptr(u), _ptr(p),
                                      _ptr(dlogits), _stream(logits.device))
    if s != BTX_OK:
        raise BtxError(s, "btx_lb_loss_noalloc")


def btx_merge_workspace_size(n_models, n_items):
    sz = C.c_size_t(0)
    s = lib().btx_merge_workspace_size(n_models, n_items, C.byref(sz))
    if s != BTX_OK:
        raise BtxError(s, "btx_merge_workspace_size")
    return sz.value


def btx_merge(models, outputs, workspace=None):
    """models: list of N dicts name -> tensor; outputs: dict name -> tensor ([N, ...] for names
    containing '.ffn.', same shape as the sources otherwise).  Builds the item table and calls
    the library once; returns the workspace (keep it alive until the stream has run)."""
    n = len(models)
    names = list(models[0].keys())
    items = (MergeItem * len(names))()
    keep = []
    dtype = None
    for i, name in enumerate(names):
        srcs = [m[name] for m in models]
        dtype = srcs[0].dtype
        arr = (C.c_void_p * n)(*[_ptr(s).value for s in srcs])
        keep.append(arr)
        items[i].kind = PARAM_FFN if ".ffn." in name else PARAM_AVERAGE
        items[i].layer = 0
        items[i].numel = srcs[0].numel()
        items[i].src = C.cast(arr, C.POINTER(C.c_void_p))
        items[i].dst = _ptr(outputs[name]).value
    device = models[0][names[0]].device
    if workspace is None:
        workspace = torch.empty(btx_merge_workspace_size(n, len(names)), dtype=torch.uint8, device=device)
    with _on(device):
        s = lib().btx_merge(n, _dtype_code(dtype), items, len(names), _ptr(workspace), workspace.numel(),
                            _stream(device))
    if s != BTX_OK:
        raise BtxError(s, "btx_merge")
    return workspace


def btx_merge_ffn(w1s, w3s, w2s, layout, chunks, w1_dst, w3_dst, w2_dst, workspace=None):
    """One layer's FFN matrices of N models (lists of [F,d], [F,d], [d,F] tensors) into expert tensors in
    the STACK, SPLIT or BLEND layout; see btx.h."""
    n = len(w1s)
    F, d = w1s[0].shape
    arr = lambda ts: (C.c_void_p * n)(*[_ptr(t).value for t in ts])
    a1, a3, a2 = arr(w1s), arr(w3s), arr(w2s)
    device = w1s[0].device
    if workspace is None:
        sz = C.c_size_t(0)
        s = lib().btx_merge_ffn_workspace_size(n, max(1, chunks), C.byref(sz))
        if s != BTX_OK:
            raise BtxError(s, "btx_merge_ffn_workspace_size")
        workspace = torch.empty(sz.value, dtype=torch.uint8, device=device)
    with _on(device):
        s = lib().btx_merge_ffn(n, _dtype_code(w1s[0].dtype), layout, chunks, d, F, a1, a3, a2, _ptr(w1_dst),
                                _ptr(w3_dst), _ptr(w2_dst), _ptr(workspace), workspace.numel(), _stream(device))
    if s != BTX_OK:
        raise BtxError(s, "btx_merge_ffn")
    return workspace


def _bad(t, name, shape, dtype, dev):
    if t is None:
        raise ValueError(f"btx: {name} is missing")
    if tuple(t.shape) == tuple(shape) and t.dtype is dtype and t.get_device() == dev:
        raise RuntimeError(f"btx: {name} must be contiguous")
    raise ValueError(f"btx: {name} must be {tuple(shape)} {dtype} on device {dev}, not {tuple(t.shape)} {t.dtype} on {t.device}")


def _arg(t, name, shape, dtype, dev):
    """Address of a contiguous tensor argument of the given shape and type on device number `dev`: the library sees
    only the address."""
    if t is None or t.shape != shape or t.dtype is not dtype or t.get_device() != dev or not t.is_contiguous():
        _bad(t, name, shape, dtype, dev)
    return t.data_ptr()


def _opt(t, name, shape, dtype, dev):
    return None if t is None else _arg(t, name, shape, dtype, dev)


def _rows(t, name, shape, dtype, dev):
    """Address and row stride of a matrix argument whose rows are contiguous (any row stride)."""
    if t.shape != shape or t.dtype is not dtype or t.get_device() != dev:
        _bad(t, name, shape, dtype, dev)
    rs, cs = t.stride()
    width = shape[1]
    if (cs != 1 and width > 1) or (rs < width and shape[0] > 1):
        raise RuntimeError(f"btx: the rows of {name} must be contiguous and must not overlap")
    return t.data_ptr(), rs if rs > width else width


def _device(t):
    """Number of the CUDA device that a tensor lives on."""
    dev = t.get_device()
    if dev < 0:
        raise RuntimeError("btx: tensors must live on a CUDA device (there is no CPU path)")
    return dev


def _launch(name, dev, *args):
    """Calls a library function that takes the current stream last, with the tensors' device current.  The usual case,
    in which it is, costs no context switch: these calls run for a few microseconds on the device."""
    fn = getattr(_lib or lib(), name)
    if torch._C._cuda_getDevice() == dev:
        s = fn(*args, torch._C._cuda_getCurrentRawStream(dev))
    else:
        with torch.cuda.device(dev):
            s = fn(*args, torch._C._cuda_getCurrentRawStream(dev))
    if s != BTX_OK:
        raise BtxError(s, name)


_DTYPE = {BTX_F32: torch.float32, BTX_BF16: torch.bfloat16}
_U8, _I32, _F32 = torch.uint8, torch.int32, torch.float32


def make_route_desc(T, E, k, dtype, score=SCORE_SOFTMAX, n_group=1, topk_group=1, group_score=GROUP_MAX, renorm=True,
                    scale=1.0) -> RouteDesc:
    code = _dtype_code(dtype) if isinstance(dtype, torch.dtype) else int(dtype)
    return RouteDesc(T, E, k, code, score, n_group, topk_group, group_score, int(renorm), float(scale))


def btx_route(desc, logits, bias, topk_idx, gates, scores=None, counts=None, row_valid=None):
    """Expert choice and weights from router logits [T,E] (rows may be strided); see btx.h."""
    T, E, k, dev = desc.T, desc.E, desc.k, _device(logits)
    rows, stride = _rows(logits, "logits", (T, E), _DTYPE.get(desc.dtype), dev)
    if row_valid is not None and row_valid.dtype is torch.bool:
        row_valid = row_valid.view(torch.uint8)
    _launch("btx_route", dev, C.byref(desc), rows, stride, _opt(bias, "bias", (E,), _F32, dev),
            _opt(row_valid, "row_valid", (T,), _U8, dev), _arg(topk_idx, "topk_idx", (T, k), _I32, dev),
            _arg(gates, "gates", (T, k), _F32, dev), _opt(scores, "scores", (T, E), _F32, dev),
            _opt(counts, "counts", (E,), _I32, dev))


def btx_route_backward(desc, logits, topk_idx, dgates, dlogits):
    """d logits from d gates (fp32 [T,k]) and the choice btx_route made; see btx.h."""
    T, E, k, dev = desc.T, desc.E, desc.k, _device(logits)
    rows, stride = _rows(logits, "logits", (T, E), _DTYPE.get(desc.dtype), dev)
    out, out_stride = _rows(dlogits, "dlogits", (T, E), _DTYPE.get(desc.dtype), dev)
    _launch("btx_route_backward", dev, C.byref(desc), rows, stride, _arg(topk_idx, "topk_idx", (T, k), _I32, dev),
            _arg(dgates, "dgates", (T, k), _F32, dev), out, out_stride)


@dataclass
class Mx4:
    """A batch of matrices [batch, rows, K] held as MXFP4 codes and scale tiles (layout in btx.h)."""
    codes: torch.Tensor
    scales: torch.Tensor

    @staticmethod
    def empty(batch, rows, K, device):
        btx_mx4_sizes(batch, rows, K)
        return Mx4(torch.empty((batch, rows, K // 2), dtype=_U8, device=device),
                   torch.empty((batch, (rows + 127) // 128, (K + 127) // 128, 512), dtype=_U8, device=device))

    @property
    def shape(self):
        b, r, c = self.codes.shape
        return b, r, 2 * c


def _mx4(q, name, dev):
    """Shape (batch, rows, K) and addresses of an Mx4 argument."""
    codes, scales = q.codes, q.scales
    batch, rows, half = codes.shape
    if (codes.dtype is not _U8 or codes.get_device() != dev or not codes.is_contiguous() or scales.dtype is not _U8
            or scales.get_device() != dev or not scales.is_contiguous()
            or scales.shape != (batch, (rows + 127) // 128, (half + 63) // 64, 512)):
        _arg(codes, name + ".codes", (batch, rows, half), _U8, dev)
        _arg(scales, name + ".scales", (batch, (rows + 127) // 128, (half + 63) // 64, 512), _U8, dev)
    return batch, rows, 2 * half, codes.data_ptr(), scales.data_ptr()


def _workspace(ws, dev):
    n = ws.numel()
    if ws.dtype is not _U8 or ws.dim() != 1 or ws.get_device() != dev or not ws.is_contiguous():
        _bad(ws, "workspace", (n,), _U8, dev)
    return ws.data_ptr(), n


def btx_mx4_sizes(batch, rows, K):
    """Bytes of the codes and of the scales of a batch of MXFP4 matrices."""
    codes, scales = C.c_size_t(0), C.c_size_t(0)
    s = lib().btx_mx4_sizes(batch, rows, K, C.byref(codes), C.byref(scales))
    if s != BTX_OK:
        raise BtxError(s, "btx_mx4_sizes")
    return codes.value, scales.value


def btx_mx4_quantize(src, out, row_first=0, row_step=1):
    """src [batch, rows, K] or [rows, K] (contiguous rows, any row and batch stride) cast into the Mx4 `out`; row r
    becomes row row_first + r * row_step."""
    dev = _device(src)
    shape, stride = src.shape, src.stride()
    if len(shape) == 2:
        (rows, K), (row_stride, col), batch, batch_stride = shape, stride, 1, 0
    else:
        (batch, rows, K), (batch_stride, row_stride, col) = shape, stride
    ob, out_rows, oK, codes, scales = _mx4(out, "out", dev)
    if ob != batch or oK != K:
        raise ValueError(f"btx: src is {tuple(shape)}, out is {out.shape}")
    if col != 1 and K > 1:
        raise RuntimeError("btx: the rows of src must be contiguous")
    _launch("btx_mx4_quantize", dev, _dtype_code(src.dtype), src.data_ptr(), row_stride, batch_stride, batch, rows, K, out_rows,
            row_first, row_step, codes, scales)


def btx_mx4_dequantize(q, dst):
    """The values of the Mx4 `q` into dst (contiguous, [batch, rows, K] or [rows, K] for one matrix)."""
    dev = _device(dst)
    batch, rows, K, codes, scales = _mx4(q, "q", dev)
    shape = (rows, K) if batch == 1 and dst.dim() == 2 else (batch, rows, K)
    _launch("btx_mx4_dequantize", dev, _dtype_code(dst.dtype), codes, scales, batch, rows, K, _arg(dst, "dst", shape, dst.dtype, dev))


def btx_mx4_matmul_workspace_size(M, N, K, dtype, batch=1):
    sz = C.c_size_t(0)
    s = lib().btx_mx4_matmul_workspace_size(_dtype_code(dtype), batch, M, N, K, C.byref(sz))
    if s != BTX_OK:
        raise BtxError(s, "btx_mx4_matmul_workspace_size")
    return sz.value


def btx_mx4_matmul(a, b, y, workspace):
    """y = a b^T of two Mx4 of the same batch and K; y is [batch, M, N], or [M, N] for one matrix."""
    dev = _device(y)
    batch, M, K, ac, asc = _mx4(a, "a", dev)
    bb, N, bK, bc, bsc = _mx4(b, "b", dev)
    if bb != batch or bK != K:
        raise ValueError(f"btx: a is {a.shape}, b is {b.shape}")
    shape = (M, N) if batch == 1 and y.dim() == 2 else (batch, M, N)
    ws, ws_bytes = _workspace(workspace, dev)
    _launch("btx_mx4_matmul", dev, _dtype_code(y.dtype), batch, M, N, K, ac, asc, bc, bsc, _arg(y, "y", shape, y.dtype, dev), ws,
            ws_bytes)


def make_mx4_moe_desc(T, d_model, d_ff, E, k, dtype) -> Mx4MoeDesc:
    return Mx4MoeDesc(T, d_model, d_ff, E, k, _dtype_code(dtype) if isinstance(dtype, torch.dtype) else int(dtype))


def btx_mx4_moe_workspace_size(desc):
    sz = C.c_size_t(0)
    s = lib().btx_mx4_moe_workspace_size(C.byref(desc), C.byref(sz))
    if s != BTX_OK:
        raise BtxError(s, "btx_mx4_moe_workspace_size")
    return sz.value


def btx_mx4_moe_forward(desc, x, topk_idx, gates, w13, w2, y, workspace):
    """The expert layer on MXFP4 experts under a given routing; w13 holds the rows of W1 and W3 in turn; see btx.h."""
    T, d, F, E, k, dev = desc.T, desc.d_model, desc.d_ff, desc.E, desc.k, _device(x)
    dt = _DTYPE.get(desc.dtype)
    *s13, c13, sc13 = _mx4(w13, "w13", dev)
    *s2, c2, sc2 = _mx4(w2, "w2", dev)
    if s13 != [E, 2 * F, d] or s2 != [E, d, F]:
        raise ValueError(f"btx: w13 is {w13.shape}, w2 is {w2.shape}; the layer has E, d_ff, d_model = {E}, {F}, {d}")
    ws, ws_bytes = _workspace(workspace, dev)
    _launch("btx_mx4_moe_forward", dev, C.byref(desc), _arg(x, "x", (T, d), dt, dev),
            _arg(topk_idx, "topk_idx", (T, k), _I32, dev), _arg(gates, "gates", (T, k), _F32, dev), c13, sc13, c2, sc2,
            _arg(y, "y", (T, d), dt, dev), ws, ws_bytes)


class Fp8:
    """A batch of matrices [batch, rows, K] held as FP8 codes and scale tiles (layout in btx.h).  The tensors are checked here, once,
    and the attributes are read-only, so that calls of a few microseconds need only see that nobody has resized them."""
    __slots__ = ("codes", "scales", "K", "shape", "device", "sizes")

    def __init__(self, codes, scales, K):
        dev, K = _device(codes), index(K)
        batch, rows, _ = codes.shape
        _arg(codes, "codes", (batch, rows, (K + 31) // 32 * 32), _U8, dev)
        _arg(scales, "scales", (batch, (rows + 127) // 128, (K + 511) // 512, 512), _U8, dev)
        if (batch | rows | K) >> 31:
            raise ValueError("btx: the sizes of an Fp8 must fit 32 bits")
        for name, value in zip(self.__slots__, (codes, scales, K, (batch, rows, K), dev, (codes.numel(), scales.numel()))):
            object.__setattr__(self, name, value)

    def __setattr__(self, name, value):
        raise AttributeError(f"btx: the {name} of an Fp8 cannot be changed: make another one of its tensors")

    __delattr__ = lambda self, name: self.__setattr__(name, None)

    def __reduce__(self):
        return Fp8, (self.codes, self.scales, self.K)

    @staticmethod
    def empty(batch, rows, K, device):
        btx_fp8_sizes(batch, rows, K)
        return Fp8(torch.empty((batch, rows, (K + 31) // 32 * 32), dtype=_U8, device=device),
                   torch.empty((batch, (rows + 127) // 128, (K + 511) // 512, 512), dtype=_U8, device=device), K)


def _fp8(q, name, shape, dev):
    """Addresses of the codes and scales of an Fp8 argument of the given shape."""
    if q.shape != shape or q.device != dev:
        raise ValueError(f"btx: {name} must hold {shape} on device {dev}, not {q.shape} on device {q.device}")
    codes, scales = q.codes, q.scales
    if (codes.numel(), scales.numel()) != q.sizes:
        raise ValueError(f"btx: the tensors of {name} have been resized since it was made")
    return codes.data_ptr(), scales.data_ptr()


def btx_fp8_sizes(batch, rows, K):
    """Bytes of the codes and of the scales of a batch of FP8 matrices."""
    codes, scales = C.c_size_t(0), C.c_size_t(0)
    s = lib().btx_fp8_sizes(batch, rows, K, C.byref(codes), C.byref(scales))
    if s != BTX_OK:
        raise BtxError(s, "btx_fp8_sizes")
    return codes.value, scales.value


def btx_fp8_quantize(src, out, block_rows=1, row_first=0, row_step=1, out_t=None):
    """src [batch, rows, K] or [rows, K] (contiguous rows, any row and batch stride) cast into the Fp8 `out` (row r becomes row
    row_first + r * row_step) and, transposed, into the Fp8 `out_t` [batch, K, rows]; either may be None; see btx.h."""
    dev = _device(src)
    shape, stride = src.shape, src.stride()
    if len(shape) == 2:
        (rows, K), (row_stride, col), batch, batch_stride = shape, stride, 1, 0
    else:
        (batch, rows, K), (batch_stride, row_stride, col) = shape, stride
    out_rows, codes, scales, codes_t, scales_t = rows, None, None, None, None
    if out is not None:
        out_rows = out.shape[1]
        codes, scales = _fp8(out, "out", (batch, out_rows, K), dev)
    if out_t is not None:
        codes_t, scales_t = _fp8(out_t, "out_t", (batch, K, rows), dev)
    if col != 1 and K > 1:
        raise RuntimeError("btx: the rows of src must be contiguous")
    block_rows, row_first, row_step = index(block_rows), index(row_first), index(row_step)
    if (batch | rows | K | block_rows | row_first | row_step) >> 31 not in (0, -1):      # (negative ones the library refuses)
        raise ValueError("btx: the sizes of a cast must fit 32 bits")
    _launch("btx_fp8_quantize", dev, _dtype_code(src.dtype), src.data_ptr(), row_stride, batch_stride, batch, rows, K, block_rows,
            out_rows, row_first, row_step, codes, scales, codes_t, scales_t)


def btx_fp8_dequantize(q, dst):
    """The values of the Fp8 `q` into dst (contiguous, [batch, rows, K] or [rows, K] for one matrix)."""
    dev = _device(dst)
    batch, rows, K = q.shape
    shape = (rows, K) if batch == 1 and dst.dim() == 2 else q.shape
    _launch("btx_fp8_dequantize", dev, _dtype_code(dst.dtype), *_fp8(q, "q", q.shape, dev), batch, rows, K,
            _arg(dst, "dst", shape, dst.dtype, dev))


def btx_fp8_matmul_workspace_size(M, N, K, dtype, batch=1):
    sz = C.c_size_t(0)
    s = lib().btx_fp8_matmul_workspace_size(_dtype_code(dtype), batch, M, N, K, C.byref(sz))
    if s != BTX_OK:
        raise BtxError(s, "btx_fp8_matmul_workspace_size")
    return sz.value


def btx_fp8_matmul(a, b, y, workspace, accumulate=False):
    """y = a b^T (fp32 y: or added to y) of two Fp8 of the same batch and K; y is [batch, M, N], or [M, N] for one matrix."""
    dev = _device(y)
    batch, M, K = a.shape
    N = b.shape[1]
    _launch("btx_fp8_matmul", dev, _dtype_code(y.dtype), batch, M, N, K, *_fp8(a, "a", a.shape, dev), *_fp8(b, "b", (batch, N, K), dev),
            _arg(y, "y", (M, N) if batch == 1 and y.dim() == 2 else (batch, M, N), y.dtype, dev), int(accumulate),
            *_workspace(workspace, dev))


def make_fp8_moe_desc(T, d_model, d_ff, E, k, dtype) -> Fp8MoeDesc:
    return Fp8MoeDesc(T, d_model, d_ff, E, k, _dtype_code(dtype) if isinstance(dtype, torch.dtype) else int(dtype))


def btx_fp8_moe_workspace_size(desc):
    sz = C.c_size_t(0)
    s = lib().btx_fp8_moe_workspace_size(C.byref(desc), C.byref(sz))
    if s != BTX_OK:
        raise BtxError(s, "btx_fp8_moe_workspace_size")
    return sz.value


def btx_fp8_moe_forward(desc, x, topk_idx, gates, w13, w2, y, workspace):
    """The expert layer on FP8 experts under a given routing; x is a tensor or an Fp8 of its rows, w13 holds the rows of W1
    and W3 in turn; see btx.h."""
    T, d, F, E, k, dev = desc.T, desc.d_model, desc.d_ff, desc.E, desc.k, _device(y)
    dt, x_scales = _DTYPE.get(desc.dtype), None
    if isinstance(x, Fp8):
        x, x_scales = _fp8(x, "x", (1, T, d), dev)
    else:
        x = _arg(x, "x", (T, d), dt, dev)
    _launch("btx_fp8_moe_forward", dev, C.byref(desc), x, x_scales, _arg(topk_idx, "topk_idx", (T, k), _I32, dev),
            _arg(gates, "gates", (T, k), _F32, dev), *_fp8(w13, "w13", (E, 2 * F, d), dev), *_fp8(w2, "w2", (E, d, F), dev),
            _arg(y, "y", (T, d), dt, dev), *_workspace(workspace, dev))


def make_norm_desc(T, d_model, dtype, eps=1e-5) -> NormDesc:
    return NormDesc(T, d_model, _dtype_code(dtype) if isinstance(dtype, torch.dtype) else int(dtype), float(eps))


def _opt_rows(t, name, shape, dtype, dev):
    return (None, 0) if t is None else _rows(t, name, shape, dtype, dev)


def btx_rms_norm(desc, x, weight, residual=None, h=None, y=None, q=None):
    """h = x + residual and its norm, into y and the Fp8 `q` (each None to skip); rows may be strided; see btx.h."""
    d, dev = desc.d_model, _device(x)
    dt, shape = _DTYPE.get(desc.dtype), (desc.T, d)
    codes, scales = (None, None) if q is None else _fp8(q, "q", (1, *shape), dev)
    _launch("btx_rms_norm", dev, C.byref(desc), *_rows(x, "x", shape, dt, dev), *_opt_rows(residual, "residual", shape, dt, dev),
            _opt(weight, "weight", (d,), dt, dev), *_opt_rows(h, "h", shape, dt, dev), *_opt_rows(y, "y", shape, dt, dev), codes, scales)


def btx_rms_norm_backward_workspace_size(desc):
    sz = C.c_size_t(0)
    s = lib().btx_rms_norm_backward_workspace_size(C.byref(desc), C.byref(sz))
    if s != BTX_OK:
        raise BtxError(s, "btx_rms_norm_backward_workspace_size")
    return sz.value


def btx_rms_norm_backward(desc, h, weight, dy, dx, dweight, workspace, dh=None, accumulate=False):
    """Gradients of btx_rms_norm: dx in the tensors' type, dweight fp32 (None: not wanted); see btx.h."""
    d, dev = desc.d_model, _device(h)
    dt, shape = _DTYPE.get(desc.dtype), (desc.T, d)
    _launch("btx_rms_norm_backward", dev, C.byref(desc), *_rows(h, "h", shape, dt, dev), _opt(weight, "weight", (d,), dt, dev),
            *_rows(dy, "dy", shape, dt, dev), *_opt_rows(dh, "dh", shape, dt, dev), *_rows(dx, "dx", shape, dt, dev),
            _opt(dweight, "dweight", (d,), _F32, dev), int(accumulate), *_workspace(workspace, dev))


def btx_selftest_wait_expiry(workspace):
    """Makes one bounded device-side wait run out on purpose; see btx.h."""
    with _on(workspace.device):
        s = lib().btx_selftest_wait_expiry(_ptr(workspace), workspace.numel() * workspace.element_size(),
                                           _stream(workspace.device))
    if s != BTX_OK:
        raise BtxError(s, "btx_selftest_wait_expiry")


def btx_selftest_separate_launches(on):
    """Takes the separate launches of btx_mx4_moe_forward for every batch of this thread; see btx.h."""
    s = lib().btx_selftest_separate_launches(int(on))
    if s != BTX_OK:
        raise BtxError(s, "btx_selftest_separate_launches")


def btx_device_status(workspace):
    st = C.c_int32(0)
    with _on(workspace.device):
        s = lib().btx_device_status(_ptr(workspace), _stream(workspace.device), C.byref(st))
    if s != BTX_OK:
        raise BtxError(s, "btx_device_status")
    return st.value
