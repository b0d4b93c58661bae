"""Thin ctypes binding of ``libmoe_mi355x.so`` (declared in include/moe.h).

Argument marshalling only: every step of the layer runs in the library's HIP
kernels.  torch supplies device memory and the current HIP stream.  There is no
fallback of any kind: a missing library or a non-OK status raises.
"""
from __future__ import annotations

import ctypes
import functools
import os

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libmoe_mi355x.so")

MOE_OK = 0
MOE_ERR_NULL, MOE_ERR_SHAPE, MOE_ERR_UNSUPPORTED, MOE_ERR_ALIGN, MOE_ERR_WORKSPACE, MOE_ERR_HIP = range(1, 7)
STATUS_NAMES = {0: "MOE_OK", 1: "MOE_ERR_NULL", 2: "MOE_ERR_SHAPE", 3: "MOE_ERR_UNSUPPORTED",
                4: "MOE_ERR_ALIGN", 5: "MOE_ERR_WORKSPACE", 6: "MOE_ERR_HIP"}
SCORE = {"softmax": 0, "sigmoid": 1}
WFMT = {"bf16": 0, "fp8": 1, "int4": 2, "fp8a16": 3, "mxfp4": 4, "mxfp4x8": 5}
OFMT = {"f32": 0, "bf16": 1}
DTYPE = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
NORM = {"layer": 0, "rms": 1}
ACT = {"silu": 0, "gelu": 1}

EXPORTED = ("moe_status_str", "moe_permute_capacity", "moe_permute_workspace_bytes",
            "moe_gate_topk", "moe_router_gate_topk", "moe_router_workspace_bytes", "moe_permute", "moe_act_quant_fp8", "moe_workspace_bytes",
            "moe_workspace_layout", "moe_forward", "moe_forward_profiled", "moe_forward_static_ws",
            "moe_norm_forward", "moe_norm_backward", "moe_norm_backward_workspace_bytes",
            "moe_ffn_forward", "moe_ffn_backward", "moe_ffn_workspace_bytes", "moe_ffn_backward_workspace_bytes",
            # include/moe_peaks.h: achievable-peak probes
            "moe_peak_mfma_flops_per_launch", "moe_peak_sink_elems", "moe_peak_mfma", "moe_peak_read", "moe_peak_copy",
            "moe_peak_lds_copy_bytes_per_launch", "moe_peak_lds_copy", "moe_peak_lds_read_bytes_per_launch",
            "moe_peak_lds_read")
STATIC_WS_BYTES = 256 << 20  # MOE_STATIC_WS_BYTES: the library's own per-GPU workspace
NUM_STAGES = 6
STAGES = ("gate", "permute", "act_quant", "gemm1", "gemm2", "combine")


class MoeError(RuntimeError):
    def __init__(self, status: int, where: str):
        super().__init__(f"{where}: {STATUS_NAMES.get(status, status)}")
        self.status = status


class MoeArgs(ctypes.Structure):
    _fields_ = [
        ("T", ctypes.c_int32), ("H", ctypes.c_int32), ("E", ctypes.c_int32),
        ("I", ctypes.c_int32), ("top_k", ctypes.c_int32),
        ("score_mode", ctypes.c_int32), ("renormalize", ctypes.c_int32),
        ("routed_scale", ctypes.c_float), ("wfmt", ctypes.c_int32), ("ofmt", ctypes.c_int32),
        ("sel_bias", ctypes.c_void_p), ("hidden", ctypes.c_void_p), ("logits", ctypes.c_void_p),
        ("w1", ctypes.c_void_p), ("w2", ctypes.c_void_p),
        ("w1_scale", ctypes.c_void_p), ("w2_scale", ctypes.c_void_p),
        ("out", ctypes.c_void_p), ("topk_ids_out", ctypes.c_void_p), ("topk_w_out", ctypes.c_void_p),
        ("w_router", ctypes.c_void_p), ("logits_out", ctypes.c_void_p),
    ]


class MoeWsLayout(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in (
        "topk_ids", "topk_w", "expert_offsets", "sorted_ids", "inv_pos", "act_q", "act_s",
        "inter", "inter_s", "y", "permute_ws", "router_ws")] + [
        ("block_m", ctypes.c_int32), ("cap", ctypes.c_int32), ("total", ctypes.c_int64)]


class MoeFfnArgs(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("T", "H", "I", "dtype", "act")] + [
        (n, ctypes.c_void_p) for n in ("x", "w1", "w2", "add", "y", "pre", "dy", "dx", "dw1", "dw2")]


_lib = None


def lib() -> ctypes.CDLL:
    """Load the library once; raise if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build it with "
                              "`python -m paper_2607_12875_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, f32, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
        L.moe_status_str.restype = ctypes.c_char_p
        L.moe_status_str.argtypes = [i32]
        L.moe_permute_capacity.restype = sz
        L.moe_permute_capacity.argtypes = [i32, i32, i32, i32]
        L.moe_permute_workspace_bytes.restype = sz
        L.moe_permute_workspace_bytes.argtypes = [i32, i32, i32]
        L.moe_gate_topk.restype = i32
        L.moe_gate_topk.argtypes = [vp, vp, i32, i32, i32, i32, i32, f32, vp, vp, vp]
        L.moe_router_gate_topk.restype = i32
        L.moe_router_gate_topk.argtypes = [vp, vp, i32, i32, i32, i32, i32, i32, f32, vp, vp, vp, vp, vp, sz, vp]
        L.moe_router_workspace_bytes.restype = sz
        L.moe_router_workspace_bytes.argtypes = [i32, i32, i32]
        L.moe_permute.restype = i32
        L.moe_permute.argtypes = [vp, i32, i32, i32, i32, vp, vp, vp, i32, vp, sz, vp]
        L.moe_act_quant_fp8.restype = i32
        L.moe_act_quant_fp8.argtypes = [vp, i32, i32, vp, vp, vp]
        L.moe_workspace_bytes.restype = sz
        L.moe_workspace_bytes.argtypes = [ctypes.POINTER(MoeArgs)]
        L.moe_workspace_layout.restype = i32
        L.moe_workspace_layout.argtypes = [ctypes.POINTER(MoeArgs), ctypes.POINTER(MoeWsLayout)]
        L.moe_forward.restype = i32
        L.moe_forward.argtypes = [ctypes.POINTER(MoeArgs), vp, sz, vp]
        L.moe_forward_static_ws.restype = i32
        L.moe_forward_static_ws.argtypes = [ctypes.POINTER(MoeArgs), vp]
        L.moe_peak_mfma_flops_per_launch.restype = ctypes.c_longlong
        L.moe_peak_mfma_flops_per_launch.argtypes = [i32, i32]
        L.moe_peak_sink_elems.restype = i32
        L.moe_peak_sink_elems.argtypes = []
        L.moe_peak_read.restype = i32
        L.moe_peak_read.argtypes = [vp, sz, vp, vp]
        L.moe_peak_mfma.restype = i32
        L.moe_peak_mfma.argtypes = [i32, i32, vp, vp]
        L.moe_peak_copy.restype = i32
        L.moe_peak_copy.argtypes = [vp, vp, sz, vp]
        L.moe_peak_lds_copy_bytes_per_launch.restype = ctypes.c_longlong
        L.moe_peak_lds_copy_bytes_per_launch.argtypes = [i32, i32, i32]
        L.moe_peak_lds_copy.restype = i32
        L.moe_peak_lds_copy.argtypes = [vp, sz, i32, i32, i32, vp]
        L.moe_peak_lds_read_bytes_per_launch.restype = ctypes.c_longlong
        L.moe_peak_lds_read_bytes_per_launch.argtypes = [i32, i32]
        L.moe_peak_lds_read.restype = i32
        L.moe_peak_lds_read.argtypes = [i32, i32, vp, vp]
        L.moe_forward_profiled.restype = i32
        L.moe_forward_profiled.argtypes = [ctypes.POINTER(MoeArgs), vp, sz,
                                           ctypes.POINTER(ctypes.c_void_p), vp]
        L.moe_norm_forward.restype = i32
        L.moe_norm_forward.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, f32, vp, vp, vp, vp, vp]
        L.moe_norm_backward_workspace_bytes.restype = sz
        L.moe_norm_backward_workspace_bytes.argtypes = [i32, i32]
        L.moe_norm_backward.restype = i32
        L.moe_norm_backward.argtypes = [vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, vp, vp, vp, vp, sz, vp]
        for f in (L.moe_ffn_workspace_bytes, L.moe_ffn_backward_workspace_bytes):
            f.restype = sz
            f.argtypes = [ctypes.POINTER(MoeFfnArgs)]
        for f in (L.moe_ffn_forward, L.moe_ffn_backward):
            f.restype = i32
            f.argtypes = [ctypes.POINTER(MoeFfnArgs), vp, sz, vp]
        _lib = L
    return _lib


def _check(status: int, where: str):
    if status != MOE_OK:
        raise MoeError(status, where)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(stream=None):
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def _dev(*ts):
    for t in ts:
        if t is not None and (not t.is_cuda or not t.is_contiguous()):
            raise ValueError("tensors must be contiguous device tensors")


# ------------------------------------------------------------------ entry points
def moe_permute_capacity(T: int, top_k: int, E: int, block_m: int) -> int:
    return lib().moe_permute_capacity(T, top_k, E, block_m)


def moe_permute_workspace_bytes(T: int, top_k: int, E: int) -> int:
    return lib().moe_permute_workspace_bytes(T, top_k, E)


def moe_gate_topk(logits, top_k, mode="softmax", renormalize=True, routed_scale=1.0,
                  sel_bias=None, topk_ids=None, topk_w=None, stream=None):
    """MoE Gate: returns (topk_ids int32 [T,k], topk_w fp32 [T,k])."""
    _dev(logits, sel_bias)
    T, E = logits.shape
    if topk_ids is None:
        topk_ids = torch.empty((T, top_k), dtype=torch.int32, device=logits.device)
    if topk_w is None:
        topk_w = torch.empty((T, top_k), dtype=torch.float32, device=logits.device)
    _check(lib().moe_gate_topk(_ptr(logits), _ptr(sel_bias), T, E, top_k, SCORE[mode],
                               int(renormalize), float(routed_scale), _ptr(topk_ids),
                               _ptr(topk_w), _stream(stream)), "moe_gate_topk")
    return topk_ids, topk_w


def moe_router_gate_topk(hidden, w_router, top_k, mode="softmax", renormalize=True, routed_scale=1.0,
                         sel_bias=None, logits=None, topk_ids=None, topk_w=None, stream=None):
    """Router GEMM (bf16 hidden [T,H] x w_router [E,H]^T, fp32) then the
    gate: returns (topk_ids int32 [T,k], topk_w fp32 [T,k]); logits, if given
    (fp32 [T,E]), receives the logits the selection used."""
    _dev(hidden, w_router, sel_bias, logits)
    T, H = hidden.shape
    E = w_router.shape[0]
    if topk_ids is None:
        topk_ids = torch.empty((T, top_k), dtype=torch.int32, device=hidden.device)
    if topk_w is None:
        topk_w = torch.empty((T, top_k), dtype=torch.float32, device=hidden.device)
    nws = lib().moe_router_workspace_bytes(T, H, E)
    ws = torch.empty(max(nws, 16), dtype=torch.uint8, device=hidden.device)
    _check(lib().moe_router_gate_topk(_ptr(hidden), _ptr(w_router), T, H, E, top_k, SCORE[mode],
                                      int(renormalize), float(routed_scale), _ptr(sel_bias),
                                      _ptr(logits), _ptr(topk_ids), _ptr(topk_w), _ptr(ws), ws.numel(),
                                      _stream(stream)),
           "moe_router_gate_topk")
    return topk_ids, topk_w


def moe_permute(topk_ids, E: int, block_m: int, stream=None):
    """Permute/align: returns (expert_offsets [E+1], sorted_ids [cap], inv_pos [T*k])."""
    _dev(topk_ids)
    T, k = topk_ids.shape
    dev = topk_ids.device
    cap = moe_permute_capacity(T, k, E, block_m)
    offsets = torch.empty(E + 1, dtype=torch.int32, device=dev)
    sorted_ids = torch.empty(max(cap, 1), dtype=torch.int32, device=dev)
    inv_pos = torch.empty(max(T * k, 1), dtype=torch.int32, device=dev)
    nws = moe_permute_workspace_bytes(T, k, E)
    ws = torch.empty(max(nws, 16), dtype=torch.uint8, device=dev)
    _check(lib().moe_permute(_ptr(topk_ids), T, k, E, block_m, _ptr(offsets), _ptr(sorted_ids),
                             _ptr(inv_pos), cap, _ptr(ws), nws, _stream(stream)), "moe_permute")
    return offsets, sorted_ids[:cap], inv_pos[:T * k]


def moe_act_quant_fp8(x, stream=None):
    """Per (row, 128-column) e4m3 quantisation of bf16 x [M,K] -> (codes uint8, scales fp32)."""
    _dev(x)
    M, K = x.shape
    q = torch.empty((M, K), dtype=torch.uint8, device=x.device)
    s = torch.empty((M, max(K // 128, 1)), dtype=torch.float32, device=x.device)
    _check(lib().moe_act_quant_fp8(_ptr(x), M, K, _ptr(q), _ptr(s), _stream(stream)),
           "moe_act_quant_fp8")
    return q, s


def make_args(T, H, E, I, top_k, *, mode="softmax", renormalize=True, routed_scale=1.0,
              wfmt="bf16", out_dtype="f32", hidden=None, logits=None, w1=None, w2=None,
              w1_scale=None, w2_scale=None, sel_bias=None, out=None, topk_ids_out=None,
              topk_w_out=None, w_router=None, logits_out=None) -> MoeArgs:
    return MoeArgs(T, H, E, I, top_k, SCORE[mode], int(renormalize), float(routed_scale),
                   WFMT[wfmt], OFMT[out_dtype], _ptr(sel_bias), _ptr(hidden), _ptr(logits),
                   _ptr(w1), _ptr(w2), _ptr(w1_scale), _ptr(w2_scale), _ptr(out),
                   _ptr(topk_ids_out), _ptr(topk_w_out), _ptr(w_router), _ptr(logits_out))


def moe_workspace_bytes(args: MoeArgs) -> int:
    return lib().moe_workspace_bytes(ctypes.byref(args))


def moe_workspace_layout(args: MoeArgs) -> dict:
    L = MoeWsLayout()
    _check(lib().moe_workspace_layout(ctypes.byref(args), ctypes.byref(L)), "moe_workspace_layout")
    return {name: getattr(L, name) for name, _ in MoeWsLayout._fields_}


def moe_forward_args(args: MoeArgs, workspace, stream=None):
    """Run the layer on a prepared MoeArgs with a caller-owned uint8 workspace."""
    _check(lib().moe_forward(ctypes.byref(args), _ptr(workspace), workspace.numel(),
                             _stream(stream)), "moe_forward")


def moe_forward_static_ws(args: MoeArgs, stream=None):
    """Run the layer on a prepared MoeArgs in the library's own per-GPU
    workspace (no workspace argument, nothing allocated); the workspace the
    sizes need must not exceed STATIC_WS_BYTES."""
    _check(lib().moe_forward_static_ws(ctypes.byref(args), _stream(stream)), "moe_forward_static_ws")


def moe_forward_profiled(args: MoeArgs, workspace, events, stream=None):
    """moe_forward with hipEvent_t handles (ints) recorded around each stage."""
    arr = (ctypes.c_void_p * (NUM_STAGES + 1))(*events)
    _check(lib().moe_forward_profiled(ctypes.byref(args), _ptr(workspace), workspace.numel(),
                                      arr, _stream(stream)), "moe_forward_profiled")


def moe_forward(hidden, logits, w1, w2, top_k, *, mode="softmax", renormalize=True,
                routed_scale=1.0, wfmt="bf16", sel_bias=None, w1_scale=None, w2_scale=None,
                out_dtype="f32", out=None, workspace=None, topk_ids_out=None, topk_w_out=None,
                w_router=None, logits_out=None, stream=None):
    """The whole layer on device tensors; returns (out [T,H], workspace).

    hidden bf16 [T,H]; logits fp32 [T,E]; weights in the wfmt storage:
    bf16 [E,2I,H] / [E,H,I]; fp8 uint8 codes with fp32 block scales
    [E,2I/128,H/128] / [E,H/128,I/128]; int4 int32 [E,2I,H/8] / [E,H,I/8] with
    bf16 scales [E,2I,H/128] / [E,H,I/128]; "fp8a16" (weight-only fp8, a decode
    route) takes the fp8 storage with bf16 activations; "mxfp4" uint8
    [E,2I,H/2] / [E,H,I/2] two E2M1 codes per byte with uint8 E8M0 scales
    [E,2I,H/32] / [E,H,I/32] (bf16 activations); "mxfp4x8" the same storage
    with MXFP8 activations quantised in-layer.  With w_router (bf16
    [E,H]) the layer computes its own logits (pass logits=None); logits_out
    (fp32 [T,E]) then receives them."""
    _dev(hidden, logits, w1, w2, sel_bias, w1_scale, w2_scale, out, topk_ids_out, topk_w_out,
         w_router, logits_out)
    T, H = hidden.shape
    E = (w_router if w_router is not None else logits).shape[0 if w_router is not None else 1]
    I = w2.shape[2] * {"int4": 8, "mxfp4": 2, "mxfp4x8": 2}.get(wfmt, 1)
    if out is None:
        out = torch.empty((T, H), dtype=torch.float32 if out_dtype == "f32" else torch.bfloat16,
                          device=hidden.device)
    args = make_args(T, H, E, I, top_k, mode=mode, renormalize=renormalize,
                     routed_scale=routed_scale, wfmt=wfmt, out_dtype=out_dtype, hidden=hidden,
                     logits=logits, w1=w1, w2=w2, w1_scale=w1_scale, w2_scale=w2_scale,
                     sel_bias=sel_bias, out=out, topk_ids_out=topk_ids_out, topk_w_out=topk_w_out,
                     w_router=w_router, logits_out=logits_out)
    need = moe_workspace_bytes(args)
    if workspace is None or workspace.numel() < need:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=hidden.device)
    moe_forward_args(args, workspace, stream)
    return out, workspace


# ------------------------------------------------- norm, feed-forward block
# As under torch.cuda.stream, a caller who frees inputs that another stream allocated
# before stream= has run the call tells the allocator (Tensor.record_stream).
def _sizes(where, *n):
    """Refuse a size that a C int would cut, as the library refuses one past its limits."""
    if min(n) < -1 << 31 or max(n) >= 1 << 31:
        raise MoeError(MOE_ERR_SHAPE, where)


def _rows(x, name):
    """Shape and device index of a contiguous [T, width] device tensor."""
    i = x.get_device()
    if i < 0 or x.dim() != 2 or not x.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous two-dimensional device tensor")
    shape = x.shape
    if (shape[0] | shape[1]) >> 31:
        _sizes(name, *shape)
    return shape, i


def _dtype(x, name):
    d = DTYPE.get(x.dtype)
    if d is None:
        raise ValueError(f"{name}: {x.dtype} is not supported")
    return d


def _at(t, name, shape, dtype, index):
    """The address of t: None, or a contiguous tensor of that shape and type on device `index`."""
    if t is None:
        return None
    if t.shape != shape or t.dtype != dtype or t.get_device() != index or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous {dtype} tensor of shape {tuple(shape)} on cuda:{index}")
    return t.data_ptr()


def _on_stream(f):
    """With stream=, the whole call runs with that as the current stream, so that
    what it allocates belongs to it too."""
    first = f.__code__.co_varnames[0]

    @functools.wraps(f)
    def call(*args, stream=None, **kw):
        if stream is None:
            return f(*args, **kw)
        if (args[0] if args else kw[first]).get_device() != stream.device_index:
            raise ValueError(f"{first}: expected a tensor on the stream's device, cuda:{stream.device_index}")
        with torch.cuda.stream(stream):
            return f(*args, **kw)
    return call


def _call(f, where, index, *args):
    """f(*args, stream) on device `index` and its current stream."""
    s = torch._C._cuda_getCurrentRawStream(index)
    if index == torch._C._cuda_getDevice():
        status = f(*args, s)
    else:
        with torch.cuda.device(index):
            status = f(*args, s)
    if status != MOE_OK:
        raise MoeError(status, where)


@_on_stream
def moe_norm_forward(x, weight, *, bias=None, residual=None, kind="layer", eps=1e-5, y=None, sum_out=None,
                     stats=True):
    """Layer or rms norm of the rows of x [T,H] (fp32, bf16, fp16), or of x +
    residual: returns (y, s, mean, rstd).

    s is what was normalised: x itself, or the sum rounded to the type (in
    sum_out where given).  mean and rstd (fp32 [T], for moe_norm_backward) are
    None without stats, mean also for "rms".  weight and bias [H] in x's type.
    Results carry no autograd graph: moe_norm_backward is a call of its own."""
    shape, i = _rows(x, "x")
    T, H = shape
    dt, dtype = x.dtype, _dtype(x, "x")
    pw, pb = _at(weight, "weight", (H,), dt, i), _at(bias, "bias", (H,), dt, i)
    pr = _at(residual, "residual", shape, dt, i)
    if y is None:
        y = torch.empty_like(x)
    if residual is None:
        sum_out = None
    elif sum_out is None:
        sum_out = torch.empty_like(x)
    py, ps = _at(y, "y", shape, dt, i), _at(sum_out, "sum_out", shape, dt, i)
    mean = rstd = None
    if stats:
        rstd = torch.empty(T, dtype=torch.float32, device=x.device)
        if kind != "rms":
            mean = torch.empty_like(rstd)
    _call(lib().moe_norm_forward, "moe_norm_forward", i, x.data_ptr(), pr, pw, pb, T, H, NORM[kind], dtype,
          eps, py, ps, _ptr(mean), _ptr(rstd))
    return y, x if residual is None else sum_out, mean, rstd


@_on_stream
def moe_norm_backward(dy, x, weight, mean, rstd, *, kind="layer", dsum=None, dx=None, need_dweight=True,
                      need_dbias=False, workspace=None):
    """Backward pass of moe_norm_forward: returns (dx, dweight, dbias), the last
    two fp32 [H] or None.

    x is the s that the forward pass returned, mean and rstd its statistics
    (mean None for "rms"); dsum (or None) the gradient that reaches s on its
    other way, added to dx.  workspace: a uint8 tensor of
    moe_norm_backward_workspace_bytes; without, or with fewer, the call allocates
    one for itself."""
    shape, i = _rows(x, "x")
    T, H = shape
    dt, dtype, f32 = x.dtype, _dtype(x, "x"), torch.float32
    pdy, pw, pds = _at(dy, "dy", shape, dt, i), _at(weight, "weight", (H,), dt, i), _at(dsum, "dsum", shape, dt, i)
    pm, prs = _at(mean, "mean", (T,), f32, i), _at(rstd, "rstd", (T,), f32, i)
    if dx is None:
        dx = torch.empty_like(x)
    pdx = _at(dx, "dx", shape, dt, i)
    dweight = torch.empty(H, dtype=f32, device=x.device) if need_dweight else None
    dbias = torch.empty(H, dtype=f32, device=x.device) if need_dbias else None
    nws = lib().moe_norm_backward_workspace_bytes(T, H) if need_dweight or need_dbias else 0
    workspace = _workspace(workspace, nws, x) if nws else None
    _call(lib().moe_norm_backward, "moe_norm_backward", i, pdy, x.data_ptr(), pw, pm, prs, pds, T, H,
          NORM[kind], dtype, pdx, _ptr(dweight), _ptr(dbias), _ptr(workspace), nws)
    return dx, dweight, dbias


def moe_norm_backward_workspace_bytes(T: int, H: int) -> int:
    _sizes("moe_norm_backward_workspace_bytes", T, H)
    return lib().moe_norm_backward_workspace_bytes(T, H)


def _workspace(ws, need, ref):
    """ws if it holds need bytes on ref's device, else a new one."""
    if ws is None or ws.numel() * ws.element_size() < need or ws.get_device() != ref.get_device():
        return torch.empty(max(need, 256), dtype=torch.uint8, device=ref.device)
    if not ws.is_contiguous():
        raise ValueError("workspace: expected a contiguous tensor")
    return ws


def make_ffn_args(T, H, I, *, dtype=torch.bfloat16, act="silu", x=None, w1=None, w2=None, add=None, y=None, pre=None,
                  dy=None, dx=None, dw1=None, dw2=None) -> MoeFfnArgs:
    _sizes("make_ffn_args", T, H, I)
    return MoeFfnArgs(T, H, I, DTYPE[dtype], ACT[act], _ptr(x), _ptr(w1), _ptr(w2), _ptr(add), _ptr(y), _ptr(pre),
                      _ptr(dy), _ptr(dx), _ptr(dw1), _ptr(dw2))


def moe_ffn_workspace_bytes(args: MoeFfnArgs) -> int:
    return lib().moe_ffn_workspace_bytes(ctypes.byref(args))


def moe_ffn_backward_workspace_bytes(args: MoeFfnArgs) -> int:
    return lib().moe_ffn_backward_workspace_bytes(ctypes.byref(args))


@_on_stream
def moe_ffn_forward(x, w1, w2, *, act="silu", add=None, save=False, y=None, pre=None, workspace=None):
    """Gated feed-forward block y = (act(x w1[:I]^T) * (x w1[I:]^T)) w2^T + add on
    bf16 or fp16 x [T,H], w1 [2I,H], w2 [H,I] (H and I multiples of 8): returns
    (y, pre, workspace).

    With save, or into a pre that is given, pre (fp32 [T,2I]) keeps both
    projections for moe_ffn_backward, else it is None.  add [T,H] may be y itself.
    workspace: a uint8 tensor, kept from call to call; without, or with fewer than
    moe_ffn_workspace_bytes, a new one, which is returned.  Results carry no
    autograd graph: moe_ffn_backward is a call of its own."""
    shape, i = _rows(x, "x")
    T, H = shape
    I, dt = w2.shape[-1], x.dtype
    if I >> 31:
        _sizes("w2", I)
    if y is None:
        y = torch.empty_like(x)
    if save and pre is None:
        pre = torch.empty((T, 2 * I), dtype=torch.float32, device=x.device)
    args = MoeFfnArgs(T, H, I, _dtype(x, "x"), ACT[act], x.data_ptr(), _at(w1, "w1", (2 * I, H), dt, i),
                      _at(w2, "w2", (H, I), dt, i), _at(add, "add", shape, dt, i), _at(y, "y", shape, dt, i),
                      _at(pre, "pre", (T, 2 * I), torch.float32, i))
    at = ctypes.byref(args)
    workspace = _workspace(workspace, lib().moe_ffn_workspace_bytes(at), x)
    _call(lib().moe_ffn_forward, "moe_ffn_forward", i, at, workspace.data_ptr(),
          workspace.numel() * workspace.element_size())
    return y, pre, workspace


@_on_stream
def moe_ffn_backward(dy, x, w1, w2, pre, *, act="silu", dx=None, dw1=None, dw2=None, need=(True, True, True),
                     workspace=None):
    """Backward pass of moe_ffn_forward from its pre: returns (dx, dw1, dw2,
    workspace), the gradients in x's type.  need says which of them are
    computed; the others are None.  workspace as for moe_ffn_forward, of
    moe_ffn_backward_workspace_bytes."""
    shape, i = _rows(x, "x")
    T, H = shape
    I, dt = w2.shape[-1], x.dtype
    if I >> 31:
        _sizes("w2", I)
    dx = None if not need[0] else torch.empty_like(x) if dx is None else dx
    dw1 = None if not need[1] else torch.empty_like(w1) if dw1 is None else dw1
    dw2 = None if not need[2] else torch.empty_like(w2) if dw2 is None else dw2
    args = MoeFfnArgs(T, H, I, _dtype(x, "x"), ACT[act], x.data_ptr(), _at(w1, "w1", (2 * I, H), dt, i),
                      _at(w2, "w2", (H, I), dt, i), None, None, _at(pre, "pre", (T, 2 * I), torch.float32, i),
                      _at(dy, "dy", shape, dt, i), _at(dx, "dx", shape, dt, i), _at(dw1, "dw1", (2 * I, H), dt, i),
                      _at(dw2, "dw2", (H, I), dt, i))
    at = ctypes.byref(args)
    workspace = _workspace(workspace, lib().moe_ffn_backward_workspace_bytes(at), x)
    _call(lib().moe_ffn_backward, "moe_ffn_backward", i, at, workspace.data_ptr(),
          workspace.numel() * workspace.element_size())
    return dx, dw1, dw2, workspace


# ------------------------------------------------------------ peak probes
def moe_peak_mfma_flops_per_launch(fp8: bool, iters: int) -> int:
    return lib().moe_peak_mfma_flops_per_launch(int(bool(fp8)), iters)


def moe_peak_sink_elems() -> int:
    return lib().moe_peak_sink_elems()


def moe_peak_mfma(fp8: bool, iters: int, sink, stream=None):
    """One launch of the MFMA-only probe; sink: float32 device tensor of at
    least moe_peak_sink_elems() elements."""
    _dev(sink)
    if sink.dtype != torch.float32 or sink.numel() < moe_peak_sink_elems():
        raise ValueError("sink: float32, moe_peak_sink_elems() elements")
    _check(lib().moe_peak_mfma(int(bool(fp8)), iters, _ptr(sink), _stream(stream)), "moe_peak_mfma")


def moe_peak_read(src, sink, stream=None):
    """Read src once with the streaming probe; sink: int32 device tensor of at
    least moe_peak_sink_elems() zeroed elements, XORed with per-workgroup folds."""
    _dev(src, sink)
    if sink.dtype != torch.int32 or sink.numel() < moe_peak_sink_elems():
        raise ValueError("sink: int32, moe_peak_sink_elems() elements")
    n = src.numel() * src.element_size()
    _check(lib().moe_peak_read(_ptr(src), n, _ptr(sink), _stream(stream)), "moe_peak_read")


def moe_peak_copy(src, dst, stream=None):
    """dst[:] = src[:] (same byte size, 16-byte multiple) with the streaming copy probe."""
    _dev(src, dst)
    n = src.numel() * src.element_size()
    if dst.numel() * dst.element_size() != n:
        raise ValueError("src and dst must have the same size in bytes")
    _check(lib().moe_peak_copy(_ptr(src), _ptr(dst), n, _stream(stream)), "moe_peak_copy")


def moe_peak_lds_copy_bytes_per_launch(waves: int, copies: int, steps: int) -> int:
    return lib().moe_peak_lds_copy_bytes_per_launch(waves, copies, steps)


def moe_peak_lds_copy(src, region_bytes: int, waves: int, copies: int, steps: int, stream=None):
    """One launch of the global -> LDS copy probe over region b % 8 of src per
    workgroup b; src must hold 8 * region_bytes bytes."""
    _dev(src)
    if src.numel() * src.element_size() < 8 * region_bytes:
        raise ValueError("src must hold 8 * region_bytes bytes")
    _check(lib().moe_peak_lds_copy(_ptr(src), region_bytes, waves, copies, steps, _stream(stream)),
           "moe_peak_lds_copy")


def moe_peak_lds_read_bytes_per_launch(waves: int, iters: int) -> int:
    return lib().moe_peak_lds_read_bytes_per_launch(waves, iters)


def moe_peak_lds_read(waves: int, iters: int, sink, stream=None):
    """One launch of the LDS fragment-read probe; sink: int32 device tensor of
    at least moe_peak_sink_elems() elements."""
    _dev(sink)
    if sink.dtype != torch.int32 or sink.numel() < moe_peak_sink_elems():
        raise ValueError("sink: int32, moe_peak_sink_elems() elements")
    _check(lib().moe_peak_lds_read(waves, iters, _ptr(sink), _stream(stream)), "moe_peak_lds_read")
