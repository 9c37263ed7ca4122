"""Thin ctypes binding of libbpdq.so: same names as the C ABI (include/bpdq.h).

Only argument marshalling happens here: torch tensors supply device memory and the
current HIP stream; every step of the pass runs inside the library's kernels.  There is
no CPU fallback -- a missing library raises.
"""
from __future__ import annotations

import ctypes
import math
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libbpdq.so")
_lib = None

EXPORTS = [
    "bpdq_version",
    "bpdq_hessian_workspace_bytes", "bpdq_hessian_accumulate_f32", "bpdq_hessian_accumulate",
    "bpdq_hessian_accumulate_bf16x3", "bpdq_hessian_accumulate_timed",
    "bpdq_prepare_workspace_bytes", "bpdq_prepare",
    "bpdq_quantize_workspace_bytes", "bpdq_quantize_layer", "bpdq_quantize_layers", "bpdq_block_update",
    "bpdq_pack_planes", "bpdq_dequant", "bpdq_coefs_to_fp16", "bpdq_dequant_fp16",
    "bpdq_channel_order_workspace_bytes", "bpdq_channel_order", "bpdq_channel_order_noalloc",
    "bpdq_gather_columns",
    "bpdq_scatter_columns", "bpdq_gather_symmetric", "bpdq_gemv",
    "bpdq_linear_workspace_bytes", "bpdq_linear", "bpdq_gated_linear", "bpdq_rms_norm", "bpdq_rms_norm_q8", "bpdq_rotary_frequencies",
    "bpdq_rotary", "bpdq_sample_workspace_bytes", "bpdq_sample", "bpdq_kv_write", "bpdq_kv_read", "bpdq_kv_attention_workspace_bytes", "bpdq_kv_attention",
    "bpdq_probe_mfma", "bpdq_probe_copy",
]


class BpdqParams(ctypes.Structure):
    _fields_ = [("bits", ctypes.c_int), ("group", ctypes.c_int), ("block", ctypes.c_int),
                ("refine_iters", ctypes.c_int), ("alpha", ctypes.c_float),
                ("grid", ctypes.c_int), ("coef_fp16", ctypes.c_int)]


class BpdqKvCache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p), ("n_pages", ctypes.c_int), ("n_kv", ctypes.c_int),
                ("page", ctypes.c_int), ("head_dim", ctypes.c_int)]


class BpdqError(RuntimeError):
    pass


def load():
    """Load libbpdq.so (built by `python -m paper_2602_04163_amd.build`)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise BpdqError(f"{LIB_PATH} is missing: build it with "
                        "`python -m paper_2602_04163_amd.build` (there is no fallback path)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, ci, cf, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
    pp = ctypes.POINTER(BpdqParams)
    lib.bpdq_version.restype = ci
    lib.bpdq_version.argtypes = []
    lib.bpdq_hessian_workspace_bytes.restype = sz
    lib.bpdq_hessian_workspace_bytes.argtypes = [ci, ci]
    lib.bpdq_hessian_accumulate_f32.restype = ci
    lib.bpdq_hessian_accumulate_f32.argtypes = [vp, ci, ci, ci, cf, vp, ci, vp, sz, vp]
    for name in ("bpdq_hessian_accumulate", "bpdq_hessian_accumulate_bf16x3"):
        getattr(lib, name).restype = ci
        getattr(lib, name).argtypes = [vp, ci, ci, ci, cf, vp, ci, vp, sz, vp]
    lib.bpdq_hessian_accumulate_timed.restype = ci
    lib.bpdq_hessian_accumulate_timed.argtypes = [ci, vp, ci, ci, ci, cf, vp, ci, vp, sz, vp, vp, vp]
    lib.bpdq_prepare_workspace_bytes.restype = sz
    lib.bpdq_prepare_workspace_bytes.argtypes = [ci]
    lib.bpdq_prepare.restype = ci
    lib.bpdq_prepare.argtypes = [vp, ci, cf, vp, vp, vp, vp, sz, vp]
    lib.bpdq_quantize_workspace_bytes.restype = sz
    lib.bpdq_quantize_workspace_bytes.argtypes = [ci, ci, pp]
    lib.bpdq_quantize_layer.restype = ci
    lib.bpdq_quantize_layer.argtypes = [vp, ci, ci, vp, vp, pp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.bpdq_quantize_layers.restype = ci
    lib.bpdq_quantize_layers.argtypes = [vp, ci, ci, vp, vp, pp, ci, ctypes.POINTER(ci), vp, vp, vp,
                                         vp, vp, vp, sz, vp]
    lib.bpdq_block_update.restype = ci
    lib.bpdq_block_update.argtypes = [vp, ci, ci, vp, ci, ci, vp, ci, ci, ci, ci, vp]
    lib.bpdq_pack_planes.restype = ci
    lib.bpdq_pack_planes.argtypes = [vp, ci, ci, ci, vp, vp]
    lib.bpdq_dequant.restype = ci
    lib.bpdq_dequant.argtypes = [vp, vp, ci, ci, ci, ci, vp, vp]
    lib.bpdq_dequant_fp16.restype = ci
    lib.bpdq_dequant_fp16.argtypes = [vp, vp, ci, ci, ci, ci, vp, vp]
    lib.bpdq_coefs_to_fp16.restype = ci
    lib.bpdq_coefs_to_fp16.argtypes = [vp, ctypes.c_long, vp, vp]
    lib.bpdq_gemv.restype = ci
    lib.bpdq_gemv.argtypes = [vp, vp, ci, ci, ci, ci, vp, vp, vp]
    cl, kv = ctypes.c_long, ctypes.POINTER(BpdqKvCache)
    lib.bpdq_linear.restype = ci
    lib.bpdq_linear.argtypes = [vp, vp, ci, ci, ci, ci, vp, ci, cl, ci, vp, ci, vp, cl, vp, cl, vp, sz, vp]
    lib.bpdq_linear_workspace_bytes.restype = sz
    lib.bpdq_linear_workspace_bytes.argtypes = [ci, ci]
    lib.bpdq_gated_linear.restype = ci
    lib.bpdq_gated_linear.argtypes = [vp, vp, ci, ci, ci, ci, vp, ci, cl, ci, vp, ci, vp, cl, vp, sz, vp]
    lib.bpdq_rms_norm.restype = ci
    lib.bpdq_rms_norm.argtypes = [vp, ci, ci, cl, ci, vp, cl, ci, vp, cl, vp, cf, cf, vp, cl, vp]
    lib.bpdq_rms_norm_q8.restype = ci
    lib.bpdq_rms_norm_q8.argtypes = [vp, ci, ci, cl, ci, vp, cl, ci, vp, cl, vp, cf, cf, ci, vp, cl, vp, vp]
    cd = ctypes.c_double
    lib.bpdq_rotary_frequencies.restype = ci
    lib.bpdq_rotary_frequencies.argtypes = [ci, cd, ci, cd, cd, cd, ci, vp, vp]
    lib.bpdq_rotary.restype = ci
    lib.bpdq_rotary.argtypes = [vp, ci, ci, cf, ci, vp, vp, ci, ci, ci, vp, cl, ci, vp, cl, ci, ci, ci, vp, cl, vp, cl, vp]
    lib.bpdq_sample_workspace_bytes.restype = sz
    lib.bpdq_sample_workspace_bytes.argtypes = [ci, ci]
    lib.bpdq_sample.restype = ci
    lib.bpdq_sample.argtypes = [vp, ci, ci, cl, ci, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    for name in ("bpdq_kv_write", "bpdq_kv_read"):
        getattr(lib, name).restype = ci
        getattr(lib, name).argtypes = [kv, vp, ci, ci, vp, vp, ci, ci, vp, cl, vp, cl, ci, vp]
    lib.bpdq_kv_attention_workspace_bytes.restype = sz
    lib.bpdq_kv_attention_workspace_bytes.argtypes = [ci, ci, ci, ci, ci, ci, ci]
    lib.bpdq_kv_attention.restype = ci
    lib.bpdq_kv_attention.argtypes = [kv, vp, ci, ci, vp, vp, ci, ci, ci, vp, cl, ci, ci, cf, ci, ci, vp, cl, vp, vp, sz, vp]
    lib.bpdq_channel_order_workspace_bytes.restype = sz
    lib.bpdq_channel_order_workspace_bytes.argtypes = [ci]
    lib.bpdq_channel_order.restype = ci
    lib.bpdq_channel_order.argtypes = [vp, ci, ci, vp, vp, sz, vp]
    lib.bpdq_channel_order_noalloc.restype = ci
    lib.bpdq_channel_order_noalloc.argtypes = [vp, ci, ci, vp, vp]
    lib.bpdq_gather_columns.restype = ci
    lib.bpdq_gather_columns.argtypes = [vp, ci, ci, vp, vp, vp]
    lib.bpdq_scatter_columns.restype = ci
    lib.bpdq_scatter_columns.argtypes = [vp, ci, ci, vp, vp, vp]
    lib.bpdq_gather_symmetric.restype = ci
    lib.bpdq_gather_symmetric.argtypes = [vp, ci, vp, vp, vp]
    lib.bpdq_probe_mfma.restype = ci
    lib.bpdq_probe_mfma.argtypes = [ci, ci, ci, ci, ci, vp, ctypes.POINTER(ctypes.c_double), vp]
    lib.bpdq_probe_copy.restype = ci
    lib.bpdq_probe_copy.argtypes = [vp, vp, ctypes.c_long, vp]
    _lib = lib
    return lib


# private to torch; where a torch lacks it the handle comes by way of a Stream object
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream():
    # the current stream's handle without the Stream object that torch.cuda.current_stream() builds
    # (2.8 of the 8.4 us of host time of a bpdq_gemv call)
    if _raw_stream is None:
        return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    return ctypes.c_void_p(_raw_stream(torch.cuda.current_device()))


def _ptr(t):
    return ctypes.c_void_p(0 if t is None else t.data_ptr())


def _check(rc, name):
    if rc != 0:
        raise BpdqError(f"{name} returned {rc}" + (f" (argument {-rc} invalid)" if -99 < rc < 0 else ""))


def _dev(t, dtype, name):
    if not (t.is_cuda and t.dtype == dtype and t.is_contiguous()):
        raise BpdqError(f"{name}: expected a contiguous {dtype} tensor on the GPU")


def _workspace(nbytes, device):
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def _ws(ws):
    """Address and bytes of a workspace, which may be a caller's: a contiguous tensor of any type on the GPU, or None."""
    if ws is None:
        return None, 0
    if not (ws.is_cuda and ws.is_contiguous()):
        raise BpdqError("ws: expected a contiguous tensor on the GPU")
    return ws.data_ptr(), ws.numel() * ws.element_size()


def bpdq_version() -> int:
    return load().bpdq_version()


def bpdq_hessian_workspace_bytes(n_tok: int, d_in: int) -> int:
    return load().bpdq_hessian_workspace_bytes(n_tok, d_in)


def bpdq_hessian_accumulate(Xc, H, scale=2.0, symmetrize=False, ws=None, _entry="bpdq_hessian_accumulate"):
    """H += scale * Xc^T Xc (upper triangle; mirrored when symmetrize), on the fp16 matrix cores
    with two fp16 halves per channel-scaled value; small calls in one launch on the fp32 matrix cores."""
    lib = load()
    _dev(H, torch.float32, "H")
    if not (Xc.is_cuda and Xc.dtype == torch.float32 and Xc.dim() == 2 and Xc.stride(1) == 1):
        raise BpdqError("Xc: expected a float32 GPU matrix with unit column stride")
    n_tok, d_in = Xc.shape
    if H.shape != (d_in, d_in):
        raise BpdqError("H: expected d_in x d_in")
    if ws is None:
        ws = _workspace(lib.bpdq_hessian_workspace_bytes(n_tok, d_in), H.device)
    rc = getattr(lib, _entry)(_ptr(Xc), n_tok, d_in, Xc.stride(0) if n_tok > 1 else d_in,
                              scale, _ptr(H), int(bool(symmetrize)), *_ws(ws),
                              _stream())
    _check(rc, _entry)
    return H


def bpdq_hessian_accumulate_f32(Xc, H, scale=2.0, symmetrize=False, ws=None):
    """bpdq_hessian_accumulate on the fp32 matrix cores."""
    return bpdq_hessian_accumulate(Xc, H, scale, symmetrize, ws, _entry="bpdq_hessian_accumulate_f32")


def bpdq_hessian_accumulate_bf16x3(Xc, H, scale=2.0, symmetrize=False, ws=None):
    """bpdq_hessian_accumulate on the bf16 matrix cores, three bf16 pieces per value."""
    return bpdq_hessian_accumulate(Xc, H, scale, symmetrize, ws, _entry="bpdq_hessian_accumulate_bf16x3")


HESSIAN_KERNELS = {"f16x2": 0, "bf16x3": 1, "f32": 2}


def bpdq_hessian_accumulate_timed(kernel, Xc, H, scale=2.0, symmetrize=False, ws=None, ev_begin=None,
                                  ev_end=None):
    """bpdq_hessian_accumulate with the kernel chosen by name; ev_begin / ev_end are torch.cuda.Event
    objects (timing enabled, recorded at least once before so that they exist) that the library
    records right around the tile-product kernel."""
    lib = load()
    _dev(H, torch.float32, "H")
    n_tok, d_in = Xc.shape
    if ws is None:
        ws = _workspace(lib.bpdq_hessian_workspace_bytes(n_tok, d_in), H.device)
    ev = [ctypes.c_void_p(0 if e is None else e.cuda_event) for e in (ev_begin, ev_end)]
    rc = lib.bpdq_hessian_accumulate_timed(HESSIAN_KERNELS[kernel], _ptr(Xc), n_tok, d_in,
                                           Xc.stride(0) if n_tok > 1 else d_in, scale, _ptr(H),
                                           int(bool(symmetrize)), *_ws(ws), _stream(), ev[0], ev[1])
    _check(rc, "bpdq_hessian_accumulate_timed")
    return H


def bpdq_prepare_workspace_bytes(d_in: int) -> int:
    return load().bpdq_prepare_workspace_bytes(d_in)


def bpdq_prepare(H, damp=0.01, U=None, ws=None):
    """Returns (U, dead, info): U = chol_upper((H + damp*mean(diag H) I)^-1)."""
    lib = load()
    _dev(H, torch.float32, "H")
    d_in = H.shape[0]
    if U is None:
        U = torch.empty_like(H)
    _dev(U, torch.float32, "U")
    dead = torch.empty(d_in, dtype=torch.uint8, device=H.device)
    info = torch.empty(1, dtype=torch.int32, device=H.device)
    if ws is None:
        ws = _workspace(lib.bpdq_prepare_workspace_bytes(d_in), H.device)
    rc = lib.bpdq_prepare(_ptr(H), d_in, damp, _ptr(U), _ptr(dead), _ptr(info), *_ws(ws), _stream())
    _check(rc, "bpdq_prepare")
    return U, dead, info


GRID_VARIABLE, GRID_UNIFORM = 0, 1


def make_params(bits, group, block, refine_iters, alpha=1e-4, grid=GRID_VARIABLE,
                coef_fp16=False) -> BpdqParams:
    return BpdqParams(bits, group, block, refine_iters, alpha, grid, int(bool(coef_fp16)))


def bpdq_quantize_workspace_bytes(d_out, d_in, params: BpdqParams) -> int:
    return load().bpdq_quantize_workspace_bytes(d_out, d_in, ctypes.byref(params))


def bpdq_quantize_layer(W, U, dead, params: BpdqParams, want_w_hat=True, ws=None, out=None):
    """Returns dict(planes, coefs, W_hat, grp_err, grp_iter) of device tensors."""
    lib = load()
    _dev(W, torch.float32, "W")
    _dev(U, torch.float32, "U")
    d_out, d_in = W.shape
    k, g = params.bits, params.group
    dev = W.device
    if out is None:
        out = dict(
            planes=torch.empty((k, d_out, d_in // 32), dtype=torch.int32, device=dev),
            coefs=torch.empty((k + 1, d_out, d_in // g), dtype=torch.float32, device=dev),
            W_hat=torch.empty((d_out, d_in), dtype=torch.float32, device=dev) if want_w_hat else None,
            grp_err=torch.empty(d_in // g, dtype=torch.float64, device=dev),
            grp_iter=torch.empty(d_in // g, dtype=torch.int32, device=dev),
        )
    if ws is None:
        need = lib.bpdq_quantize_workspace_bytes(d_out, d_in, ctypes.byref(params))
        if need == 0:
            raise BpdqError("bpdq_quantize_workspace_bytes: invalid parameters")
        ws = _workspace(need, dev)
    rc = lib.bpdq_quantize_layer(_ptr(W), d_out, d_in, _ptr(U), _ptr(dead), ctypes.byref(params),
                                 _ptr(out["planes"]), _ptr(out["coefs"]), _ptr(out["W_hat"]),
                                 _ptr(out["grp_err"]), _ptr(out["grp_iter"]), *_ws(ws),
                                 _stream())
    _check(rc, "bpdq_quantize_layer")
    return out


def bpdq_quantize_layers(W, seg_end, U, dead, params: BpdqParams, want_w_hat=True, ws=None):
    """Layers sharing one U, stacked by rows (seg_end = ascending row boundaries).  Returns the
    same dict as bpdq_quantize_layer with grp_err / grp_iter of shape (n_seg, d_in/g)."""
    lib = load()
    _dev(W, torch.float32, "W")
    _dev(U, torch.float32, "U")
    d_out, d_in = W.shape
    k, g = params.bits, params.group
    dev = W.device
    n_seg = len(seg_end)
    out = dict(
        planes=torch.empty((k, d_out, d_in // 32), dtype=torch.int32, device=dev),
        coefs=torch.empty((k + 1, d_out, d_in // g), dtype=torch.float32, device=dev),
        W_hat=torch.empty((d_out, d_in), dtype=torch.float32, device=dev) if want_w_hat else None,
        grp_err=torch.empty((n_seg, d_in // g), dtype=torch.float64, device=dev),
        grp_iter=torch.empty((n_seg, d_in // g), dtype=torch.int32, device=dev),
    )
    if ws is None:
        need = lib.bpdq_quantize_workspace_bytes(d_out, d_in, ctypes.byref(params))
        if need == 0:
            raise BpdqError("bpdq_quantize_workspace_bytes: invalid parameters")
        ws = _workspace(need, dev)
    seg = (ctypes.c_int * n_seg)(*[int(e) for e in seg_end])
    rc = lib.bpdq_quantize_layers(_ptr(W), d_out, d_in, _ptr(U), _ptr(dead), ctypes.byref(params),
                                  n_seg, seg, _ptr(out["planes"]), _ptr(out["coefs"]),
                                  _ptr(out["W_hat"]), _ptr(out["grp_err"]), _ptr(out["grp_iter"]),
                                  *_ws(ws), _stream())
    _check(rc, "bpdq_quantize_layers")
    return out


def bpdq_block_update(Et, U, k0, Wp, c_begin, c_end, d_out=None):
    """Wp[:, c_begin:c_end] -= Et^T U[k0:k0+Kd, c_begin:c_end] in place (Et: Kd x lde, K-major)."""
    lib = load()
    _dev(Et, torch.float32, "Et")
    _dev(U, torch.float32, "U")
    _dev(Wp, torch.float32, "Wp")
    Kd, lde = Et.shape
    d_out = Wp.shape[0] if d_out is None else d_out
    _check(lib.bpdq_block_update(_ptr(Et), lde, Kd, _ptr(U), U.shape[1], k0, _ptr(Wp), Wp.shape[1], d_out,
                                 c_begin, c_end, _stream()), "bpdq_block_update")
    return Wp


def bpdq_pack_planes(codes, bits):
    lib = load()
    _dev(codes, torch.uint8, "codes")
    d_out, d_in = codes.shape
    planes = torch.empty((bits, d_out, d_in // 32), dtype=torch.int32, device=codes.device)
    _check(lib.bpdq_pack_planes(_ptr(codes), d_out, d_in, bits, _ptr(planes), _stream()),
           "bpdq_pack_planes")
    return planes


def bpdq_dequant(planes, coefs, group):
    lib = load()
    _dev(planes, torch.int32, "planes")
    _dev(coefs, torch.float32, "coefs")
    bits, d_out, nw = planes.shape
    d_in = nw * 32
    W_hat = torch.empty((d_out, d_in), dtype=torch.float32, device=planes.device)
    _check(lib.bpdq_dequant(_ptr(planes), _ptr(coefs), d_out, d_in, bits, group, _ptr(W_hat),
                            _stream()), "bpdq_dequant")
    return W_hat


def bpdq_coefs_to_fp16(coefs):
    """Half-precision copy of the coefficients (same shape, torch.float16)."""
    lib = load()
    _dev(coefs, torch.float32, "coefs")
    out = torch.empty(coefs.shape, dtype=torch.float16, device=coefs.device)
    _check(lib.bpdq_coefs_to_fp16(_ptr(coefs), coefs.numel(), _ptr(out), _stream()),
           "bpdq_coefs_to_fp16")
    return out


def bpdq_dequant_fp16(planes, coefs_h, group):
    lib = load()
    _dev(planes, torch.int32, "planes")
    _dev(coefs_h, torch.float16, "coefs_h")
    bits, d_out, nw = planes.shape
    d_in = nw * 32
    W_hat = torch.empty((d_out, d_in), dtype=torch.float32, device=planes.device)
    _check(lib.bpdq_dequant_fp16(_ptr(planes), _ptr(coefs_h), d_out, d_in, bits, group, _ptr(W_hat),
                                 _stream()), "bpdq_dequant_fp16")
    return W_hat


def bpdq_channel_order(H, group_size=1):
    """perm (int32, d_in): channels by descending H_jj, or blocks of group_size channels by
    descending block sum."""
    lib = load()
    _dev(H, torch.float32, "H")
    d_in = H.shape[0]
    perm = torch.empty(d_in, dtype=torch.int32, device=H.device)
    ws = _workspace(lib.bpdq_channel_order_workspace_bytes(d_in), H.device)
    _check(lib.bpdq_channel_order(_ptr(H), d_in, group_size, _ptr(perm), *_ws(ws),
                                  _stream()), "bpdq_channel_order")
    return perm


def bpdq_channel_order_noalloc(H, group_size=1, perm=None):
    """bpdq_channel_order without a workspace: the library's built-in scratch holds the keys.
    `perm` may be passed in, so that the call allocates nothing at all."""
    lib = load()
    _dev(H, torch.float32, "H")
    d_in = H.shape[0]
    if perm is None:
        perm = torch.empty(d_in, dtype=torch.int32, device=H.device)
    _dev(perm, torch.int32, "perm")
    _check(lib.bpdq_channel_order_noalloc(_ptr(H), d_in, group_size, _ptr(perm), _stream()),
           "bpdq_channel_order_noalloc")
    return perm


def bpdq_gather_columns(W, perm):
    lib = load()
    _dev(W, torch.float32, "W")
    _dev(perm, torch.int32, "perm")
    out = torch.empty_like(W)
    _check(lib.bpdq_gather_columns(_ptr(W), W.shape[0], W.shape[1], _ptr(perm), _ptr(out), _stream()),
           "bpdq_gather_columns")
    return out


def bpdq_scatter_columns(Wp, perm):
    lib = load()
    _dev(Wp, torch.float32, "Wp")
    _dev(perm, torch.int32, "perm")
    out = torch.empty_like(Wp)
    _check(lib.bpdq_scatter_columns(_ptr(Wp), Wp.shape[0], Wp.shape[1], _ptr(perm), _ptr(out),
                                    _stream()), "bpdq_scatter_columns")
    return out


def bpdq_gather_symmetric(H, perm):
    lib = load()
    _dev(H, torch.float32, "H")
    _dev(perm, torch.int32, "perm")
    out = torch.empty_like(H)
    _check(lib.bpdq_gather_symmetric(_ptr(H), H.shape[0], _ptr(perm), _ptr(out), _stream()),
           "bpdq_gather_symmetric")
    return out


def bpdq_gemv(planes, coefs_h, group, x, y=None):
    """y = What x for one token from the stored format (planes int32, coefficients float16)."""
    lib = load()
    _dev(planes, torch.int32, "planes")
    _dev(coefs_h, torch.float16, "coefs_h")
    _dev(x, torch.float32, "x")
    bits, d_out, nw = planes.shape
    d_in = nw * 32
    if x.numel() != d_in:
        raise BpdqError("x: expected d_in values")
    if y is None:
        y = torch.empty(d_out, dtype=torch.float32, device=planes.device)
    _check(lib.bpdq_gemv(_ptr(planes), _ptr(coefs_h), d_out, d_in, bits, group, _ptr(x), _ptr(y),
                         _stream()), "bpdq_gemv")
    return y


DTYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
ACTS = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}


def _rows(t, dtype, shape, name):
    """The row stride of a tensor of the given shape on the GPU whose rows (all axes but the first) are dense and do not overlap (one row that
    is expanded to several does)."""
    if t.dtype is not dtype or t.shape != shape or not t.is_cuda:
        raise BpdqError(f"{name}: expected a {dtype} tensor of shape {tuple(shape)} on the GPU")
    if t.is_contiguous():
        return t.numel() // shape[0] if shape[0] else math.prod(shape[1:])
    strides = t.stride()
    step = 1
    for axis in range(len(shape) - 1, 0, -1):
        if strides[axis] != step and shape[axis] > 1:
            raise BpdqError(f"{name}: its rows must be dense")
        step *= shape[axis]
    if shape[0] <= 1:
        return step
    if strides[0] < step:
        raise BpdqError(f"{name}: its rows must not overlap")
    return strides[0]


def _call(name, rc):
    if rc:
        _check(rc, name)


def _here(*tensors):
    """Refuses tensors on another GPU than the current one, on whose stream the kernels run."""
    here = torch.cuda.current_device()
    for t in tensors:
        if t is not None and t.get_device() != here:
            raise BpdqError(f"a tensor on GPU {t.get_device()}, and the current one is {here}")


def _like(t):
    """A new tensor of dense rows."""
    return torch.empty_like(t, memory_format=torch.contiguous_format)


def _scratch(nbytes, device):
    """A workspace, or None where none is asked for."""
    return torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None


def bpdq_linear_workspace_bytes(n_tok, d_in):
    return load().bpdq_linear_workspace_bytes(n_tok, d_in)


def bpdq_linear(planes, coefs_h, group, X, bias=None, act="none", residual=None, Y=None, ws=None):
    """Y = act(X What^T + bias) + residual from the stored format, for any number of tokens; X, bias, residual and Y float16 or
    bfloat16.  Y may be the residual."""
    lib = _lib or load()
    _dev(planes, torch.int32, "planes")
    _dev(coefs_h, torch.float16, "coefs_h")
    bits, d_out, nw = planes.shape
    d_in, dtype = nw * 32, X.dtype
    if group <= 0 or coefs_h.shape != (bits + 1, d_out, d_in // group):
        raise BpdqError("coefs_h: expected (bits + 1) x d_out x (d_in / group)")
    if X.dim() != 2 or (dtype is not torch.bfloat16 and dtype is not torch.float16):
        raise BpdqError("X: expected a float16 or bfloat16 matrix")
    code = ACTS.get(act)
    if code is None:
        raise BpdqError(f"act: expected one of {sorted(ACTS)}")
    n_tok = X.shape[0]
    ldx = _rows(X, dtype, (n_tok, d_in), "X")
    rows = (n_tok, d_out)
    if Y is None:
        Y = torch.empty(rows, dtype=dtype, device=X.device)
        ldy = d_out
    else:
        ldy = _rows(Y, dtype, rows, "Y")
    if bias is not None and (bias.dtype is not dtype or bias.shape != (d_out,) or not bias.is_cuda or not bias.is_contiguous()):
        raise BpdqError(f"bias: expected a contiguous {dtype} vector of d_out values on the GPU")
    ldr = 0 if residual is None else _rows(residual, dtype, rows, "residual")
    if ws is None:
        ws = _scratch(lib.bpdq_linear_workspace_bytes(n_tok, d_in), X.device)
    _call("bpdq_linear", lib.bpdq_linear(
        planes.data_ptr(), coefs_h.data_ptr(), d_out, d_in, bits, group, X.data_ptr(), n_tok, ldx, DTYPES[dtype],
        None if bias is None else bias.data_ptr(), code, None if residual is None else residual.data_ptr(), ldr, Y.data_ptr(), ldy,
        *_ws(ws), _stream()))
    return Y


def bpdq_gated_linear(planes, coefs_h, group, X, bias=None, act="silu", Y=None, ws=None):
    """Y = act(X Wgate^T + bias[:d_out]) * (X Wup^T + bias[d_out:]) from the stored format: two layers stacked by rows, gate first, as
    bpdq_quantize_layers leaves them (2 d_out rows); X, bias and Y float16 or bfloat16, for any number of tokens."""
    lib = _lib or load()
    _dev(planes, torch.int32, "planes")
    _dev(coefs_h, torch.float16, "coefs_h")
    bits, rows, nw = planes.shape
    d_out, d_in, dtype = rows // 2, nw * 32, X.dtype
    if rows % 2:
        raise BpdqError("planes: expected an even number of rows, those of the gate and as many of the other projection")
    if group <= 0 or coefs_h.shape != (bits + 1, rows, d_in // group):
        raise BpdqError("coefs_h: expected (bits + 1) x (2 d_out) x (d_in / group)")
    if X.dim() != 2 or (dtype is not torch.bfloat16 and dtype is not torch.float16):
        raise BpdqError("X: expected a float16 or bfloat16 matrix")
    code = ACTS.get(act)
    if code is None:
        raise BpdqError(f"act: expected one of {sorted(ACTS)}")
    n_tok = X.shape[0]
    ldx = _rows(X, dtype, (n_tok, d_in), "X")
    if Y is None:
        Y = torch.empty((n_tok, d_out), dtype=dtype, device=X.device)
        ldy = d_out
    else:
        ldy = _rows(Y, dtype, (n_tok, d_out), "Y")
    if bias is not None and (bias.dtype is not dtype or bias.shape != (rows,) or not bias.is_cuda or not bias.is_contiguous()):
        raise BpdqError(f"bias: expected a contiguous {dtype} vector of 2 d_out values on the GPU")
    if ws is None:
        ws = _scratch(lib.bpdq_linear_workspace_bytes(n_tok, d_in), X.device)
    _here(X, planes, coefs_h, bias, Y, ws)
    _call("bpdq_gated_linear", lib.bpdq_gated_linear(
        planes.data_ptr(), coefs_h.data_ptr(), d_out, d_in, bits, group, X.data_ptr(), n_tok, ldx, DTYPES[dtype],
        None if bias is None else bias.data_ptr(), code, Y.data_ptr(), ldy, *_ws(ws), _stream()))
    return Y


def _norm(X, weight, residual, S):
    """The arguments that both norms begin with, and S."""
    dtype = X.dtype
    if X.dim() != 2 or dtype not in DTYPES:
        raise BpdqError("X: expected a float32, float16 or bfloat16 matrix")
    shape = n_tok, d = X.shape
    ldx, ldr, lds, wide = _rows(X, dtype, shape, "X"), 0, 0, dtype
    if weight is not None and (weight.dtype is not dtype or weight.shape != (d,) or not weight.is_cuda or not weight.is_contiguous()):
        raise BpdqError(f"weight: expected a contiguous {dtype} vector of d values on the GPU")
    if residual is not None:
        wide = residual.dtype
        if wide is not dtype and wide is not torch.float32:
            raise BpdqError(f"residual: expected {dtype} or float32")
        ldr = _rows(residual, wide, shape, "residual")
        if S is None:
            S, lds = _like(residual), d
        else:
            lds = _rows(S, wide, shape, "S")
    elif S is not None:
        raise BpdqError("S: the sum, only with a residual")
    return (X.data_ptr(), n_tok, d, ldx, DTYPES[dtype], None if residual is None else residual.data_ptr(), ldr, DTYPES[wide],
            None if S is None else S.data_ptr(), lds, None if weight is None else weight.data_ptr()), S


def bpdq_rms_norm(X, weight=None, eps=1e-6, residual=None, S=None, offset=0.0, Y=None):
    """Returns (Y, S): S = X + residual (None without a residual), in the residual's type (X's or float32), and
    Y = S / sqrt(mean(S^2) + eps) * (offset + weight) in X's.  S may be the residual, Y may be X."""
    args, S = _norm(X, weight, residual, S)
    if Y is None:
        Y, ldy = _like(X), X.shape[1]
    else:
        ldy = _rows(Y, X.dtype, X.shape, "Y")
    _here(X, weight, residual, S, Y)
    _call("bpdq_rms_norm", (_lib or load()).bpdq_rms_norm(*args, offset, eps, Y.data_ptr(), ldy, _stream()))
    return Y, S


def bpdq_rms_norm_q8(X, weight=None, eps=1e-6, residual=None, S=None, offset=0.0, group=0, codes=None, scales=None):
    """bpdq_rms_norm with Y in 8 bits: returns (codes, scales, S), codes int8, scales float32 of n_tok x (d / group), one a row for group 0."""
    args, S = _norm(X, weight, residual, S)
    n_tok, d = X.shape
    if codes is None:
        codes = torch.empty((n_tok, d), dtype=torch.int8, device=X.device)
    ldc = _rows(codes, torch.int8, (n_tok, d), "codes")
    shape = (n_tok, d // group if group > 0 else 1)
    if scales is None:
        scales = torch.empty(shape, dtype=torch.float32, device=X.device)
    _dev(scales, torch.float32, "scales")
    if scales.shape != shape:
        raise BpdqError("scales: expected n_tok x (d / group)")
    _here(X, weight, residual, S, codes, scales)
    _call("bpdq_rms_norm_q8", (_lib or load()).bpdq_rms_norm_q8(*args, offset, eps, group, codes.data_ptr(), ldc, scales.data_ptr(),
                                                                _stream()))
    return codes, scales, S


ROTARY_LAYOUTS = {"half": 0, "interleaved": 1}
ROTARY_SCALINGS = {"plain": 0, "linear": 1, "ntk": 2, "yarn": 3, "bands": 4}


def bpdq_rotary_frequencies(rot, base=10000.0, scaling="plain", factor=1.0, low=1.0, high=32.0, original=4096):
    """Radians per position of the rot / 2 pairs of channels (a float64 tensor on the host), and the factor on cosine and sine that goes with
    them.  scaling: plain, linear, ntk, yarn or bands (include/bpdq.h); factor, low, high and original are those of the scaling."""
    code = ROTARY_SCALINGS.get(scaling)
    if code is None:
        raise BpdqError(f"scaling: expected one of {sorted(ROTARY_SCALINGS)}")
    freq, mscale = torch.empty(max(rot // 2, 1), dtype=torch.float64), ctypes.c_double()
    _call("bpdq_rotary_frequencies", (_lib or load()).bpdq_rotary_frequencies(
        rot, base, code, factor, low, high, original, freq.data_ptr(), ctypes.addressof(mscale)))
    return freq, mscale.value


def bpdq_rotary(freq, pos, tok_start, Q, K=None, max_tok=None, layout="half", mscale=1.0, inverse=False, Q_out=None, K_out=None):
    """Rotary positions on Q (n_tok, n_q, head_dim) and K (n_tok, n_kv, head_dim): row tok_start[b] + i is at position pos[b] + i.  freq: float64
    on the GPU, rot / 2 frequencies (bpdq_rotary_frequencies); channels from rot on pass.  Returns (Q_out, K_out), new unless given; Q_out may
    be Q and K_out may be K.  max_tok: at least the largest count of a sequence (all rows, if it is not given)."""
    _dev(freq, torch.float64, "freq")
    _dev(pos, torch.int32, "pos")
    _dev(tok_start, torch.int32, "tok_start")
    n_seq, dtype = pos.numel(), Q.dtype
    if tok_start.numel() != n_seq + 1:
        raise BpdqError("tok_start: expected n_seq + 1 starts")
    code = ROTARY_LAYOUTS.get(layout)
    if code is None:
        raise BpdqError(f"layout: expected one of {sorted(ROTARY_LAYOUTS)}")
    if Q.dim() != 3 or dtype not in DTYPES:
        raise BpdqError("Q: expected a float32, float16 or bfloat16 tensor of n_tok x n_q x head_dim")
    n_tok, n_q, dim = Q.shape
    ldq, ldqo = _rows(Q, dtype, Q.shape, "Q"), n_q * dim
    if Q_out is None:
        Q_out = _like(Q)
    else:
        ldqo = _rows(Q_out, dtype, Q.shape, "Q_out")
    n_kv = ldk = ldko = 0
    k = k_out = None
    if K is not None:
        if K.dim() != 3 or K.shape[0] != n_tok or K.shape[2] != dim:
            raise BpdqError("K: expected n_tok x n_kv x head_dim")
        n_kv = K.shape[1]
        ldk, ldko = _rows(K, dtype, K.shape, "K"), n_kv * dim
        if K_out is None:
            K_out = _like(K)
        else:
            ldko = _rows(K_out, dtype, K.shape, "K_out")
        k, k_out = K.data_ptr(), K_out.data_ptr()
    elif K_out is not None:
        raise BpdqError("K_out: only with K")
    _here(Q, freq, pos, tok_start, Q_out, K, K_out)
    _call("bpdq_rotary", (_lib or load()).bpdq_rotary(
        freq.data_ptr(), 2 * freq.numel(), code, mscale, 1 if inverse else 0, pos.data_ptr(), tok_start.data_ptr(), n_seq, n_tok,
        n_tok if max_tok is None else max_tok, Q.data_ptr(), ldq, n_q, k, ldk, n_kv, dim, DTYPES[dtype], Q_out.data_ptr(), ldqo, k_out,
        ldko, _stream()))
    return Q_out, K_out


def bpdq_sample_workspace_bytes(n_tok, n_vocab):
    return load().bpdq_sample_workspace_bytes(n_tok, n_vocab)


def bpdq_sample(logits, u, temperature=None, top_k=None, top_p=None, min_p=None, token=None, prob=None, want_prob=False, ws=None):
    """The next token of each row of logits (float32, float16 or bfloat16, n_tok x n_vocab) from the random numbers u (float32, n_tok, in [0, 1)):
    temperature, top_p, min_p float32 and top_k int32, n_tok values each, or None.  Returns token (int32), or (token, prob) where prob (float32)
    is given or wanted."""
    lib = _lib or load()
    dtype = logits.dtype
    if logits.dim() != 2 or dtype not in DTYPES:
        raise BpdqError("logits: expected a float32, float16 or bfloat16 matrix")
    n_tok, n_vocab = logits.shape
    ldl = _rows(logits, dtype, logits.shape, "logits")
    if token is None:
        token = torch.empty(n_tok, dtype=torch.int32, device=logits.device)
    if prob is None and want_prob:
        prob = torch.empty(n_tok, dtype=torch.float32, device=logits.device)
    vectors = []
    for t, kind, name in ((temperature, torch.float32, "temperature"), (top_k, torch.int32, "top_k"), (top_p, torch.float32, "top_p"),
                          (min_p, torch.float32, "min_p"), (u, torch.float32, "u"), (token, torch.int32, "token"),
                          (prob, torch.float32, "prob")):
        if t is None:
            vectors.append(None)
            continue
        if t.dtype is not kind or t.shape != (n_tok,) or not t.is_cuda or not t.is_contiguous():
            raise BpdqError(f"{name}: expected a contiguous {kind} vector of n_tok values on the GPU")
        vectors.append(t.data_ptr())
    if ws is None:
        ws = _scratch(lib.bpdq_sample_workspace_bytes(n_tok, n_vocab), logits.device)
    _here(logits, temperature, top_k, top_p, min_p, u, token, prob, ws)
    _call("bpdq_sample", lib.bpdq_sample(logits.data_ptr(), n_tok, n_vocab, ldl, DTYPES[dtype], *vectors, *_ws(ws), _stream()))
    return token if prob is None else (token, prob)


class KvCache:
    """Keys and values in 8 bits: k, v uint8 (n_pages, n_kv, page, head_dim) in the layout of include/bpdq.h, k_scale, v_scale
    float32 (n_pages, n_kv).  KvCache.empty(...) makes one."""
    __slots__ = ("k", "v", "k_scale", "v_scale", "n_kv", "page", "head_dim", "device", "_c", "_ref")

    def __init__(self, k, v, k_scale, v_scale):
        if k.dim() != 4:
            raise BpdqError("k: expected n_pages x n_kv x page x head_dim")
        _dev(k, torch.uint8, "k")
        _dev(v, torch.uint8, "v")
        _dev(k_scale, torch.float32, "k_scale")
        _dev(v_scale, torch.float32, "v_scale")
        n_pages, self.n_kv, self.page, self.head_dim = shape = k.shape
        if v.shape != shape or k_scale.shape != (n_pages, self.n_kv) or v_scale.shape != (n_pages, self.n_kv):
            raise BpdqError("v as k, and scales of n_pages x n_kv, are expected")
        self.k, self.v, self.k_scale, self.v_scale, self.device = k, v, k_scale, v_scale, k.device
        self._c = BpdqKvCache(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), *shape[:1], self.n_kv,
                              self.page, self.head_dim)
        self._ref = ctypes.byref(self._c)

    @classmethod
    def empty(cls, n_pages, n_kv, head_dim, page=64, device="cuda"):
        shape = (n_pages, n_kv, page, head_dim)
        return cls(torch.empty(shape, dtype=torch.uint8, device=device), torch.empty(shape, dtype=torch.uint8, device=device),
                   torch.empty(shape[:2], device=device), torch.empty(shape[:2], device=device))


def _sequences(page_table, at, start):
    """Checks of what describes the sequences of a call; their number and the table's width."""
    _dev(page_table, torch.int32, "page_table")
    _dev(at, torch.int32, "pos / kv_len")
    _dev(start, torch.int32, "tok_start / q_start")
    n_seq = at.numel()
    shape = page_table.shape
    if len(shape) != 2 or shape[0] != n_seq or start.numel() != n_seq + 1:
        raise BpdqError("page_table: expected n_seq x max_pages, and n_seq + 1 starts")
    return n_seq, shape[1]


def bpdq_kv_write(cache, page_table, pos, tok_start, K, V, max_tok=None):
    """Quantizes rows tok_start[b] .. tok_start[b+1]-1 of K and V (n_tok, n_kv, head_dim) into the cache as tokens pos[b] .. of
    sequence b.  max_tok: at least the largest count of a sequence (all rows, if it is not given)."""
    n_seq, max_pages = _sequences(page_table, pos, tok_start)
    dtype = K.dtype
    n_tok = K.shape[0]
    shape = (n_tok, cache.n_kv, cache.head_dim)
    if dtype not in DTYPES:
        raise BpdqError("K: expected float32, float16 or bfloat16")
    ldk, ldv = _rows(K, dtype, shape, "K"), _rows(V, dtype, shape, "V")
    _call("bpdq_kv_write", (_lib or load()).bpdq_kv_write(
        cache._ref, page_table.data_ptr(), max_pages, n_seq, pos.data_ptr(), tok_start.data_ptr(), n_tok,
        n_tok if max_tok is None else max_tok, K.data_ptr(), ldk, V.data_ptr(), ldv, DTYPES[dtype], _stream()))


def bpdq_kv_read(cache, page_table, pos, tok_start, n_tok, max_tok=None, dtype=torch.float32, K=None, V=None):
    """Tokens pos[b] .. of sequence b from the cache into rows tok_start[b] .. tok_start[b+1]-1 of K and V; returns both."""
    n_seq, max_pages = _sequences(page_table, pos, tok_start)
    shape = (n_tok, cache.n_kv, cache.head_dim)
    if dtype not in DTYPES:
        raise BpdqError("dtype: expected float32, float16 or bfloat16")
    if K is None:
        K = torch.empty(shape, dtype=dtype, device=cache.device)
    if V is None:
        V = torch.empty(shape, dtype=dtype, device=cache.device)
    ldk, ldv = _rows(K, dtype, shape, "K"), _rows(V, dtype, shape, "V")
    _call("bpdq_kv_read", (_lib or load()).bpdq_kv_read(
        cache._ref, page_table.data_ptr(), max_pages, n_seq, pos.data_ptr(), tok_start.data_ptr(), n_tok,
        n_tok if max_tok is None else max_tok, K.data_ptr(), ldk, V.data_ptr(), ldv, DTYPES[dtype], _stream()))
    return K, V


def bpdq_kv_attention_workspace_bytes(n_seq, max_q, max_kv, n_q, n_kv, head_dim, window=0):
    return load().bpdq_kv_attention_workspace_bytes(n_seq, max_q, max_kv, n_q, n_kv, head_dim, window)


def bpdq_kv_attention(cache, page_table, kv_len, q_start, Q, max_q=None, max_kv=None, scale=None, causal=True, window=0,
                      out=None, lse=None, ws=None):
    """Attention of rows q_start[b] .. q_start[b+1]-1 of Q (n_tok, n_q, head_dim), the last of them at position kv_len[b] - 1, over
    the kv_len[b] cached tokens of sequence b.  max_q, max_kv: at least the largest counts (all rows and all of the table's
    pages, if they are not given: right, but laid out for one long chunk, which takes 31 single tokens over caches of up to 16384 4.5 times
    as long); scale: 1 / sqrt(head_dim) by default; lse: float32 (n_tok, n_q), filled if given."""
    lib = _lib or load()
    n_seq, max_pages = _sequences(page_table, kv_len, q_start)
    dtype, dim = Q.dtype, cache.head_dim
    if Q.dim() != 3 or (dtype is not torch.bfloat16 and dtype is not torch.float16):
        raise BpdqError("Q: expected a float16 or bfloat16 tensor of n_tok x n_q x head_dim")
    n_tok, n_q = Q.shape[:2]
    shape = (n_tok, n_q, dim)
    ldq = _rows(Q, dtype, shape, "Q")
    if max_q is None:
        max_q = n_tok
    if max_kv is None:
        max_kv = max_pages * cache.page
    if out is None:
        out = torch.empty(shape, dtype=dtype, device=Q.device)
        ldo = n_q * dim
    else:
        ldo = _rows(out, dtype, shape, "out")
    if lse is not None:
        _dev(lse, torch.float32, "lse")
        if lse.shape != (n_tok, n_q):
            raise BpdqError("lse: expected n_tok x n_q")
    if ws is None:
        ws = _scratch(lib.bpdq_kv_attention_workspace_bytes(n_seq, max_q, max_kv, n_q, cache.n_kv, dim, window), Q.device)
    _call("bpdq_kv_attention", lib.bpdq_kv_attention(
        cache._ref, page_table.data_ptr(), max_pages, n_seq, kv_len.data_ptr(), q_start.data_ptr(), n_tok, max_q, max_kv,
        Q.data_ptr(), ldq, n_q, DTYPES[dtype], dim ** -0.5 if scale is None else scale, 1 if causal else 0, window,
        out.data_ptr(), ldo, None if lse is None else lse.data_ptr(), *_ws(ws), _stream()))
    return out


PROBE_KINDS = {"f32": 0, "bf16": 1, "f16": 2, "f64": 3, "i8": 4}
PROBE_DATA = {"zeros": 0, "ones": 1, "normal": 2}


def bpdq_probe_mfma(kind, data, waves_per_simd, groups, iters, out):
    """Enqueue one register-only matrix-core loop; returns the flops it performs."""
    lib = load()
    _dev(out, torch.float32, "out")
    if out.numel() < groups * 256 * waves_per_simd:
        raise BpdqError("out: too small")
    flops = ctypes.c_double(0.0)
    _check(lib.bpdq_probe_mfma(PROBE_KINDS[kind], PROBE_DATA[data], waves_per_simd, groups, iters,
                               _ptr(out), ctypes.byref(flops), _stream()), "bpdq_probe_mfma")
    return flops.value


def bpdq_probe_copy(src, dst):
    lib = load()
    _dev(src, torch.float32, "src")
    _dev(dst, torch.float32, "dst")
    _check(lib.bpdq_probe_copy(_ptr(src), _ptr(dst), min(src.numel(), dst.numel()), _stream()),
           "bpdq_probe_copy")
    return dst
