"""LC-VQ linear layer (LC-QAT, arXiv 2606.10531) on MI355X (gfx950).

Thin torch binding of liblcvq.so: every function checks devices, dtypes and
contiguity, allocates outputs and workspace with torch, and passes raw device
pointers plus the current HIP stream to the C ABI.  All arithmetic runs in the
library's HIP kernels; there is no CPU or PyTorch fallback.
"""
from __future__ import annotations

import ctypes

import torch

from . import _lib
from ._lib import (BF16, EST_DGE, EST_STE, F32, KV_BF16, KV_E4M3, MASK_LATENT, MASK_ROUNDED, OP_BWD, OP_FWD, OP_FWD_PACKED,  # noqa: F401
                   SCALES_BY_GROUP, SCALES_BY_ROW, SRC_CODES_U8, SRC_LATENT, SRC_PACKED2, LcvqError)

__all__ = ["linear_fwd", "linear_fwd_packed", "linear_fwd_packed_noalloc", "linear_bwd", "linear_bwd_dge", "xavier_quantizer", "xavier_init",
           "pack2bit", "dequant", "encode", "adamw_step", "kv_cache", "kv_write", "kv_read",
           "attn_paged", "attn_workspace_bytes", "linear_fwd_int4", "int4_workspace_bytes", "workspace_bytes", "saved_bytes", "new_saved", "LcvqError", "MASK_ROUNDED", "MASK_LATENT",
           "SRC_LATENT", "SRC_CODES_U8", "SRC_PACKED2", "EST_STE", "EST_DGE"]

_DT = {torch.float32: F32, torch.bfloat16: BF16}


def _dtype_code(t: torch.Tensor) -> int:
    code = _DT.get(t.dtype)
    if code is None:
        raise TypeError(f"unsupported dtype {t.dtype} (float32 or bfloat16)")
    return code


def _check(t, name: str, shape=None, dtype=None) -> None:
    """Shape and dtype of one argument, checked before anything reaches the library
    (a mis-shaped buffer would be read or written out of bounds by the kernels, and
    a wrong dtype silently reinterpreted)."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a tensor, got {type(t).__name__}")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if dtype is not None and t.dtype is not dtype:
        if not (isinstance(dtype, tuple) and t.dtype in dtype):
            raise TypeError(f"{name} has dtype {t.dtype}, expected {dtype}")


def _check_map(A, b, d: int) -> None:
    if d not in (4, 8):
        raise ValueError(f"group size d={d} (4 or 8)")
    _check(A, "A", (d, d), torch.float32)
    _check(b, "b", (d,), torch.float32)


def _check_2d(t, name: str) -> tuple:
    _check(t, name)
    shape = t.shape
    if len(shape) != 2:
        raise ValueError(f"{name} must be 2-D, got shape {tuple(shape)}")
    return tuple(shape)


def _dev(t: torch.Tensor, name: str) -> int:
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be on the GPU (got {t.device})")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _opt(t, name):
    return None if t is None else _dev(t, name)


def _stream(device) -> int:
    """The current stream's handle: torch.cuda.current_stream(device).cuda_stream without
    building the stream object (1.9 -> 0.1 us a call)."""
    return torch._C._cuda_getCurrentRawStream(device.index)


def saved_bytes(N: int, m: int, n: int, d: int, dtype: torch.dtype) -> int:
    """Size of the saved state of the training pair (0 for float32, which needs none)."""
    return int(_lib.load().lcvq_saved_bytes(N, m, n, d, _DT[dtype]))


def new_saved(N: int, m: int, n: int, d: int, dtype: torch.dtype, device) -> torch.Tensor:
    """A buffer for the saved state of linear_fwd(..., saved=...) / linear_bwd(..., saved=...)."""
    return torch.empty(max(saved_bytes(N, m, n, d, dtype), 16), dtype=torch.uint8, device=device)


def _saved_arg(saved, N, m, n, d, dtype):
    _check(saved, "saved", dtype=torch.uint8)
    if saved.dim() != 1:
        raise ValueError("saved must be a 1-D uint8 tensor")
    need = saved_bytes(N, m, n, d, dtype)
    if saved.numel() < need:
        raise ValueError(f"saved has {saved.numel()} bytes, need {need}")
    return _dev(saved, "saved"), saved.numel()


def workspace_bytes(op: int, N: int, m: int, n: int, d: int, dtype: torch.dtype) -> int:
    return int(_lib.load().lcvq_workspace_bytes(op, N, m, n, d, _DT[dtype]))


def _workspace(op, N, m, n, d, dtype, device, workspace):
    return _bytes(workspace, workspace_bytes(op, N, m, n, d, dtype), device)


def _bytes(workspace, need, device):
    if workspace is None:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=device)
    elif workspace.dtype != torch.uint8 or workspace.dim() != 1:
        raise TypeError(f"workspace must be a 1-D uint8 tensor (got {workspace.dtype}, {workspace.dim()}-D)")
    elif workspace.numel() < need:
        raise ValueError(f"workspace has {workspace.numel()} bytes, need {need}")
    return workspace


def pack2bit(src: torch.Tensor, out: torch.Tensor | None = None) -> torch.Tensor:
    """Packed 2-bit codes (m x n/4 uint8) of a latent tensor (fp32/bf16) or of uint8 codes."""
    m, n = _check_2d(src, "src")
    if src.dtype == torch.uint8:
        kind, sdt = SRC_CODES_U8, F32
    else:
        kind, sdt = SRC_LATENT, _dtype_code(src)
    if n % 4 != 0:
        raise ValueError(f"n={n} is not a multiple of 4")
    if out is not None:
        _check(out, "out", (m, n // 4), torch.uint8)
    else:
        out = torch.empty((m, n // 4), dtype=torch.uint8, device=src.device)
    _lib.check(_lib.load().lcvq_pack2bit(_dev(src, "src"), kind, sdt, m, n, _dev(out, "out"),
                                         _stream(src.device)), "lcvq_pack2bit")
    return out


def dequant(src: torch.Tensor, A: torch.Tensor, b: torch.Tensor, d: int, n: int | None = None,
            src_kind: int | None = None, out_dtype: torch.dtype = torch.bfloat16,
            out: torch.Tensor | None = None) -> torch.Tensor:
    """Dense W_hat (m x n) from latents, uint8 codes or packed 2-bit codes (pass n for packed)."""
    _check_2d(src, "src")
    if src_kind is None:
        src_kind = SRC_CODES_U8 if src.dtype == torch.uint8 else SRC_LATENT
    m = src.shape[0]
    if n is None:
        n = src.shape[1] * (4 if src_kind == SRC_PACKED2 else 1)
    if src_kind == SRC_PACKED2:
        _check(src, "src", (m, n // 4), torch.uint8)
        if n % 4 != 0:
            raise ValueError(f"n={n} is not a multiple of 4")
    elif src_kind == SRC_CODES_U8:
        _check(src, "src", (m, n), torch.uint8)
    else:
        _check(src, "src", (m, n), (torch.float32, torch.bfloat16))
    _check_map(A, b, d)
    sdt = _dtype_code(src) if src_kind == SRC_LATENT else F32
    if out is not None:
        _check(out, "out", (m, n), (torch.float32, torch.bfloat16))
    else:
        out = torch.empty((m, n), dtype=out_dtype, device=src.device)
    _lib.check(_lib.load().lcvq_dequant(m, n, d, src_kind, sdt, _dev(src, "src"), _dev(A, "A"), _dev(b, "b"),
                                        _dev(out, "out"), _DT[out.dtype], _stream(src.device)), "lcvq_dequant")
    return out


def encode(W: torch.Tensor, A: torch.Tensor, b: torch.Tensor, d: int, codes: bool = True, packed: bool = False):
    """LC encode of a dense weight W (m x n, fp32 or bf16): per group the codes
    clip(round(A^-1 (w_g - b)), 0, 3), the nearest codewords when A is a scaled
    orthogonal matrix.  Returns (codes m x n uint8 or None, packed m x n/4 uint8 or None)."""
    m, n = _check_2d(W, "W")
    _check(W, "W", dtype=(torch.float32, torch.bfloat16))
    _check_map(A, b, d)
    c = torch.empty((m, n), dtype=torch.uint8, device=W.device) if codes else None
    p = torch.empty((m, n // 4), dtype=torch.uint8, device=W.device) if packed else None
    _lib.check(_lib.load().lcvq_encode(m, n, d, _dev(W, "W"), _dtype_code(W), _dev(A, "A"), _dev(b, "b"),
                                       _opt(c, "codes"), _opt(p, "packed"), _stream(W.device)), "lcvq_encode")
    return c, p


def xavier_quantizer(m: int, n: int) -> tuple[float, float]:
    """(q_scale, q_shift) = (1 / s', t) of the Xavier reparameterisation (Sec. 3.4,
    eq. xavier_preprocess) for 2-bit codes, from lcvq_xavier_quantizer."""
    qs, qb = ctypes.c_float(), ctypes.c_float()
    _lib.check(_lib.load().lcvq_xavier_quantizer(m, n, ctypes.byref(qs), ctypes.byref(qb)),
               "lcvq_xavier_quantizer")
    return qs.value, qb.value


def xavier_init(codes: torch.Tensor, m: int, n: int, src_kind: int | None = None,
                out_dtype: torch.dtype = torch.float32, out: torch.Tensor | None = None) -> torch.Tensor:
    """Initial proxy weights W_p = s' (W_z - t) (Sec. 3.4, eq. xavier_preprocess) of
    uint8 (m x n) or packed (m x n/4) codes, from lcvq_xavier_init."""
    if src_kind is None:
        src_kind = SRC_CODES_U8 if tuple(codes.shape) == (m, n) else SRC_PACKED2
    _check(codes, "codes", (m, n) if src_kind == SRC_CODES_U8 else (m, n // 4), torch.uint8)
    if out is not None:
        _check(out, "out", (m, n), (torch.float32, torch.bfloat16))
    else:
        out = torch.empty((m, n), dtype=out_dtype, device=codes.device)
    _lib.check(_lib.load().lcvq_xavier_init(m, n, src_kind, _dev(codes, "codes"), _dev(out, "out"), _DT[out.dtype],
                                            _stream(codes.device)), "lcvq_xavier_init")
    return out


def adamw_step(theta: torch.Tensor, grad: torch.Tensor, m1: torch.Tensor, m2: torch.Tensor, step: int,
               lr: float, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
               weight_decay: float = 0.0, shadow: torch.Tensor | None = None) -> None:
    """One in-place AdamW update of fp32 `theta`, `m1`, `m2` from `grad` (fp32 or bf16);
    `shadow` (fp32 or bf16, optional) receives the updated theta."""
    for t, nm in ((theta, "theta"), (m1, "m1"), (m2, "m2")):
        _check(t, nm, dtype=torch.float32)
    _check(grad, "grad", dtype=(torch.float32, torch.bfloat16))
    if shadow is not None:
        _check(shadow, "shadow", dtype=(torch.float32, torch.bfloat16))
    numel = theta.numel()
    for t, nm in ((grad, "grad"), (m1, "m1"), (m2, "m2")) + (((shadow, "shadow"),) if shadow is not None else ()):
        if t.numel() != numel:
            raise ValueError(f"{nm} has {t.numel()} elements, theta has {numel}")
    sdt = _dtype_code(shadow) if shadow is not None else F32
    _lib.check(_lib.load().lcvq_adamw_step(_dev(theta, "theta"), _dev(grad, "grad"), _dtype_code(grad),
                                           _dev(m1, "m1"), _dev(m2, "m2"), _opt(shadow, "shadow"), sdt, numel,
                                           lr, beta1, beta2, eps, weight_decay, step, _stream(theta.device)),
               "lcvq_adamw_step")


def linear_fwd(Z: torch.Tensor, A: torch.Tensor, b: torch.Tensor, X: torch.Tensor, d: int,
               packed_out: torch.Tensor | None = None, workspace: torch.Tensor | None = None,
               out: torch.Tensor | None = None, q_scale: float = 1.0, q_shift: float = 0.0,
               saved: torch.Tensor | None = None) -> torch.Tensor:
    """Y = X W_hat^T (N x m) for latents Z (m x n), map A (d x d fp32), offset b (d fp32).

    q_scale, q_shift: the quantiser rounds Z * q_scale + q_shift (see xavier_quantizer);
    the default is the code domain.  saved: a buffer from new_saved(); the forward then
    also writes what linear_bwd(..., saved=...) of the same layer needs (the training
    pair, lcvq_linear_fwd_train)."""
    m, n = _check_2d(Z, "Z")
    dt = _dtype_code(Z)
    N = _check_2d(X, "X")[0]
    _check(X, "X", (N, n), Z.dtype)
    _check_map(A, b, d)
    if packed_out is not None:
        if n % 4 != 0:
            raise ValueError(f"packed codes need n % 4 == 0 (n={n})")
        _check(packed_out, "packed_out", (m, n // 4), torch.uint8)
    if out is not None:
        _check(out, "out", (N, m), Z.dtype)
    else:
        out = torch.empty((N, m), dtype=X.dtype, device=X.device)
    ws = _workspace(OP_FWD, N, m, n, d, X.dtype, X.device, workspace)
    tail = (_dev(A, "A"), _dev(b, "b"), _dev(X, "X"), _dev(out, "Y"), _opt(packed_out, "packed_out"),
            _dev(ws, "workspace"), ws.numel(), _stream(X.device))
    if saved is not None:
        sp, sn = _saved_arg(saved, N, m, n, d, Z.dtype)
        _lib.check(_lib.load().lcvq_linear_fwd_train(N, m, n, d, dt, _dev(Z, "Z"), q_scale, q_shift, *tail[:5], sp, sn,
                                                     *tail[5:]), "lcvq_linear_fwd_train")
    elif q_scale == 1.0 and q_shift == 0.0:
        _lib.check(_lib.load().lcvq_linear_fwd(N, m, n, d, dt, _dev(Z, "Z"), *tail), "lcvq_linear_fwd")
    else:
        _lib.check(_lib.load().lcvq_linear_fwd_ex(N, m, n, d, dt, _dev(Z, "Z"), q_scale, q_shift, *tail),
                   "lcvq_linear_fwd_ex")
    return out


def linear_fwd_packed(packed: torch.Tensor, A: torch.Tensor, b: torch.Tensor, X: torch.Tensor, d: int,
                      out_dtype: torch.dtype = torch.bfloat16, workspace: torch.Tensor | None = None,
                      out: torch.Tensor | None = None) -> torch.Tensor:
    """Y = X W_hat^T (N x m, bf16 or fp32) from packed 2-bit codes (m x n/4 uint8) and bf16 X (N x n).

    A workspace of workspace_bytes(OP_FWD_PACKED, N, ...) takes all N tokens in as few passes as
    it can; any workspace sized for one token is accepted."""
    m, n4 = _check_2d(packed, "packed")
    n = 4 * n4
    _check(packed, "packed", dtype=torch.uint8)
    N = _check_2d(X, "X")[0]
    _check(X, "X", (N, n), torch.bfloat16)
    _check_map(A, b, d)
    if out is not None:
        _check(out, "out", (N, m), (torch.float32, torch.bfloat16))
    else:
        out = torch.empty((N, m), dtype=out_dtype, device=X.device)
    # a workspace for one token will do; one for N tokens needs the fewest passes
    ws = _workspace(OP_FWD_PACKED, N if workspace is None else 1, m, n, d, torch.bfloat16, X.device, workspace)
    _lib.check(_lib.load().lcvq_linear_fwd_packed(N, m, n, d, _dev(packed, "packed"), _dev(A, "A"), _dev(b, "b"),
                                                  _dev(X, "X"), _dev(out, "Y"), _DT[out.dtype],
                                                  _dev(ws, "workspace"), ws.numel(), _stream(X.device)),
               "lcvq_linear_fwd_packed")
    return out


def linear_fwd_packed_noalloc(packed: torch.Tensor, A: torch.Tensor, b: torch.Tensor, X: torch.Tensor, d: int,
                              out: torch.Tensor) -> torch.Tensor:
    """linear_fwd_packed without a workspace: the library's fixed per-device scratch
    array takes its place (for callers that cannot allocate).  `out` (N x m, bf16 or
    fp32) is the caller's; calls that overlap on one device race."""
    m, n4 = _check_2d(packed, "packed")
    n = 4 * n4
    _check(packed, "packed", dtype=torch.uint8)
    N = _check_2d(X, "X")[0]
    _check(X, "X", (N, n), torch.bfloat16)
    _check_map(A, b, d)
    _check(out, "out", (N, m), (torch.float32, torch.bfloat16))
    _lib.check(_lib.load().lcvq_linear_fwd_packed_noalloc(N, m, n, d, _dev(packed, "packed"), _dev(A, "A"),
                                                          _dev(b, "b"), _dev(X, "X"), _dev(out, "Y"),
                                                          _DT[out.dtype], _stream(X.device)),
               "lcvq_linear_fwd_packed_noalloc")
    return out


def linear_bwd(Z: torch.Tensor, A: torch.Tensor, b: torch.Tensor, X: torch.Tensor, dY: torch.Tensor, d: int,
               mask_mode: int = MASK_ROUNDED, accumulate: bool = False, need_dX: bool = True,
               need_dZ: bool = True, need_map: bool = True, dz_dtype: torch.dtype | None = None,
               dX: torch.Tensor | None = None, dZ: torch.Tensor | None = None, dA: torch.Tensor | None = None,
               db: torch.Tensor | None = None, workspace: torch.Tensor | None = None, q_scale: float = 1.0,
               q_shift: float = 0.0, saved: torch.Tensor | None = None):
    """Straight-through backward: returns (dX, dZ, dA, db); skipped outputs are None.
    saved: the buffer a linear_fwd(..., saved=...) of the same layer and inputs filled."""
    return _linear_bwd(None, Z, A, b, X, dY, d, mask_mode, accumulate, need_dX, need_dZ, need_map, dz_dtype,
                       dX, dZ, dA, db, workspace, q_scale, q_shift, saved)


def linear_bwd_dge(Z: torch.Tensor, A: torch.Tensor, b: torch.Tensor, X: torch.Tensor, dY: torch.Tensor,
                   d: int, k: float = 5.0, cap: float = 3.0, mask_mode: int = MASK_LATENT,
                   accumulate: bool = False, need_dX: bool = True, need_dZ: bool = True, need_map: bool = True,
                   dz_dtype: torch.dtype | None = None, dX: torch.Tensor | None = None,
                   dZ: torch.Tensor | None = None, dA: torch.Tensor | None = None, db: torch.Tensor | None = None,
                   workspace: torch.Tensor | None = None, q_scale: float = 1.0, q_shift: float = 0.0,
                   saved: torch.Tensor | None = None):
    """Backward with the differentiable gradient estimator (k, slope cap): returns (dX, dZ, dA, db).

    The default mask is the latent one, [0 <= Z <= 3], which the chain rule
    gives through clip(f(Z), 0, 3)."""
    return _linear_bwd((float(k), float(cap)), Z, A, b, X, dY, d, mask_mode, accumulate, need_dX, need_dZ,
                       need_map, dz_dtype, dX, dZ, dA, db, workspace, q_scale, q_shift, saved)


def _linear_bwd(dge, Z, A, b, X, dY, d, mask_mode, accumulate, need_dX, need_dZ, need_map, dz_dtype, dX, dZ, dA,
                db, workspace, q_scale=1.0, q_shift=0.0, saved=None):
    m, n = _check_2d(Z, "Z")
    dt = _dtype_code(Z)
    N = _check_2d(X, "X")[0]
    _check(X, "X", (N, n), Z.dtype)
    _check(dY, "dY", (N, m), Z.dtype)
    _check_map(A, b, d)
    dev = X.device
    if dz_dtype is None:
        dz_dtype = dZ.dtype if dZ is not None else Z.dtype
    if dz_dtype not in (torch.float32, Z.dtype):
        raise TypeError(f"dZ dtype {dz_dtype}: float32 or the latent's dtype {Z.dtype}")
    if dX is not None:
        _check(dX, "dX", (N, n), Z.dtype)
    if dZ is not None:
        _check(dZ, "dZ", (m, n), dz_dtype)
    if (dA is None) != (db is None):
        raise ValueError("dA and db are given together or not at all")
    if dA is not None:
        _check(dA, "dA", (d, d), torch.float32)
        _check(db, "db", (d,), torch.float32)
    if need_dX and dX is None:
        dX = torch.empty((N, n), dtype=X.dtype, device=dev)
    if need_dZ and dZ is None:
        dZ = (torch.zeros if accumulate else torch.empty)((m, n), dtype=dz_dtype, device=dev)
    if need_map and dA is None:  # (not accumulating: the library writes every entry)
        dA = (torch.zeros if accumulate else torch.empty)((d, d), dtype=torch.float32, device=dev)
        db = (torch.zeros if accumulate else torch.empty)((d,), dtype=torch.float32, device=dev)
    ws = _workspace(OP_BWD, N, m, n, d, X.dtype, dev, workspace)
    head = (N, m, n, d, dt, _dev(Z, "Z"), _dev(A, "A"), _dev(b, "b"), _dev(X, "X"), _dev(dY, "dY"), mask_mode)
    tail = (1 if accumulate else 0, _opt(dX if need_dX else None, "dX"), _opt(dZ if need_dZ else None, "dZ"),
            _DT[dz_dtype], _opt(dA if need_map else None, "dA"), _opt(db if need_map else None, "db"),
            _dev(ws, "workspace"), ws.numel(), _stream(dev))
    if saved is not None:
        sp, sn = _saved_arg(saved, N, m, n, d, Z.dtype)
        est = (EST_STE, 0.0, 0.0) if dge is None else (EST_DGE, *dge)
        head_ex = head[:6] + (q_scale, q_shift) + head[6:]
        _lib.check(_lib.load().lcvq_linear_bwd_train(*head_ex, *est, *tail[:6], sp, sn, *tail[6:]),
                   "lcvq_linear_bwd_train")
    elif q_scale != 1.0 or q_shift != 0.0:
        est = (EST_STE, 0.0, 0.0) if dge is None else (EST_DGE, *dge)
        head_ex = head[:6] + (q_scale, q_shift) + head[6:]
        _lib.check(_lib.load().lcvq_linear_bwd_ex(*head_ex, *est, *tail), "lcvq_linear_bwd_ex")
    elif dge is None:
        _lib.check(_lib.load().lcvq_linear_bwd(*head, *tail), "lcvq_linear_bwd")
    else:
        _lib.check(_lib.load().lcvq_linear_bwd_dge(*head, *dge, *tail), "lcvq_linear_bwd_dge")
    return (dX if need_dX else None, dZ if need_dZ else None, dA if need_map else None,
            db if need_map else None)


# ------------------------------------------------------ serving: cache, attention --

def kv_cache(pages: int, page_size: int, heads: int, head_dim: int, dtype: torch.dtype = torch.uint8, device="cuda"):
    """An empty paged cache: (data, scales).

    data is 2 (keys, values) x pages x heads x page_size x head_dim, uint8 for the 8-bit
    format (e4m3 codes) or bfloat16; scales is 2 x pages x heads x page_size uint8, the
    codes' factor 2^(scale - 127) per token and head, or None for bfloat16.  Token slot s
    is entry s % page_size of page s // page_size."""
    if dtype not in (torch.uint8, torch.bfloat16):
        raise TypeError(f"cache dtype {dtype} (uint8 for e4m3 codes, or bfloat16)")
    data = torch.zeros((2, pages, heads, page_size, head_dim), dtype=dtype, device=device)
    scales = torch.full((2, pages, heads, page_size), 127, dtype=torch.uint8, device=device) if dtype == torch.uint8 else None
    return data, scales


def _arg(t, name, shape, dtype, device) -> int:
    """The address of a dense tensor of that shape, type and device.  For calls whose host side
    is most of their time: one look at a tensor that is right, the checks that say why at others."""
    if (isinstance(t, torch.Tensor) and t.dtype is dtype and t.get_device() == device.index and t.shape == shape
            and t.is_contiguous()):
        return t.data_ptr()
    _check(t, name, shape, dtype)
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, expected {device}")
    return _dev(t, name)


def _fits(x: int, name: str) -> None:
    """For numbers of the caller's that the library takes in 32 bits (ctypes would cut them off)."""
    if not -0x80000000 <= x < 0x80000000:
        raise ValueError(f"{name}={x} does not fit 32 bits")


def _cache(data, scales):
    """(format, pages, Hkv, page_size, D) and the four device pointers of a cache."""
    _check(data, "data", dtype=(torch.uint8, torch.bfloat16))
    shape = data.shape
    if len(shape) != 5 or shape[0] != 2:
        raise ValueError(f"data must be 2 x pages x heads x page_size x head_dim, got shape {tuple(shape)}")
    _, pages, H, page, D = shape
    p, rows = _dev(data, "data"), pages * H * page
    if data.dtype is torch.bfloat16:
        if scales is not None:
            raise ValueError("a bfloat16 cache has no scales")
        return KV_BF16, pages, H, page, D, (p, p + 2 * rows * D, None, None)
    s = _arg(scales, "scales", shape[:4], torch.uint8, data.device)
    return KV_E4M3, pages, H, page, D, (p, p + rows * D, s, s + rows)


def _heads_view(t, name, H, D, dtype, device):
    """Pointer and strides (token, head) of T x H x D heads whose last dimension is dense: a
    slice of a fused projection's output passes as it is."""
    _check(t, name, dtype=dtype)
    shape = t.shape
    if len(shape) != 3 or shape[1] != H or shape[2] != D:
        raise ValueError(f"{name} has shape {tuple(shape)}, expected (T, {H}, {D})")
    if t.get_device() != device.index:
        raise ValueError(f"{name} must be on the GPU, with the cache (got {t.device})")
    token, head, one = t.stride()
    if one != 1:
        raise ValueError(f"{name}: the head's elements must be contiguous")
    # (the stride of a dimension of one has no meaning)
    return t.data_ptr(), token if shape[0] > 1 else 0, head if H > 1 else 0


def kv_write(K: torch.Tensor, V: torch.Tensor, slots: torch.Tensor, data: torch.Tensor,
             scales: torch.Tensor | None = None) -> None:
    """Writes the keys and values of T tokens (T x heads x head_dim, fp32 or bf16, any token
    and head strides) into the slots (int64) of a cache from kv_cache, quantising them for an
    8-bit one.  A slot outside the cache (-1) is skipped; no two tokens may share one."""
    fmt, pages, H, page, D, ptr = _cache(data, scales)
    dev = data.device
    kp, kt, kh = _heads_view(K, "K", H, D, (torch.float32, torch.bfloat16), dev)
    vp, vt, vh = _heads_view(V, "V", H, D, K.dtype, dev)
    T = K.shape[0]
    if V.shape[0] != T:
        raise ValueError(f"V has {V.shape[0]} tokens, K has {T}")
    sp = _arg(slots, "slots", (T,), torch.int64, dev)
    _lib.check(_lib.load().lcvq_kv_write(T, H, D, kp, vp, _dtype_code(K), kt, kh, vt, vh, sp, fmt, pages, page, *ptr,
                                         _stream(dev)), "lcvq_kv_write")


def kv_read(data: torch.Tensor, slots: torch.Tensor, scales: torch.Tensor | None = None,
            out_dtype: torch.dtype = torch.bfloat16):
    """(K, V), T x heads x head_dim each (bf16, exact, or fp32): what the slots (int64) of the
    cache hold, zeros for a slot outside it."""
    fmt, pages, H, page, D, ptr = _cache(data, scales)
    if out_dtype not in _DT:
        raise TypeError(f"unsupported dtype {out_dtype} (float32 or bfloat16)")
    _check(slots, "slots", dtype=torch.int64)
    T, dev = slots.numel(), data.device
    sp = _arg(slots, "slots", (T,), torch.int64, dev)
    K = torch.empty((T, H, D), dtype=out_dtype, device=dev)
    V = torch.empty_like(K)
    _lib.check(_lib.load().lcvq_kv_read(T, H, D, sp, fmt, pages, page, *ptr, K.data_ptr(), V.data_ptr(), _DT[out_dtype],
                                        _stream(dev)), "lcvq_kv_read")
    return K, V


def attn_workspace_bytes(T: int, B: int, Hq: int, Hkv: int, D: int, max_q: int) -> int:
    """Workspace of attn_paged for calls of at most T rows, B sequences and max_q new tokens each."""
    for x, name in ((B, "B"), (Hq, "Hq"), (Hkv, "Hkv"), (D, "D"), (max_q, "max_q")):
        _fits(x, name)
    return int(_lib.load().lcvq_attn_workspace_bytes(T, B, Hq, Hkv, D, max_q))


def attn_paged(q: torch.Tensor, data: torch.Tensor, table: torch.Tensor, kv_lens: torch.Tensor, q_starts: torch.Tensor,
               scales: torch.Tensor | None = None, scale: float | None = None, causal: bool = True, window: int = 0,
               max_q: int | None = None, need_lse: bool = False, workspace: torch.Tensor | None = None,
               out: torch.Tensor | None = None, lse: torch.Tensor | None = None):
    """Attention of B sequences' new tokens over a cache from kv_cache that holds them already.

    q (T x query heads x head_dim bf16, any token and head strides) has sequence b's new tokens
    in rows q_starts[b] .. q_starts[b + 1] - 1 (int32, B + 1); kv_lens (int32, B) counts its
    cached tokens, table (int32, B x width) names their pages.  New token i of n, at position
    p = kv_lens - n + i, sees the cached tokens up to p (all of them with causal=False), the
    last `window` of these if window > 0.  scale defaults to head_dim ** -0.5.  max_q: the most
    new tokens of any sequence (default T); with it few-token calls choose their kernel.

    Returns (out, lse): T x query heads x head_dim bf16, and the log-sum-exp of the scaled
    scores, T x query heads fp32, or None unless need_lse or lse.  A row that sees nothing
    gives 0 and -inf."""
    _fits(window, "window")
    B, width = _check_2d(table, "table")
    _fits(B, "sequences")
    if max_q is not None:
        _fits(max_q, "max_q")
    fmt, pages, H, page, D, ptr = _cache(data, scales)
    _check(q, "q", dtype=torch.bfloat16)
    if q.dim() != 3:
        raise ValueError(f"q must be T x heads x head_dim, got shape {tuple(q.shape)}")
    T, Hq, dev = q.shape[0], q.shape[1], data.device
    qp, qt, qh = _heads_view(q, "q", Hq, D, torch.bfloat16, dev)
    if H == 0 or Hq % H != 0 or Hq == 0:
        raise ValueError(f"{Hq} query heads on {H} cached heads")
    tp = _arg(table, "table", table.shape, torch.int32, dev)
    lp = _arg(kv_lens, "kv_lens", (B,), torch.int32, dev)
    sp = _arg(q_starts, "q_starts", (B + 1,), torch.int32, dev)
    if max_q is None:
        max_q = T
    if out is None:
        out = torch.empty((T, Hq, D), dtype=torch.bfloat16, device=dev)
    op = _arg(out, "out", (T, Hq, D), torch.bfloat16, dev)
    if lse is None and need_lse:
        lse = torch.empty((T, Hq), dtype=torch.float32, device=dev)
    ep = None if lse is None else _arg(lse, "lse", (T, Hq), torch.float32, dev)
    lib = _lib.load()
    workspace = _bytes(workspace, lib.lcvq_attn_workspace_bytes(T, B, Hq, H, D, max_q), dev)
    _lib.check(lib.lcvq_attn_paged(T, B, Hq, H, D, qp, qt, qh, fmt, pages, page, *ptr, tp, width, lp, sp, max_q,
                                   D ** -0.5 if scale is None else scale, 1 if causal else 0, window, op, ep,
                                   _dev(workspace, "workspace"), workspace.numel(), _stream(dev)), "lcvq_attn_paged")
    return out, lse


# ------------------------------------------------------------ serving: 4-bit weights --

def int4_workspace_bytes(N: int, m: int, n: int) -> int:
    """Workspace of linear_fwd_int4 (0 where it needs none); it never falls as N grows."""
    return int(_lib.load().lcvq_int4_workspace_bytes(N, m, n))


def linear_fwd_int4(packed: torch.Tensor, scales: torch.Tensor, X: torch.Tensor, group: int,
                    zeros: torch.Tensor | None = None, out_dtype: torch.dtype = torch.bfloat16,
                    workspace: torch.Tensor | None = None, out: torch.Tensor | None = None,
                    by_group: bool | None = None) -> torch.Tensor:
    """Y = X W^T (N x m, bf16 or fp32) for W[r, c] = scales[r, c // group] (code[r, c] - zero).

    packed (m x n/2 uint8) holds two codes a byte, the even column in the low half; scales and
    zeros (bf16, zero points, 8 if not given) are m x n/group for groups of 32, 64 or a multiple
    of 128 columns, or both n/group x m, which large layers read up to 13 % faster.  The shape
    tells which; where m is n/group, by_group has to.  X is N x n bf16.  For few tokens: the
    weights are read once per 16."""
    _fits(group, "group")
    m, n2 = _check_2d(packed, "packed")
    n = 2 * n2
    N, dev = _check_2d(X, "X")[0], X.device
    xp = _arg(X, "X", (N, n), torch.bfloat16, dev)
    wp = _arg(packed, "packed", (m, n2), torch.uint8, dev)
    if group <= 0 or n % group != 0:
        raise ValueError(f"n={n} is not a multiple of group={group}")
    K = n // group
    if by_group is None:
        if K == m > 1:
            raise ValueError(f"{m} rows and as many groups: by_group must say whether scales has a row per group or per weight row")
        by_group = isinstance(scales, torch.Tensor) and scales.shape == (K, m)
    shape = (K, m) if by_group else (m, K)
    sp = _arg(scales, "scales", shape, torch.bfloat16, dev)
    zp = None if zeros is None else _arg(zeros, "zeros", shape, torch.bfloat16, dev)
    if out is None:
        if out_dtype not in _DT:
            raise TypeError(f"unsupported dtype {out_dtype} (float32 or bfloat16)")
        out = torch.empty((N, m), dtype=out_dtype, device=dev)
    else:
        _check(out, "out", dtype=(torch.float32, torch.bfloat16))
    op = _arg(out, "out", (N, m), out.dtype, dev)
    lib, ws, size = _lib.load(), None, 0
    need = lib.lcvq_int4_workspace_bytes(N, m, n)
    if need > 0:
        workspace = _bytes(workspace, need, dev)
        ws, size = _dev(workspace, "workspace"), workspace.numel()
    _lib.check(lib.lcvq_linear_fwd_int4_ex(N, m, n, group, wp, sp, zp, SCALES_BY_GROUP if by_group else SCALES_BY_ROW, xp, op,
                                           _DT[out.dtype], ws, size, _stream(dev)), "lcvq_linear_fwd_int4")
    return out
