"""Python binding of libjab (the MI355X JAB-loss library).

Argument marshalling only: tensors provide device memory (``data_ptr``) and the
current HIP stream; every step of the computation runs in the library's HIP
kernels.  Importing this module does not touch the GPU; the first call loads
``libjab.so`` and raises if it was not built -- there is no fallback path.

Function names follow the C ABI in ``include/jab.h``.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass
from typing import Optional, Sequence, Tuple

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libjab.so")

JAB_OK, JAB_E_INVALID, JAB_E_UNSUPPORTED, JAB_E_WORKSPACE, JAB_E_HIP = 0, -1, -2, -3, -4
F32, F16, BF16 = 0, 1, 2
ASYM, SYM = 0, 1
OP_FWD, OP_SWEEP, OP_BWD, OP_REF, OP_QUANTIZE, OP_PROJECT, OP_FWD_KL, OP_CURVATURE, OP_FISHER, OP_STE = range(10)
KT_NAMES = ("quant", "gemm", "attn", "reduce", "attn_bwd", "dw_gemm", "misc", "gemm_vt", "kl")

_DTYPE_CODE = {torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16}
_CODE_DTYPE = {v: k for k, v in _DTYPE_CODE.items()}


class JabError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{msg} (status {status})")
        self.status = status


class Problem(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("seq_len", ctypes.c_int32), ("d_model", ctypes.c_int32),
                ("n_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("group_size", ctypes.c_int32), ("dtype", ctypes.c_int32), ("scheme", ctypes.c_int32),
                ("rope_theta", ctypes.c_float)]

    @property
    def rows(self) -> int:
        return (self.n_heads + 2 * self.n_kv_heads) * self.head_dim

    @property
    def torch_dtype(self) -> torch.dtype:
        return _CODE_DTYPE[self.dtype]

    def with_batch(self, batch: int) -> "Problem":
        p = Problem()
        ctypes.pointer(p)[0] = self
        p.batch = batch
        return p


class Quant(ctypes.Structure):
    _fields_ = [("bits", ctypes.c_int32 * 3), ("scale", ctypes.c_void_p), ("zero", ctypes.c_void_p)]


class SteConfig(ctypes.Structure):
    _fields_ = [("n_steps", ctypes.c_int32), ("eval_every", ctypes.c_int32), ("alpha_w", ctypes.c_float),
                ("alpha_s", ctypes.c_float), ("beta1", ctypes.c_float), ("beta2", ctypes.c_float),
                ("adam_eps", ctypes.c_float), ("scale_floor", ctypes.c_float), ("lambda_kl", ctypes.c_float)]


class _CacheStruct(ctypes.Structure):
    _fields_ = [("bits", ctypes.c_int32), ("page_size", ctypes.c_int32), ("n_pages", ctypes.c_int32),
                ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p), ("k_zero", ctypes.c_void_p), ("v_zero", ctypes.c_void_p)]


class _CacheRowsStruct(ctypes.Structure):
    _fields_ = [("n_seq", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("max_new", ctypes.c_int32),
                ("pages", ctypes.c_void_p), ("past", ctypes.c_void_p), ("start", ctypes.c_void_p)]


def problem(batch, seq_len, d_model, n_heads, n_kv_heads, head_dim, group_size, dtype,
            scheme: int = ASYM, rope_theta: float = 0.0) -> Problem:
    code = _DTYPE_CODE[dtype] if isinstance(dtype, torch.dtype) else int(dtype)
    return Problem(batch, seq_len, d_model, n_heads, n_kv_heads, head_dim, group_size, code, scheme, rope_theta)


def problem_of(wl, batch: Optional[int] = None) -> Problem:
    """Problem for a workload of ``paper_2609_34866_amd.inputs``."""
    return problem(wl.batch if batch is None else batch, wl.seq_len, wl.d_model, wl.n_heads,
                   wl.n_kv_heads, wl.head_dim, wl.group_size, wl.torch_dtype,
                   SYM if wl.symmetric else ASYM, wl.rope_theta)


_LIB = None


def lib() -> ctypes.CDLL:
    global _LIB
    if _LIB is not None:
        return _LIB
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"libjab.so is not built ({LIB_PATH}); run __graft_entry__.build()")
    L = ctypes.CDLL(LIB_PATH)
    vp, sz, i32, P = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32, ctypes.POINTER(Problem)
    Q, C, R = ctypes.POINTER(Quant), ctypes.POINTER(_CacheStruct), ctypes.POINTER(_CacheRowsStruct)
    sig = {
        "jab_workspace_size": (sz, [P, i32, i32]),
        "jab_quant_init": (i32, [P, vp, vp, vp, vp, vp]),
        "jab_quantize": (i32, [P, vp, Q, vp, vp, vp, vp, sz, vp]),
        "jab_attn_ref": (i32, [P, vp, vp, vp, vp, sz, vp]),
        "jab_loss_fwd": (i32, [P, vp, vp, Q, vp, vp, vp, sz, vp]),
        "jab_loss_fwd_noalloc": (i32, [P, vp, vp, Q, vp, vp, vp]),
        "jab_attn_ref_kl": (i32, [P, vp, vp, vp, vp, vp, vp, sz, vp]),
        "jab_loss_fwd_kl": (i32, [P, vp, vp, Q, vp, vp, vp, vp, vp, sz, vp]),
        "jab_loss_sweep": (i32, [P, vp, vp, i32, vp, vp, vp, i32, vp, vp, vp, vp, vp, sz, vp]),
        "jab_loss_bwd": (i32, [P, vp, vp, Q, vp, vp, vp, vp, vp, vp, sz, vp]),
        "jab_project": (i32, [P, vp, vp, Q, vp, vp, sz, vp]),
        "jab_allocate": (i32, [i32, i32, vp, vp, vp, ctypes.c_double, i32, i32, vp, vp]),
        "jab_omega": (i32, [i32, i32, vp, i32, vp, i32, i32, vp]),
        "jab_curvature": (i32, [P, vp, vp, ctypes.c_float, i32, vp, vp, vp, sz, vp]),
        "jab_fisher": (i32, [P, vp, vp, Q, vp, vp, vp, ctypes.c_float, vp, vp, sz, vp]),
        "jab_loss_bwd_kl": (i32, [P, vp, vp, Q, vp, vp, vp, vp, ctypes.c_float, vp, vp, vp, vp, sz, vp]),
        "jab_ste_stats_len": (i32, [i32, i32]),
        "jab_ste_finetune": (i32, [P, ctypes.POINTER(SteConfig), vp, vp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp,
                                   vp, vp, vp, vp, vp, sz, vp]),
        "jab_quant_rows": (i32, [P, ctypes.c_int64, vp, vp, vp, vp]),
        "jab_project_int": (i32, [P, vp, vp, vp, vp, vp, vp]),
        "jab_cache_write": (i32, [P, C, R, vp, vp]),
        "jab_cache_read": (i32, [P, C, R, vp, vp, vp]),
        "jab_attn_cache": (i32, [P, C, R, vp, vp, vp, sz, vp]),
        "jab_attn_cache_workspace": (sz, [P, C, R]),
        "jab_status_string": (ctypes.c_char_p, [i32]),
        "jab_last_error": (ctypes.c_char_p, []),
        "jab_set_bwd_ds_limit": (i32, [ctypes.c_size_t]),
        "jab_timing_enable": (i32, [i32]),
        "jab_timing_read": (i32, [vp, vp]),
    }
    for name, (res, args) in sig.items():
        f = getattr(L, name)
        f.restype, f.argtypes = res, args
    _LIB = L
    return L


EXPORTED = ("jab_workspace_size", "jab_quant_init", "jab_quantize", "jab_attn_ref", "jab_loss_fwd",
            "jab_loss_fwd_noalloc",
            "jab_attn_ref_kl", "jab_loss_fwd_kl", "jab_loss_sweep", "jab_loss_bwd", "jab_project",
            "jab_allocate", "jab_omega", "jab_curvature", "jab_fisher", "jab_loss_bwd_kl", "jab_ste_stats_len", "jab_ste_finetune",
            "jab_quant_rows", "jab_project_int", "jab_cache_write", "jab_cache_read", "jab_attn_cache",
            "jab_attn_cache_workspace", "jab_status_string", "jab_last_error", "jab_set_bwd_ds_limit", "jab_timing_enable",
            "jab_timing_read")
ALLOC_GREEDY, ALLOC_PARETO = 0, 1
TRACE_BLOCK, TRACE_UNIT = 0, 1
OMEGA_C1, OMEGA_C2 = 0, 1


def _check(status: int) -> None:
    if status != JAB_OK:
        L = lib()
        raise JabError(status, f"{L.jab_status_string(status).decode()}: {L.jab_last_error().decode()}")


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream() -> ctypes.c_void_p:
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _quant(bits: Sequence[int], scale: Optional[torch.Tensor], zero: Optional[torch.Tensor]) -> Quant:
    q = Quant()
    for i in range(3):
        q.bits[i] = int(bits[i])
    q.scale = None if scale is None else scale.data_ptr()
    q.zero = None if zero is None else zero.data_ptr()
    return q


def workspace_size(p: Problem, op: int, n_bits: int = 0) -> int:
    return int(lib().jab_workspace_size(ctypes.byref(p), op, n_bits))


def workspace(p: Problem, op: int, n_bits: int = 0, device="cuda") -> torch.Tensor:
    n = workspace_size(p, op, n_bits)
    if n == 0:
        raise JabError(JAB_E_INVALID, "invalid problem for workspace_size")
    return torch.empty(n, dtype=torch.uint8, device=device)


# --------------------------------------------------------------------------- entry points
def quant_init(p: Problem, w: torch.Tensor, bits: Sequence[int]) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    ng = p.d_model // p.group_size
    scale = torch.empty((p.rows, ng), dtype=torch.float32, device=w.device)
    zero = torch.empty((p.rows, ng), dtype=torch.uint8, device=w.device) if p.scheme == ASYM else None
    b = (ctypes.c_int32 * 3)(*[int(v) for v in bits])
    _check(lib().jab_quant_init(ctypes.byref(p), _ptr(w), ctypes.cast(b, ctypes.c_void_p), _ptr(scale),
                                _ptr(zero), _stream()))
    return scale, zero


def quantize(p: Problem, w: torch.Tensor, bits, scale, zero, want_codes=True, want_w_hat=True,
             want_werr=True, out: Optional[dict] = None, ws: Optional[torch.Tensor] = None) -> dict:
    """Codes, fake-quantized fp32 weights and eps^W sums; `out` may hold preallocated "codes",
    "w_hat" and "werr" tensors (then the want_* flags are ignored)."""
    dev = w.device
    if out is not None:
        codes, w_hat, werr = out.get("codes"), out.get("w_hat"), out.get("werr")
    else:
        codes = torch.empty((p.rows, p.d_model), dtype=torch.uint8, device=dev) if want_codes else None
        w_hat = torch.empty((p.rows, p.d_model), dtype=torch.float32, device=dev) if want_w_hat else None
        werr = torch.empty((3, 2), dtype=torch.float64, device=dev) if want_werr else None
    if werr is not None and ws is None:
        ws = workspace(p, OP_QUANTIZE, device=dev)
    q = _quant(bits, scale, zero)
    _check(lib().jab_quantize(ctypes.byref(p), _ptr(w), ctypes.byref(q), _ptr(codes), _ptr(w_hat), _ptr(werr),
                              _ptr(ws), 0 if ws is None else ws.numel(), _stream()))
    return {"codes": codes, "w_hat": w_hat, "werr": werr}


def project(p: Problem, x: torch.Tensor, w: torch.Tensor, bits=None, scale=None, zero=None,
            ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    y = torch.empty((p.batch, p.seq_len, p.rows), dtype=x.dtype, device=x.device)
    q = None if bits is None else _quant(bits, scale, zero)
    if q is not None and ws is None:
        ws = workspace(p, OP_PROJECT, device=x.device)
    _check(lib().jab_project(ctypes.byref(p), _ptr(x), _ptr(w), None if q is None else ctypes.byref(q), _ptr(y),
                             _ptr(ws), 0 if ws is None else ws.numel(), _stream()))
    return y


def attn_ref(p: Problem, x: torch.Tensor, w: torch.Tensor, ws: Optional[torch.Tensor] = None,
             out: Optional[torch.Tensor] = None) -> torch.Tensor:
    a = out if out is not None else torch.empty((p.batch, p.seq_len, p.n_heads * p.head_dim),
                                                dtype=torch.float32, device=x.device)
    if ws is None:
        ws = workspace(p, OP_REF, device=x.device)
    _check(lib().jab_attn_ref(ctypes.byref(p), _ptr(x), _ptr(w), _ptr(a), _ptr(ws), ws.numel(), _stream()))
    return a


def loss_fwd(p: Problem, x, w, bits, scale, zero, a_ref, ws: Optional[torch.Tensor] = None,
             out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """-> float64 [3 + B]: sse, mse, sum a_ref^2, sse per sequence."""
    if out is None:
        out = torch.empty(3 + p.batch, dtype=torch.float64, device=x.device)
    if ws is None:
        ws = workspace(p, OP_FWD, device=x.device)
    q = _quant(bits, scale, zero)
    _check(lib().jab_loss_fwd(ctypes.byref(p), _ptr(x), _ptr(w), ctypes.byref(q), _ptr(a_ref), _ptr(out),
                              _ptr(ws), ws.numel(), _stream()))
    return out


NOALLOC_SCRATCH_BYTES = 64 << 20      # JAB_NOALLOC_SCRATCH_BYTES


def loss_fwd_noalloc(p: Problem, x, w, bits, scale, zero, a_ref, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """jab_loss_fwd on the library's own device scratch (no workspace argument) -> float64 [3 + B]."""
    if out is None:
        out = torch.empty(3 + p.batch, dtype=torch.float64, device=x.device)
    q = _quant(bits, scale, zero)
    _check(lib().jab_loss_fwd_noalloc(ctypes.byref(p), _ptr(x), _ptr(w), ctypes.byref(q), _ptr(a_ref), _ptr(out),
                                      _stream()))
    return out


def attn_ref_kl(p: Problem, x: torch.Tensor, w: torch.Tensor, ws: Optional[torch.Tensor] = None):
    """Teacher pass keeping the KL term's inputs -> (a_ref fp32 [B][T][Hq*dh], qk_ref dtype
    [B*T][(Hq+Hkv)*dh], lse_ref fp32 [B][Hq][T], base 2)."""
    a = torch.empty((p.batch, p.seq_len, p.n_heads * p.head_dim), dtype=torch.float32, device=x.device)
    qk = torch.empty((p.batch * p.seq_len, (p.n_heads + p.n_kv_heads) * p.head_dim), dtype=x.dtype,
                     device=x.device)
    lse = torch.empty((p.batch, p.n_heads, p.seq_len), dtype=torch.float32, device=x.device)
    if ws is None:
        ws = workspace(p, OP_REF, device=x.device)
    _check(lib().jab_attn_ref_kl(ctypes.byref(p), _ptr(x), _ptr(w), _ptr(a), _ptr(qk), _ptr(lse), _ptr(ws),
                                 ws.numel(), _stream()))
    return a, qk, lse


def loss_fwd_kl(p: Problem, x, w, bits, scale, zero, a_ref, qk_ref, lse_ref, ws: Optional[torch.Tensor] = None,
                out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """-> float64 [2 (3 + B)]: loss_fwd's [3 + B], then kl, kl / B, teacher map mass defect,
    kl per sequence."""
    if out is None:
        out = torch.empty(2 * (3 + p.batch), dtype=torch.float64, device=x.device)
    if ws is None:
        ws = workspace(p, OP_FWD_KL, device=x.device)
    q = _quant(bits, scale, zero)
    _check(lib().jab_loss_fwd_kl(ctypes.byref(p), _ptr(x), _ptr(w), ctypes.byref(q), _ptr(a_ref), _ptr(qk_ref),
                                 _ptr(lse_ref), _ptr(out), _ptr(ws), ws.numel(), _stream()))
    return out


def loss_sweep(p: Problem, x, w, bits: Sequence[int], scales: Sequence[torch.Tensor],
               zeros: Optional[Sequence[Optional[torch.Tensor]]], triples: Sequence[Sequence[int]], a_ref,
               ws: Optional[torch.Tensor] = None, per_seq: bool = True):
    """-> (loss [n_triples] float64, loss_per_seq [n_triples][B] float64 or None)."""
    nb, nt = len(bits), len(triples)
    loss = torch.empty(nt, dtype=torch.float64, device=x.device)
    lps = torch.empty((nt, p.batch), dtype=torch.float64, device=x.device) if per_seq else None
    if ws is None:
        ws = workspace(p, OP_SWEEP, nb, device=x.device)
    cb = (ctypes.c_int32 * nb)(*[int(b) for b in bits])
    cs = (ctypes.c_void_p * nb)(*[s.data_ptr() for s in scales])
    cz = None
    if zeros is not None:
        cz = (ctypes.c_void_p * nb)(*[None if z is None else z.data_ptr() for z in zeros])
    flat = [int(v) for t in triples for v in t]
    ct = (ctypes.c_int32 * len(flat))(*flat)
    _check(lib().jab_loss_sweep(ctypes.byref(p), _ptr(x), _ptr(w), nb, ctypes.cast(cb, ctypes.c_void_p),
                                ctypes.cast(cs, ctypes.c_void_p),
                                None if cz is None else ctypes.cast(cz, ctypes.c_void_p), nt,
                                ctypes.cast(ct, ctypes.c_void_p), _ptr(a_ref), _ptr(loss), _ptr(lps), _ptr(ws),
                                ws.numel(), _stream()))
    return loss, lps


def loss_bwd(p: Problem, x, w, bits, scale, zero, a_ref, gscale: Sequence[float],
             ws: Optional[torch.Tensor] = None):
    """-> (out [3 + B] float64, dw [R][d] fp32, dscale [R][d/g] fp32)."""
    dev = x.device
    out = torch.empty(3 + p.batch, dtype=torch.float64, device=dev)
    dw = torch.empty((p.rows, p.d_model), dtype=torch.float32, device=dev)
    ds = torch.empty((p.rows, p.d_model // p.group_size), dtype=torch.float32, device=dev)
    if ws is None:
        ws = workspace(p, OP_BWD, device=dev)
    g = (ctypes.c_float * 3)(*[float(v) for v in gscale])
    q = _quant(bits, scale, zero)
    _check(lib().jab_loss_bwd(ctypes.byref(p), _ptr(x), _ptr(w), ctypes.byref(q), _ptr(a_ref),
                              ctypes.cast(g, ctypes.c_void_p), _ptr(out), _ptr(dw), _ptr(ds), _ptr(ws),
                              ws.numel(), _stream()))
    return out, dw, ds


def fisher(p: Problem, x, w, bits, scale, zero, a_ref, ws: Optional[torch.Tensor] = None,
           out: Optional[torch.Tensor] = None, lambda_kl: float = 0.0, kl_cache=None) -> torch.Tensor:
    """Fisher-coupling scores at the probe (bits, scale, zero) -> float64 [4]: the squared
    straight-through gradient norms of W_Q, W_K, W_V and the mse."""
    if out is None:
        out = torch.empty(4, dtype=torch.float64, device=x.device)
    if ws is None:
        ws = workspace(p, OP_FISHER, device=x.device)
    q = _quant(bits, scale, zero)
    qk_t, lse_t = kl_cache if kl_cache is not None else (None, None)
    _check(lib().jab_fisher(ctypes.byref(p), _ptr(x), _ptr(w), ctypes.byref(q), _ptr(a_ref), _ptr(qk_t), _ptr(lse_t),
                            float(lambda_kl), _ptr(out), _ptr(ws), ws.numel(), _stream()))
    return out


def ste_finetune(p: Problem, x, a_ref, x_held, a_ref_held, bits, w_master, scale, zero, gscale=None,
                 n_steps: int = 200, eval_every: int = 10, alpha_w: float = 0.05, alpha_s: float = 0.02,
                 beta1: float = 0.9, beta2: float = 0.999, adam_eps: float = 1e-8, scale_floor: float = 1e-12,
                 ws: Optional[torch.Tensor] = None, w: Optional[torch.Tensor] = None, lambda_kl: float = 0.0,
                 kl_cache=None, kl_cache_held=None):
    """Joint STE fine-tuning; w_master (fp32) and scale are updated in place to the best
    checkpoint -> (w in the dtype, stats float64; see jab_ste_stats_len for the layout)."""
    dev = x.device
    cfg = SteConfig(n_steps, eval_every, alpha_w, alpha_s, beta1, beta2, adam_eps, scale_floor, lambda_kl)
    qk_t, lse_t = kl_cache if kl_cache is not None else (None, None)
    qk_h, lse_h = kl_cache_held if kl_cache_held is not None else (None, None)
    n = lib().jab_ste_stats_len(n_steps, eval_every)
    if n <= 0:
        raise JabError(JAB_E_INVALID, "invalid n_steps / eval_every")
    stats = torch.empty(n, dtype=torch.float64, device=dev)
    if w is None:
        w = torch.empty((p.rows, p.d_model), dtype=x.dtype, device=dev)
    if ws is None:
        ws = workspace(p, OP_STE, device=dev)
    if gscale is None:
        gscale = lsq_gscale(bits, p.group_size)
    b = (ctypes.c_int32 * 3)(*[int(v) for v in bits])
    g = (ctypes.c_float * 3)(*[float(v) for v in gscale])
    _check(lib().jab_ste_finetune(ctypes.byref(p), ctypes.byref(cfg), _ptr(x), _ptr(a_ref), int(x_held.shape[0]),
                                  _ptr(x_held), _ptr(a_ref_held), _ptr(qk_t), _ptr(lse_t), _ptr(qk_h), _ptr(lse_h),
                                  ctypes.cast(b, ctypes.c_void_p),
                                  ctypes.cast(g, ctypes.c_void_p), _ptr(w_master), _ptr(w), _ptr(scale),
                                  _ptr(zero), _ptr(stats), _ptr(ws), ws.numel(),
                                  _stream()))
    return w, stats


def loss_bwd_kl(p: Problem, x, w, bits, scale, zero, a_ref, qk_ref, lse_ref, gscale: Sequence[float],
                lambda_kl: float, ws: Optional[torch.Tensor] = None):
    """Backward of mse + lambda_kl * kl / B -> (out [2 (3 + B)] float64, dw, dscale)."""
    dev = x.device
    out = torch.empty(2 * (3 + p.batch), dtype=torch.float64, device=dev)
    dw = torch.empty((p.rows, p.d_model), dtype=torch.float32, device=dev)
    ds = torch.empty((p.rows, p.d_model // p.group_size), dtype=torch.float32, device=dev)
    if ws is None:
        ws = workspace(p, OP_BWD, device=dev)
    g = (ctypes.c_float * 3)(*[float(v) for v in gscale])
    q = _quant(bits, scale, zero)
    _check(lib().jab_loss_bwd_kl(ctypes.byref(p), _ptr(x), _ptr(w), ctypes.byref(q), _ptr(a_ref), _ptr(qk_ref),
                                 _ptr(lse_ref), ctypes.cast(g, ctypes.c_void_p), float(lambda_kl), _ptr(out),
                                 _ptr(dw), _ptr(ds), _ptr(ws), ws.numel(), _stream()))
    return out, dw, ds


# --------------------------------------------------------------------------- the block in use
# A decoding step is a few microseconds on the device, so these calls keep what the host does short: the tensors'
# dtype, shape, layout and device are checked here, everything else in the library.
_current = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_raw_stream = torch._C._cuda_getCurrentRawStream if hasattr(torch._C, "_cuda_getCurrentRawStream") else None


def _here(t: torch.Tensor) -> int:
    """The current GPU, on which the call's tensors have to be (t: one of them)."""
    if not t.is_cuda:
        raise JabError(JAB_E_INVALID, f"a tensor is on {t.device}, not on the current GPU")
    return _current()


def _stream_of(dev: int) -> int:
    return _raw_stream(dev) if _raw_stream is not None else torch.cuda.current_stream(dev).cuda_stream


def _arg(name: str, t: torch.Tensor, dtype: torch.dtype, shape: tuple, dev: int) -> int:
    """The address of a contiguous tensor of this dtype and shape on GPU `dev`."""
    if t.dtype != dtype or t.shape != shape or not t.is_contiguous():
        raise JabError(JAB_E_INVALID, f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)}, not "
                                      f"{t.dtype} {tuple(t.shape)}{'' if t.is_contiguous() else ' with strides'}")
    if t.get_device() != dev:
        raise JabError(JAB_E_INVALID, f"{name} is on {t.device}, not on GPU {dev}")
    return t.data_ptr()


def quant_rows(p: Problem, src: torch.Tensor, codes: Optional[torch.Tensor] = None,
               scale: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Rows of d_model values (any leading dimensions) onto the symmetric 8-bit grid, a scale per row ->
    (codes int8 of src's shape, scale fp32 of its leading dimensions)."""
    d, shape = p.d_model, src.shape
    if len(shape) < 1 or shape[-1] != d:
        raise JabError(JAB_E_INVALID, f"src must have rows of d_model = {d} values, not shape {tuple(shape)}")
    dev = _here(src)
    sp = _arg("src", src, _CODE_DTYPE[p.dtype], shape, dev)
    if codes is None:
        codes = torch.empty_like(src, dtype=torch.int8)
        cp = codes.data_ptr()
    else:
        cp = _arg("codes", codes, torch.int8, shape, dev)
    if scale is None:
        scale = src.new_empty(shape[:-1], dtype=torch.float32)
        ap = scale.data_ptr()
    else:
        ap = _arg("scale", scale, torch.float32, shape[:-1], dev)
    _check(lib().jab_quant_rows(ctypes.byref(p), src.numel() // d, sp, cp, ap, _stream_of(dev)))
    return codes, scale


def project_int(p: Problem, xq: torch.Tensor, sx: torch.Tensor, wq: torch.Tensor, sw: torch.Tensor,
                out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The fused projection on 8-bit integers: codes xq [B][T][d_model], wq [R][d_model] and their rows'
    scales (quant_rows) -> y [B][T][R]."""
    B, T, d, R, dt, dev = p.batch, p.seq_len, p.d_model, p.rows, _CODE_DTYPE[p.dtype], _here(xq)
    if out is None:
        out = xq.new_empty((B, T, R), dtype=dt)
        yp = out.data_ptr()
    else:
        yp = _arg("out", out, dt, (B, T, R), dev)
    _check(lib().jab_project_int(ctypes.byref(p), _arg("xq", xq, torch.int8, (B, T, d), dev),
                                 _arg("sx", sx, torch.float32, (B, T), dev), _arg("wq", wq, torch.int8, (R, d), dev),
                                 _arg("sw", sw, torch.float32, (R,), dev), yp, _stream_of(dev)))
    return out


class Cache:
    """The paged cache of quantized keys and values of one block: the caller's tensors (jab_cache has the layouts)."""

    def __init__(self, p: Problem, bits: int, page_size: int, k, v, k_scale, v_scale, k_zero=None, v_zero=None):
        if bits not in (4, 8) or page_size not in (32, 64, 128, 256):
            raise JabError(JAB_E_INVALID, "bits must be 4 or 8 and page_size 32, 64, 128 or 256")
        n, h, dhb = k.shape[0], p.n_kv_heads, p.head_dim * bits // 8
        if (p.scheme == ASYM) != (k_zero is not None) or (k_zero is None) != (v_zero is None):
            raise JabError(JAB_E_INVALID, "zero-points go with the asymmetric scheme")
        self.tensors = (k, v, k_scale, v_scale, k_zero, v_zero)      # kept alive with the struct's addresses
        self.geometry = (h, p.head_dim, p.scheme)
        if not k.is_cuda:
            raise JabError(JAB_E_INVALID, f"the cache is on {k.device}, not on a GPU")
        self.device = dev = k.get_device()
        rows = (n, h, page_size)
        self.struct = _CacheStruct(
            bits, page_size, n, _arg("k", k, torch.uint8, rows + (dhb,), dev),
            _arg("v", v, torch.uint8, (n, h, page_size // 32, dhb, 32), dev),
            _arg("k_scale", k_scale, torch.float32, rows, dev), _arg("v_scale", v_scale, torch.float32, rows, dev),
            None if k_zero is None else _arg("k_zero", k_zero, torch.uint8, rows, dev),
            None if v_zero is None else _arg("v_zero", v_zero, torch.uint8, rows, dev))
        self.ref = ctypes.byref(self.struct)

    @classmethod
    def empty(cls, p: Problem, bits: int, page_size: int, n_pages: int, device="cuda") -> "Cache":
        """A cache of n_pages unwritten pages."""
        h, dhb = p.n_kv_heads, p.head_dim * bits // 8
        rows = (n_pages, h, page_size)

        def buf(shape, dtype):
            return torch.empty(shape, dtype=dtype, device=device)

        z = p.scheme == ASYM
        return cls(p, bits, page_size, buf(rows + (dhb,), torch.uint8),
                   buf((n_pages, h, page_size // 32, dhb, 32), torch.uint8), buf(rows, torch.float32),
                   buf(rows, torch.float32), buf(rows, torch.uint8) if z else None, buf(rows, torch.uint8) if z else None)


class CacheRows:
    """Which rows of a batch belong to which sequence (jab_cache_rows): pages int32 [n_seq][max_pages], past
    int32 [n_seq], start int32 [n_seq + 1], and the most new tokens of a sequence."""

    def __init__(self, pages: torch.Tensor, past: torch.Tensor, start: torch.Tensor, max_new: int):
        if pages.dim() != 2:
            raise JabError(JAB_E_INVALID, "pages must be [n_seq][max_pages]")
        n = pages.shape[0]
        if not pages.is_cuda:
            raise JabError(JAB_E_INVALID, f"pages is on {pages.device}, not on a GPU")
        self.device = dev = pages.get_device()
        self.tensors = (pages, past, start)
        self.struct = _CacheRowsStruct(n, pages.shape[1], int(max_new),
                                       _arg("pages", pages, torch.int32, pages.shape, dev),
                                       _arg("past", past, torch.int32, (n,), dev),
                                       _arg("start", start, torch.int32, (n + 1,), dev))
        self.ref = ctypes.byref(self.struct)


def _cache_call(p: Problem, cache: Cache, rows: CacheRows) -> int:
    """The GPU of a call on this cache and these rows."""
    if cache.geometry != (p.n_kv_heads, p.head_dim, p.scheme):
        raise JabError(JAB_E_INVALID, "the cache was laid out for other heads or another scheme")
    dev = _current()
    if cache.device != dev or rows.device != dev:
        raise JabError(JAB_E_INVALID, "the cache and its rows must be on the current GPU")
    return dev


def cache_write(p: Problem, cache: Cache, rows: CacheRows, y: torch.Tensor) -> None:
    """The key (turned by the rotary embedding) and value columns of y [B][T][R] into the cache."""
    dev = _cache_call(p, cache, rows)
    _check(lib().jab_cache_write(ctypes.byref(p), cache.ref, rows.ref,
                                 _arg("y", y, _CODE_DTYPE[p.dtype], (p.batch, p.seq_len, p.rows), dev), _stream_of(dev)))


def cache_read(p: Problem, cache: Cache, rows: CacheRows, k: Optional[torch.Tensor] = None,
               v: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """What cache_write stored for these rows -> (k, v) [B][T][n_kv_heads * head_dim] in the dtype."""
    dev, dt, shape = _cache_call(p, cache, rows), _CODE_DTYPE[p.dtype], (p.batch, p.seq_len, p.n_kv_heads * p.head_dim)
    if k is None:
        k = cache.tensors[0].new_empty(shape, dtype=dt)
        kp = k.data_ptr()
    else:
        kp = _arg("k", k, dt, shape, dev)
    if v is None:
        v = cache.tensors[0].new_empty(shape, dtype=dt)
        vp = v.data_ptr()
    else:
        vp = _arg("v", v, dt, shape, dev)
    _check(lib().jab_cache_read(ctypes.byref(p), cache.ref, rows.ref, kp, vp, _stream_of(dev)))
    return k, v


def attn_cache_workspace(p: Problem, cache: Cache, rows: CacheRows) -> torch.Tensor:
    """The workspace attn_cache needs for this cache and these rows' sizes (possibly empty)."""
    n = lib().jab_attn_cache_workspace(ctypes.byref(p), cache.ref, rows.ref)
    if n == ctypes.c_size_t(-1).value:
        raise JabError(JAB_E_INVALID, lib().jab_last_error().decode())
    return torch.empty(n, dtype=torch.uint8, device=cache.tensors[0].device)


def attn_cache(p: Problem, cache: Cache, rows: CacheRows, y: torch.Tensor, ws: Optional[torch.Tensor] = None,
               out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Attention of y's query columns over the cache -> [B][T][n_heads * head_dim] in the dtype."""
    dev, dt, B, T = _cache_call(p, cache, rows), _CODE_DTYPE[p.dtype], p.batch, p.seq_len
    shape = (B, T, p.n_heads * p.head_dim)
    yp = _arg("y", y, dt, (B, T, p.rows), dev)
    if out is None:
        out = y.new_empty(shape)
        ap = out.data_ptr()
    else:
        ap = _arg("out", out, dt, shape, dev)
    if ws is None:
        ws = attn_cache_workspace(p, cache, rows)
    _check(lib().jab_attn_cache(ctypes.byref(p), cache.ref, rows.ref, yp, ap, _arg("ws", ws, torch.uint8, ws.shape, dev),
                                ws.numel(), _stream_of(dev)))
    return out


CURVATURE_FORMS = ("t_Q", "t_K", "t_V", "pooled", "h_QQ", "h_KK", "h_VV")


def curvature(p: Problem, x, w, probes: torch.Tensor, lambda_kl: float = 0.0, ws: Optional[torch.Tensor] = None,
              out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Hutchinson terms of eq. gn's Hessian at the float point -> float64 [n_probes][7] in the order of
    CURVATURE_FORMS (per-unit partition t_u, pooled v^T H v, diagonal blocks h_uu).
    probes: int8 [n_probes][R][d_model] in {-1, +1}."""
    n_probes = probes.shape[0]
    if out is None:
        out = torch.empty((n_probes, 7), dtype=torch.float64, device=x.device)
    if ws is None:
        ws = workspace(p, OP_CURVATURE, device=x.device)
    _check(lib().jab_curvature(ctypes.byref(p), _ptr(x), _ptr(w), float(lambda_kl), n_probes, _ptr(probes),
                               _ptr(out), _ptr(ws), ws.numel(), _stream()))
    return out


def allocate(omega, widths: Sequence[int], params: Sequence[float], budget_bits: float, min_bits: int = 0,
             method: int = ALLOC_GREEDY) -> Tuple[list, float]:
    """Bit allocation of eq. mckp (host-only) -> (width index per unit, objective)."""
    rows = [list(map(float, r)) for r in omega]
    n, k = len(rows), len(widths)
    if any(len(r) != k for r in rows) or len(params) != n:
        raise JabError(JAB_E_INVALID, "omega must be [n_units][n_widths] and params [n_units]")
    om = (ctypes.c_double * (n * k))(*[v for r in rows for v in r])
    wd = (ctypes.c_int32 * k)(*[int(v) for v in widths])
    pr = (ctypes.c_double * n)(*[float(v) for v in params])
    ch = (ctypes.c_int32 * n)()
    obj = ctypes.c_double(0.0)
    _check(lib().jab_allocate(n, k, ctypes.addressof(wd), ctypes.addressof(om), ctypes.addressof(pr),
                              float(budget_bits), int(min_bits), int(method), ctypes.addressof(ch),
                              ctypes.addressof(obj)))
    return list(ch), obj.value


def omega(curv, werr, trace: int = TRACE_BLOCK, criterion: int = OMEGA_C1) -> torch.Tensor:
    """Sensitivity table of eq. omega (host-only): curv [n_layers][n_probes][7] (jab_curvature's
    output per block), werr [n_layers][n_widths][3][2] (jab_quantize's per width) ->
    omega [3 n_layers][n_widths] (float64, host) for jab_allocate."""
    c = torch.as_tensor(curv, dtype=torch.float64).cpu().contiguous()
    e = torch.as_tensor(werr, dtype=torch.float64).cpu().contiguous()
    if c.dim() != 3 or c.shape[2] != 7 or e.dim() != 4 or e.shape[0] != c.shape[0] or tuple(e.shape[2:]) != (3, 2):
        raise JabError(JAB_E_INVALID, "curv must be [n_layers][n_probes][7] and werr [n_layers][n_widths][3][2]")
    out = torch.empty((3 * c.shape[0], e.shape[1]), dtype=torch.float64)
    _check(lib().jab_omega(c.shape[0], c.shape[1], c.data_ptr(), e.shape[1], e.data_ptr(), int(trace),
                           int(criterion), out.data_ptr()))
    return out


def set_bwd_ds_limit(max_bytes: int) -> None:
    """Largest stored-dS buffer the attention backward keeps in its workspace (default
    8 GiB; 0 recomputes dS in the dQ pass).  Set before sizing workspaces."""
    _check(lib().jab_set_bwd_ds_limit(int(max_bytes)))


def timing_enable(on: bool = True) -> None:
    _check(lib().jab_timing_enable(1 if on else 0))


def timing_read() -> dict:
    """Per kernel family: (summed milliseconds, launches) since the last read."""
    ms = (ctypes.c_double * len(KT_NAMES))()
    n = (ctypes.c_int64 * len(KT_NAMES))()
    _check(lib().jab_timing_read(ctypes.cast(ms, ctypes.c_void_p), ctypes.cast(n, ctypes.c_void_p)))
    return {k: (ms[i], n[i]) for i, k in enumerate(KT_NAMES)}


def lsq_gscale(bits: Sequence[int], group: int, scheme: int = ASYM):
    """LSQ's gradient factor (n_w q_max)^(-1/2) per matrix, n_w = weights sharing a scale."""
    out = []
    for b in bits:
        if b == 0:
            out.append(0.0)
            continue
        qmax = (1 << b) - 1 if scheme == ASYM else (1 << (b - 1)) - 1
        out.append(float((group * qmax) ** -0.5))
    return out
