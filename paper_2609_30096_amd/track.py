"""Python binding of libtrack.so (the C ABI declared in include/track.h).

Argument marshalling only: every step of the denoiser, the sampler loops and
the routing run inside the library.  torch provides device memory and the
current stream.  The library must have been built (``__graft_entry__.build()``
or ``python -m paper_2609_30096_amd.build``); without it every call raises.
"""
from __future__ import annotations

import ctypes
import dataclasses
import os
from typing import Dict, List, Optional, Sequence, Tuple

import numpy as np

from . import synth

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libtrack.so")
_lib = None

OK, E_INVALID, E_SHAPE, E_INCOMPATIBLE, E_DEVICE, E_NOMEM, E_UNSUPPORTED = range(7)
DTYPE_F32, DTYPE_BF16 = 0, 1
EPI_BIAS, EPI_BIAS_GELU, EPI_GATE_RESID, EPI_RESID, EPI_BIAS_F32 = range(5)
PROF_ATTN_SELF, PROF_ATTN_CROSS, PROF_GEMM, PROF_NORM, PROF_STEP, PROF_OTHER = range(6)

EXPORTS = [
    "track_weight_count", "track_weights_bytes", "track_weight_info", "track_model_create", "track_model_destroy",
    "track_workspace_bytes", "track_model_set_workspace", "track_dit_forward", "track_calibrate",
    "track_calibrate_bands", "track_band_workspace_bytes", "track_op_band_energy",
    "track_route_policy", "track_route_threshold", "track_route_baseline", "track_sample", "track_last_error",
    "track_op_linear", "track_op_linear_vt", "track_op_attention", "track_op_attention_log2q",
    "track_op_layernorm", "track_rope_table_len", "track_op_rmsnorm_rope", "track_op_rmsnorm_rope_qk", "track_step_partial_count",
    "track_op_step", "track_op_step_noalloc", "track_hbm_stream", "track_mfma_stream", "track_unipc_coefficients", "track_op_unipc_step", "track_profile_enable", "track_profile_reset", "track_profile_read", "track_set_progress",
    "track_rope_freqs", "track_op_rope", "track_op_headnorm_rope", "track_attention_window_workspace_bytes",
    "track_op_attention_window",
]


class TrackError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"[track status {status}] {msg}")
        self.status = status


class DitConfigC(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "blocks", "dim", "heads", "head_dim", "ffn_dim", "in_ch", "patch_t", "patch_h", "patch_w",
        "text_dim", "freq_dim", "dtype")]


class LatentShapeC(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("channels", "frames", "height", "width", "text_len")]


class SamplerConfigC(ctypes.Structure):
    _fields_ = [("steps", ctypes.c_int32), ("use_cfg", ctypes.c_int32), ("shift", ctypes.c_double),
                ("guidance", ctypes.c_double), ("eps", ctypes.c_double), ("solver", ctypes.c_int32),
                ("order", ctypes.c_int32)]


class RopeConfigC(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("head_dim", "rot_dim", "layout", "axes")] +
                [("section", ctypes.c_int32 * 3), ("scaling", ctypes.c_int32)] +
                [(n, ctypes.c_double) for n in ("base", "factor", "orig_len", "beta_fast", "beta_slow")])


class HeadRowsC(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("ldx", ctypes.c_int64), ("sx", ctypes.c_int64),
                ("y", ctypes.c_void_p), ("ldy", ctypes.c_int64), ("sy", ctypes.c_int64), ("heads", ctypes.c_int32)]


class WindowC(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("left", "right", "sink", "group")] + [("scale", ctypes.c_double)]


SOLVERS = {"euler": 0, "unipc": 1}
ROPE_LAYOUTS = {"interleaved": 0, "half": 1}
ROPE_SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "yarn": 3}


_vp, _i32, _i64, _f32, _f64, _sz = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float,
                                    ctypes.c_double, ctypes.c_size_t)
PROGRESS_FN = ctypes.CFUNCTYPE(None, ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32)
_progress_ref = None


def _declare(L):
    P = ctypes.POINTER
    sig = {
        "track_weight_count": (_i32, [P(DitConfigC)]),
        "track_weights_bytes": (_sz, [P(DitConfigC)]),
        "track_weight_info": (_i32, [P(DitConfigC), _i32, P(ctypes.c_char_p), P(_i32), P(_i64), P(_sz)]),
        "track_model_create": (_i32, [P(DitConfigC), _vp, _sz, P(_vp)]),
        "track_model_destroy": (None, [_vp]),
        "track_workspace_bytes": (_sz, [_vp, P(LatentShapeC), _i32]),
        "track_model_set_workspace": (_i32, [_vp, _vp, _sz]),
        "track_dit_forward": (_i32, [_vp, P(LatentShapeC), _vp, _f64, _vp, _vp, _f32, _vp, _vp]),
        "track_calibrate": (_i32, [_vp, _vp, P(LatentShapeC), _i32, P(_vp), P(_vp), _vp, P(SamplerConfigC),
                                   P(_f64), P(_f64), P(_vp), _vp]),
        "track_calibrate_bands": (_i32, [_vp, _vp, P(LatentShapeC), _i32, P(_vp), P(_vp), _vp, P(SamplerConfigC),
                                         P(_f64), P(_f64), P(_f64), P(_f64), P(_vp), _vp]),
        "track_band_workspace_bytes": (_sz, [P(LatentShapeC), _i32, _i32, _i32]),
        "track_op_band_energy": (_i32, [P(LatentShapeC), _i32, _i32, _i32, _i32, _f32, _vp, _vp, _vp, _sz, P(_f64),
                                        _vp]),
        "track_route_policy": (_i32, [P(_f64), _i32, _i32, P(_i32)]),
        "track_route_threshold": (_i32, [P(_f64), _i32, _f64, P(_i32), P(_i32)]),
        "track_route_baseline": (_i32, [_i32, _i32, _i32, ctypes.c_uint64, P(_i32)]),
        "track_sample": (_i32, [_vp, _vp, P(ctypes.c_uint8), P(LatentShapeC), P(SamplerConfigC), _vp, _vp, _vp,
                                _vp, _vp]),
        "track_last_error": (ctypes.c_char_p, []),
        "track_op_linear": (_i32, [_i32, _i32, _i64, _i64, _i64, _vp, _i64, _vp, _vp, _vp, _vp, _i64, _vp]),
        "track_op_linear_vt": (_i32, [_i32, _i64, _i64, _i64, _vp, _i64, _vp, _vp, _i64, _vp, _i64, _vp]),
        "track_op_attention": (_i32, [_i32, _i32, _i32, _i32, _i64, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _vp,
                                      _i64, _vp]),
        "track_op_attention_log2q": (_i32, [_i32, _i32, _i32, _i32, _i64, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _vp,
                                      _i64, _vp]),
        "track_op_layernorm": (_i32, [_i32, _i64, _i32, _vp, _vp, _vp, _vp, _vp]),
        "track_rope_table_len": (_i64, [_i32, P(_i32)]),
        "track_op_rmsnorm_rope": (_i32, [_i32, _i64, _i32, _i32, _vp, _i64, _i64, _vp, P(_i32), _vp, _vp]),
        "track_op_rmsnorm_rope_qk": (_i32, [_i32, _i64, _i32, _i32, _vp, _i64, _i64, _vp, _vp, P(_i32), _vp, _vp]),
        "track_rope_freqs": (_i32, [P(RopeConfigC), P(_f64), P(_f32)]),
        "track_op_rope": (_i32, [_i32, P(RopeConfigC), _i64, _i64, P(HeadRowsC), P(HeadRowsC), _vp, _vp, _f32, _i32,
                                 _vp]),
        "track_op_headnorm_rope": (_i32, [_i32, P(RopeConfigC), _i64, _i64, P(HeadRowsC), P(HeadRowsC), _vp, _vp, _f32,
                                          _f32, _vp, _vp, _f32, _vp]),
        "track_attention_window_workspace_bytes": (_i64, [_i32, P(WindowC), _i32, _i32, _i32, _i32, _i64, _i64]),
        "track_op_attention_window": (_i32, [_i32, P(WindowC), _i32, _i32, _i32, _i32, _i64, _i64] +
                                      [_vp, _i64, _i64] * 4 + [_vp] * 5 + [_sz, _vp]),
        "track_step_partial_count": (_i64, [_i64]),
        "track_op_step": (_i32, [_i64, _i32, _f32, _f32, _vp, _vp, _vp, _vp, _f64, _vp, _vp]),
        "track_op_step_noalloc": (_i32, [_i64, _i32, _f32, _f32, _vp, _vp, _vp, _f64, _vp, _vp]),
        "track_unipc_coefficients": (_i32, [_i32, _f64, _i32, _i32, P(_f64)]),
        "track_op_unipc_step": (_i32, [_i64, _i32, _f32, _f32, P(_f64), _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                       _f64, _vp, _vp]),
        "track_hbm_stream": (_i32, [_i32, _vp, _vp, _i64, _vp]),
        "track_mfma_stream": (_i32, [_vp, _i64, _vp, ctypes.POINTER(ctypes.c_int64), _vp]),
        "track_profile_enable": (_i32, [_i32]),
        "track_profile_reset": (_i32, []),
        "track_profile_read": (_i32, [_i32, P(_i64), P(_f64)]),
        "track_set_progress": (_i32, [PROGRESS_FN, _vp]),
    }
    for name, (res, args) in sig.items():
        f = getattr(L, name)
        f.restype = res
        f.argtypes = args


def lib():
    """The loaded library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(f"{_LIB_PATH} is missing: build it with `python -m paper_2609_30096_amd.build`")
        L = ctypes.CDLL(_LIB_PATH)
        _declare(L)
        _lib = L
    return _lib


def _check(status: int):
    if status != OK:
        raise TrackError(status, lib().track_last_error().decode())


def _torch():
    import torch
    return torch


def _stream():
    torch = _torch()
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _ptr(t) -> ctypes.c_void_p:
    return ctypes.c_void_p(0 if t is None else t.data_ptr())


def dtype_code(dtype: str) -> int:
    return DTYPE_BF16 if dtype == synth.BF16 else DTYPE_F32


def torch_dtype(dtype: str):
    torch = _torch()
    return torch.bfloat16 if dtype == synth.BF16 else torch.float32


def config_c(cfg: synth.DiTConfig) -> DitConfigC:
    pt, ph, pw = cfg.patch
    return DitConfigC(cfg.blocks, cfg.dim, cfg.heads, cfg.head_dim, cfg.ffn_dim, cfg.in_ch, pt, ph, pw,
                      cfg.text_dim, cfg.freq_dim, dtype_code(cfg.dtype))


def shape_c(shape: synth.LatentShape) -> LatentShapeC:
    return LatentShapeC(shape.channels, shape.frames, shape.height, shape.width, shape.text_len)


def sampler_c(scfg: synth.SamplerConfig) -> SamplerConfigC:
    return SamplerConfigC(scfg.steps, 1 if scfg.use_cfg else 0, scfg.shift, scfg.guidance, scfg.eps,
                          SOLVERS[scfg.solver], scfg.order)


# ---------------------------------------------------------------- weights and models
def weight_table(cfg: synth.DiTConfig) -> Tuple[List[Tuple[str, Tuple[int, ...], int]], int]:
    """[(name, shape, byte offset)] in buffer order, and the buffer size."""
    L = lib()
    c = config_c(cfg)
    n = L.track_weight_count(ctypes.byref(c))
    if n < 0:
        raise TrackError(E_INVALID, "invalid config: " + L.track_last_error().decode())
    out = []
    for i in range(n):
        name = ctypes.c_char_p()
        nd = _i32()
        shp = (_i64 * 2)()
        off = _sz()
        _check(L.track_weight_info(ctypes.byref(c), i, ctypes.byref(name), ctypes.byref(nd), shp, ctypes.byref(off)))
        out.append((name.value.decode(), tuple(shp[:nd.value]), off.value))
    return out, L.track_weights_bytes(ctypes.byref(c))


def pack_weights(cfg: synth.DiTConfig, params: Dict[str, np.ndarray], device="cuda"):
    """Device weight buffer (uint8 tensor) holding ``params`` in the library's layout."""
    torch = _torch()
    table, total = weight_table(cfg)
    buf = torch.empty(total, dtype=torch.uint8, device=device)
    tdt = torch_dtype(cfg.dtype)
    es = 2 if cfg.dtype == synth.BF16 else 4
    for name, shape, off in table:
        a = params[name]
        if tuple(a.shape) != shape:
            raise ValueError(f"{name}: shape {a.shape} != {shape}")
        t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(device).to(tdt).reshape(-1)
        buf[off:off + t.numel() * es].view(tdt).copy_(t)
    return buf


def gen_weights_on_device(cfg: synth.DiTConfig, model_seed: int, device="cuda", threads: int = 16):
    """pack_weights of the seeded recipe; drawn on host threads chunk by chunk, one block at a time."""
    import concurrent.futures as cf
    torch = _torch()
    table, total = weight_table(cfg)
    specs = synth.param_specs(cfg)
    for i, (name, _, _) in enumerate(table):
        if specs[i][0] != name:
            raise ValueError(f"tensor order mismatch at {i}: {specs[i][0]} vs {name}")
    buf = torch.empty(total, dtype=torch.uint8, device=device)
    tdt = torch_dtype(cfg.dtype)
    es = 2 if cfg.dtype == synth.BF16 else 4
    # groups of tensors generated together: the globals, each block, the head
    groups, cur, prefix = [], [], None
    for i, (name, _, _) in enumerate(table):
        p = name.split(".")[0] if name.startswith("blk") else ("head" if name.startswith("head") else "global")
        if p != prefix and cur:
            groups.append(cur)
            cur = []
        prefix = p
        cur.append(i)
    groups.append(cur)
    with cf.ThreadPoolExecutor(max_workers=threads) as ex:
        for g in groups:
            arrs = synth.gen_param_set(cfg, model_seed, g, ex, round_to_dtype=False)
            for i in g:
                name, shape, off = table[i]
                # float32 -> bf16 rounds to nearest even on the device
                t = torch.from_numpy(arrs[name]).reshape(-1).to(device).to(tdt)
                buf[off:off + t.numel() * es].view(tdt).copy_(t)
    return buf


class Model:
    """A model handle over a device weight buffer, with a torch-allocated workspace."""

    def __init__(self, cfg: synth.DiTConfig, weights):
        self.cfg = cfg
        self.weights = weights
        self._c = config_c(cfg)
        h = _vp()
        _check(lib().track_model_create(ctypes.byref(self._c), _ptr(weights), weights.numel(), ctypes.byref(h)))
        self.handle = h
        self.workspace = None

    def workspace_bytes(self, shape: synth.LatentShape, batch: int) -> int:
        n = lib().track_workspace_bytes(self.handle, ctypes.byref(shape_c(shape)), batch)
        if n == 0:
            raise TrackError(E_SHAPE, f"latent shape {shape} is invalid for this model")
        return n

    def ensure_workspace(self, shape: synth.LatentShape, batch: int):
        need = self.workspace_bytes(shape, batch)
        if self.workspace is None or self.workspace.numel() < need:
            torch = _torch()
            self.workspace = None
            self.workspace = torch.empty(need, dtype=torch.uint8, device=self.weights.device)
            _check(lib().track_model_set_workspace(self.handle, _ptr(self.workspace), need))

    def close(self):
        if getattr(self, "handle", None):
            lib().track_model_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ---------------------------------------------------------------- the four calls
def dit_forward(model: Model, shape: synth.LatentShape, x_t, t: float, cond, uncond=None, guidance: float = 1.0):
    """Guided prediction p(x_t, t) (Eq. 1); x_t: device [C, F, H, W] float32."""
    torch = _torch()
    model.ensure_workspace(shape, 2 if uncond is not None else 1)
    out = torch.empty_like(x_t)
    _check(lib().track_dit_forward(model.handle, ctypes.byref(shape_c(shape)), _ptr(x_t), float(t), _ptr(cond),
                                   _ptr(uncond), float(guidance), _ptr(out), _stream()))
    return out


def calibrate(large: Model, small: Model, shape: synth.LatentShape, x_T: Sequence, conds: Sequence, uncond,
              scfg: synth.SamplerConfig, return_x0: bool = False, bands: bool = False):
    """Reference-trajectory calibration; returns (r [M, N], q [N]) as float64 numpy arrays.

    With bands, also the band scores (rb [M, N, 6], qb [N, 6]: spatial low,
    mid, high, temporal low, mid, high).  With return_x0, also the list of
    each sample's all-large endpoint (device tensors), last.
    """
    torch = _torch()
    B = 2 if scfg.use_cfg else 1
    large.ensure_workspace(shape, B)
    small.ensure_workspace(shape, B)
    M, N = len(x_T), scfg.steps
    xs = (_vp * M)(*[t.data_ptr() for t in x_T])
    cs = (_vp * M)(*[t.data_ptr() for t in conds])
    r = np.zeros((M, N), dtype=np.float64)
    q = np.zeros(N, dtype=np.float64)
    sc = sampler_c(scfg)
    x0 = [torch.empty_like(t) for t in x_T] if return_x0 else None
    x0p = (_vp * M)(*[t.data_ptr() for t in x0]) if return_x0 else None
    if bands:
        rb = np.zeros((M, N, 6), dtype=np.float64)
        qb = np.zeros((N, 6), dtype=np.float64)
        _check(lib().track_calibrate_bands(large.handle, small.handle, ctypes.byref(shape_c(shape)), M, xs, cs,
                                           _ptr(uncond), ctypes.byref(sc), r.ctypes.data_as(ctypes.POINTER(_f64)),
                                           q.ctypes.data_as(ctypes.POINTER(_f64)),
                                           rb.ctypes.data_as(ctypes.POINTER(_f64)),
                                           qb.ctypes.data_as(ctypes.POINTER(_f64)), x0p, _stream()))
        out = (r, q, rb, qb)
    else:
        _check(lib().track_calibrate(large.handle, small.handle, ctypes.byref(shape_c(shape)), M, xs, cs,
                                     _ptr(uncond), ctypes.byref(sc), r.ctypes.data_as(ctypes.POINTER(_f64)),
                                     q.ctypes.data_as(ctypes.POINTER(_f64)), x0p, _stream()))
        out = (r, q)
    return out + (x0,) if return_x0 else out


def route_policy(q, K: int) -> np.ndarray:
    """Indices of the K lowest scores, ascending (ties to the lower index)."""
    q = np.ascontiguousarray(q, dtype=np.float64)
    out = np.zeros(max(K, 1), dtype=np.int32)
    _check(lib().track_route_policy(q.ctypes.data_as(ctypes.POINTER(_f64)), len(q), int(K),
                                    out.ctypes.data_as(ctypes.POINTER(_i32))))
    return out[:K].copy()


def route_threshold(q, C0: float) -> np.ndarray:
    """Steps with q_k^2 < C0 (Eqs. 6-7, C_0 form), ascending."""
    q = np.ascontiguousarray(q, dtype=np.float64)
    out = np.zeros(len(q), dtype=np.int32)
    n = _i32(0)
    _check(lib().track_route_threshold(q.ctypes.data_as(ctypes.POINTER(_f64)), len(q), float(C0),
                                       out.ctypes.data_as(ctypes.POINTER(_i32)), ctypes.byref(n)))
    return out[:n.value].copy()


POLICY_FIRST_K, POLICY_LAST_K, POLICY_RANDOM_K = 0, 1, 2


def route_baseline(kind: int, N: int, K: int, seed: int = 0) -> np.ndarray:
    """Equal-budget baseline policy (First-K, Last-K, Random-K): K step indices, ascending."""
    out = np.zeros(max(K, 1), dtype=np.int32)
    _check(lib().track_route_baseline(int(kind), int(N), int(K), int(seed) & (2**64 - 1),
                                      out.ctypes.data_as(ctypes.POINTER(_i32))))
    return out[:K].copy()


def sample(large: Model, small: Optional[Model], use_small, shape: synth.LatentShape, scfg: synth.SamplerConfig,
           x_T, cond, uncond=None, out=None):
    """Routed sampling (Eq. 3); returns x_0 as a device tensor [C, F, H, W] (in `out` if given,
    which may be x_T itself)."""
    torch = _torch()
    B = 2 if scfg.use_cfg else 1
    large.ensure_workspace(shape, B)
    if small is not None:
        small.ensure_workspace(shape, B)
    pol = np.ascontiguousarray(np.asarray(use_small, dtype=bool).astype(np.uint8))
    if pol.shape != (scfg.steps,):
        raise ValueError("use_small must have one entry per step")
    out = torch.empty_like(x_T) if out is None else out
    sc = sampler_c(scfg)
    _check(lib().track_sample(large.handle, None if small is None else small.handle,
                              pol.ctypes.data_as(ctypes.POINTER(ctypes.c_uint8)), ctypes.byref(shape_c(shape)),
                              ctypes.byref(sc), _ptr(x_T), _ptr(cond), _ptr(uncond), _ptr(out), _stream()))
    return out


# ---------------------------------------------------------------- component entry points
def op_linear(dtype: int, epilogue: int, A, W, bias, out, gate=None, M=None, N=None, K=None, lda=None, ldo=None):
    M = A.shape[0] if M is None else M
    K = W.shape[1] if K is None else K
    N = W.shape[0] if N is None else N
    lda = A.stride(0) if lda is None else lda
    ldo = out.stride(0) if ldo is None else ldo
    _check(lib().track_op_linear(dtype, epilogue, M, N, K, _ptr(A), lda, _ptr(W), _ptr(bias), _ptr(gate), _ptr(out),
                                 ldo, _stream()))


def op_linear_vt(A, W, bias, L: int, vt, ldv: int, dtype: int = DTYPE_BF16):
    """A W^T + bias written transposed per batch of L rows into vt (the V^T layout of op_attention)."""
    M, K = A.shape
    N = W.shape[0]
    _check(lib().track_op_linear_vt(dtype, M, N, K, _ptr(A), A.stride(0), _ptr(W), _ptr(bias), L, _ptr(vt), ldv,
                                    _stream()))


def op_attention(dtype: int, B: int, H: int, head_dim: int, Lq: int, Lk: int, q, ldq: int, k, ldk: int, vt, ldv: int,
                 out, ldo: int, q_log2: bool = False):
    """q_log2: q is given times log2(e) / sqrt(head_dim) (track_op_attention_log2q)."""
    fn = lib().track_op_attention_log2q if q_log2 else lib().track_op_attention
    _check(fn(dtype, B, H, head_dim, Lq, Lk, _ptr(q), ldq, _ptr(k), ldk, _ptr(vt), ldv, _ptr(out), ldo, _stream()))


def op_layernorm(dtype: int, x, y, scale=None, shift=None):
    rows, d = x.shape
    _check(lib().track_op_layernorm(dtype, rows, d, _ptr(x), _ptr(scale), _ptr(shift), _ptr(y), _stream()))


def op_rmsnorm_rope(dtype: int, buf, heads: int, head_dim: int, g, col0: int = 0, grid=None, rows=None, ld=None):
    torch = _torch()
    rows = buf.shape[0] if rows is None else rows
    ld = buf.stride(0) if ld is None else ld
    ws = None
    gp = None
    if grid is not None:
        gp = (_i32 * 3)(*grid)
        n = lib().track_rope_table_len(head_dim, gp)
        ws = torch.empty(2 * n, dtype=torch.float32, device=buf.device)
    _check(lib().track_op_rmsnorm_rope(dtype, rows, heads, head_dim, _ptr(buf), ld, col0, _ptr(g), gp, _ptr(ws),
                                       _stream()))


def op_rmsnorm_rope_qk(dtype: int, buf, heads: int, head_dim: int, g_q, g_k, col0: int = 0, grid=None, rows=None,
                       ld=None):
    """op_rmsnorm_rope on the two adjacent segments (q with g_q, then k with g_k) of every row, one launch."""
    torch = _torch()
    rows = buf.shape[0] if rows is None else rows
    ld = buf.stride(0) if ld is None else ld
    ws = None
    gp = None
    if grid is not None:
        gp = (_i32 * 3)(*grid)
        n = lib().track_rope_table_len(head_dim, gp)
        ws = torch.empty(2 * n, dtype=torch.float32, device=buf.device)
    _check(lib().track_op_rmsnorm_rope_qk(dtype, rows, heads, head_dim, _ptr(buf), ld, col0, _ptr(g_q), _ptr(g_k), gp,
                                          _ptr(ws), _stream()))


@dataclasses.dataclass(frozen=True)
class RopeConfig:
    """Rotary positions (track_rope_config): sections are the rotated pairs of each axis."""
    head_dim: int
    rot_dim: Optional[int] = None            # head_dim
    layout: str = "interleaved"              # or "half"
    sections: Optional[Tuple[int, ...]] = None  # one axis
    base: float = 10000.0
    scaling: str = "none"                    # "linear", "ntk", "yarn"
    factor: float = 1.0
    orig_len: float = 4096.0
    beta_fast: float = 32.0
    beta_slow: float = 1.0

    def c(self) -> RopeConfigC:
        rot = self.head_dim if self.rot_dim is None else self.rot_dim
        sec = (rot // 2,) if self.sections is None else tuple(self.sections)
        if len(sec) > 3:
            raise ValueError("rotary positions have at most 3 axes")
        if self.layout not in ROPE_LAYOUTS or self.scaling not in ROPE_SCALINGS:
            raise ValueError(f"layout {self.layout!r} of {list(ROPE_LAYOUTS)}, scaling {self.scaling!r} of "
                             f"{list(ROPE_SCALINGS)}")
        return RopeConfigC(self.head_dim, rot, ROPE_LAYOUTS[self.layout], len(sec),
                           (ctypes.c_int32 * 3)(*sec), ROPE_SCALINGS[self.scaling], self.base, self.factor,
                           self.orig_len, self.beta_fast, self.beta_slow)


def rope_freqs(cfg: RopeConfig) -> Tuple[np.ndarray, float]:
    """Radians a position of every rotated pair (float64), and the amplitude."""
    c = cfg.c()
    out = np.zeros(max(c.rot_dim // 2, 1), dtype=np.float64)
    amp = ctypes.c_float(0.0)
    _check(lib().track_rope_freqs(ctypes.byref(c), out.ctypes.data_as(ctypes.POINTER(_f64)), ctypes.byref(amp)))
    return out, float(amp.value)


class Rope:
    """A configuration with its frequencies on the device (made once, used by every call)."""

    def __init__(self, cfg: RopeConfig, device="cuda"):
        freqs, self.amplitude = rope_freqs(cfg)
        self.cfg = cfg
        self.c = cfg.c()
        self.axes = self.c.axes
        self.layouts = {}
        self.check = _rope_layout(self)
        self.freqs = _torch().from_numpy(freqs).to(device)


def _float_dtype(t) -> int:
    d = str(t.dtype)
    if d == "torch.bfloat16":
        return DTYPE_BF16
    if d == "torch.float32":
        return DTYPE_F32
    raise TypeError(f"float32 or bfloat16 tensor expected, got {d}")


def _like(t, other, what):
    if t.dtype != other.dtype or t.get_device() != other.get_device():
        raise TypeError(f"{what}: {t.dtype} on {t.device} beside {other.dtype} on {other.device}")


def _ints(t, shape, ref, what):
    """An int32 tensor of the given shape, contiguous, on ref's device (None passes)."""
    if t is not None and (t.shape != shape or str(t.dtype) != "torch.int32" or not t.is_contiguous() or
                          t.get_device() != ref.get_device()):
        raise ValueError(f"{what}: contiguous int32 {tuple(shape)} on {ref.device} expected")


def _seq_heads(t, what):
    """[sequences, tokens, heads, channels] with heads side by side: (row stride, sequence stride)."""
    shape = t.shape
    if len(shape) != 4:
        raise ValueError(f"{what}: [sequences, tokens, heads, channels] expected, got {tuple(shape)}")
    B, L, H, D = shape
    s0, s1, s2, s3 = t.stride()
    if ((s3 != 1 and D > 1) or (s2 != D and H > 1)) and t.numel():
        raise ValueError(f"{what}: heads of a token must lie side by side")
    ld = s1 if L > 1 else H * D
    return ld, s0 if B > 1 else ld * L


def _on_device(fn, t, *args):
    """fn(*args, stream) on t's device and its current stream (the raw handle: the Stream object around it takes a
    third of a small call's time)."""
    torch = _torch()
    at = t.get_device()
    if at < 0:
        raise ValueError(f"GPU tensors expected, got {t.device}")
    if at == torch.cuda.current_device():
        _check(fn(*args, torch._C._cuda_getCurrentRawStream(at)))
    else:
        with torch.cuda.device(at):
            _check(fn(*args, torch._C._cuda_getCurrentRawStream(at)))


_LAYOUTS_KEPT = 512


def _layout(kept: dict, tensors, check):
    """What `check` makes of the layouts of these tensors (None among them), checked once for each combination of
    shapes, strides, types and devices: for a single token the checks took longer than the kernel."""
    key = tuple([None if t is None else (t.shape, t.stride(), t.dtype, t.get_device()) for t in tensors])
    got = kept.get(key)
    if got is None:
        got = check(*tensors)
        if len(kept) >= _LAYOUTS_KEPT:
            kept.clear()
        kept[key] = got
    return got


def _head_rows(x, y, what):
    """(strides of x, strides of y, heads) as track_head_rows takes them."""
    if y.shape != x.shape:
        raise ValueError(f"{what}: output of shape {tuple(y.shape)} for {tuple(x.shape)}")
    _like(y, x, what)
    return _seq_heads(x, what) + _seq_heads(y, what) + (x.shape[2],)


def _rope_layout(rope):
    def check(q, k, q_out, k_out, pos, g_q, g_k):
        rq, rk = _head_rows(q, q_out, "q"), None
        B, L, _, D = q.shape
        if D != rope.c.head_dim:
            raise ValueError(f"q: heads of {D} channels, {rope.c.head_dim} configured")
        if k is not None:
            rk = _head_rows(k, k_out, "k")
            if k.shape[0] != B or k.shape[1] != L or k.shape[3] != D:
                raise ValueError(f"k of shape {tuple(k.shape)} beside q of {tuple(q.shape)}")
            _like(k, q, "k")
        elif k_out is not None or g_k is not None:
            raise ValueError("k_out or g_k without k")
        if pos is None:
            raise ValueError("pos: positions are needed")
        _ints(pos, (rope.axes, B, L), q, "pos")
        if rope.freqs.get_device() != q.get_device():
            raise ValueError(f"rope on {rope.freqs.device}, q on {q.device}")
        for g, what in ((g_q, "g_q"), (g_k, "g_k")):
            if g is not None:
                if g.shape != q.shape[3:] or not g.is_contiguous():
                    raise ValueError(f"{what}: [{D}] expected")
                _like(g, q, what)
        return _float_dtype(q), B, L, rq, rk
    return check


def _rows_c(layout, x, y) -> HeadRowsC:
    ldx, sx, ldy, sy, heads = layout
    return HeadRowsC(x.data_ptr(), ldx, sx, y.data_ptr(), ldy, sy, heads)


def op_rope(rope: Rope, q, k, pos, q_out=None, k_out=None, inverse: bool = False):
    """Rotates q [B, L, H, D] and k [B, L, Hk, D] (or None) by positions pos (int32 [axes, B, L]), in place or
    into q_out and k_out; returns the outputs.  Strides of tokens and sequences are free."""
    q_out = q if q_out is None else q_out
    k_out = k if k_out is None else k_out
    dtype, B, L, rq, rk = _layout(rope.layouts, (q, k, q_out, k_out, pos, None, None), rope.check)
    _on_device(lib().track_op_rope, q, dtype, rope.c, B, L, _rows_c(rq, q, q_out),
               None if k is None else _rows_c(rk, k, k_out), pos.data_ptr(), rope.freqs.data_ptr(), rope.amplitude,
               1 if inverse else 0)
    return q_out, k_out


def op_headnorm_rope(rope: Rope, q, k, g_q, g_k, pos, q_out=None, k_out=None, eps: float = 1e-6,
                     q_scale: float = 1.0):
    """op_rope behind the RMSNorm of every head, with gains g_q and g_k [D]; q times q_scale."""
    q_out = q if q_out is None else q_out
    k_out = k if k_out is None else k_out
    dtype, B, L, rq, rk = _layout(rope.layouts, (q, k, q_out, k_out, pos, g_q, g_k), rope.check)
    _on_device(lib().track_op_headnorm_rope, q, dtype, rope.c, B, L, _rows_c(rq, q, q_out),
               None if k is None else _rows_c(rk, k, k_out), 0 if g_q is None else g_q.data_ptr(),
               0 if g_k is None else g_k.data_ptr(), eps, q_scale, pos.data_ptr(), rope.freqs.data_ptr(),
               rope.amplitude)
    return q_out, k_out


@dataclasses.dataclass(frozen=True)
class Window:
    """What a query sees (track_window): groups before and after its own (-1: all), and the first tokens."""
    left: int = -1
    right: int = 0
    sink: int = 0
    group: int = 1
    scale: Optional[float] = None  # 1 / sqrt(head_dim)

    def __post_init__(self):
        if self.scale == 0.0:  # the library's mark for 1 / sqrt(head_dim), which is None here
            raise ValueError("window: a scale of 0")
        object.__setattr__(self, "_c", WindowC(self.left, self.right, self.sink, self.group,
                                               0.0 if self.scale is None else self.scale))

    def c(self) -> WindowC:
        return self._c


def attention_window_workspace_bytes(window: Window, dtype: int, B: int, H: int, Hk: int, head_dim: int, Lq: int,
                                     Lk: int) -> int:
    n = lib().track_attention_window_workspace_bytes(dtype, window.c(), B, H, Hk, head_dim, Lq, Lk)
    if n < 0:
        raise TrackError(E_INVALID, lib().track_last_error().decode())
    return n


def attention_window_workspace(window: Window, q, k):
    """The workspace of op_attention_window on tensors of these shapes (None where it needs none); it serves calls of the
    same q on fewer keys too."""
    torch = _torch()
    with torch.cuda.device(q.device):
        n = attention_window_workspace_bytes(window, _float_dtype(q), q.shape[0], q.shape[2], k.shape[2], q.shape[3],
                                             q.shape[1], k.shape[1])
        return torch.empty(n, dtype=torch.uint8, device=q.device) if n else None


_window_layouts: dict = {}


def _check_window(q, k, vt, out, lse, q_len, k_len, q_start, workspace):
    ldq, sq = _seq_heads(q, "q")
    ldk, sk = _seq_heads(k, "k")
    ldo, so = _seq_heads(out, "out")
    B, Lq, H, D = q.shape
    Bk, Lk, Hk, Dk = k.shape
    if out.shape != q.shape or Bk != B or Dk != D:
        raise ValueError(f"q {tuple(q.shape)}, k {tuple(k.shape)}, out {tuple(out.shape)} do not match")
    for t, what in ((k, "k"), (vt, "vt"), (out, "out")):
        _like(t, q, what)
    if vt.dim() != 4 or vt.shape[:3] != (B, Hk, D) or vt.shape[3] < Lk:
        raise ValueError(f"vt: [{B}, {Hk}, {D}, >= {Lk}] expected, got {tuple(vt.shape)}")
    sv, s1, ldv, s3 = vt.stride()
    if ((s3 != 1 and vt.shape[3] > 1) or (s1 != D * ldv and Hk > 1)) and vt.numel():
        raise ValueError("vt: rows of keys, D of them a head, heads one after another")
    if Lk == 0:  # no key is read, whatever strides an empty tensor has
        ldk, sk, ldv, sv = Hk * D, 0, 8, 0
    for t, what in ((q_len, "q_len"), (k_len, "k_len"), (q_start, "q_start")):
        _ints(t, (B,), q, what)
    if lse is not None and (str(lse.dtype) != "torch.float32" or lse.shape != (B, H, Lq) or
                            not lse.is_contiguous() or lse.get_device() != q.get_device()):
        raise ValueError(f"lse: contiguous float32 [{B}, {H}, {Lq}] on {q.device} expected")
    nbytes = 0
    if workspace is not None:
        if workspace.get_device() != q.get_device() or not workspace.is_contiguous():
            raise ValueError(f"workspace: contiguous, on {q.device} expected")
        nbytes = workspace.numel() * workspace.element_size()
    return (_float_dtype(q), B, H, Hk, D, Lq, Lk, ldq, sq, ldk, sk, ldv, sv if B > 1 else 0, ldo, so, nbytes)


def op_attention_window(window: Window, q, k, vt, out, lse=None, q_len=None, k_len=None, q_start=None,
                        workspace=None):
    """Window attention of q [B, Lq, H, D] on k [B, Lk, Hk, D] and vt [B, Hk, D, >= Lk] into out (like q); returns
    out.  k may be a view into a longer cache; a sequence stride of 0 in k and vt shares them.  lse: float32
    [B, H, Lq]; q_len, k_len, q_start: int32 [B].  Layouts are checked once for each combination of shapes and strides:
    a view that grows by a token a call is checked every time, a cache of one length with k_len is not."""
    (dtype, B, H, Hk, D, Lq, Lk, ldq, sq, ldk, sk, ldv, sv, ldo, so, nbytes) = _layout(
        _window_layouts, (q, k, vt, out, lse, q_len, k_len, q_start, workspace), _check_window)
    _on_device(lib().track_op_attention_window, q, dtype, window.c(), B, H, Hk, D, Lq, Lk, q.data_ptr(), ldq, sq,
               k.data_ptr(), ldk, sk, vt.data_ptr(), ldv, sv, out.data_ptr(), ldo, so,
               *[0 if t is None else t.data_ptr() for t in (lse, q_len, k_len, q_start, workspace)], nbytes)
    return out


def step_partial_count(n: int) -> int:
    return lib().track_step_partial_count(n)


def op_step(n: int, B: int, guidance: float, dsigma: float, vel_L, x, vel_S=None, partial=None, eps: float = 1e-8,
            r_out=None):
    _check(lib().track_op_step(n, B, float(guidance), float(dsigma), _ptr(vel_L), _ptr(vel_S), _ptr(x),
                               _ptr(partial), float(eps), _ptr(r_out), _stream()))


def op_step_noalloc(n: int, B: int, guidance: float, dsigma: float, vel_L, x, vel_S=None, eps: float = 1e-8,
                    r_out=None):
    """op_step with the calibration partials in the library's static device scratch (allocates nothing)."""
    _check(lib().track_op_step_noalloc(n, B, float(guidance), float(dsigma), _ptr(vel_L), _ptr(vel_S), _ptr(x),
                                       float(eps), _ptr(r_out), _stream()))


def unipc_coefficients(N: int, shift: float, order: int, step: int) -> np.ndarray:
    """The 12 weights of step `step` of the fused UniPC update (see include/track.h)."""
    out = np.zeros(12, dtype=np.float64)
    _check(lib().track_unipc_coefficients(int(N), float(shift), int(order), int(step),
                                          out.ctypes.data_as(ctypes.POINTER(_f64))))
    return out


def op_unipc_step(n: int, B: int, guidance: float, sigma: float, coef, vel_L, x, x_last, m_out, h0=None, h1=None,
                  h2=None, vel_S=None, partial=None, eps: float = 1e-8, r_out=None):
    coef = np.ascontiguousarray(coef, dtype=np.float64)
    _check(lib().track_op_unipc_step(int(n), int(B), float(guidance), float(sigma),
                                     coef.ctypes.data_as(ctypes.POINTER(_f64)), _ptr(vel_L), _ptr(vel_S), _ptr(x),
                                     _ptr(x_last), _ptr(h0), _ptr(h1), _ptr(h2), _ptr(m_out), _ptr(partial),
                                     float(eps), _ptr(r_out), _stream()))


def band_workspace_bytes(shape: synth.LatentShape, patch=(1, 2, 2)) -> int:
    return int(lib().track_band_workspace_bytes(ctypes.byref(shape_c(shape)), *patch))


def op_band_energy(shape: synth.LatentShape, B: int, guidance: float, vel_L, vel_S, workspace, patch=(1, 2, 2)):
    """Six band energies of the guided difference of two token-layout velocity buffers (synchronous)."""
    out = np.zeros(6, dtype=np.float64)
    nbytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _check(lib().track_op_band_energy(ctypes.byref(shape_c(shape)), *patch, int(B), float(guidance), _ptr(vel_L),
                                      _ptr(vel_S), _ptr(workspace), nbytes, out.ctypes.data_as(ctypes.POINTER(_f64)),
                                      _stream()))
    return out


def set_progress(fn=None):
    """Call fn(sample, step, steps) after each completed step of calibrate/sample (None: off)."""
    global _progress_ref
    if fn is None:
        _check(lib().track_set_progress(PROGRESS_FN(), None))
        _progress_ref = None
        return
    cb = PROGRESS_FN(lambda user, j, k, n: fn(j, k, n))
    _check(lib().track_set_progress(cb, None))
    _progress_ref = cb


HBM_COPY, HBM_READ, HBM_WRITE = 0, 1, 2


def hbm_stream(kind: int, src, dst, nbytes: int):
    """Plain copy / read / write stream over nbytes (the HBM reference kernels)."""
    _check(lib().track_hbm_stream(int(kind), _ptr(src), _ptr(dst), int(nbytes), _stream()))


def mfma_stream(operands, iters: int, sink) -> int:
    """Independent bf16 MFMA chains on every CU from 64 KiB of operands (the
    sustained matrix-core reference); returns the launch's FLOP count."""
    flop = ctypes.c_int64(0)
    _check(lib().track_mfma_stream(_ptr(operands), int(iters), _ptr(sink), ctypes.byref(flop), _stream()))
    return int(flop.value)


# ---------------------------------------------------------------- profiling
def profile_enable(kinds=(PROF_ATTN_SELF, PROF_ATTN_CROSS, PROF_GEMM, PROF_NORM, PROF_STEP, PROF_OTHER)):
    """Bracket launches of the given kernel classes with HIP events (empty: off)."""
    mask = 0
    for k in kinds:
        mask |= 1 << k
    _check(lib().track_profile_enable(mask))


def profile_reset():
    _check(lib().track_profile_reset())


def profile_read(kind: int) -> Tuple[int, float]:
    n = _i64()
    ms = _f64()
    _check(lib().track_profile_read(kind, ctypes.byref(n), ctypes.byref(ms)))
    return n.value, ms.value
