"""ctypes binding of libtlq.so: same names as the C ABI (include/tlq.h), argument marshalling only.

Tensors are torch CUDA tensors used purely as device-memory handles (bf16 tensors may be passed as
torch.bfloat16 or as int16/uint16 bit patterns); the stream is torch's current stream unless given.
Every step of the path runs in the library's kernels.  Importing this module loads the library and
raises if it has not been built: there is no fallback implementation.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import Optional

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libtlq.so")

OK = 0
ERR_INVALID_ARG, ERR_SHAPE, ERR_ALIGN, ERR_UNSUPPORTED = -1, -2, -3, -4
ERR_WORKSPACE, ERR_CUDA, ERR_TIMEOUT, ERR_NONFINITE, ERR_OVERRUN = -5, -6, -7, -8, -9
W4A16_ASYM_GROUP, W8A8_SYM = 0, 1
WA_SYM_CHANNEL = W8A8_SYM     # symmetric per-channel weights / per-token activations, w_bits and a_bits in 2..8
STAT_MEAN_ABS, STAT_MAX_ABS, STAT_MASKED_MAX = 0, 1, 2
NORM_MEAN_ABS, NORM_L2 = 0, 1
DTYPE_BF16, DTYPE_F32 = 0, 1
N_STAGES = 4
STAGE_NAMES = ("stats", "fakequant", "gemm", "reduce")

EXPORTS = (
    "tlq_status_string", "tlq_version", "tlq_token_importance", "tlq_scale_candidates_workspace_bytes",
    "tlq_scale_candidates", "tlq_scale_candidates_noalloc", "tlq_quantize_weights", "tlq_pack_codes4", "tlq_quantize_activations", "tlq_scale_search_workspace_bytes", "tlq_scale_search_layer", "tlq_scale_search_layer_two_stream",
    "tlq_apply_layer_workspace_bytes", "tlq_apply_layer", "tlq_read_status", "tlq_stage_timing_enable",
    "tlq_stage_timing_drain", "tlq_kernel_launch_count", "tlq_selftest_bounded_wait", "tlq_debug_tile_walk", "tlq_debug_resident_walk", "tlq_l2_partition_info", "tlq_debug_canary_offsets",
    "tlq_debug_check_canaries", "tlq_linear_i8_workspace_bytes", "tlq_linear_i8", "tlq_kv_workspace_bytes", "tlq_kv_store",
    "tlq_kv_attention", "tlq_linear_i8_act", "tlq_norm_quantize", "tlq_token_logprobs", "tlq_distill_loss",
)


class TlqError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {status_string(status)} ({status})")


class Config(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("mode", ctypes.c_int32), ("w_bits", ctypes.c_int32),
                ("a_bits", ctypes.c_int32), ("group_size", ctypes.c_int32), ("n_grid", ctypes.c_int32),
                ("stat_mode", ctypes.c_int32), ("flags", ctypes.c_uint32)]


class _KvCacheStruct(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("n_blocks", ctypes.c_int32), ("k_codes", ctypes.c_void_p), ("v_codes", ctypes.c_void_p),
                ("k_steps", ctypes.c_void_p), ("v_steps", ctypes.c_void_p)]


class _KvBatchStruct(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("n_requests", ctypes.c_int32), ("max_q_len", ctypes.c_int32),
                ("max_blocks", ctypes.c_int32), ("cu_q", ctypes.c_void_p), ("kv_len", ctypes.c_void_p),
                ("block_table", ctypes.c_void_p)]


KV_BLOCK = 64                 # tokens of one cache block
ACT_NONE, ACT_SILU, ACT_GELU, ACT_GELU_TANH = 0, 1, 2, 3
MAX_TOP = 128                 # alternatives of a token, or teacher's logits of a row

FLAG_SKIP_ZERO_WEIGHT_TOKENS = 1
FLAG_GEMM_CTA_PAIRS = 2
FLAG_GEMM_NARROW_TILES = 4
FLAG_NO_REFINE = 8
FLAG_DEBUG_CANARIES = 16


def config(mode: int = W4A16_ASYM_GROUP, w_bits: Optional[int] = None, a_bits: Optional[int] = None,
           group_size: int = 128, n_grid: int = 20, stat_mode: int = STAT_MEAN_ABS, flags: int = 0) -> Config:
    if w_bits is None:
        w_bits = 4 if mode == W4A16_ASYM_GROUP else 8
    if a_bits is None:
        a_bits = 16 if mode == W4A16_ASYM_GROUP else 8
    return Config(ctypes.sizeof(Config), mode, w_bits, a_bits, group_size, n_grid, stat_mode, flags)


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2602_07899_b200.build` "
                          "(there is no fallback implementation)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i64, i32, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_size_t
    cfgp = ctypes.POINTER(Config)
    lib.tlq_status_string.restype = ctypes.c_char_p
    lib.tlq_status_string.argtypes = [i32]
    lib.tlq_version.restype = i32
    lib.tlq_kernel_launch_count.restype = i64
    lib.tlq_token_importance.argtypes = [vp, i32, i64, i64, i64, i32, ctypes.c_float, vp, vp, vp]
    lib.tlq_scale_candidates_workspace_bytes.restype = sz
    lib.tlq_scale_candidates_workspace_bytes.argtypes = [i64, i64]
    lib.tlq_scale_candidates.argtypes = [vp, i64, i64, vp, cfgp, vp, sz, vp, vp, vp]
    lib.tlq_scale_candidates_noalloc.argtypes = [vp, i64, i64, vp, cfgp, vp, vp, vp]
    lib.tlq_scale_candidates_noalloc.restype = i32
    lib.tlq_quantize_weights.argtypes = [vp, vp, i64, i64, cfgp, vp, vp, vp, vp, vp]
    lib.tlq_pack_codes4.argtypes = [vp, i64, i64, vp, vp]
    lib.tlq_pack_codes4.restype = i32
    lib.tlq_quantize_activations.argtypes = [vp, vp, i64, i64, cfgp, vp, vp, vp]
    lib.tlq_quantize_activations.restype = i32
    lib.tlq_scale_search_workspace_bytes.restype = sz
    lib.tlq_scale_search_workspace_bytes.argtypes = [i64, i64, i64, cfgp]
    lib.tlq_scale_search_layer.argtypes = [vp, i64, i64, vp, i64, vp, vp, cfgp, vp, sz, vp, vp, vp, vp, vp]
    lib.tlq_scale_search_layer_two_stream.argtypes = [vp, vp, i64, i64, vp, i64, vp, vp, cfgp, vp, sz, vp, vp, vp, vp, vp]
    lib.tlq_scale_search_layer_two_stream.restype = i32
    lib.tlq_apply_layer_workspace_bytes.restype = sz
    lib.tlq_apply_layer_workspace_bytes.argtypes = [i64, i64, i64, cfgp]
    lib.tlq_apply_layer.argtypes = [vp, i64, i64, vp, i64, vp, vp, cfgp, vp, sz, vp, vp, vp, vp, vp]
    lib.tlq_read_status.argtypes = [vp, vp]
    lib.tlq_selftest_bounded_wait.argtypes = [vp, sz, i64, vp]
    lib.tlq_selftest_bounded_wait.restype = i32
    lib.tlq_debug_tile_walk.argtypes = [i64, i64, i32, i32, i32, i32, i32, vp]
    lib.tlq_debug_tile_walk.restype = i32
    lib.tlq_debug_canary_offsets.argtypes = [i32, i64, i64, i64, vp, vp, i32]
    lib.tlq_debug_canary_offsets.restype = i32
    lib.tlq_debug_check_canaries.argtypes = [i32, i64, i64, i64, vp, vp, sz, vp]
    lib.tlq_debug_check_canaries.restype = i32
    lib.tlq_l2_partition_info.argtypes = [vp, vp]
    lib.tlq_l2_partition_info.restype = i32
    lib.tlq_debug_resident_walk.argtypes = [i64, i64, i32, i32, i32, vp]
    lib.tlq_debug_resident_walk.restype = i32
    lib.tlq_stage_timing_enable.argtypes = [i32]
    lib.tlq_stage_timing_drain.argtypes = [ctypes.POINTER(ctypes.c_float), i32]
    kvp, kbp = ctypes.POINTER(_KvCacheStruct), ctypes.POINTER(_KvBatchStruct)
    lib.tlq_linear_i8_workspace_bytes.restype = sz
    lib.tlq_linear_i8_workspace_bytes.argtypes = [i64, i64, i64]
    lib.tlq_linear_i8.restype = i32
    lib.tlq_linear_i8.argtypes = [vp, vp, i64, i64, vp, vp, i64, vp, vp, sz, vp, vp]
    lib.tlq_kv_workspace_bytes.restype = sz
    lib.tlq_kv_workspace_bytes.argtypes = [kvp, kbp, i32, i64]
    lib.tlq_kv_store.restype = i32
    lib.tlq_kv_store.argtypes = [vp, i64, i64, i32, kvp, kbp, vp, i32, ctypes.POINTER(ctypes.c_int32), vp, i64, vp, vp,
                                 ctypes.c_float, vp, vp, vp, vp, sz, vp]
    lib.tlq_kv_attention.restype = i32
    lib.tlq_kv_attention.argtypes = [vp, i64, i64, i32, kvp, kbp, ctypes.c_float, i32, vp, sz, vp, vp, vp]
    f32 = ctypes.c_float
    lib.tlq_linear_i8_act.restype = i32
    lib.tlq_linear_i8_act.argtypes = [vp, vp, i64, i64, vp, vp, i64, vp, i32, i32, vp, i64, vp, sz, vp, vp]
    lib.tlq_norm_quantize.restype = i32
    lib.tlq_norm_quantize.argtypes = [vp, i64, i64, i64, vp, i64, vp, f32, vp, cfgp, vp, i64, vp, vp, vp, vp, vp]
    lib.tlq_token_logprobs.restype = i32
    lib.tlq_token_logprobs.argtypes = [vp, i32, i64, i64, i64, f32, vp, i32, vp, vp, vp, vp, vp, vp]
    lib.tlq_distill_loss.restype = i32
    lib.tlq_distill_loss.argtypes = [vp, i32, i64, i64, i64, f32, vp, vp, i32, vp, vp, vp, i64, vp]
    for fn in ("tlq_token_importance", "tlq_scale_candidates", "tlq_scale_candidates_noalloc", "tlq_quantize_weights", "tlq_pack_codes4", "tlq_quantize_activations", "tlq_scale_search_layer",
               "tlq_apply_layer", "tlq_read_status", "tlq_stage_timing_enable", "tlq_stage_timing_drain"):
        getattr(lib, fn).restype = i32
    return lib


lib = _load()


def status_string(status: int) -> str:
    return lib.tlq_status_string(int(status)).decode()


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("tensor must be contiguous")
    return t.data_ptr()


# the raw handle of the current stream, without a Stream object (a microsecond per call)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _stream(stream, dev: Optional[int] = None) -> Optional[int]:
    """`dev`: number of the current device, where the caller has asked for it."""
    if stream is None:
        if _raw_stream is not None:
            return _raw_stream(_raw_device() if dev is None else dev)
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _check(status: int, what: str) -> None:
    if status != OK:
        raise TlqError(status, what)


def tlq_token_importance(G: torch.Tensor, norm_kind: int = NORM_MEAN_ABS, top_frac: float = 0.0,
                         imp_out: Optional[torch.Tensor] = None, mask_out: Optional[torch.Tensor] = None, stream=None):
    """G [B,N,C] (bf16 / int16 bits / float32) -> (imp float32 [N], mask uint8 [N] or None)."""
    if G.dim() == 2:
        G = G.unsqueeze(0)
    B, N, C = G.shape
    dt = DTYPE_F32 if G.dtype == torch.float32 else DTYPE_BF16
    if imp_out is None:
        imp_out = torch.empty(N, dtype=torch.float32, device=G.device)
    if mask_out is None and top_frac > 0:
        mask_out = torch.empty(N, dtype=torch.uint8, device=G.device)
    _check(lib.tlq_token_importance(_ptr(G), dt, B, N, C, norm_kind, float(top_frac), _ptr(imp_out), _ptr(mask_out),
                                    _stream(stream)), "tlq_token_importance")
    return imp_out, mask_out


def tlq_scale_candidates(X: torch.Tensor, cfg: Config, mask: Optional[torch.Tensor] = None, stream=None):
    """X [N,C1] bf16 -> (x_stat float64 [C1], s bf16 [K,C1])."""
    N, C1 = X.shape
    nbytes = lib.tlq_scale_candidates_workspace_bytes(N, C1)
    ws = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=X.device)
    x_stat = torch.empty(C1, dtype=torch.float64, device=X.device)
    s = torch.empty((cfg.n_grid, C1), dtype=torch.bfloat16, device=X.device)
    _check(lib.tlq_scale_candidates(_ptr(X), N, C1, _ptr(mask), ctypes.byref(cfg), _ptr(ws), nbytes, _ptr(x_stat),
                                    _ptr(s), _stream(stream)), "tlq_scale_candidates")
    return x_stat, s


def tlq_scale_candidates_noalloc(X: torch.Tensor, cfg: Config, x_stat: torch.Tensor, s: torch.Tensor,
                                 mask: Optional[torch.Tensor] = None, stream=None) -> None:
    """Same result as tlq_scale_candidates, written into the caller's x_stat [C1] float64 and s [K,C1] bf16;
    the library uses its built-in scratch array, so nothing is allocated here or in the library."""
    N, C1 = X.shape
    _check(lib.tlq_scale_candidates_noalloc(_ptr(X), N, C1, _ptr(mask), ctypes.byref(cfg), _ptr(x_stat), _ptr(s),
                                            _stream(stream)), "tlq_scale_candidates_noalloc")


def tlq_quantize_weights(W: torch.Tensor, s: Optional[torch.Tensor], cfg: Config, want_dw: bool = False, stream=None):
    """W [C2,C1] bf16, s [C1] bf16 or None -> dict(codes, steps, zeros, dW)."""
    C2, C1 = W.shape
    dev = W.device
    if cfg.mode == W4A16_ASYM_GROUP:
        ng = C1 // cfg.group_size
        codes = torch.empty((C2, C1), dtype=torch.uint8, device=dev)
        steps = torch.empty((C2, ng), dtype=torch.float32, device=dev)
        zeros = torch.empty((C2, ng), dtype=torch.int32, device=dev)
        dW = torch.empty((C2, C1), dtype=torch.bfloat16, device=dev) if want_dw else None
    else:
        codes = torch.empty((C2, C1), dtype=torch.int8, device=dev)
        steps = torch.empty((C2,), dtype=torch.float32, device=dev)
        zeros, dW = None, None
    _check(lib.tlq_quantize_weights(_ptr(W), _ptr(s), C2, C1, ctypes.byref(cfg), _ptr(codes), _ptr(steps), _ptr(zeros),
                                    _ptr(dW), _stream(stream)), "tlq_quantize_weights")
    return dict(codes=codes, steps=steps, zeros=zeros, dW=dW)


def tlq_pack_codes4(codes: torch.Tensor, stream=None) -> torch.Tensor:
    """codes uint8/int8 [R,C] (one 4-bit code per byte) -> uint8 [R,C/2], even channel in the low nibble."""
    R, C = codes.shape
    packed = torch.empty((R, C // 2), dtype=torch.uint8, device=codes.device)
    _check(lib.tlq_pack_codes4(_ptr(codes), R, C, _ptr(packed), _stream(stream)), "tlq_pack_codes4")
    return packed


def tlq_quantize_activations(X: torch.Tensor, s: Optional[torch.Tensor], cfg: Config, stream=None):
    """X [N,C1] bf16, s [C1] bf16 or None -> (codes int8 [N,C1], steps float32 [N]) (W8A8 mode)."""
    N, C1 = X.shape
    codes = torch.empty((N, C1), dtype=torch.int8, device=X.device)
    steps = torch.empty((N,), dtype=torch.float32, device=X.device)
    _check(lib.tlq_quantize_activations(_ptr(X), _ptr(s), N, C1, ctypes.byref(cfg), _ptr(codes), _ptr(steps),
                                        _stream(stream)), "tlq_quantize_activations")
    return codes, steps


def tlq_scale_search_workspace_bytes(N: int, C1: int, C2: int, cfg: Config) -> int:
    return int(lib.tlq_scale_search_workspace_bytes(N, C1, C2, ctypes.byref(cfg)))


class SearchBuffers:
    """Caller-owned device buffers of one tlq_scale_search_layer call (reusable across calls)."""

    def __init__(self, N: int, C1: int, C2: int, cfg: Config, device, per_token: bool = False,
                 workspace: Optional[torch.Tensor] = None):
        self.nbytes = tlq_scale_search_workspace_bytes(N, C1, C2, cfg)
        if self.nbytes == 0:
            raise TlqError(ERR_SHAPE, "tlq_scale_search_workspace_bytes")
        if workspace is None or workspace.numel() < self.nbytes:
            workspace = torch.empty(self.nbytes, dtype=torch.uint8, device=device)
        self.workspace = workspace
        self.best_idx = torch.empty(1, dtype=torch.int32, device=device)
        self.losses = torch.empty(cfg.n_grid, dtype=torch.float64, device=device)
        self.s_best = torch.empty(C1, dtype=torch.bfloat16, device=device)
        self.per_token = torch.empty((cfg.n_grid, N), dtype=torch.float32, device=device) if per_token else None


def tlq_scale_search_layer(X: torch.Tensor, W: torch.Tensor, w_imp: Optional[torch.Tensor], cfg: Config,
                           buffers: Optional[SearchBuffers] = None, mask: Optional[torch.Tensor] = None,
                           per_token: bool = False, stream=None, check: bool = True,
                           X_fp: Optional[torch.Tensor] = None) -> SearchBuffers:
    """Enqueue the search; with check=True also synchronise and raise on a device-side error.
    X_fp selects tlq_scale_search_layer_two_stream (X is then the quantized stream)."""
    N, C1 = X.shape
    C2 = W.shape[0]
    if buffers is None:
        buffers = SearchBuffers(N, C1, C2, cfg, X.device, per_token)
    st = _stream(stream)
    if X_fp is None:
        _check(lib.tlq_scale_search_layer(_ptr(X), N, C1, _ptr(W), C2, _ptr(w_imp), _ptr(mask), ctypes.byref(cfg),
                                          _ptr(buffers.workspace), buffers.nbytes, _ptr(buffers.best_idx),
                                          _ptr(buffers.losses), _ptr(buffers.s_best), _ptr(buffers.per_token), st),
               "tlq_scale_search_layer")
    else:
        if X_fp.shape != X.shape:
            raise ValueError("X_fp must have the shape of X")
        _check(lib.tlq_scale_search_layer_two_stream(_ptr(X), _ptr(X_fp), N, C1, _ptr(W), C2, _ptr(w_imp), _ptr(mask),
                                                     ctypes.byref(cfg), _ptr(buffers.workspace), buffers.nbytes,
                                                     _ptr(buffers.best_idx), _ptr(buffers.losses), _ptr(buffers.s_best),
                                                     _ptr(buffers.per_token), st),
               "tlq_scale_search_layer_two_stream")
    if check:
        _check(lib.tlq_read_status(_ptr(buffers.workspace), st), "tlq_scale_search_layer (device)")
    return buffers


def tlq_apply_layer(X: torch.Tensor, W: torch.Tensor, s: Optional[torch.Tensor], bias: Optional[torch.Tensor],
                    cfg: Config, want_codes: bool = True, stream=None, check: bool = True):
    """-> dict(Yq bf16 [N,C2], codes, steps, zeros)."""
    N, C1 = X.shape
    C2 = W.shape[0]
    dev = X.device
    nbytes = int(lib.tlq_apply_layer_workspace_bytes(N, C1, C2, ctypes.byref(cfg)))
    if nbytes == 0:
        raise TlqError(ERR_SHAPE, "tlq_apply_layer_workspace_bytes")
    ws = torch.empty(nbytes, dtype=torch.uint8, device=dev)
    Yq = torch.empty((N, C2), dtype=torch.bfloat16, device=dev)
    codes = steps = zeros = None
    if want_codes:
        if cfg.mode == W4A16_ASYM_GROUP:
            ng = C1 // cfg.group_size
            codes = torch.empty((C2, C1), dtype=torch.uint8, device=dev)
            steps = torch.empty((C2, ng), dtype=torch.float32, device=dev)
            zeros = torch.empty((C2, ng), dtype=torch.int32, device=dev)
        else:
            codes = torch.empty((C2, C1), dtype=torch.int8, device=dev)
            steps = torch.empty((C2,), dtype=torch.float32, device=dev)
    st = _stream(stream)
    _check(lib.tlq_apply_layer(_ptr(X), N, C1, _ptr(W), C2, _ptr(s), _ptr(bias), ctypes.byref(cfg), _ptr(ws), nbytes,
                               _ptr(codes), _ptr(steps), _ptr(zeros), _ptr(Yq), st), "tlq_apply_layer")
    if check:
        _check(lib.tlq_read_status(_ptr(ws), st), "tlq_apply_layer (device)")
    return dict(Yq=Yq, codes=codes, steps=steps, zeros=zeros)


# ----------------------------------------------------------------------------------------------- serving
# What runs a calibrated layer: see the serving part of include/tlq.h.  These calls never synchronise; read the status
# word of their workspace with tlq_read_status when a step's results are fetched.  With `stream` given, the results belong to that
# stream, as if the call had been made with it current.


_I8, _I32, _F32, _BF16 = torch.int8, torch.int32, torch.float32, torch.bfloat16


def _typed(t: torch.Tensor, dtype: torch.dtype, shape, what: str) -> torch.Tensor:
    if t.dtype is not dtype or t.shape != shape:
        raise ValueError(f"{what} must be {dtype} of shape {tuple(shape)}, got {t.dtype} {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    return t


def _one_device(what: str, first, *rest) -> int:
    """Number of the device that all of them lie on (-1: host memory)."""
    dev = first.get_device()
    for t in rest:
        if t is not None and t.get_device() != dev:
            raise ValueError(f"{what}: all tensors must lie on one device")
    return dev


def _on_device(what: str, first, *rest) -> None:
    """The kernels run on the current device, and a pointer to anywhere else is a memory fault there: refused here.  (The calls ask
    what concerns them themselves first, which takes a microsecond less, and come here when something is wrong.)"""
    dev = _one_device(what, first, *rest)
    if dev < 0 or dev != _raw_device():
        raise ValueError(f"{what}: tensors must lie on the current CUDA device, got {'host memory' if dev < 0 else f'device {dev}'}")


def _rows(t: torch.Tensor, what: str) -> int:
    """Row pitch in elements of a bf16 tensor whose rows are contiguous."""
    if t.dtype is not _BF16:
        raise ValueError(f"{what} must be torch.bfloat16, got {t.dtype}")
    if t.is_contiguous():
        return t.shape[1] if t.ndim == 2 else t.shape[1] * t.shape[2]
    inner = t.shape[-1]
    if t.stride(-1) != 1 or (t.ndim == 3 and t.shape[1] > 1 and t.stride(1) != inner):
        raise ValueError(f"{what}: the heads and channels of a token must be contiguous")
    return t.stride(0) if t.shape[0] > 1 else t.shape[1:].numel()


class KvCache:
    """The 8-bit cache of one layer: k_codes int8 [blocks, kv heads, 64, head_dim] (token by channel), v_codes int8
    [blocks, kv heads, head_dim, 64] (channel by token), k_steps and v_steps float32 [blocks, kv heads]."""

    def __init__(self, k_codes: torch.Tensor, v_codes: torch.Tensor, k_steps: torch.Tensor, v_steps: torch.Tensor):
        blocks, heads, _, dim = k_codes.shape
        _typed(k_codes, torch.int8, (blocks, heads, KV_BLOCK, dim), "k_codes")
        _typed(v_codes, torch.int8, (blocks, heads, dim, KV_BLOCK), "v_codes")
        _typed(k_steps, torch.float32, (blocks, heads), "k_steps")
        _typed(v_steps, torch.float32, (blocks, heads), "v_steps")
        self.k_codes, self.v_codes, self.k_steps, self.v_steps = k_codes, v_codes, k_steps, v_steps
        self.n_blocks, self.n_kv_heads, self.head_dim, self.device = blocks, heads, dim, k_codes.device
        self._device = _one_device("KvCache", k_codes, v_codes, k_steps, v_steps)
        self._c = _KvCacheStruct(ctypes.sizeof(_KvCacheStruct), heads, dim, blocks, k_codes.data_ptr(), v_codes.data_ptr(),
                                 k_steps.data_ptr(), v_steps.data_ptr())
        self._p = ctypes.addressof(self._c)

    def get_device(self) -> int:
        """As of a tensor: the number of its device, -1 in host memory (which the calls refuse)."""
        return self._device

    @classmethod
    def empty(cls, n_blocks: int, n_kv_heads: int, head_dim: int, device) -> "KvCache":
        return cls(torch.zeros((n_blocks, n_kv_heads, KV_BLOCK, head_dim), dtype=torch.int8, device=device),
                   torch.zeros((n_blocks, n_kv_heads, head_dim, KV_BLOCK), dtype=torch.int8, device=device),
                   torch.zeros((n_blocks, n_kv_heads), dtype=torch.float32, device=device),
                   torch.zeros((n_blocks, n_kv_heads), dtype=torch.float32, device=device))


class KvBatch:
    """The requests of one step, on the device: cu_q int32 [n + 1], kv_len int32 [n] (with the step's tokens),
    block_table int32 [n, max_blocks]; max_q_len bounds the new tokens of a request (host)."""

    def __init__(self, cu_q: torch.Tensor, kv_len: torch.Tensor, block_table: torch.Tensor, max_q_len: int):
        n = kv_len.shape[0]
        _typed(cu_q, torch.int32, (n + 1,), "cu_q")
        _typed(kv_len, torch.int32, (n,), "kv_len")
        _typed(block_table, torch.int32, (n, block_table.shape[-1]), "block_table")
        self.cu_q, self.kv_len, self.block_table, self.max_q_len = cu_q, kv_len, block_table, int(max_q_len)
        self._device = _one_device("KvBatch", cu_q, kv_len, block_table)
        self._c = _KvBatchStruct(ctypes.sizeof(_KvBatchStruct), n, self.max_q_len, block_table.shape[1], cu_q.data_ptr(),
                                 kv_len.data_ptr(), block_table.data_ptr())
        self._p = ctypes.addressof(self._c)

    def get_device(self) -> int:
        return self._device


def _by_address(name: str):
    """The call with its structures passed as addresses, which ctypes converts faster than structure objects."""
    typed, fn = getattr(lib, name), lib[name]
    fn.restype = typed.restype
    fn.argtypes = [ctypes.c_void_p if hasattr(t, "_type_") and hasattr(t, "contents") else t for t in typed.argtypes]
    return fn


_kv_store, _kv_attention = _by_address("tlq_kv_store"), _by_address("tlq_kv_attention")


def _made_on(stream, make, *args, **kw) -> torch.Tensor:
    """A tensor of one call, made (and a workspace zeroed) on the stream that the call runs on: memory of another stream's pool may still
    be in use there, and is given away there as soon as it is dropped."""
    if stream is None:
        return make(*args, **kw)
    with torch.cuda.stream(stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(int(stream))):
        return make(*args, **kw)


@functools.lru_cache(maxsize=64)
def _host_ints(values: tuple):
    return (ctypes.c_int32 * len(values))(*values)


def linear_workspace(N: int, C1: int, C2: int, device) -> torch.Tensor:
    """A zeroed workspace for tlq_linear_i8 of up to N tokens (kept by the caller, one per stream)."""
    n = int(lib.tlq_linear_i8_workspace_bytes(N, C1, C2))
    if n == 0:
        raise TlqError(ERR_SHAPE, "tlq_linear_i8_workspace_bytes")
    return torch.zeros(n, dtype=torch.uint8, device=device)


def kv_workspace(cache: KvCache, n_heads: int, T: int, batch: KvBatch) -> torch.Tensor:
    """A zeroed workspace for tlq_kv_store and tlq_kv_attention of up to T tokens (kept by the caller, one per stream)."""
    n = int(lib.tlq_kv_workspace_bytes(cache._c, batch._c, n_heads, T))
    if n == 0:
        raise TlqError(ERR_SHAPE, "tlq_kv_workspace_bytes")
    return torch.zeros(n, dtype=torch.uint8, device=cache.device)


def tlq_linear_i8(Xq: torch.Tensor, t: torch.Tensor, Wq: torch.Tensor, u: torch.Tensor, bias: Optional[torch.Tensor] = None,
                  workspace: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Xq int8 [N,C1] with steps t [N], Wq int8 [C2,C1] with steps u [C2], bias bf16 [C2] or None -> bf16 [N,C2]."""
    N, C1 = Xq.shape
    C2, W1 = Wq.shape
    if (W1 != C1 or Xq.dtype is not _I8 or Wq.dtype is not _I8 or t.dtype is not _F32 or u.dtype is not _F32
            or t.ndim != 1 or u.ndim != 1 or t.numel() != N or u.numel() != C2 or not Xq.is_contiguous() or not Wq.is_contiguous()
            or not t.is_contiguous() or not u.is_contiguous()):
        _typed(Xq, _I8, (N, C1), "Xq")
        _typed(Wq, _I8, (C2, C1), "Wq")
        _typed(t, _F32, (N,), "t")
        _typed(u, _F32, (C2,), "u")
    if bias is not None and (bias.dtype is not _BF16 or bias.shape != (C2,) or not bias.is_contiguous()):
        _typed(bias, _BF16, (C2,), "bias")
    # (a workspace's elements count as bytes: a view that repeats memory has fewer)
    if workspace is not None and not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    dev = Xq.get_device()
    if (dev < 0 or dev != _raw_device() or t.get_device() != dev or Wq.get_device() != dev or u.get_device() != dev
            or bias is not None and bias.get_device() != dev or workspace is not None and workspace.get_device() != dev
            or out is not None and out.get_device() != dev):
        _on_device("tlq_linear_i8", Xq, t, Wq, u, bias, workspace, out)
    if workspace is None:
        workspace = _made_on(stream, linear_workspace, N, C1, C2, Xq.device)
    if out is None:
        out = Xq.new_empty((N, C2), dtype=_BF16) if stream is None else _made_on(stream, Xq.new_empty, (N, C2), dtype=_BF16)
    else:
        _typed(out, _BF16, (N, C2), "out")
    status = lib.tlq_linear_i8(Xq.data_ptr(), t.data_ptr(), N, C1, Wq.data_ptr(), u.data_ptr(), C2,
                               None if bias is None else bias.data_ptr(), workspace.data_ptr(), workspace.numel(),
                               out.data_ptr(), _stream(stream, dev))
    if status:
        raise TlqError(status, "tlq_linear_i8")
    return out


def tlq_kv_store(qkv: torch.Tensor, n_heads: int, cache: KvCache, batch: KvBatch, positions: Optional[torch.Tensor] = None,
                 cos_sin: Optional[torch.Tensor] = None, sections=None, q_norm: Optional[torch.Tensor] = None,
                 k_norm: Optional[torch.Tensor] = None, eps: float = 1e-6, want_values: bool = False,
                 workspace: Optional[torch.Tensor] = None, stream=None):
    """qkv bf16 [T, >= (n_heads + 2 kv heads) * head_dim] (rows may be strided) -> (q bf16 [T, n_heads, head_dim], k values,
    v values): normed (q_norm, k_norm bf16 [head_dim]) and rotated (positions int32 [T], [1,T] or [3,T]; cos_sin float32
    [positions, head_dim]; sections: pairs of each axis) queries; keys and values go into the cache, and come back as the
    values their codes stand for (bf16 [T, kv heads, head_dim]) with want_values."""
    T, d = qkv.shape[0], cache.head_dim
    ld = _rows(qkv, "qkv")
    if qkv.dim() != 2 or qkv.shape[1] < (n_heads + 2 * cache.n_kv_heads) * d:
        raise ValueError("qkv must be [T, (n_heads + 2 * n_kv_heads) * head_dim]")
    axes, sec, limit = 1, None, 0
    if positions is not None:
        axes = 1 if positions.ndim == 1 else positions.shape[0]
        if positions.dtype is not _I32 or positions.ndim > 2 or positions.shape[-1] != T or not positions.is_contiguous():
            _typed(positions, _I32, (T,) if positions.ndim == 1 else (axes, T), "positions")
        if cos_sin is None:
            raise ValueError("positions need cos_sin")
        limit = cos_sin.shape[0]
        if cos_sin.dtype is not _F32 or cos_sin.ndim != 2 or cos_sin.shape[1] != d or not cos_sin.is_contiguous():
            _typed(cos_sin, _F32, (limit, d), "cos_sin")
        if sections is not None:
            if len(sections) != axes:
                raise ValueError("one section for each position axis")
            sec = _host_ints(tuple(sections))
    if q_norm is not None and (q_norm.dtype is not _BF16 or q_norm.shape != (d,) or not q_norm.is_contiguous()):
        _typed(q_norm, _BF16, (d,), "q_norm")
    if k_norm is not None and (k_norm.dtype is not _BF16 or k_norm.shape != (d,) or not k_norm.is_contiguous()):
        _typed(k_norm, _BF16, (d,), "k_norm")
    if workspace is not None and not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    dev = qkv.get_device()
    if (dev < 0 or dev != _raw_device() or cache._device != dev or batch._device != dev
            or positions is not None and (positions.get_device() != dev or cos_sin.get_device() != dev)
            or q_norm is not None and q_norm.get_device() != dev or k_norm is not None and k_norm.get_device() != dev
            or workspace is not None and workspace.get_device() != dev):
        _on_device("tlq_kv_store", qkv, cache, batch, positions, cos_sin, q_norm, k_norm, workspace)
    if workspace is None:
        workspace = _made_on(stream, kv_workspace, cache, n_heads, T, batch)
    empty = qkv.new_empty if stream is None else functools.partial(_made_on, stream, qkv.new_empty)
    q = empty((T, n_heads, d))
    k = v = None
    if want_values:
        k, v = empty((T, cache.n_kv_heads, d)), empty((T, cache.n_kv_heads, d))
    _check(_kv_store(qkv.data_ptr(), T, ld, n_heads, cache._p, batch._p,
                            None if positions is None else positions.data_ptr(), axes, sec,
                            None if cos_sin is None else cos_sin.data_ptr(), limit,
                            None if q_norm is None else q_norm.data_ptr(), None if k_norm is None else k_norm.data_ptr(),
                            eps, q.data_ptr(), None if k is None else k.data_ptr(), None if v is None else v.data_ptr(),
                            workspace.data_ptr(), workspace.numel(), _stream(stream, dev)), "tlq_kv_store")
    return q, k, v


def tlq_kv_attention(q: torch.Tensor, cache: KvCache, batch: KvBatch, scale: float, causal: bool = True,
                     want_lse: bool = False, workspace: Optional[torch.Tensor] = None, stream=None):
    """q bf16 [T, n_heads, head_dim] (rows may be strided) -> (out bf16 [T, n_heads, head_dim], lse float32 [T, n_heads] or
    None): attention of a step's rows over the cached tokens of their requests."""
    T, n_heads, d = q.shape
    if d != cache.head_dim:
        raise ValueError("q and the cache differ in head_dim")
    ldq = _rows(q, "q")
    if workspace is not None and not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    dev = q.get_device()
    if (dev < 0 or dev != _raw_device() or cache._device != dev or batch._device != dev
            or workspace is not None and workspace.get_device() != dev):
        _on_device("tlq_kv_attention", q, cache, batch, workspace)
    if workspace is None:
        workspace = _made_on(stream, kv_workspace, cache, n_heads, T, batch)
    empty = q.new_empty if stream is None else functools.partial(_made_on, stream, q.new_empty)
    out = empty((T, n_heads, d))
    lse = empty((T, n_heads), dtype=_F32) if want_lse else None
    _check(_kv_attention(q.data_ptr(), T, ldq, n_heads, cache._p, batch._p, scale, 1 if causal else 0,
                                workspace.data_ptr(), workspace.numel(), out.data_ptr(),
                                None if lse is None else lse.data_ptr(), _stream(stream, dev)), "tlq_kv_attention")
    return out, lse


def _empty_on(like: torch.Tensor, stream):
    return like.new_empty if stream is None else functools.partial(_made_on, stream, like.new_empty)


def tlq_linear_i8_act(Xq: torch.Tensor, t: torch.Tensor, Wq: torch.Tensor, u: torch.Tensor, bias: Optional[torch.Tensor] = None,
                      act: int = ACT_NONE, gated: bool = False, residual: Optional[torch.Tensor] = None,
                      workspace: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """tlq_linear_i8 with act (ACT_*), gate and residual before the rounding -> bf16 [N, C2], or [N, C2 / 2] with `gated`, where rows
    2j and 2j + 1 of Wq, u and bias make channel j (gated_rows lays them out).  residual bf16 of the result's shape (rows may be
    strided); it may be `out` itself.  Workspace as of tlq_linear_i8."""
    N, C1 = Xq.shape
    C2 = Wq.shape[0]
    width = C2 // 2 if gated else C2
    if (Wq.shape[1] != C1 or Xq.dtype is not _I8 or Wq.dtype is not _I8 or t.dtype is not _F32 or u.dtype is not _F32
            or t.ndim != 1 or u.ndim != 1 or t.numel() != N or u.numel() != C2 or not Xq.is_contiguous() or not Wq.is_contiguous()
            or not t.is_contiguous() or not u.is_contiguous()):
        _typed(Xq, _I8, (N, C1), "Xq")
        _typed(Wq, _I8, (C2, C1), "Wq")
        _typed(t, _F32, (N,), "t")
        _typed(u, _F32, (C2,), "u")
    if bias is not None and (bias.dtype is not _BF16 or bias.shape != (C2,) or not bias.is_contiguous()):
        _typed(bias, _BF16, (C2,), "bias")
    ldr = 0
    if residual is not None:
        if residual.shape != (N, width):
            raise ValueError(f"residual must have the result's shape {(N, width)}, got {tuple(residual.shape)}")
        ldr = _rows(residual, "residual")
    if workspace is not None and not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    dev = Xq.get_device()
    if (dev < 0 or dev != _raw_device() or t.get_device() != dev or Wq.get_device() != dev or u.get_device() != dev
            or bias is not None and bias.get_device() != dev or residual is not None and residual.get_device() != dev
            or workspace is not None and workspace.get_device() != dev or out is not None and out.get_device() != dev):
        _on_device("tlq_linear_i8_act", Xq, t, Wq, u, bias, residual, workspace, out)
    if workspace is None:
        workspace = _made_on(stream, linear_workspace, N, C1, C2, Xq.device)
    if out is None:
        out = _empty_on(Xq, stream)(N, width, dtype=_BF16)
    else:
        _typed(out, _BF16, (N, width), "out")
    status = lib.tlq_linear_i8_act(Xq.data_ptr(), t.data_ptr(), N, C1, Wq.data_ptr(), u.data_ptr(), C2,
                                   None if bias is None else bias.data_ptr(), act, 1 if gated else 0,
                                   None if residual is None else residual.data_ptr(), ldr, workspace.data_ptr(), workspace.numel(),
                                   out.data_ptr(), _stream(stream, dev))
    if status:
        raise TlqError(status, "tlq_linear_i8_act")
    return out


def gated_rows(gate: torch.Tensor, up: torch.Tensor) -> torch.Tensor:
    """Rows of a gate and an up projection (codes, steps or biases) in the order that tlq_linear_i8_act takes: 2j gate, 2j + 1 up."""
    if gate.shape != up.shape or gate.dtype is not up.dtype:
        raise ValueError("gate and up must have one shape and type")
    return torch.stack((gate, up), 1).flatten(0, 1)


def tlq_norm_quantize(x: torch.Tensor, w: Optional[torch.Tensor], cfg: Optional[Config] = None, residual: Optional[torch.Tensor] = None,
                      s: Optional[torch.Tensor] = None, eps: float = 1e-6, want_codes: bool = True, want_values: bool = False,
                      want_y: bool = False, h: Optional[torch.Tensor] = None, stream=None):
    """x bf16 [N,C], residual bf16 [N,C] or None (rows of both may be strided), w bf16 [C] or None, s bf16 [C] or None ->
    dict(h, codes, steps, values, y): the sum x + residual (x itself without one), int8 codes [N,C] with steps [N] of its norm times
    w / s, with want_values the values they stand for (bf16), with want_y the norm times w (bf16).  `h`: where the sum goes (x and
    residual are allowed).  cfg: symmetric mode, 8 bits by default."""
    shape = x.shape
    N, C = shape
    ldx = C if x.dtype is _BF16 and x.is_contiguous() else _rows(x, "x")
    ldr = ldh = 0
    dev = x.get_device()
    here = dev >= 0 and dev == _raw_device()
    if residual is not None:
        if residual.shape != shape:
            raise ValueError("x and residual must have one shape")
        ldr = C if residual.dtype is _BF16 and residual.is_contiguous() else _rows(residual, "residual")
        here = here and residual.get_device() == dev
    if w is not None:
        if w.dtype is not _BF16 or w.ndim != 1 or w.numel() != C or not w.is_contiguous():
            _typed(w, _BF16, (C,), "w")
        here = here and w.get_device() == dev
    if s is not None:
        if s.dtype is not _BF16 or s.ndim != 1 or s.numel() != C or not s.is_contiguous():
            _typed(s, _BF16, (C,), "s")
        here = here and s.get_device() == dev
    if not want_codes and (want_values or s is not None):
        raise ValueError("values and s belong to codes")
    if not here or h is not None and h.get_device() != dev:
        _on_device("tlq_norm_quantize", x, residual, w, s, h)
    # (a tensor like another one is made in two thirds of the time of one of given sizes)
    like, empty = (torch.empty_like, x.new_empty) if stream is None else (functools.partial(_made_on, stream, torch.empty_like),
                                                                          functools.partial(_made_on, stream, x.new_empty))
    if h is not None:
        if h.shape != shape:
            raise ValueError("h must have the shape of x")
        ldh = _rows(h, "h")
    elif residual is not None:
        h, ldh = like(x), C
    codes = steps = values = y = None
    if want_codes:
        codes, steps = like(x, dtype=_I8), empty(N, dtype=_F32)
        if cfg is None:
            cfg = _default_cfg()
        if want_values:
            values = like(x)
    if want_y:
        y = like(x)
    status = _norm_quantize(x.data_ptr(), N, C, ldx, None if residual is None else residual.data_ptr(), ldr,
                            None if w is None else w.data_ptr(), eps, None if s is None else s.data_ptr(),
                            None if cfg is None else ctypes.addressof(cfg), None if h is None else h.data_ptr(), ldh,
                            None if codes is None else codes.data_ptr(), None if steps is None else steps.data_ptr(),
                            None if values is None else values.data_ptr(), None if y is None else y.data_ptr(), _stream(stream, dev))
    if status:
        raise TlqError(status, "tlq_norm_quantize")
    return dict(h=x if h is None else h, codes=codes, steps=steps, values=values, y=y)


@functools.lru_cache(maxsize=1)
def _default_cfg() -> Config:
    return config(W8A8_SYM)


_norm_quantize = _by_address("tlq_norm_quantize")


# ----------------------------------------------------------------------------------------------- scoring
# A model by its logits: see the scoring part of include/tlq.h.

def _logits(t: torch.Tensor, what: str):
    """Type number and row pitch of logits [N,V]."""
    if t.dtype is not _BF16 and t.dtype is not _F32:
        raise ValueError(f"{what} must be torch.bfloat16 or torch.float32, got {t.dtype}")
    if t.ndim == 2 and t.is_contiguous():
        return (DTYPE_F32 if t.dtype is _F32 else DTYPE_BF16), t.shape[1]
    if t.ndim != 2 or t.shape[1] > 1 and t.stride(1) != 1:
        raise ValueError(f"{what} must be [N,V] with the logits of a row one after another")
    return (DTYPE_F32 if t.dtype is _F32 else DTYPE_BF16), (t.stride(0) if t.shape[0] > 1 else t.shape[1])


def tlq_token_logprobs(logits: torch.Tensor, ids: Optional[torch.Tensor] = None, top_k: int = 0, scale: float = 1.0,
                       want_entropy: bool = False, want_lse: bool = False, stream=None):
    """logits bf16 or float32 [N,V] (rows may be strided), ids int32 [N] or None (negative: no token) -> dict(logp, entropy, lse: float32 [N],
    top_ids int32 [N,K], top_logp float32 [N,K]), None where not asked for: log probabilities of the given tokens under
    softmax(scale * logits), its entropy and normaliser, and the top_k largest logits, largest first."""
    kind, ld = _logits(logits, "logits")
    N, V = logits.shape
    dev = logits.get_device()
    if ids is not None and (ids.dtype is not _I32 or ids.ndim != 1 or ids.numel() != N or not ids.is_contiguous()):
        _typed(ids, _I32, (N,), "ids")
    if not 0 <= top_k <= MAX_TOP:
        raise ValueError(f"top_k must be 0 to {MAX_TOP}")
    if dev < 0 or dev != _raw_device() or ids is not None and ids.get_device() != dev:
        _on_device("tlq_token_logprobs", logits, ids)
    like, empty = (torch.empty_like, logits.new_empty) if stream is None else (functools.partial(_made_on, stream, torch.empty_like),
                                                                               functools.partial(_made_on, stream, logits.new_empty))
    logp = entropy = lse = top_ids = top_logp = None
    if ids is not None:
        logp = like(ids, dtype=_F32)
    if want_entropy:
        entropy = empty(N, dtype=_F32) if logp is None else like(logp)
    if want_lse:
        one = entropy if logp is None else logp
        lse = empty(N, dtype=_F32) if one is None else like(one)
    if top_k:
        top_ids = empty(N, top_k, dtype=_I32)
        top_logp = like(top_ids, dtype=_F32)
    status = lib.tlq_token_logprobs(logits.data_ptr(), kind, N, V, ld, scale, None if ids is None else ids.data_ptr(), top_k,
                                    None if logp is None else logp.data_ptr(), None if entropy is None else entropy.data_ptr(),
                                    None if lse is None else lse.data_ptr(), None if top_ids is None else top_ids.data_ptr(),
                                    None if top_logp is None else top_logp.data_ptr(), _stream(stream, dev))
    if status:
        raise TlqError(status, "tlq_token_logprobs")
    return dict(logp=logp, entropy=entropy, lse=lse, top_ids=top_ids, top_logp=top_logp)


def tlq_distill_loss(logits: torch.Tensor, top_ids: torch.Tensor, top_logits: torch.Tensor, weights: Optional[torch.Tensor] = None,
                     scale: float = 1.0, want_grad: bool = True, grad: Optional[torch.Tensor] = None, stream=None):
    """logits bf16 or float32 [N,V] (rows may be strided), a teacher's top_ids int32 [N,K] (negative: empty place) and top_logits float32
    [N,K], weights float32 [N] or None -> (loss float32 [N], grad of the logits' type [N,V] or None): weights times the divergence of
    softmax(scale * logits) from the teacher's softmax(scale * top_logits) over its K places, and the gradient of that by the logits.
    top_logits may be tlq_token_logprobs' top_logp of scale 1 (of another scale they have it in them already: a temperature belongs
    here alone).  `grad`: where it goes (the logits themselves are allowed)."""
    kind, ld = _logits(logits, "logits")
    N, V = logits.shape
    K = top_ids.shape[-1]
    if top_ids.dtype is not _I32 or top_ids.shape != (N, K) or not top_ids.is_contiguous():
        _typed(top_ids, _I32, (N, K), "top_ids")
    if top_logits.dtype is not _F32 or top_logits.shape != (N, K) or not top_logits.is_contiguous():
        _typed(top_logits, _F32, (N, K), "top_logits")
    if weights is not None and (weights.dtype is not _F32 or weights.shape != (N,) or not weights.is_contiguous()):
        _typed(weights, _F32, (N,), "weights")
    dev = logits.get_device()
    if (dev < 0 or dev != _raw_device() or top_ids.get_device() != dev or top_logits.get_device() != dev
            or weights is not None and weights.get_device() != dev or grad is not None and grad.get_device() != dev):
        _on_device("tlq_distill_loss", logits, top_ids, top_logits, weights, grad)
    empty = _empty_on(logits, stream)
    ldg = V
    if grad is not None:
        if grad.dtype is not logits.dtype or grad.shape != logits.shape:
            raise ValueError("grad must have the type and shape of the logits")
        ldg = _logits(grad, "grad")[1]
    elif want_grad:
        grad = empty(N, V)
    loss = empty(N, dtype=_F32)
    status = lib.tlq_distill_loss(logits.data_ptr(), kind, N, V, ld, scale, top_ids.data_ptr(), top_logits.data_ptr(), K,
                                  None if weights is None else weights.data_ptr(), loss.data_ptr(), None if grad is None else grad.data_ptr(),
                                  ldg, _stream(stream, dev))
    if status:
        raise TlqError(status, "tlq_distill_loss")
    return loss, grad


def tlq_read_status(workspace: torch.Tensor, stream=None) -> int:
    return int(lib.tlq_read_status(_ptr(workspace), _stream(stream)))


def tlq_selftest_bounded_wait(workspace: torch.Tensor, limit_cycles: int = 2_000_000, stream=None) -> int:
    """Run the bounded-wait self-test on `workspace` and return the device status it left (TLQ_ERR_TIMEOUT when
    the error path works).  Synchronises the stream."""
    st = _stream(stream)
    _check(lib.tlq_selftest_bounded_wait(_ptr(workspace), workspace.numel() * workspace.element_size(), int(limit_cycles), st),
           "tlq_selftest_bounded_wait")
    return int(lib.tlq_read_status(_ptr(workspace), st))


def tlq_debug_canary_offsets(kind: int, N: int, C1: int, C2: int, cfg: Config):
    """-> list of byte offsets of the guard words of a workspace laid out with FLAG_DEBUG_CANARIES (host only)."""
    buf = (ctypes.c_uint64 * 32)()
    n = int(lib.tlq_debug_canary_offsets(kind, N, C1, C2, ctypes.byref(cfg), buf, 32))
    _check(min(n, 0), "tlq_debug_canary_offsets")
    return [int(buf[i]) for i in range(n)]


def tlq_debug_check_canaries(kind: int, N: int, C1: int, C2: int, cfg: Config, workspace: torch.Tensor,
                             stream=None) -> None:
    """Enqueue one more comparison of the guard words; read the outcome with tlq_read_status."""
    _check(lib.tlq_debug_check_canaries(kind, N, C1, C2, ctypes.byref(cfg), _ptr(workspace), workspace.numel(),
                                        _stream(stream)), "tlq_debug_check_canaries")


def tlq_l2_partition_info():
    """-> dict(valid, n_sms, count=(n0, n1), part=numpy uint8 [256]): the current device's SM -> L2 partition table."""
    import numpy as np
    info = (ctypes.c_int32 * 4)()
    part = np.zeros(256, dtype=np.uint8)
    _check(lib.tlq_l2_partition_info(info, part.ctypes.data_as(ctypes.c_void_p)), "tlq_l2_partition_info")
    return dict(valid=bool(info[0]), n_sms=int(info[1]), count=(int(info[2]), int(info[3])), part=part)


def tlq_debug_tile_walk(mtiles: int, otiles: int, K: int, n0: int, n1: int = 0, blocked: bool = False, block_a: int = 8):
    """Host-side replay of the fused GEMM's tile walk -> numpy int32 [K, otiles, mtiles] of visit counts."""
    import numpy as np
    visits = np.zeros((K, otiles, mtiles), dtype=np.int32)
    _check(lib.tlq_debug_tile_walk(mtiles, otiles, K, n0, n1, 1 if blocked else 0, block_a,
                                   visits.ctypes.data_as(ctypes.c_void_p)), "tlq_debug_tile_walk")
    return visits


def tlq_debug_resident_walk(mtiles: int, otiles: int, K: int, grid: int, blocked: bool = True):
    """Host-side replay of the tile-resident kernels' work items -> numpy int32 [K, otiles, mtiles] of visit counts."""
    import numpy as np
    visits = np.zeros((K, otiles, mtiles), dtype=np.int32)
    _check(lib.tlq_debug_resident_walk(mtiles, otiles, K, grid, 1 if blocked else 0,
                                       visits.ctypes.data_as(ctypes.c_void_p)), "tlq_debug_resident_walk")
    return visits


def tlq_stage_timing_enable(on: bool) -> None:
    _check(lib.tlq_stage_timing_enable(1 if on else 0), "tlq_stage_timing_enable")


def tlq_stage_timing_drain(max_calls: int = 512):
    """-> list of per-call [stats, fakequant, gemm, reduce] milliseconds, oldest call first."""
    arr = (ctypes.c_float * (N_STAGES * max_calls))()
    n = lib.tlq_stage_timing_drain(arr, max_calls)
    if n < 0:
        raise TlqError(n, "tlq_stage_timing_drain")
    return [[float(arr[c * N_STAGES + i]) for i in range(N_STAGES)] for c in range(n)]


def tlq_kernel_launch_count() -> int:
    return int(lib.tlq_kernel_launch_count())


def bf16_from_bits(bits, device="cuda") -> torch.Tensor:
    """numpy uint16 bit patterns -> torch.bfloat16 device tensor (no arithmetic)."""
    import numpy as np
    t = torch.from_numpy(np.ascontiguousarray(bits).view(np.int16))
    return t.to(device).view(torch.bfloat16)
