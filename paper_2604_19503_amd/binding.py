"""ctypes binding of include/realb.h: argument marshalling only."""
from __future__ import annotations

import ctypes as C
import os

import numpy as np
import torch

BF16, FP4, FORCE_NONE = 0, 1, -1
_PKG = os.path.dirname(os.path.abspath(__file__))
_LIB = None

EXPORTS = [
    "realb_default_config", "realb_create", "realb_destroy", "realb_last_error", "realb_get_M", "realb_set_M",
    "realb_route_stats", "realb_select_precision", "realb_select_precision_host", "realb_quantize_experts_fp4",
    "realb_quantize_rows_fp4", "realb_permute", "realb_grouped_moe_ffn", "realb_grouped_moe_ffn_gate_up",
    "realb_grouped_moe_ffn_down", "realb_set_gemm_tile", "realb_set_gemm_tile_shape", "realb_combine", "realb_layer_forward", "realb_rank_forward",
    "realb_quantize_rows_nvfp4", "realb_amax_bf16", "realb_route_stats_static",
    "realb_workspace_bytes", "realb_scale_offset", "realb_scale_index_map", "realb_prefetch_join", "realb_stage_timing", "realb_stage_ms",
    "realb_quantize_rows_fp8", "realb_quantize_blocks_fp8", "realb_residual_norm", "realb_linear_fp8", "realb_gated_ffn_fp8",
    "realb_gated_ffn_workspace_bytes",
]


class RealbError(RuntimeError):
    pass


class Config(C.Structure):
    _fields_ = [("T_max", C.c_int), ("E", C.c_int), ("k", C.c_int), ("D", C.c_int), ("H", C.c_int), ("I", C.c_int),
                ("C", C.c_double), ("tau", C.c_double), ("M_init", C.c_double), ("aimd_mul", C.c_double),
                ("aimd_add", C.c_double), ("Gamma", C.c_longlong), ("aimd_enabled", C.c_int), ("update_first", C.c_int)]


class LayerIO(C.Structure):
    _fields_ = [("logits", C.c_void_p), ("is_vision", C.c_void_p), ("x", C.c_void_p), ("T", C.c_int),
                ("w13", C.c_void_p), ("w2", C.c_void_p), ("rank", C.c_int), ("force", C.c_int), ("overlap", C.c_int),
                ("max_rows", C.c_longlong),
                ("next_w13", C.c_void_p), ("next_w2", C.c_void_p), ("next_w13_q", C.c_void_p), ("next_w13_s", C.c_void_p),
                ("next_w2_q", C.c_void_p), ("next_w2_s", C.c_void_p), ("reserve_cus", C.c_int),
                ("topk_ids", C.c_void_p), ("topk_w", C.c_void_p), ("expert_cnt", C.c_void_p), ("expert_vis", C.c_void_p),
                ("rank_load", C.c_void_p), ("rank_vis", C.c_void_p),
                ("expert_offsets", C.c_void_p), ("row_to_assign", C.c_void_p), ("assign_to_row", C.c_void_p),
                ("x_perm", C.c_void_p), ("x_q", C.c_void_p), ("x_s", C.c_void_p),
                ("w13_q", C.c_void_p), ("w13_s", C.c_void_p), ("w2_q", C.c_void_p), ("w2_s", C.c_void_p),
                ("h_mid", C.c_void_p), ("h_s", C.c_void_p), ("y_rows", C.c_void_p), ("out", C.c_void_p),
                ("prec_host", C.c_int32 * 64), ("ib_global", C.c_double), ("M_after", C.c_double)]


class NormIO(C.Structure):
    _fields_ = [("T", C.c_int), ("H", C.c_int), ("eps", C.c_float), ("scale", C.c_float), ("res_type", C.c_int),
                ("res", C.c_void_p), ("ld_res", C.c_longlong), ("y", C.c_void_p), ("ld_y", C.c_longlong), ("post_w", C.c_void_p),
                ("gate", C.c_void_p), ("ld_gate", C.c_longlong), ("gate_step", C.c_int),
                ("res_out", C.c_void_p), ("ld_res_out", C.c_longlong), ("pre_w", C.c_void_p), ("out", C.c_void_p), ("ld_out", C.c_longlong),
                ("out_q", C.c_void_p), ("ld_q", C.c_longlong), ("out_s", C.c_void_p), ("ld_s", C.c_longlong)]
    _gpu = None                                          # the tensors' GPU


class LinearIO(C.Structure):
    _fields_ = [("M", C.c_int), ("N", C.c_int), ("K", C.c_int),
                ("x_q", C.c_void_p), ("ld_x", C.c_longlong), ("x_s", C.c_void_p), ("ld_xs", C.c_longlong),
                ("w_q", C.c_void_p), ("w_s", C.c_void_p), ("bias", C.c_void_p), ("add", C.c_void_p), ("ld_add", C.c_longlong),
                ("out_type", C.c_int), ("out", C.c_void_p), ("ld_out", C.c_longlong)]
    _gpu = None


class FfnIO(C.Structure):
    _fields_ = [("T", C.c_int), ("H", C.c_int), ("I", C.c_int), ("sums", C.c_int),
                ("x_q", C.c_void_p), ("ld_x", C.c_longlong), ("x_s", C.c_void_p), ("ld_xs", C.c_longlong),
                ("w13_q", C.c_void_p), ("w13_s", C.c_void_p), ("w2_q", C.c_void_p), ("w2_s", C.c_void_p),
                ("add", C.c_void_p), ("ld_add", C.c_longlong), ("out", C.c_void_p), ("ld_out", C.c_longlong),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t)]
    _gpu = None
    _workspaces = _workspace_of = None                   # stream -> workspace allocated there (None: the caller's), the stream of the present one


def library_path() -> str:
    return os.path.join(_PKG, "librealb.so")


def load_library() -> C.CDLL:
    """Loads librealb.so from the package directory; raises if it is not built."""
    global _LIB
    if _LIB is not None:
        return _LIB
    path = library_path()
    if not os.path.exists(path):
        raise RealbError(f"{path} is missing: run `python -m paper_2604_19503_amd.build` (or __graft_entry__.build()) first")
    lib = C.CDLL(path)
    for name in EXPORTS:
        if not hasattr(lib, name):
            raise RealbError(f"{path} does not export {name}")
    lib.realb_last_error.restype = C.c_char_p
    lib.realb_get_M.restype = C.c_double
    lib.realb_get_M.argtypes = [C.c_void_p]
    lib.realb_set_M.argtypes = [C.c_void_p, C.c_double]
    lib.realb_default_config.restype = None
    lib.realb_default_config.argtypes = [C.POINTER(Config)] + [C.c_int] * 6
    lib.realb_workspace_bytes.restype = C.c_size_t
    lib.realb_workspace_bytes.argtypes = [C.POINTER(Config)]
    lib.realb_scale_offset.restype = C.c_size_t
    lib.realb_scale_offset.argtypes = [C.c_longlong, C.c_int, C.c_int]
    lib.realb_scale_index_map.argtypes = [C.c_longlong, C.c_int, C.c_void_p]
    lib.realb_create.argtypes = [C.POINTER(Config), C.POINTER(C.c_void_p)]
    lib.realb_destroy.argtypes = [C.c_void_p]
    lib.realb_set_gemm_tile_shape.argtypes = [C.c_void_p, C.c_int]
    vp = C.c_void_p
    lib.realb_route_stats.argtypes = [vp, vp, vp, C.c_int, vp, vp, vp, vp, vp, vp, vp]
    lib.realb_route_stats_static.argtypes = [vp, vp, C.c_int, C.c_int, C.c_int, C.c_int, vp, vp, vp, vp, vp, vp, vp]
    lib.realb_select_precision.argtypes = [vp, vp, vp, C.c_int, C.c_int, vp, vp, vp, vp]
    lib.realb_select_precision_host.argtypes = [C.POINTER(Config), vp, vp, C.c_int, C.c_int, vp, vp, vp]
    lib.realb_quantize_experts_fp4.argtypes = [vp, vp, vp, C.c_int, vp, vp, vp, vp, vp]
    lib.realb_quantize_rows_fp4.argtypes = [vp, C.c_longlong, C.c_int, vp, vp, vp]
    lib.realb_permute.argtypes = [vp, vp, vp, C.c_int, C.c_int, C.c_int, C.c_longlong, vp, vp, vp, vp, vp, vp, vp]
    lib.realb_grouped_moe_ffn.argtypes = [vp, C.c_int, vp, C.c_int, C.c_longlong, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.realb_grouped_moe_ffn_gate_up.argtypes = [vp, C.c_int, vp, C.c_int, C.c_longlong, vp, vp, vp, vp, vp, vp, vp]
    lib.realb_grouped_moe_ffn_down.argtypes = [vp, C.c_int, vp, C.c_int, C.c_longlong, vp, vp, vp, vp, vp, vp]
    lib.realb_combine.argtypes = [vp, vp, vp, vp, C.c_int, vp, vp]
    lib.realb_layer_forward.argtypes = [vp, C.POINTER(LayerIO), vp]
    lib.realb_rank_forward.argtypes = [vp, C.POINTER(LayerIO), C.c_int, vp]
    lib.realb_prefetch_join.argtypes = [vp, vp]
    lib.realb_stage_timing.argtypes = [vp, C.c_int]
    lib.realb_stage_ms.argtypes = [vp, vp]
    lib.realb_quantize_rows_nvfp4.argtypes = [vp, C.c_longlong, C.c_int, C.c_float, vp, vp, vp]
    lib.realb_amax_bf16.argtypes = [vp, C.c_longlong, vp, vp]
    ll = C.c_longlong
    lib.realb_quantize_rows_fp8.argtypes = [vp, ll, ll, C.c_int, vp, ll, vp, ll, vp]
    lib.realb_quantize_blocks_fp8.argtypes = [vp, C.c_int, C.c_int, C.c_int, vp, vp, vp]
    lib.realb_residual_norm.argtypes = [C.POINTER(NormIO), vp]
    lib.realb_linear_fp8.argtypes = [C.POINTER(LinearIO), vp]
    lib.realb_gated_ffn_fp8.argtypes = [C.POINTER(FfnIO), vp]
    lib.realb_gated_ffn_workspace_bytes.argtypes = [C.c_int, C.c_int]
    lib.realb_gated_ffn_workspace_bytes.restype = C.c_size_t
    _LIB = lib
    return lib


def _check(rc: int):
    if rc != 0:
        raise RealbError(f"realb error {rc}: {load_library().realb_last_error().decode()}")


def _p(t):
    if t is None:
        return None
    if isinstance(t, torch.Tensor):
        assert t.is_contiguous()
        return C.c_void_p(t.data_ptr())
    return t


def _stream(stream=None):
    s = torch.cuda.current_stream() if stream is None else stream
    return C.c_void_p(s.cuda_stream)


def _on(stream):
    """What a call allocates comes from the pool of the stream that it runs on: memory of another stream's pool may still be in use there, and
    would go back there while this call runs."""
    return torch.cuda.stream(stream)


def bf16_from_bits(bits: np.ndarray, device="cuda") -> torch.Tensor:
    """numpy uint16 bf16 patterns -> torch.bfloat16 tensor on the device."""
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).to(device).view(torch.bfloat16)


def scale_index_map(rows: int, K: int) -> np.ndarray:
    """realb_scale_index_map: int64 [rows, K/32] byte offsets into a K-step-tiled scale tensor."""
    idx = np.empty((rows, K // 32), dtype=np.int64)
    _check(load_library().realb_scale_index_map(rows, K, idx.ctypes.data))
    return idx


def workspace_bytes(cfg: Config) -> int:
    return int(load_library().realb_workspace_bytes(C.byref(cfg)))


def scales_to_canonical(s, rows: int, K: int) -> np.ndarray:
    """Pure index permutation (no arithmetic): a K-step-tiled scale tensor, as the library reads
    and writes it, rearranged to the plain [rows, K/32] order through the library's own index map."""
    flat = (s.detach().cpu().numpy() if isinstance(s, torch.Tensor) else np.asarray(s)).reshape(-1)
    return flat[scale_index_map(rows, K)]


def bits_from_bf16(t: torch.Tensor) -> np.ndarray:
    return t.detach().contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


def set_gemm_tile(wn: int):
    _check(load_library().realb_set_gemm_tile(int(wn)))


def default_config(T_max, E, k, D, H, I) -> Config:
    cfg = Config()
    load_library().realb_default_config(C.byref(cfg), T_max, E, k, D, H, I)
    return cfg


def select_precision_host(cfg: Config, rank_load, rank_vis, T: int, M: float, force: int = FORCE_NONE):
    """realb_select_precision_host: returns (prec[D], ib_global, M_after).  No GPU."""
    load = np.ascontiguousarray(rank_load, dtype=np.int32)
    vis = np.ascontiguousarray(rank_vis, dtype=np.int32)
    prec = np.zeros(cfg.D, dtype=np.int32)
    Mio, ib = C.c_double(M), C.c_double(0)
    _check(load_library().realb_select_precision_host(C.byref(cfg), load.ctypes.data, vis.ctypes.data, T, force,
                                                      C.addressof(Mio), prec.ctypes.data, C.addressof(ib)))
    return prec, ib.value, Mio.value


def quantize_rows_fp4(x: torch.Tensor, stream=None):
    """realb_quantize_rows_fp4 on a bf16 [rows,K] tensor -> (q u8 [rows,K/2], s u8 K-step-tiled,
    ceil(rows/32)*32 * K/32 bytes; see scales_to_canonical)."""
    rows, K = x.shape
    with _on(stream):
        q = torch.empty((rows, K // 2), dtype=torch.uint8, device=x.device)
        s = torch.zeros((-(-rows // 32) * 32, K // 32), dtype=torch.uint8, device=x.device)
    _check(load_library().realb_quantize_rows_fp4(_p(x), rows, K, _p(q), _p(s), _stream(stream)))
    return q, s


def amax_bf16(x: torch.Tensor, stream=None) -> torch.Tensor:
    """realb_amax_bf16: max |x| of a bf16 tensor (element count a multiple of 8) as a 1-element float tensor."""
    with _on(stream):
        out = torch.empty(1, dtype=torch.float32, device=x.device)
    _check(load_library().realb_amax_bf16(_p(x), x.numel(), _p(out), _stream(stream)))
    return out


def quantize_rows_nvfp4(x: torch.Tensor, global_scale: float, stream=None):
    """realb_quantize_rows_nvfp4 on a bf16 [rows,K] tensor -> (q u8 [rows,K/2], s u8 [rows,K/16] E4M3 bytes)."""
    rows, K = x.shape
    with _on(stream):
        q = torch.empty((rows, K // 2), dtype=torch.uint8, device=x.device)
        s = torch.empty((rows, K // 16), dtype=torch.uint8, device=x.device)
    _check(load_library().realb_quantize_rows_nvfp4(_p(x), rows, K, C.c_float(global_scale), _p(q), _p(s), _stream(stream)))
    return q, s


def route_stats_static(logits, is_vision, E: int, k: int, D: int, b, T=None, stream=None):
    """realb_route_stats_static: the routing call that allocates nothing and needs no context; writes into
    the caller's buffers b (topk_ids, topk_w, expert_cnt, expert_vis, rank_load, rank_vis)."""
    T = logits.shape[0] if T is None else T
    _check(load_library().realb_route_stats_static(_p(logits), _p(is_vision), T, E, k, D, _p(b.topk_ids), _p(b.topk_w),
                                                   _p(b.expert_cnt), _p(b.expert_vis), _p(b.rank_load), _p(b.rank_vis),
                                                   _stream(stream)))


# ---- the operators around the MoE layer.  The make_*_io functions check types and shapes once and keep the tensors alive; a call
# then only passes the block of addresses on.
_TYPES = {torch.bfloat16: 0, torch.float32: 1}
_BF16_ONLY, _CODES = (torch.bfloat16,), (torch.uint8,)


def _require(cond: bool, what: str):
    if not cond:
        raise RealbError(what)


def _rows(t: torch.Tensor, name: str, shape, dtypes) -> int:
    """Row pitch of a matrix whose rows are dense; checks its shape and type."""
    if t.shape != shape:
        raise RealbError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.dtype not in dtypes:
        raise RealbError(f"{name} has type {t.dtype}")
    rows, cols = shape
    if rows == 0:
        return -(-cols // 16) * 16
    ld, step = t.stride()
    if step != 1 and cols != 1:
        raise RealbError(f"the rows of {name} are not dense")
    return ld if rows > 1 else -(-cols // 16) * 16                               # (one row has no pitch)


def _vector(t, name: str, n: int):
    if t is None:
        return None
    _require(t.dtype == torch.bfloat16 and t.is_contiguous() and tuple(t.shape) == (n,), f"{name} must be a dense bfloat16 vector of {n}")
    return t.data_ptr()


def _same_device(first, *others) -> int:
    gpu = first.get_device()
    for t in others:
        if t is not None and t.get_device() != gpu:
            gpu = -1
    _require(gpu >= 0, "tensors are not on one GPU")
    return gpu


def _raw_stream(stream, gpu):
    """As _stream, a plain number: these calls are short enough for the difference to show.  gpu: the tensors' one (None: arguments that were not
    made here).  Kernels are launched on the current GPU, so all three have to agree."""
    s = torch.cuda.current_stream() if stream is None else stream
    if gpu is not None and (s.device_index != gpu or (stream is not None and torch.cuda.current_device() != gpu)):
        raise RealbError(f"the tensors are on GPU {gpu}, the stream on {s.device_index}, the current one is {torch.cuda.current_device()}")
    return s.cuda_stream


class Fp8Rows:
    """Activation rows in E4M3: codes q u8 [rows, K] (rows may be a slice of wider ones) and scales s f32 [ceil(K/128), >= rows]."""

    def __init__(self, q: torch.Tensor, s: torch.Tensor):
        if q.dim() != 2 or s.dim() != 2:
            raise RealbError("q and s must be matrices")
        self.q, self.s = q, s
        self.rows, self.K = q.shape
        self.ld = _rows(q, "q", q.shape, _CODES)
        blocks, room = s.shape
        if s.dtype is not torch.float32 or blocks != -(-self.K // 128) or room < self.rows or (s.stride(1) != 1 and room > 1):
            raise RealbError(f"s must be float32 [{-(-self.K // 128)}, >= {self.rows}] with dense rows")
        self.ld_s = s.stride(0) if blocks > 1 else room

    @classmethod
    def empty(cls, rows: int, K: int, device="cuda") -> "Fp8Rows":
        return cls(torch.empty((rows, K), dtype=torch.uint8, device=device),
                   torch.empty((-(-K // 128), max(4, -(-rows // 4) * 4)), dtype=torch.float32, device=device))


class Fp8Weight:
    """Weights in E4M3: codes q u8 [.., N, K] and a scale per 128 x 128 block, s f32 [.., ceil(N/128), ceil(K/128)]."""

    def __init__(self, q: torch.Tensor, s: torch.Tensor):
        if q.dim() < 2:
            raise RealbError("q must have rows and columns")
        self.q, self.s = q, s
        self.N, self.K = q.shape[-2:]
        if q.dtype is not torch.uint8 or not q.is_contiguous():
            raise RealbError("q must be dense uint8")
        want = (*q.shape[:-2], -(-self.N // 128), -(-self.K // 128))
        if s.dtype is not torch.float32 or not s.is_contiguous() or s.shape != want:
            raise RealbError(f"s must be dense float32 {want}")

    @classmethod
    def empty(cls, *shape: int, device="cuda") -> "Fp8Weight":
        return cls(torch.empty(shape, dtype=torch.uint8, device=device),
                   torch.empty((*shape[:-2], -(-shape[-2] // 128), -(-shape[-1] // 128)), dtype=torch.float32, device=device))


def quantize_rows_fp8(x: torch.Tensor, out: "Fp8Rows | None" = None, stream=None) -> Fp8Rows:
    """realb_quantize_rows_fp8 on a bf16 [rows, K] tensor with dense rows of any pitch."""
    if out is None:
        with _on(stream):
            out = Fp8Rows.empty(*x.shape, device=x.device)
    ld = _rows(x, "x", (out.rows, out.K), _BF16_ONLY)
    raw = _raw_stream(stream, _same_device(x, out.q, out.s))
    _check(load_library().realb_quantize_rows_fp8(x.data_ptr(), ld, out.rows, out.K, out.q.data_ptr(), out.ld, out.s.data_ptr(), out.ld_s, raw))
    return out


def quantize_blocks_fp8(w: torch.Tensor, out: "Fp8Weight | None" = None, stream=None) -> Fp8Weight:
    """realb_quantize_blocks_fp8 on a dense bf16 [.., N, K] tensor."""
    if out is None:
        with _on(stream):
            out = Fp8Weight.empty(*w.shape, device=w.device)
    if w.dtype is not torch.bfloat16 or not w.is_contiguous() or w.shape != out.q.shape:
        raise RealbError(f"w must be dense bfloat16 {tuple(out.q.shape)}")
    raw = _raw_stream(stream, _same_device(w, out.q, out.s))
    mats = w.numel() // max(1, out.N * out.K) if w.dim() > 2 else 1
    _check(load_library().realb_quantize_blocks_fp8(w.data_ptr(), mats, out.N, out.K, out.q.data_ptr(), out.s.data_ptr(), raw))
    return out


def make_norm_io(res, y=None, res_out=None, post_weight=None, gate=None, scale: float = 1.0, pre_weight=None, eps: float = 1e-6, out=None,
                 out_fp8: "Fp8Rows | None" = None) -> NormIO:
    """Arguments of residual_norm: res [T,H] bf16 or f32; y bf16 [T,H]; gate bf16 [1,H] (per channel), [T,1] (per token) or [T,H];
    res_out of res's type (may be res); out bf16 [T,H] and / or out_fp8 for the norm with pre_weight."""
    T, H = res.shape
    io = NormIO()
    io.T, io.H, io.eps, io.scale = T, H, eps, scale
    io.ld_res = _rows(res, "res", (T, H), _TYPES)
    io.res, io.res_type = res.data_ptr(), _TYPES[res.dtype]
    if y is not None:
        io.y, io.ld_y = y.data_ptr(), _rows(y, "y", (T, H), (torch.bfloat16,))
    io.post_w, io.pre_w = _vector(post_weight, "post_weight", H), _vector(pre_weight, "pre_weight", H)
    if gate is not None:
        _require(gate.dim() == 2 and gate.dtype == torch.bfloat16 and gate.shape[0] in (1, T) and gate.shape[1] in (1, H),
                 f"gate must be bfloat16 [1 or {T}, 1 or {H}]")
        io.gate, io.gate_step = gate.data_ptr(), int(gate.shape[1] == H)
        io.ld_gate = 0 if gate.shape[0] == 1 else gate.stride(0)
        _require(gate.shape[1] == 1 or gate.stride(1) == 1, "the rows of gate are not dense")
    if res_out is not None:
        io.res_out, io.ld_res_out = res_out.data_ptr(), _rows(res_out, "res_out", (T, H), (res.dtype,))
    if out is not None:
        io.out, io.ld_out = out.data_ptr(), _rows(out, "out", (T, H), (torch.bfloat16,))
    if out_fp8 is not None:
        _require((out_fp8.rows, out_fp8.K) == (T, H), f"out_fp8 is [{out_fp8.rows}, {out_fp8.K}], expected [{T}, {H}]")
        io.out_q, io.ld_q, io.out_s, io.ld_s = out_fp8.q.data_ptr(), out_fp8.ld, out_fp8.s.data_ptr(), out_fp8.ld_s
    io._gpu = _same_device(res, y, post_weight, pre_weight, gate, res_out, out, *((out_fp8.q, out_fp8.s) if out_fp8 else ()))
    io._keep = (res, y, res_out, post_weight, gate, pre_weight, out, out_fp8)
    return io


def residual_norm(io: NormIO, stream=None):
    rc = (_LIB or load_library()).realb_residual_norm(C.byref(io), _raw_stream(stream, io._gpu))
    if rc:
        _check(rc)


def make_linear_io(x: Fp8Rows, w: Fp8Weight, out: torch.Tensor, bias=None, add=None) -> LinearIO:
    """Arguments of linear_fp8: out [rows, N] bf16 or f32; bias bf16 [N]; add of out's type (may be out)."""
    _require(w.q.dim() == 2 and w.K == x.K, f"weights {tuple(w.q.shape)} do not go with rows of {x.K}")
    io = LinearIO()
    io.M, io.N, io.K = x.rows, w.N, x.K
    io.x_q, io.ld_x, io.x_s, io.ld_xs = x.q.data_ptr(), x.ld, x.s.data_ptr(), x.ld_s
    io.w_q, io.w_s, io.bias = w.q.data_ptr(), w.s.data_ptr(), _vector(bias, "bias", w.N)
    if add is not None:
        io.add, io.ld_add = add.data_ptr(), _rows(add, "add", (x.rows, w.N), (out.dtype,))
    io.ld_out = _rows(out, "out", (x.rows, w.N), _TYPES)
    io.out, io.out_type = out.data_ptr(), _TYPES[out.dtype]
    io._gpu = _same_device(x.q, x.s, w.q, w.s, out, bias, add)
    io._keep = (x, w, out, bias, add)
    return io


def linear_fp8(io: LinearIO, stream=None):
    rc = (_LIB or load_library()).realb_linear_fp8(C.byref(io), _raw_stream(stream, io._gpu))
    if rc:
        _check(rc)


def make_ffn_io(x: Fp8Rows, w13: Fp8Weight, w2: Fp8Weight, out: torch.Tensor, add=None, workspace=None, f32_sums: bool = False) -> FfnIO:
    """Arguments of gated_ffn_fp8: w13 [2I, H], w2 [H, I], out bf16 [rows, H], add bf16 (may be out).  workspace: dense u8 of at least
    realb_gated_ffn_workspace_bytes(rows, I), for one call at a time; if not given, allocated here for the current stream and by the first call on
    any other stream for that one, and kept with the arguments.  f32_sums: FP32 sums in both products, whatever the number of
    rows (up to 64 they always are); without it more rows take the 8-bit instruction, faster and 0.0018 to 0.0026 off the formula, not 0.0017."""
    H, I = x.K, w2.K
    _require(tuple(w13.q.shape) == (2 * I, H) and tuple(w2.q.shape) == (H, I), f"weights {tuple(w13.q.shape)} and {tuple(w2.q.shape)} do not go with rows of {H}")
    _require(workspace is None or (workspace.dtype == torch.uint8 and workspace.is_contiguous()), "workspace must be dense uint8")
    io = FfnIO()
    io.T, io.H, io.I, io.sums = x.rows, H, I, int(bool(f32_sums))
    io.x_q, io.ld_x, io.x_s, io.ld_xs = x.q.data_ptr(), x.ld, x.s.data_ptr(), x.ld_s
    io.w13_q, io.w13_s, io.w2_q, io.w2_s = (t.data_ptr() for t in (w13.q, w13.s, w2.q, w2.s))
    if add is not None:
        io.add, io.ld_add = add.data_ptr(), _rows(add, "add", (x.rows, H), (torch.bfloat16,))
    io.out, io.ld_out = out.data_ptr(), _rows(out, "out", (x.rows, H), (torch.bfloat16,))
    io._gpu = _same_device(x.q, x.s, w13.q, w13.s, w2.q, w2.s, out, add, workspace)
    io._keep = (x, w13, w2, out, add, workspace)
    if workspace is None:
        io._workspaces = {}
        _own_workspace(io, None, _raw_stream(None, None))
    else:
        io.workspace, io.workspace_bytes = workspace.data_ptr(), workspace.numel()
    return io


def _own_workspace(io: FfnIO, stream, raw: int):
    """The workspace of the stream, allocated at its first call."""
    own = io._workspaces.get(raw)
    if own is None:
        need = int((_LIB or load_library()).realb_gated_ffn_workspace_bytes(io.T, io.I))
        with _on(stream):
            own = io._workspaces[raw] = torch.empty(max(need, 16), dtype=torch.uint8, device=io._keep[0].q.device)
    io.workspace, io.workspace_bytes, io._workspace_of = own.data_ptr(), own.numel(), raw


def gated_ffn_fp8(io: FfnIO, stream=None):
    raw = _raw_stream(stream, io._gpu)
    if io._workspaces is not None and io._workspace_of != raw:
        _own_workspace(io, stream, raw)
    rc = (_LIB or load_library()).realb_gated_ffn_fp8(C.byref(io), raw)
    if rc:
        _check(rc)


class LayerBuffers:
    """Caller-side allocation of every tensor of one layer call (device memory via torch)."""

    def __init__(self, cfg: Config, T: int, device="cuda"):
        E, k, D, H, I = cfg.E, cfg.k, cfg.D, cfg.H, cfg.I
        nl = E // D
        self.T, self.n_local = T, nl
        self.max_rows = max(1, T * min(k, nl))
        R = self.max_rows
        dev = device
        i32 = dict(dtype=torch.int32, device=dev)
        u8 = dict(dtype=torch.uint8, device=dev)
        bf = dict(dtype=torch.bfloat16, device=dev)
        self.topk_ids = torch.empty((T, k), **i32)
        self.topk_w = torch.empty((T, k), dtype=torch.float32, device=dev)
        self.expert_cnt = torch.empty(E, **i32)
        self.expert_vis = torch.empty(E, **i32)
        self.rank_load = torch.empty(D, **i32)
        self.rank_vis = torch.empty(D, **i32)
        self.expert_offsets = torch.empty(nl + 1, **i32)
        self.row_to_assign = torch.empty(R, **i32)
        self.assign_to_row = torch.empty(max(1, T * k), **i32)
        self.x_perm = torch.empty((R, H), **bf)
        self.x_q = torch.empty((R, H // 2), **u8)
        R32 = -(-R // 32) * 32                           # scale tensors cover whole groups of 32 rows
        self.x_s = torch.empty((R32, H // 32), **u8)
        self.w13_q = torch.empty((nl, 2 * I, H // 2), **u8)
        self.w13_s = torch.empty((nl, 2 * I, H // 32), **u8)
        self.w2_q = torch.empty((nl, H, I // 2), **u8)
        self.w2_s = torch.empty((nl, H, I // 32), **u8)
        self.h_mid = torch.empty((R, I), **bf)          # FP4 path uses its first R*I/2 bytes as codes
        self.h_s = torch.empty((R32, I // 32), **u8)
        self.y_rows = torch.empty((R, H), **bf)
        self.out = torch.empty((T, H), **bf)


class WeightBuffers:
    """One set of FP4 weight buffers (codes and K-step-tiled scales) for a rank's experts; two of them
    serve the cross-layer prefetch as a ping-pong pair."""

    def __init__(self, cfg: Config, device="cuda"):
        nl, H, I = cfg.E // cfg.D, cfg.H, cfg.I
        u8 = dict(dtype=torch.uint8, device=device)
        self.w13_q = torch.empty((nl, 2 * I, H // 2), **u8)
        self.w13_s = torch.empty((nl, 2 * I, H // 32), **u8)
        self.w2_q = torch.empty((nl, H, I // 2), **u8)
        self.w2_s = torch.empty((nl, H, I // 32), **u8)


class Context:
    """Owns a realb_ctx.  Methods mirror the C entry points one to one."""

    def __init__(self, cfg: Config):
        self.lib = load_library()
        self.cfg = cfg
        self._h = C.c_void_p()
        _check(self.lib.realb_create(C.byref(cfg), C.byref(self._h)))

    def close(self):
        if self._h:
            self.lib.realb_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def M(self) -> float:
        return self.lib.realb_get_M(self._h)

    @M.setter
    def M(self, v: float):
        _check(self.lib.realb_set_M(self._h, float(v)))

    def route_stats(self, logits, is_vision, b: LayerBuffers, stream=None):
        _check(self.lib.realb_route_stats(self._h, _p(logits), _p(is_vision), logits.shape[0], _p(b.topk_ids), _p(b.topk_w),
                                          _p(b.expert_cnt), _p(b.expert_vis), _p(b.rank_load), _p(b.rank_vis), _stream(stream)))

    def select_precision(self, b: LayerBuffers, T: int, force: int = FORCE_NONE, stream=None):
        prec = np.zeros(self.cfg.D, dtype=np.int32)
        ib, M = C.c_double(0), C.c_double(0)
        _check(self.lib.realb_select_precision(self._h, _p(b.rank_load), _p(b.rank_vis), T, force, prec.ctypes.data,
                                               C.addressof(ib), C.addressof(M), _stream(stream)))
        return prec, ib.value, M.value

    def quantize_experts_fp4(self, w13, w2, b: LayerBuffers, stream=None):
        _check(self.lib.realb_quantize_experts_fp4(self._h, _p(w13), _p(w2), w13.shape[0], _p(b.w13_q), _p(b.w13_s),
                                                   _p(b.w2_q), _p(b.w2_s), _stream(stream)))

    def permute(self, x, b: LayerBuffers, rank: int, prec: int, stream=None):
        _check(self.lib.realb_permute(self._h, _p(x), _p(b.topk_ids), x.shape[0], rank, prec, b.max_rows,
                                      _p(b.expert_offsets), _p(b.row_to_assign), _p(b.assign_to_row),
                                      _p(b.x_perm), _p(b.x_q), _p(b.x_s), _stream(stream)))

    def grouped_moe_ffn(self, prec: int, w13, w2, b: LayerBuffers, stream=None):
        if prec == FP4:
            args = (_p(b.x_q), _p(b.x_s), _p(b.w13_q), _p(b.w13_s), _p(b.w2_q), _p(b.w2_s))
        else:
            args = (_p(b.x_perm), None, _p(w13), None, _p(w2), None)
        _check(self.lib.realb_grouped_moe_ffn(self._h, prec, _p(b.expert_offsets), b.n_local, b.max_rows, *args,
                                              _p(b.h_mid), _p(b.h_s), _p(b.y_rows), _stream(stream)))

    def grouped_moe_ffn_gate_up(self, prec: int, w13, b: LayerBuffers, stream=None):
        args = (_p(b.x_q), _p(b.x_s), _p(b.w13_q), _p(b.w13_s)) if prec == FP4 else (_p(b.x_perm), None, _p(w13), None)
        _check(self.lib.realb_grouped_moe_ffn_gate_up(self._h, prec, _p(b.expert_offsets), b.n_local, b.max_rows, *args,
                                                      _p(b.h_mid), _p(b.h_s), _stream(stream)))

    def grouped_moe_ffn_down(self, prec: int, w2, b: LayerBuffers, stream=None):
        args = (_p(b.w2_q), _p(b.w2_s)) if prec == FP4 else (_p(w2), None)
        _check(self.lib.realb_grouped_moe_ffn_down(self._h, prec, _p(b.expert_offsets), b.n_local, b.max_rows,
                                                   _p(b.h_mid), _p(b.h_s), *args, _p(b.y_rows), _stream(stream)))

    def combine(self, b: LayerBuffers, stream=None):
        _check(self.lib.realb_combine(self._h, _p(b.y_rows), _p(b.assign_to_row), _p(b.topk_w), b.T, _p(b.out), _stream(stream)))

    def make_io(self, logits, is_vision, x, w13, w2, b: LayerBuffers, rank: int, force: int = FORCE_NONE,
                overlap=True) -> LayerIO:
        """overlap: 0/False, 1/True = weight encoding in the launches of the call's routing and index kernels,
        2 = skipped (the buffers already hold this layer's encoded weights), 3 = speculative (W13 ahead of the decision),
        4 = prefetched by the previous call (see set_prefetch)."""
        io = LayerIO()
        g = lambda t: None if t is None else t.data_ptr()
        io.logits, io.is_vision, io.x, io.T = g(logits), g(is_vision), g(x), x.shape[0]
        io.w13, io.w2, io.rank, io.force, io.overlap, io.max_rows = g(w13), g(w2), rank, force, int(overlap), b.max_rows
        for name in ("topk_ids", "topk_w", "expert_cnt", "expert_vis", "rank_load", "rank_vis", "expert_offsets",
                     "row_to_assign", "assign_to_row", "x_perm", "x_q", "x_s", "w13_q", "w13_s", "w2_q", "w2_s",
                     "h_mid", "h_s", "y_rows", "out"):
            setattr(io, name, getattr(b, name).data_ptr())
        io._keep = (logits, is_vision, x, w13, w2, b)
        return io

    def layer_forward(self, io: LayerIO, stream=None):
        _check(self.lib.realb_layer_forward(self._h, C.byref(io), _stream(stream)))
        return int(io.prec_host[io.rank])

    def set_prefetch(self, io: LayerIO, next_w13, next_w2, wbuf: "WeightBuffers", reserve_cus: int):
        """Arms the cross-layer prefetch of a layer call: the next layer's weights are encoded into wbuf beside
        this layer's GEMMs, which leave reserve_cus compute units free."""
        io.next_w13, io.next_w2 = next_w13.data_ptr(), next_w2.data_ptr()
        io.next_w13_q, io.next_w13_s, io.next_w2_q, io.next_w2_s = (t.data_ptr() for t in (wbuf.w13_q, wbuf.w13_s, wbuf.w2_q, wbuf.w2_s))
        io.reserve_cus = int(reserve_cus)
        io._keep_next = (next_w13, next_w2, wbuf)

    def use_weight_buffers(self, io: LayerIO, wbuf: "WeightBuffers"):
        """Points a layer call's FP4 weight buffers at wbuf (instead of the LayerBuffers' own)."""
        io.w13_q, io.w13_s, io.w2_q, io.w2_s = (t.data_ptr() for t in (wbuf.w13_q, wbuf.w13_s, wbuf.w2_q, wbuf.w2_s))
        io._keep_w = wbuf

    def set_gemm_tile_shape(self, shape: int):
        _check(self.lib.realb_set_gemm_tile_shape(self._h, int(shape)))

    STAGES = ("route_stats", "permute_indices", "decision_and_encode", "gather", "gate_up", "down", "combine")

    def stage_timing(self, enable: bool):
        _check(self.lib.realb_stage_timing(self._h, int(bool(enable))))

    def stage_ms(self) -> dict:
        """realb_stage_ms: GPU milliseconds of each stage of the last layer call (waits for it)."""
        ms = (C.c_float * len(self.STAGES))()
        _check(self.lib.realb_stage_ms(self._h, ms))
        return dict(zip(self.STAGES, (float(v) for v in ms)))

    def prefetch_join(self, stream=None):
        _check(self.lib.realb_prefetch_join(self._h, _stream(stream)))

    def rank_forward(self, io: LayerIO, prec: int, stream=None):
        _check(self.lib.realb_rank_forward(self._h, C.byref(io), prec, _stream(stream)))
