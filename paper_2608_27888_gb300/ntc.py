"""Python binding of libntc (``include/ntc.h``): ctypes marshalling only.

The module-level ``ntc_*`` functions mirror the C ABI one to one and take raw
pointers (ints) and sizes.  ``Decoder`` wraps them for torch tensors: PyTorch
supplies device memory and streams, every step of the decode runs in libntc's
CUDA kernels.  There is no fallback: if ``_build/libntc.so`` is missing the
import of this module fails.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "_build", "libntc.so")

NTC_OK, NTC_ERR_INVALID_ARG, NTC_ERR_UNSUPPORTED, NTC_ERR_OUT_OF_MEMORY, NTC_ERR_CUDA = range(5)
NTC_PREC_TC_FP16, NTC_PREC_TC_BF16, NTC_PREC_FP32 = range(3)
NTC_MODE_BUCKETED, NTC_MODE_DIVERGENT, NTC_MODE_BUCKETED_MMA, NTC_MODE_DIVERGENT_FMA = range(4)
NTC_MAX_DECODERS = 4095
NTC_TILE_ROWS = 128

# ntc_debug_row (include/ntc.h), 512 bytes
DEBUG_ROW = np.dtype([("idx", "<u8", (2, 2, 4)), ("raw", "<u4", (2, 2, 4, 4)), ("w", "<f4", (2, 2, 4)),
                      ("t", "<f4"), ("lo", "<u4"), ("feat", "<u4", (8,)), ("pad", "<u4", (6,))])
assert DEBUG_ROW.itemsize == 512

PRECISIONS = {"fp16": NTC_PREC_TC_FP16, "bf16": NTC_PREC_TC_BF16, "fp32": NTC_PREC_FP32}
NTC_OUTPUT_FP32, NTC_OUTPUT_FP16 = 0, 1
OUTPUTS = {"fp32": NTC_OUTPUT_FP32, "fp16": NTC_OUTPUT_FP16}
MODES = {"bucketed": NTC_MODE_BUCKETED, "divergent": NTC_MODE_DIVERGENT, "bucketed_mma": NTC_MODE_BUCKETED_MMA,
         "divergent_fma": NTC_MODE_DIVERGENT_FMA}
EXPORTS = ("ntc_create", "ntc_decode", "ntc_decode_host", "ntc_destroy", "ntc_debug_taps", "ntc_debug_decode_rows",
           "ntc_debug_features", "ntc_debug_bucket", "ntc_max_tiles", "ntc_get_error_count",
           "ntc_reset_error_count", "ntc_launch_count", "ntc_set_stage_timing", "ntc_stage_times",
           "ntc_bucket_static", "ntc_kmeans_map", "ntc_debug_wait_timeout", "ntc_last_error",
           "ntc_status_string", "ntc_route", "ntc_route_backward", "ntc_expert_order",
           "ntc_expert_order_workspace", "ntc_linear", "ntc_linear_workspace", "ntc_linear_backward",
           "ntc_linear_backward_workspace", "ntc_linear_status", "ntc_combine", "ntc_combine_backward")

# routed experts
NTC_MAX_EXPERTS, NTC_MAX_TOP_K = 1024, 32
NTC_TYPE_FP32, NTC_TYPE_FP16, NTC_TYPE_BF16 = range(3)
SCORES = {"softmax": 0, "sigmoid": 1}
ACTIVATIONS = {"none": 0, "relu": 1, "leaky": 2, "gelu": 3, "silu": 4}


class ntc_desc(ctypes.Structure):
    _fields_ = [
        ("num_sets", ctypes.c_uint32),
        ("num_decoders", ctypes.c_uint32),
        ("latent_channels", ctypes.c_uint32),
        ("num_levels", ctypes.c_uint32),
        ("num_mips", ctypes.c_uint32),
        ("level_dims", ctypes.c_void_p),
        ("latent_offsets", ctypes.c_void_p),
        ("latents", ctypes.c_void_p),
        ("num_texels", ctypes.c_uint64),
        ("in_dim", ctypes.c_uint32),
        ("hidden", ctypes.c_uint32),
        ("num_hidden_layers", ctypes.c_uint32),
        ("out_dim", ctypes.c_uint32),
        ("weights", ctypes.c_void_p),
        ("set_to_decoder", ctypes.c_void_p),
        ("precision", ctypes.c_int),
        ("address_mode", ctypes.c_uint32),
        ("pe_frequencies", ctypes.c_uint32),
        ("activation", ctypes.c_uint32),
        ("leaky_slope", ctypes.c_float),
        ("output_format", ctypes.c_uint32),
    ]


class ntc_route_desc(ctypes.Structure):
    _fields_ = [(f, ctypes.c_uint32) for f in ("num_experts", "top_k", "num_groups", "top_groups", "score",
                                               "renormalize")] + [("scale", ctypes.c_float), ("type", ctypes.c_int)]


class ntc_linear_desc(ctypes.Structure):
    _fields_ = [("type", ctypes.c_int), ("in_dim", ctypes.c_uint32), ("out_dim", ctypes.c_uint32),
                ("num_experts", ctypes.c_uint32), ("activation", ctypes.c_uint32), ("leaky_slope", ctypes.c_float)] + [
                    (f, ctypes.c_uint64) for f in ("num_rows", "num_x_rows", "ld_x", "ld_w", "stride_w", "ld_y", "ld_z",
                                                   "ld_residual")]


class ntc_combine_desc(ctypes.Structure):
    _fields_ = [("type", ctypes.c_int), ("dim", ctypes.c_uint32), ("top_k", ctypes.c_uint32),
                ("num_experts", ctypes.c_uint32)] + [
                    (f, ctypes.c_uint64) for f in ("num_tokens", "num_rows", "ld_y", "ld_out", "ld_residual")]


class NtcError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__(f"{msg} (status {status})")
        self.status = status


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"libntc is not built ({LIB_PATH} missing); run __graft_entry__.build()")
    lib = ctypes.CDLL(LIB_PATH)
    P, S, I = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int
    sig = {
        "ntc_create": ([P, P], I),
        "ntc_decode": ([P, P, S, P, P, I], I),
        "ntc_decode_host": ([P, P, S, P, P, I], I),
        "ntc_destroy": ([P], I),
        "ntc_debug_taps": ([P, P, S, P, P, P, P], I),
        "ntc_debug_features": ([P, P, S, P, P], I),
        "ntc_debug_decode_rows": ([P, P, S, P, P, P], I),
        "ntc_debug_bucket": ([P, P, S, P, P, P, P, P, P], I),
        "ntc_max_tiles": ([P, S], S),
        "ntc_get_error_count": ([P, P], I),
        "ntc_reset_error_count": ([P], I),
        "ntc_debug_wait_timeout": ([P, P], I),
        "ntc_launch_count": ([P], ctypes.c_uint64),
        "ntc_set_stage_timing": ([P, I], I),
        "ntc_stage_times": ([P, P], I),
        "ntc_bucket_static": ([P, ctypes.c_uint32, ctypes.c_uint32, P, S, P, P, P], I),
        "ntc_kmeans_map": ([P, ctypes.c_uint32, ctypes.c_uint32, ctypes.c_uint32, P, ctypes.c_uint32, P, P, P], I),
        "ntc_route": ([P, S, P, S, P, P, P, P], I),
        "ntc_route_backward": ([P, S, P, S, P, P, P, P], I),
        "ntc_expert_order_workspace": ([S, ctypes.c_uint32], S),
        "ntc_expert_order": ([P, S, ctypes.c_uint32, ctypes.c_uint32, P, P, P, P, S, P], I),
        "ntc_linear_workspace": ([P, P, P], S),
        "ntc_linear": ([P, P, P, P, P, P, P, P, P, P, S, P], I),
        "ntc_linear_backward_workspace": ([P, P, P, P], S),
        "ntc_linear_backward": ([P, P, P, P, P, P, P, P, P, P, P, S, P], I),
        "ntc_linear_status": ([P], I),
        "ntc_combine": ([P, P, P, P, P, P, P, P], I),
        "ntc_combine_backward": ([P, P, P, P, P, P, P, P, P], I),
        "ntc_last_error": ([], ctypes.c_char_p),
        "ntc_status_string": ([I], ctypes.c_char_p),
    }
    for name, (args, res) in sig.items():
        f = getattr(lib, name)
        f.argtypes = args
        f.restype = res
    return lib


_lib = _load()


def _check(status):
    if status != NTC_OK:
        raise NtcError(status, _lib.ntc_last_error().decode())


# ------------------------------------------------------- 1:1 mirrors of the ABI

def ntc_create(desc: ntc_desc) -> int:
    ctx = ctypes.c_void_p()
    _check(_lib.ntc_create(ctypes.byref(desc), ctypes.byref(ctx)))
    return ctx.value


def ntc_decode(ctx, d_queries, n, d_out, stream, mode):
    _check(_lib.ntc_decode(ctx, d_queries, n, d_out, stream, mode))


def ntc_decode_host(ctx, h_queries, n, h_out, stream, mode):
    _check(_lib.ntc_decode_host(ctx, h_queries, n, h_out, stream, mode))


def ntc_destroy(ctx):
    _check(_lib.ntc_destroy(ctx))


def ntc_debug_taps(ctx, d_queries, n, d_idx, d_w, d_t, stream):
    _check(_lib.ntc_debug_taps(ctx, d_queries, n, d_idx, d_w, d_t, stream))


def ntc_debug_features(ctx, d_queries, n, d_feat, stream):
    _check(_lib.ntc_debug_features(ctx, d_queries, n, d_feat, stream))


def ntc_debug_decode_rows(ctx, d_queries, n, d_out, d_rows, stream):
    _check(_lib.ntc_debug_decode_rows(ctx, d_queries, n, d_out, d_rows, stream))


def ntc_debug_bucket(ctx, d_queries, n, d_perm, d_counts, d_tiles, d_num_tiles, d_divergence, stream):
    _check(_lib.ntc_debug_bucket(ctx, d_queries, n, d_perm, d_counts, d_tiles, d_num_tiles, d_divergence,
                                 stream))


def ntc_max_tiles(ctx, n) -> int:
    return int(_lib.ntc_max_tiles(ctx, n))


def ntc_get_error_count(ctx) -> int:
    v = ctypes.c_uint64()
    _check(_lib.ntc_get_error_count(ctx, ctypes.byref(v)))
    return int(v.value)


def ntc_reset_error_count(ctx):
    _check(_lib.ntc_reset_error_count(ctx))


def ntc_debug_wait_timeout(ctx, stream=None):
    _check(_lib.ntc_debug_wait_timeout(ctx, stream))


def ntc_launch_count(ctx) -> int:
    return int(_lib.ntc_launch_count(ctx))


def ntc_set_stage_timing(ctx, enable):
    _check(_lib.ntc_set_stage_timing(ctx, int(bool(enable))))


def ntc_stage_times(ctx):
    t = (ctypes.c_float * 2)()
    _check(_lib.ntc_stage_times(ctx, t))
    return float(t[0]), float(t[1])


def ntc_bucket_static(h_set_to_decoder, num_sets, num_decoders, d_queries, n, d_perm, d_sorted, stream):
    """Allocation-free bucketing (no context): see include/ntc.h."""
    _check(_lib.ntc_bucket_static(h_set_to_decoder, num_sets, num_decoders, d_queries, n, d_perm,
                                  d_sorted, stream))


def ntc_kmeans_map(h_features, n, dim, m, h_init, max_iters, h_map, h_centroids, iters_run):
    _check(_lib.ntc_kmeans_map(h_features, n, dim, m, h_init, max_iters, h_map, h_centroids, iters_run))


def ntc_route(desc, n, logits, ld_logits, bias, ids, weights, stream):
    _check(_lib.ntc_route(ctypes.byref(desc), n, logits, ld_logits, bias, ids, weights, stream))


def ntc_route_backward(desc, n, logits, ld_logits, ids, dweights, dlogits, stream):
    _check(_lib.ntc_route_backward(ctypes.byref(desc), n, logits, ld_logits, ids, dweights, dlogits, stream))


def ntc_expert_order_workspace(n, num_experts) -> int:
    return _lib.ntc_expert_order_workspace(n, num_experts)


def ntc_expert_order(ids, n, top_k, num_experts, rows, place, offsets, workspace, workspace_bytes, stream):
    _check(_lib.ntc_expert_order(ids, n, top_k, num_experts, rows, place, offsets, workspace, workspace_bytes, stream))


def ntc_linear_workspace(desc, x, w) -> int:
    return _lib.ntc_linear_workspace(ctypes.byref(desc), x, w)


def ntc_linear(desc, x, rows, offsets, w, bias, residual, y, z, workspace, workspace_bytes, stream):
    _check(_lib.ntc_linear(ctypes.byref(desc), x, rows, offsets, w, bias, residual, y, z, workspace, workspace_bytes,
                           stream))


def ntc_linear_backward_workspace(desc, dy, x, w) -> int:
    return _lib.ntc_linear_backward_workspace(ctypes.byref(desc), dy, x, w)


def ntc_linear_backward(desc, dy, z, x, rows, offsets, w, dx, dw, db, workspace, workspace_bytes, stream):
    _check(_lib.ntc_linear_backward(ctypes.byref(desc), dy, z, x, rows, offsets, w, dx, dw, db, workspace,
                                    workspace_bytes, stream))


def ntc_linear_status(stream=None):
    _check(_lib.ntc_linear_status(stream))


def ntc_combine(desc, y, place, weights, offsets, residual, out, stream):
    _check(_lib.ntc_combine(ctypes.byref(desc), y, place, weights, offsets, residual, out, stream))


def ntc_combine_backward(desc, dout, y, place, weights, offsets, dy, dweights, stream):
    _check(_lib.ntc_combine_backward(ctypes.byref(desc), dout, y, place, weights, offsets, dy, dweights, stream))


def kmeans_map(features, m, init, max_iters=100):
    """numpy convenience: (map [n] uint32, centroids [m, dim] float64, assignments made)."""
    F = np.ascontiguousarray(features, dtype=np.float32)
    n, dim = F.shape
    init = np.ascontiguousarray(init, dtype=np.uint32)
    out = np.empty(n, dtype=np.uint32)
    mu = np.empty((m, dim), dtype=np.float64)
    it = ctypes.c_uint32()
    ntc_kmeans_map(F.ctypes.data, n, dim, m, init.ctypes.data, max_iters, out.ctypes.data, mu.ctypes.data,
                   ctypes.byref(it))
    return out, mu, int(it.value)


def ntc_last_error() -> str:
    return _lib.ntc_last_error().decode()


# --------------------------------------------------------- torch convenience

def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(stream):
    import torch
    s = stream if stream is not None else torch.cuda.current_stream()
    return s.cuda_stream


def queries_to_device(q: np.ndarray, device="cuda"):
    """16-byte query records (numpy) -> int32 [n, 4] tensor on the device."""
    import torch
    a = np.ascontiguousarray(q).view(np.int32).reshape(-1, 4)
    return torch.from_numpy(a).to(device)


class Decoder:
    """An ntc context built from an assets object (see ``workloads.Assets``)."""

    def __init__(self, assets, precision: str = "fp16", output: str = "fp32"):
        self._keep = [
            np.ascontiguousarray(assets.level_dims, dtype=np.uint32),
            np.ascontiguousarray(assets.latent_offsets, dtype=np.uint64),
            np.ascontiguousarray(assets.latents, dtype=np.uint16),
            np.ascontiguousarray(assets.weights, dtype=np.float32),
            np.ascontiguousarray(assets.set_to_decoder, dtype=np.uint32),
        ]
        dims, offs, lat, w, m = self._keep
        d = ntc_desc()
        d.num_sets = assets.num_sets
        d.num_decoders = assets.num_decoders
        d.latent_channels = assets.channels
        d.num_levels = assets.num_levels
        d.num_mips = assets.num_mips
        d.level_dims = dims.ctypes.data
        d.latent_offsets = offs.ctypes.data
        d.latents = lat.ctypes.data
        d.num_texels = lat.size // max(1, assets.channels)
        d.in_dim = assets.in_dim
        d.hidden = assets.hidden
        d.num_hidden_layers = assets.num_hidden_layers
        d.out_dim = assets.out_dim
        d.weights = w.ctypes.data
        d.set_to_decoder = m.ctypes.data
        d.precision = PRECISIONS[precision]
        d.address_mode = assets.address_mode
        d.pe_frequencies = getattr(assets, "pe_frequencies", 0)
        d.activation = getattr(assets, "activation", 0)
        d.leaky_slope = getattr(assets, "leaky_slope", 0.0)
        d.output_format = OUTPUTS[output]
        self.desc = d
        self.output = output
        self.out_dim = assets.out_dim
        self.num_decoders = assets.num_decoders
        self.num_levels = assets.num_levels
        self.in_dim = assets.in_dim
        self.ctx = ntc_create(d)
        self._keep = None  # ntc_create copied everything

    def close(self):
        if getattr(self, "ctx", None):
            ntc_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def out_dtype(self):
        import torch
        return torch.float16 if self.output == "fp16" else torch.float32

    def decode(self, queries, out=None, mode: str = "bucketed", stream=None):
        import torch
        n = queries.shape[0]
        if out is None:
            out = torch.empty((n, self.out_dim), dtype=self.out_dtype(), device=queries.device)
        ntc_decode(self.ctx, _ptr(queries), n, _ptr(out), _stream(stream), MODES[mode])
        return out

    def decode_host(self, queries, out=None, mode: str = "bucketed", stream=None):
        import torch
        n = queries.shape[0]
        if out is None:
            out = torch.empty((n, self.out_dim), dtype=self.out_dtype(), pin_memory=True)
        ntc_decode_host(self.ctx, _ptr(queries), n, _ptr(out), _stream(stream), MODES[mode])
        return out

    def taps(self, queries, stream=None):
        import torch
        n = queries.shape[0]
        dev = queries.device
        idx = torch.empty((n, self.num_levels, 2, 4), dtype=torch.int64, device=dev)
        w = torch.empty((n, self.num_levels, 2, 4), dtype=torch.float32, device=dev)
        t = torch.empty((n,), dtype=torch.float32, device=dev)
        ntc_debug_taps(self.ctx, _ptr(queries), n, _ptr(idx), _ptr(w), _ptr(t), _stream(stream))
        return idx, w, t

    def features(self, queries, stream=None):
        import torch
        n = queries.shape[0]
        f = torch.empty((n, self.in_dim), dtype=torch.float32, device=queries.device)
        ntc_debug_features(self.ctx, _ptr(queries), n, _ptr(f), _stream(stream))
        return f

    def decode_rows(self, queries, stream=None):
        """The bucketed tensor-core decode through its debug build: (outputs,
        rows) with rows a numpy structured array of ``DEBUG_ROW`` records
        (ntc_debug_row; rows of bad queries keep their fill of 0xFF bytes)."""
        import torch
        n = queries.shape[0]
        out = torch.empty((n, self.out_dim), dtype=self.out_dtype(), device=queries.device)
        rows = torch.full((max(1, n), DEBUG_ROW.itemsize), 255, dtype=torch.uint8, device=queries.device)
        ntc_debug_decode_rows(self.ctx, _ptr(queries), n, _ptr(out), _ptr(rows), _stream(stream))
        return out, rows[:n].cpu().numpy().view(DEBUG_ROW).reshape(n)

    def bucket(self, queries, stream=None, divergence=False):
        """(perm, counts, tiles) of the bucketing; with divergence=True also
        (copied, sum over 32-query groups of distinct decoders - 1)."""
        import torch
        n = queries.shape[0]
        dev = queries.device
        mt = max(1, ntc_max_tiles(self.ctx, n))
        perm = torch.empty((max(1, n),), dtype=torch.int32, device=dev)
        counts = torch.empty((self.num_decoders + 1,), dtype=torch.int32, device=dev)
        tiles = torch.empty((mt, 3), dtype=torch.int32, device=dev)
        nt = torch.zeros((1,), dtype=torch.int32, device=dev)
        dv = torch.zeros((2,), dtype=torch.int32, device=dev)
        ntc_debug_bucket(self.ctx, _ptr(queries), n, _ptr(perm), _ptr(counts), _ptr(tiles), _ptr(nt), _ptr(dv),
                         _stream(stream))
        k = int(nt.item())
        if divergence:
            c, s = dv.cpu().numpy().astype(np.uint32).tolist()
            return perm[:n], counts, tiles[:k], (c, s)
        return perm[:n], counts, tiles[:k]

    def error_count(self) -> int:
        return ntc_get_error_count(self.ctx)

    def reset_error_count(self):
        ntc_reset_error_count(self.ctx)

    def debug_wait_timeout(self, stream=None):
        """Make one bounded wait give up (a test of the failure path): the next
        error_count() raises NtcError with NTC_ERR_CUDA until reset_error_count()."""
        ntc_debug_wait_timeout(self.ctx, _stream(stream))

    def launches(self) -> int:
        return ntc_launch_count(self.ctx)

    def set_stage_timing(self, enable=True):
        ntc_set_stage_timing(self.ctx, enable)

    def stage_times(self):
        """(bucketing ms, gather-decode ms) of the last decode."""
        return ntc_stage_times(self.ctx)


# ------------------------------------------------- routed experts, on torch tensors
#
# Each function allocates its outputs and workspace with torch and makes the one
# library call of its name.  `stream` (default: the current stream) is where the
# call is queued and where those allocations live; tensors of another stream are the
# caller's to order, as for any torch call.  Matrices may have any row stride; their
# last dimension is contiguous.

def _on(stream):
    """A context that makes `stream` current (nothing to do for None)."""
    import contextlib
    import torch
    return torch.cuda.stream(stream) if stream is not None else contextlib.nullcontext()


def _types():
    import torch
    return {torch.float32: NTC_TYPE_FP32, torch.float16: NTC_TYPE_FP16, torch.bfloat16: NTC_TYPE_BF16}


_TYPE_OF = None


def _type_of(t, name):
    global _TYPE_OF
    if _TYPE_OF is None:
        _TYPE_OF = _types()
    try:
        return _TYPE_OF[t.dtype]
    except KeyError:
        raise ValueError(f"{name} must be float32, float16 or bfloat16, not {t.dtype}") from None


def _matrix(t, name, rows, cols, dtype, device):
    """The row stride of a [rows, cols] matrix argument, after its checks."""
    if t.dtype != dtype or t.device != device:
        raise ValueError(f"{name} must be {dtype} on {device}, not {t.dtype} on {t.device}")
    if t.dim() != 2 or t.shape[0] != rows or t.shape[1] != cols:
        raise ValueError(f"{name} must have shape [{rows}, {cols}], not {list(t.shape)}")
    if cols > 1 and t.stride(1) != 1:
        raise ValueError(f"{name} must be contiguous along its last dimension")
    ld = t.stride(0) if rows > 1 else cols
    if ld < cols:
        raise ValueError(f"{name} has overlapping rows")
    return ld


def _array(t, name, shape, dtype, device):
    """The address of a contiguous array argument of this shape (None stays None), after its checks."""
    if t is None:
        return None
    if t.dtype != dtype or t.device != device:
        raise ValueError(f"{name} must be {dtype} on {device}, not {t.dtype} on {t.device}")
    if tuple(t.shape) != shape:
        raise ValueError(f"{name} must have shape {list(shape)}, not {list(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _cuda(t, name):
    import torch
    if t.device.type != "cuda":
        raise ValueError(f"{name} must be a CUDA tensor")
    if t.device.index != torch.cuda.current_device():
        raise ValueError(f"{name} is on {t.device}, which is not the current device")
    return t.device


def _choice(table, key, name):
    try:
        return table[key]
    except (KeyError, TypeError):
        raise ValueError(f"{name} must be one of {', '.join(table)}, not {key!r}") from None


def _workspace(bytes_, device):
    import torch
    return torch.empty(bytes_, dtype=torch.uint8, device=device) if bytes_ else None


def route(logits, top_k: int, *, bias=None, score: str = "softmax", groups: int = 1, top_groups: int = 1,
          renormalize: bool = True, scale: float = 1.0, stream=None):
    """ids [n, top_k] int32 and weights [n, top_k] fp32 of each row of logits [n, experts]: see ntc_route."""
    import torch
    dev = _cuda(logits, "logits")
    if logits.dim() != 2:
        raise ValueError(f"logits must have two dimensions, not {logits.dim()}")
    n, E = logits.shape
    d = ntc_route_desc(E, top_k, groups, top_groups, _choice(SCORES, score, "score"), bool(renormalize), scale,
                       _type_of(logits, "logits"))
    ld = _matrix(logits, "logits", n, E, logits.dtype, dev)
    b = _array(bias, "bias", (E,), torch.float32, dev)
    with _on(stream):
        ids = torch.empty((n, max(0, top_k)), dtype=torch.int32, device=dev)
        weights = torch.empty((n, max(0, top_k)), dtype=torch.float32, device=dev)
        ntc_route(d, n, logits.data_ptr(), ld, b, ids.data_ptr(), weights.data_ptr(), _stream(stream))
    return ids, weights


def route_backward(logits, ids, dweights, *, score: str = "softmax", renormalize: bool = True, scale: float = 1.0,
                   stream=None):
    """The gradient of route's logits for the gradient of its weights: see ntc_route_backward."""
    import torch
    dev = _cuda(logits, "logits")
    if logits.dim() != 2 or ids.dim() != 2:
        raise ValueError("logits and ids must have two dimensions")
    (n, E), k = logits.shape, ids.shape[1]
    d = ntc_route_desc(E, k, 1, 1, _choice(SCORES, score, "score"), bool(renormalize), scale,
                       _type_of(logits, "logits"))
    ld = _matrix(logits, "logits", n, E, logits.dtype, dev)
    i = _array(ids, "ids", (n, k), torch.int32, dev)
    g = _array(dweights, "dweights", (n, k), torch.float32, dev)
    with _on(stream):
        out = torch.empty((n, E), dtype=logits.dtype, device=dev)
        ntc_route_backward(d, n, logits.data_ptr(), ld, i, g, out.data_ptr(), _stream(stream))
    return out


def expert_order(ids, num_experts: int, *, stream=None):
    """rows [n * k], place [n, k] and offsets [num_experts + 1] (int32) of ids [n, k]: see ntc_expert_order."""
    import torch
    dev = _cuda(ids, "ids")
    if ids.dim() != 2:
        raise ValueError(f"ids must have two dimensions, not {ids.dim()}")
    n, k = ids.shape
    i = _array(ids, "ids", (n, k), torch.int32, dev)
    with _on(stream):
        rows = torch.empty(n * k, dtype=torch.int32, device=dev)
        place = torch.empty((n, k), dtype=torch.int32, device=dev)
        offsets = torch.empty(max(0, num_experts) + 1, dtype=torch.int32, device=dev)
        size = ntc_expert_order_workspace(n * k, num_experts)
        ws = _workspace(size, dev)
        ntc_expert_order(i, n * k, k, num_experts, rows.data_ptr(), place.data_ptr(), offsets.data_ptr(), _ptr(ws), size,
                         _stream(stream))
    return rows, place, offsets


def _linear_operands(x, w, rows, offsets, activation, leaky_slope, num_rows):
    """The descriptor of a linear call, and the addresses of rows and offsets."""
    import torch
    dev = _cuda(x, "x")
    if w.dim() == 2:
        w = w[None]
    if x.dim() != 2 or w.dim() != 3:
        raise ValueError("x must have two dimensions, w two or three")
    E, N, K = w.shape
    if w.dtype != x.dtype or w.device != dev:
        raise ValueError(f"w must be {x.dtype} on {dev}, not {w.dtype} on {w.device}")
    if K > 1 and w.stride(2) != 1:
        raise ValueError("w must be contiguous along its last dimension")
    ldw = w.stride(1) if N > 1 else K
    step = w.stride(0) if E > 1 else N * ldw
    ldx = _matrix(x, "x", x.shape[0], K, x.dtype, dev)
    r = _array(rows, "rows", (num_rows,), torch.int32, dev)
    o = _array(offsets, "offsets", (E + 1,), torch.int32, dev)
    d = ntc_linear_desc(_type_of(x, "x"), K, N, E, _choice(ACTIVATIONS, activation, "activation"), leaky_slope, num_rows,
                        x.shape[0], ldx, ldw, step, N, N, N)
    return d, w, r, o, dev


def linear(x, w, bias=None, *, rows=None, offsets=None, activation: str = "none", leaky_slope: float = 0.01,
           residual=None, save: bool = False, stream=None):
    """act(x[rows] w^T + bias) + residual, with each expert's weights for its rows: see ntc_linear.

    x [n, K]; w [E, N, K] (or [N, K]); bias fp32 [E, N] (or [N]); rows int32: the row of x of each row of the
    result (default: the same); offsets int32 [E + 1]: where each expert's rows begin; residual [rows, N].
    save=True also returns the input of the activation, which linear_backward takes as z."""
    import torch
    m = x.shape[0] if rows is None else rows.shape[0]
    d, w, r, o, dev = _linear_operands(x, w, rows, offsets, activation, leaky_slope, m)
    E, N = d.num_experts, d.out_dim
    if bias is not None and bias.dim() == 1 and E == 1:
        bias = bias[None]
    b = _array(bias, "bias", (E, N), torch.float32, dev)
    if residual is not None:
        d.ld_residual = _matrix(residual, "residual", m, N, x.dtype, dev)
    with _on(stream):
        y = torch.empty((m, N), dtype=x.dtype, device=dev)
        z = torch.empty((m, N), dtype=x.dtype, device=dev) if save else None
        size = ntc_linear_workspace(d, x.data_ptr(), w.data_ptr())
        ws = _workspace(size, dev)
        ntc_linear(d, x.data_ptr(), r, o, w.data_ptr(), b, _ptr(residual), y.data_ptr(), _ptr(z), _ptr(ws), size,
                   _stream(stream))
    return (y, z) if save else y


def linear_backward(dy, x, w, *, z=None, rows=None, offsets=None, activation: str = "none", leaky_slope: float = 0.01,
                    need=("dx", "dw", "db"), stream=None):
    """(dx, dw, db) of linear for the gradient dy of its result: see ntc_linear_backward.

    z is what linear(save=True) returned beside the result (not needed without an activation).  dx has a row per
    row of dy; where rows gathered x, combine(dx, place, None, offsets) sums a token's.  Gradients that `need`
    does not name are None."""
    import torch
    m = dy.shape[0]
    d, w, r, o, dev = _linear_operands(x, w, rows, offsets, activation, leaky_slope, m)
    E, N, K = d.num_experts, d.out_dim, d.in_dim
    d.ld_y = _matrix(dy, "dy", m, N, x.dtype, dev)
    if activation == "none":
        z = None
    elif z is None:
        raise ValueError(f"activation {activation!r} needs z")
    else:
        d.ld_z = _matrix(z, "z", m, N, x.dtype, dev)
    for name in need:
        _choice({"dx": 0, "dw": 0, "db": 0}, name, "need")
    with _on(stream):
        dx = torch.empty((m, K), dtype=x.dtype, device=dev) if "dx" in need else None
        dw = torch.empty((E, N, K), dtype=x.dtype, device=dev) if "dw" in need else None
        db = torch.empty((E, N), dtype=torch.float32, device=dev) if "db" in need else None
        size = ntc_linear_backward_workspace(d, dy.data_ptr(), x.data_ptr(), w.data_ptr())
        ws = _workspace(size, dev)
        ntc_linear_backward(d, dy.data_ptr(), _ptr(z), x.data_ptr(), r, o, w.data_ptr(), _ptr(dx), _ptr(dw), _ptr(db),
                            _ptr(ws), size, _stream(stream))
    return dx, dw, db


def _combine_desc(y, place, offsets, dim):
    dev = _cuda(y, "y")
    if y.dim() != 2 or place.dim() != 2:
        raise ValueError("y and place must have two dimensions")
    T, k = place.shape
    E = offsets.shape[0] - 1 if offsets is not None and offsets.dim() == 1 else 1
    ld = _matrix(y, "y", y.shape[0], dim, y.dtype, dev)
    return ntc_combine_desc(_type_of(y, "y"), dim, k, E, T, y.shape[0], ld, dim, dim), dev


def combine(y, place, weights=None, offsets=None, *, residual=None, stream=None):
    """residual + the sum of y[place[t, j]] times weights[t, j] (1 without weights): see ntc_combine.

    Places from offsets[-1] on (rows of no expert) are left out."""
    import torch
    D = y.shape[1]
    d, dev = _combine_desc(y, place, offsets, D)
    T, k = place.shape
    p = _array(place, "place", (T, k), torch.int32, dev)
    g = _array(weights, "weights", (T, k), torch.float32, dev)
    o = _array(offsets, "offsets", (d.num_experts + 1,), torch.int32, dev)
    if residual is not None:
        d.ld_residual = _matrix(residual, "residual", T, D, y.dtype, dev)
    with _on(stream):
        out = torch.empty((T, D), dtype=y.dtype, device=dev)
        ntc_combine(d, y.data_ptr(), p, g, o, _ptr(residual), out.data_ptr(), _stream(stream))
    return out


def combine_backward(dout, y, place, weights=None, offsets=None, *, need=("dy", "dweights"), stream=None):
    """(dy, dweights) of combine for the gradient dout of its result: see ntc_combine_backward."""
    import torch
    D = y.shape[1]
    d, dev = _combine_desc(y, place, offsets, D)
    T, k = place.shape
    p = _array(place, "place", (T, k), torch.int32, dev)
    g = _array(weights, "weights", (T, k), torch.float32, dev)
    o = _array(offsets, "offsets", (d.num_experts + 1,), torch.int32, dev)
    d.ld_out = _matrix(dout, "dout", T, D, y.dtype, dev)
    for name in need:
        _choice({"dy": 0, "dweights": 0}, name, "need")
    with _on(stream):
        dy = torch.empty((y.shape[0], D), dtype=y.dtype, device=dev) if "dy" in need else None
        dw = torch.empty((T, k), dtype=torch.float32, device=dev) if "dweights" in need else None
        ntc_combine_backward(d, dout.data_ptr(), y.data_ptr(), p, g, o, _ptr(dy), _ptr(dw), _stream(stream))
    return dy, dw
