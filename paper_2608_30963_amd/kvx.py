"""Python binding of ``libkvx.so`` (argument marshalling only).

The entry points carry the C names -- ``kvx_plan_create``,
``kvx_plan_create_factored``, ``kvx_translate``, ``kvx_plan_destroy``
(include/kvx.h) and ``kvx_fit_create``,
``kvx_fit_accumulate``, ``kvx_fit_solve``, ``kvx_fit_reset``,
``kvx_fit_destroy`` (include/kvx_fit.h), ``kvx_attn_create``,
``kvx_attn_append``, ``kvx_attn_forward``, ``kvx_attn_mass``,
``kvx_attn_evict``, ``kvx_attn_destroy`` (include/kvx_attn.h) -- and take torch
tensors for device buffers (torch provides device memory and streams; it
computes nothing here).  Every step of the translation, of the fit and of
decoding on the translated cache runs in the library's HIP kernels.

The library must have been built (``python -m paper_2608_30963_amd.build``);
loading fails loudly otherwise -- there is no fallback path.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from typing import Optional, Sequence

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libkvx.so")

KVX_OK, KVX_EINVAL, KVX_ESHAPE, KVX_EUNSUPPORTED, KVX_ENOMEM, KVX_EHIP, KVX_EDATA = range(7)
KVX_F32, KVX_BF16 = 0, 1
KVX_PREC_BF16X2, KVX_PREC_BF16, KVX_PREC_F16, KVX_PREC_BF16X2_OUTLIER = 0, 1, 2, 3
KVX_FACTORS_LOWRANK, KVX_FACTORS_MIXTURE = 1, 2
KVX_STAGE_POOL, KVX_STAGE_PROJECT, KVX_STAGE_STORE, KVX_STAGE_ALL = 1, 2, 4, 7

# Exported C symbols, as declared in include/kvx.h, kvx_fit.h and kvx_attn.h.
SYMBOLS = ("kvx_plan_create", "kvx_plan_create_factored", "kvx_translate", "kvx_plan_destroy",
           "kvx_status_string",
           "kvx_last_hip_error", "kvx_plan_query", "kvx_staged_workspace_bytes",
           "kvx_translate_staged", "kvx_fit_create", "kvx_fit_accumulate",
           "kvx_fit_solve", "kvx_fit_solve_noalloc", "kvx_fit_reset", "kvx_fit_rows",
           "kvx_fit_query", "kvx_fit_destroy", "kvx_attn_create", "kvx_attn_destroy",
           "kvx_attn_append", "kvx_attn_workspace_bytes", "kvx_attn_forward", "kvx_attn_mass",
           "kvx_attn_evict")


class KvxError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {status_string(status)} (status {status})")


class Model(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("rope_base", C.c_double), ("inv_freq", C.c_void_p)]


class PlanDesc(C.Structure):
    _fields_ = [("src", Model), ("tgt", Model), ("mix", C.c_int32),
                ("layer_map", C.c_void_p), ("dtype", C.c_int32),
                ("w_k", C.c_void_p), ("w_v", C.c_void_p),
                ("b_k", C.c_void_p), ("b_v", C.c_void_p), ("precision", C.c_int32),
                ("outlier_k", C.c_void_p), ("outlier_v", C.c_void_p)]


class Factors(C.Structure):
    _fields_ = [("kind", C.c_int32), ("rank", C.c_int32), ("u_k", C.c_void_p),
                ("u_v", C.c_void_p), ("v_k", C.c_void_p), ("v_v", C.c_void_p),
                ("n_mix", C.c_int32), ("alpha", C.c_void_p), ("w_k", C.c_void_p),
                ("w_v", C.c_void_p), ("b_k", C.c_void_p), ("b_v", C.c_void_p)]


class IO(C.Structure):
    _fields_ = [("batch", C.c_int32), ("src_tokens", C.c_int32),
                ("src_k", C.c_void_p), ("src_v", C.c_void_p), ("src_stride", C.c_int64 * 4),
                ("tgt_tokens", C.c_void_p), ("row_ptr", C.c_void_p),
                ("col_idx", C.c_void_p), ("weight", C.c_void_p),
                ("tgt_k", C.c_void_p), ("tgt_v", C.c_void_p), ("tgt_stride", C.c_int64 * 4),
                ("tgt_capacity", C.c_int32), ("block_table", C.c_void_p),
                ("block_size", C.c_int32), ("max_blocks", C.c_int32), ("num_blocks", C.c_int32)]


class FitDesc(C.Structure):
    _fields_ = [("src", Model), ("tgt", Model), ("mix", C.c_int32),
                ("layer_map", C.c_void_p), ("dtype", C.c_int32), ("fit_bias", C.c_int32)]


class FitIO(C.Structure):
    _fields_ = [("batch", C.c_int32), ("src_tokens", C.c_int32),
                ("src_k", C.c_void_p), ("src_v", C.c_void_p), ("src_stride", C.c_int64 * 4),
                ("tgt_tokens", C.c_void_p), ("row_ptr", C.c_void_p),
                ("col_idx", C.c_void_p), ("weight", C.c_void_p),
                ("tgt_k", C.c_void_p), ("tgt_v", C.c_void_p), ("tgt_stride", C.c_int64 * 4),
                ("tgt_capacity", C.c_int32)]


class FitInfo(C.Structure):
    _fields_ = [("systems", C.c_int32), ("n", C.c_int32), ("gram_blocks", C.c_int32),
                ("gram_launches", C.c_int32), ("rows", C.c_int64),
                ("device_bytes", C.c_int64), ("gram_ms", C.c_double)]


class PlanInfo(C.Structure):
    _fields_ = [("kernel", C.c_int32), ("tile_rows", C.c_int32), ("tile_cols", C.c_int32),
                ("threads", C.c_int32), ("precision", C.c_int32), ("weight_bytes", C.c_int64),
                ("split_ksteps", C.c_int64), ("ksteps", C.c_int64),
                ("tile_order", C.c_int32)]


class AttnDesc(C.Structure):
    _fields_ = [("model", Model), ("n_heads", C.c_int32), ("dtype", C.c_int32),
                ("scale", C.c_double), ("softcap", C.c_double), ("n_axes", C.c_int32),
                ("pair_axis", C.c_void_p)]


class Cache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("stride", C.c_int64 * 4),
                ("capacity", C.c_int32), ("block_table", C.c_void_p), ("block_size", C.c_int32),
                ("max_blocks", C.c_int32), ("num_blocks", C.c_int32)]


class AttnIO(C.Structure):
    _fields_ = [("batch", C.c_int32), ("layer", C.c_int32), ("rows", C.c_int32),
                ("max_new", C.c_int32), ("q_start", C.c_void_p), ("tokens", C.c_void_p),
                ("cache", Cache), ("new_q", C.c_void_p), ("new_k", C.c_void_p),
                ("new_v", C.c_void_p), ("new_q_stride", C.c_int64 * 2),
                ("new_k_stride", C.c_int64 * 2), ("new_v_stride", C.c_int64 * 2),
                ("pos", C.c_void_p), ("q", C.c_void_p), ("q_stride", C.c_int64 * 2),
                ("window", C.c_int32), ("prefix", C.c_void_p), ("out", C.c_void_p),
                ("out_stride", C.c_int64 * 2), ("lse", C.c_void_p), ("mass_in", C.c_void_p),
                ("mass", C.c_void_p), ("mass_capacity", C.c_int32)]


class EvictIO(C.Structure):
    _fields_ = [("batch", C.c_int32), ("tokens", C.c_void_p), ("keep", C.c_int32),
                ("sink", C.c_int32), ("recent", C.c_int32), ("src", Cache), ("dst", Cache),
                ("mass", C.c_void_p), ("mass_out", C.c_void_p), ("mass_capacity", C.c_int32),
                ("kept", C.c_void_p), ("tokens_out", C.c_void_p)]


_lib = None


def load(path: str = LIB_PATH):
    """Load libkvx.so; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with "
                           "`python -m paper_2608_30963_amd.build` (no fallback exists)")
    # torch provides the device memory and streams; its HIP runtime must be
    # the process's only one, so it is loaded before the library binds to
    # whichever runtime is already present
    import torch  # noqa: F401
    lib = C.CDLL(path)
    lib.kvx_plan_create.argtypes = [C.POINTER(PlanDesc), C.POINTER(C.c_void_p)]
    lib.kvx_plan_create.restype = C.c_int
    lib.kvx_plan_create_factored.argtypes = [C.POINTER(PlanDesc), C.POINTER(Factors),
                                             C.POINTER(C.c_void_p)]
    lib.kvx_plan_create_factored.restype = C.c_int
    lib.kvx_translate.argtypes = [C.c_void_p, C.POINTER(IO), C.c_void_p]
    lib.kvx_translate.restype = C.c_int
    lib.kvx_plan_destroy.argtypes = [C.c_void_p]
    lib.kvx_plan_destroy.restype = None
    lib.kvx_status_string.argtypes = [C.c_int]
    lib.kvx_status_string.restype = C.c_char_p
    lib.kvx_last_hip_error.restype = C.c_int32
    lib.kvx_plan_query.argtypes = [C.c_void_p, C.POINTER(PlanInfo)]
    lib.kvx_plan_query.restype = C.c_int
    lib.kvx_staged_workspace_bytes.argtypes = [C.c_void_p, C.POINTER(IO), C.c_int32,
                                               C.POINTER(C.c_size_t)]
    lib.kvx_staged_workspace_bytes.restype = C.c_int
    lib.kvx_translate_staged.argtypes = [C.c_void_p, C.POINTER(IO), C.c_void_p, C.c_size_t,
                                         C.c_uint32, C.c_void_p]
    lib.kvx_translate_staged.restype = C.c_int
    lib.kvx_fit_create.argtypes = [C.POINTER(FitDesc), C.POINTER(C.c_void_p)]
    lib.kvx_fit_create.restype = C.c_int
    lib.kvx_fit_accumulate.argtypes = [C.c_void_p, C.POINTER(FitIO), C.c_void_p]
    lib.kvx_fit_accumulate.restype = C.c_int
    lib.kvx_fit_solve.argtypes = [C.c_void_p, C.c_double, C.c_void_p, C.c_void_p, C.c_void_p,
                                  C.c_void_p, C.c_void_p]
    lib.kvx_fit_solve.restype = C.c_int
    lib.kvx_fit_solve_noalloc.argtypes = lib.kvx_fit_solve.argtypes
    lib.kvx_fit_solve_noalloc.restype = C.c_int
    lib.kvx_fit_reset.argtypes = [C.c_void_p, C.c_void_p]
    lib.kvx_fit_reset.restype = C.c_int
    lib.kvx_fit_rows.argtypes = [C.c_void_p]
    lib.kvx_fit_rows.restype = C.c_int64
    lib.kvx_fit_query.argtypes = [C.c_void_p, C.POINTER(FitInfo)]
    lib.kvx_fit_query.restype = C.c_int
    lib.kvx_fit_destroy.argtypes = [C.c_void_p]
    lib.kvx_fit_destroy.restype = None
    lib.kvx_attn_create.argtypes = [C.POINTER(AttnDesc), C.POINTER(C.c_void_p)]
    lib.kvx_attn_create.restype = C.c_int
    lib.kvx_attn_destroy.argtypes = [C.c_void_p]
    lib.kvx_attn_destroy.restype = None
    lib.kvx_attn_append.argtypes = [C.c_void_p, C.POINTER(AttnIO), C.c_void_p]
    lib.kvx_attn_append.restype = C.c_int
    lib.kvx_attn_workspace_bytes.argtypes = [C.c_void_p, C.POINTER(C.c_size_t)]
    lib.kvx_attn_workspace_bytes.restype = C.c_int
    lib.kvx_attn_forward.argtypes = [C.c_void_p, C.POINTER(AttnIO), C.c_void_p, C.c_size_t,
                                     C.c_void_p]
    lib.kvx_attn_forward.restype = C.c_int
    lib.kvx_attn_mass.argtypes = [C.c_void_p, C.POINTER(AttnIO), C.c_void_p]
    lib.kvx_attn_mass.restype = C.c_int
    lib.kvx_attn_evict.argtypes = [C.c_void_p, C.POINTER(EvictIO), C.c_void_p]
    lib.kvx_attn_evict.restype = C.c_int
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load().kvx_status_string(int(status)).decode()


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if hasattr(t, "data_ptr"):
        return t.data_ptr()
    return int(t)


def _host_array(values, ctype):
    if values is None:
        return None
    vals = list(values)
    return (ctype * max(1, len(vals)))(*vals)


@dataclass
class ModelShape:
    n_layers: int
    n_kv_heads: int
    head_dim: int
    rope_base: float


def _model(m, inv_freq, keep) -> Model:
    inv = None
    if inv_freq is not None:
        inv = _host_array([float(x) for x in inv_freq], C.c_double)
        keep.append(inv)
    return Model(int(m.n_layers), int(m.n_kv_heads), int(m.head_dim), float(m.rope_base),
                 C.cast(inv, C.c_void_p).value if inv is not None else None)


def _marks(arr, src, keep):
    """Host outlier marks [Ls][Hs][Ds] (any array-like, nonzero = marked) as a
    uint8 buffer, or None."""
    if arr is None:
        return None
    import numpy as np
    a = np.ascontiguousarray(np.asarray(arr) != 0, dtype=np.uint8)
    want = (int(src.n_layers), int(src.n_kv_heads), int(src.head_dim))
    if a.shape != want:
        raise ValueError(f"outlier marks have shape {a.shape}, expected {want}")
    buf = (C.c_uint8 * a.size).from_buffer_copy(a.tobytes())
    keep.append(buf)
    return C.cast(buf, C.c_void_p).value


def kvx_plan_create(src, tgt, mix: int, layer_map: Sequence[int], dtype: int, w_k, w_v,
                    b_k=None, b_v=None, precision: int = KVX_PREC_BF16X2,
                    src_inv_freq=None, tgt_inv_freq=None, outlier_k=None,
                    outlier_v=None) -> int:
    """Create a plan; returns the opaque handle (an int).  ``w_k``/``w_v``/
    ``b_k``/``b_v`` are device tensors (or raw device pointers);
    ``outlier_k``/``outlier_v`` host marks [Ls][Hs][Ds] for precision
    KVX_PREC_BF16X2_OUTLIER."""
    lib = load()
    keep = []
    lm = _host_array([int(x) for x in layer_map], C.c_int32)
    keep.append(lm)
    desc = PlanDesc(_model(src, src_inv_freq, keep), _model(tgt, tgt_inv_freq, keep),
                    int(mix), C.cast(lm, C.c_void_p).value, int(dtype), _ptr(w_k), _ptr(w_v),
                    _ptr(b_k), _ptr(b_v), int(precision), _marks(outlier_k, src, keep),
                    _marks(outlier_v, src, keep))
    h = C.c_void_p()
    st = lib.kvx_plan_create(C.byref(desc), C.byref(h))
    if st != KVX_OK:
        raise KvxError(st, "kvx_plan_create")
    return h.value


def kvx_plan_create_factored(src, tgt, mix: int, layer_map: Sequence[int], dtype: int,
                             lowrank=None, mixture=None, b_k=None, b_v=None,
                             precision: int = KVX_PREC_BF16X2, src_inv_freq=None,
                             tgt_inv_freq=None) -> int:
    """Create a plan from translator factors; returns the handle.
    ``lowrank=(u_k, v_k, u_v, v_v)`` (device [Lt][dout][r], [Lt][r][din];
    ``b_k``/``b_v`` give its bias) or ``mixture=(alpha, w_k, w_v, b_k, b_v)``
    (host alpha [K]; device [K][Lt][dout][din] and fp32 [K][Lt][dout] or
    None)."""
    lib = load()
    keep = []
    lm = _host_array([int(x) for x in layer_map], C.c_int32)
    keep.append(lm)
    f = Factors()
    if lowrank is not None:
        u_k, v_k, u_v, v_v = lowrank
        f.kind = KVX_FACTORS_LOWRANK
        f.rank = int(u_k.shape[-1]) if hasattr(u_k, "shape") else 0
        f.u_k, f.v_k, f.u_v, f.v_v = _ptr(u_k), _ptr(v_k), _ptr(u_v), _ptr(v_v)
    elif mixture is not None:
        alpha, w_k, w_v, mb_k, mb_v = mixture
        al = _host_array([float(x) for x in alpha], C.c_double)
        keep.append(al)
        f.kind = KVX_FACTORS_MIXTURE
        f.n_mix = len(alpha)
        f.alpha = C.cast(al, C.c_void_p).value
        f.w_k, f.w_v, f.b_k, f.b_v = _ptr(w_k), _ptr(w_v), _ptr(mb_k), _ptr(mb_v)
    desc = PlanDesc(_model(src, src_inv_freq, keep), _model(tgt, tgt_inv_freq, keep),
                    int(mix), C.cast(lm, C.c_void_p).value, int(dtype), None, None,
                    _ptr(b_k), _ptr(b_v), int(precision))
    h = C.c_void_p()
    st = lib.kvx_plan_create_factored(C.byref(desc), C.byref(f), C.byref(h))
    if st != KVX_OK:
        raise KvxError(st, "kvx_plan_create_factored")
    return h.value


def make_io(batch: int, src_tokens: int, src_k, src_v, tgt_k, tgt_v, tgt_capacity: int,
            tgt_tokens=None, row_ptr=None, col_idx=None, weight=None,
            src_stride=(0, 0, 0, 0), tgt_stride=(0, 0, 0, 0), block_table=None,
            block_size: int = 0, max_blocks: int = 0, num_blocks: int = 0):
    """Build the kvx_io struct; returns (io, keepalive).  ``block_table``
    (device int32 [batch][max_blocks]) selects the paged target layout."""
    keep = []
    tt = None
    if tgt_tokens is not None:
        tt = _host_array([int(x) for x in tgt_tokens], C.c_int32)
        keep.append(tt)
    io = IO(int(batch), int(src_tokens), _ptr(src_k), _ptr(src_v),
            (C.c_int64 * 4)(*[int(x) for x in src_stride]),
            C.cast(tt, C.c_void_p).value if tt is not None else None,
            _ptr(row_ptr), _ptr(col_idx), _ptr(weight), _ptr(tgt_k), _ptr(tgt_v),
            (C.c_int64 * 4)(*[int(x) for x in tgt_stride]), int(tgt_capacity),
            _ptr(block_table), int(block_size), int(max_blocks), int(num_blocks))
    return io, keep


def kvx_translate(plan: int, io: IO, stream=None) -> int:
    """Enqueue a translation; ``stream`` is a torch stream, a raw hipStream_t
    (int) or None (the current torch stream)."""
    lib = load()
    if stream is None:
        import torch
        stream = torch.cuda.current_stream()
    handle = stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
    st = lib.kvx_translate(C.c_void_p(plan), C.byref(io), C.c_void_p(handle))
    if st != KVX_OK:
        raise KvxError(st, "kvx_translate")
    return st


def kvx_translate_status(plan, io: IO, stream_handle: int = 0) -> int:
    """Raw status of kvx_translate (no exception)."""
    return int(load().kvx_translate(C.c_void_p(plan), C.byref(io), C.c_void_p(stream_handle)))


def kvx_staged_workspace_bytes(plan: int, io: IO, layers: int) -> int:
    """Device bytes the staged translation's workspace needs for `layers`
    target layers of this call."""
    n = C.c_size_t(0)
    st = load().kvx_staged_workspace_bytes(C.c_void_p(plan), C.byref(io), int(layers),
                                           C.byref(n))
    if st != KVX_OK:
        raise KvxError(st, "kvx_staged_workspace_bytes")
    return int(n.value)


def kvx_translate_staged_status(plan: int, io: IO, workspace: int, workspace_bytes: int,
                                stages: int = KVX_STAGE_ALL, stream_handle: int = 0) -> int:
    """Raw status of kvx_translate_staged (no exception); `workspace` is a
    device address."""
    return int(load().kvx_translate_staged(C.c_void_p(plan), C.byref(io), C.c_void_p(workspace),
                                           int(workspace_bytes), int(stages),
                                           C.c_void_p(stream_handle)))


def kvx_translate_staged(plan: int, io: IO, workspace, workspace_bytes: Optional[int] = None,
                         stages: int = KVX_STAGE_ALL, stream=None) -> int:
    """Enqueue the staged (three-launch) translation; `workspace` is a device
    tensor (its size is passed unless `workspace_bytes` is given) or a
    device address."""
    if hasattr(workspace, "data_ptr"):
        nbytes = workspace.numel() * workspace.element_size()
        ptr = workspace.data_ptr()
    else:
        nbytes, ptr = workspace_bytes, int(workspace)
    if workspace_bytes is not None:
        nbytes = workspace_bytes
    st = kvx_translate_staged_status(plan, io, ptr, nbytes, stages, _stream_handle(stream))
    if st != KVX_OK:
        raise KvxError(st, "kvx_translate_staged")
    return st


def kvx_plan_destroy(plan: Optional[int]) -> None:
    load().kvx_plan_destroy(C.c_void_p(plan) if plan else None)


def kvx_plan_query(plan: int) -> PlanInfo:
    info = PlanInfo()
    st = load().kvx_plan_query(C.c_void_p(plan), C.byref(info))
    if st != KVX_OK:
        raise KvxError(st, "kvx_plan_query")
    return info


class Translator:
    """RAII wrapper around a plan, for the tests and the benchmark."""

    def __init__(self, src, tgt, mix, layer_map, dtype, w_k=None, w_v=None, b_k=None,
                 b_v=None, precision=KVX_PREC_BF16X2, src_inv_freq=None, tgt_inv_freq=None,
                 lowrank=None, mixture=None, outlier_k=None, outlier_v=None):
        """Dense translator from ``w_k``/``w_v``, or a composed one from
        ``lowrank`` / ``mixture`` (see kvx_plan_create_factored)."""
        self.src, self.tgt, self.mix = src, tgt, mix
        self.dtype = dtype
        self.plan = None
        if lowrank is not None or mixture is not None:
            self.plan = kvx_plan_create_factored(src, tgt, mix, layer_map, dtype, lowrank,
                                                 mixture, b_k, b_v, precision, src_inv_freq,
                                                 tgt_inv_freq)
        else:
            self.plan = kvx_plan_create(src, tgt, mix, layer_map, dtype, w_k, w_v, b_k, b_v,
                                        precision, src_inv_freq, tgt_inv_freq, outlier_k,
                                        outlier_v)

    def info(self) -> PlanInfo:
        return kvx_plan_query(self.plan)

    def __call__(self, src_k, src_v, tgt_k, tgt_v, tgt_capacity=None, tgt_tokens=None,
                 row_ptr=None, col_idx=None, weight=None, stream=None,
                 src_stride=(0, 0, 0, 0), tgt_stride=(0, 0, 0, 0), block_table=None,
                 block_size=0):
        """Contiguous targets [Lt][B][Ht][cap][Dt]; with ``block_table``
        ([B][max_blocks] int32 on the device) paged targets
        [Lt][num_blocks][Ht][block_size][Dt] (or the given strides)."""
        batch, src_tokens = int(src_k.shape[1]), int(src_k.shape[3])
        max_blocks = num_blocks = 0
        if block_table is not None:
            max_blocks, num_blocks = int(block_table.shape[1]), int(tgt_k.shape[1])
            cap = 0 if tgt_capacity is None else int(tgt_capacity)
        else:
            cap = int(tgt_k.shape[3]) if tgt_capacity is None else int(tgt_capacity)
        io, keep = make_io(batch, src_tokens, src_k, src_v, tgt_k, tgt_v, cap, tgt_tokens,
                           row_ptr, col_idx, weight, src_stride, tgt_stride, block_table,
                           block_size, max_blocks, num_blocks)
        kvx_translate(self.plan, io, stream)
        del keep

    def close(self):
        if self.plan:
            kvx_plan_destroy(self.plan)
            self.plan = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ---------------------------------------------------------------------------
# Translator fit (include/kvx_fit.h)
# ---------------------------------------------------------------------------

def _stream_handle(stream) -> int:
    if stream is None:
        import torch
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def kvx_fit_create(src, tgt, mix: int, layer_map: Sequence[int], dtype: int,
                   fit_bias: bool = True, src_inv_freq=None, tgt_inv_freq=None) -> int:
    lib = load()
    keep = []
    lm = _host_array([int(x) for x in layer_map], C.c_int32)
    keep.append(lm)
    desc = FitDesc(_model(src, src_inv_freq, keep), _model(tgt, tgt_inv_freq, keep), int(mix),
                   C.cast(lm, C.c_void_p).value, int(dtype), 1 if fit_bias else 0)
    h = C.c_void_p()
    st = lib.kvx_fit_create(C.byref(desc), C.byref(h))
    if st != KVX_OK:
        raise KvxError(st, "kvx_fit_create")
    return h.value


def make_fit_io(batch: int, src_tokens: int, src_k, src_v, tgt_k, tgt_v, tgt_capacity: int,
                tgt_tokens=None, row_ptr=None, col_idx=None, weight=None,
                src_stride=(0, 0, 0, 0), tgt_stride=(0, 0, 0, 0)):
    keep = []
    tt = None
    if tgt_tokens is not None:
        tt = _host_array([int(x) for x in tgt_tokens], C.c_int32)
        keep.append(tt)
    io = FitIO(int(batch), int(src_tokens), _ptr(src_k), _ptr(src_v),
               (C.c_int64 * 4)(*[int(x) for x in src_stride]),
               C.cast(tt, C.c_void_p).value if tt is not None else None,
               _ptr(row_ptr), _ptr(col_idx), _ptr(weight), _ptr(tgt_k), _ptr(tgt_v),
               (C.c_int64 * 4)(*[int(x) for x in tgt_stride]), int(tgt_capacity))
    return io, keep


def kvx_fit_accumulate(fit: int, io: FitIO, stream=None) -> int:
    st = load().kvx_fit_accumulate(C.c_void_p(fit), C.byref(io), C.c_void_p(_stream_handle(stream)))
    if st != KVX_OK:
        raise KvxError(st, "kvx_fit_accumulate")
    return st


def kvx_fit_solve(fit: int, lam: float, w_k, w_v, b_k=None, b_v=None, stream=None) -> int:
    st = load().kvx_fit_solve(C.c_void_p(fit), float(lam), _ptr(w_k), _ptr(w_v), _ptr(b_k),
                              _ptr(b_v), C.c_void_p(_stream_handle(stream)))
    if st != KVX_OK:
        raise KvxError(st, "kvx_fit_solve")
    return st


def kvx_fit_solve_noalloc(fit: int, lam: float, w_k, w_v, b_k=None, b_v=None,
                          stream=None) -> int:
    st = load().kvx_fit_solve_noalloc(C.c_void_p(fit), float(lam), _ptr(w_k), _ptr(w_v),
                                      _ptr(b_k), _ptr(b_v), C.c_void_p(_stream_handle(stream)))
    if st != KVX_OK:
        raise KvxError(st, "kvx_fit_solve_noalloc")
    return st


def kvx_fit_reset(fit: int, stream=None) -> int:
    st = load().kvx_fit_reset(C.c_void_p(fit), C.c_void_p(_stream_handle(stream)))
    if st != KVX_OK:
        raise KvxError(st, "kvx_fit_reset")
    return st


def kvx_fit_rows(fit: int) -> int:
    return int(load().kvx_fit_rows(C.c_void_p(fit)))


def kvx_fit_query(fit: int) -> FitInfo:
    info = FitInfo()
    st = load().kvx_fit_query(C.c_void_p(fit), C.byref(info))
    if st != KVX_OK:
        raise KvxError(st, "kvx_fit_query")
    return info


def kvx_fit_destroy(fit: Optional[int]) -> None:
    load().kvx_fit_destroy(C.c_void_p(fit) if fit else None)


class Fitter:
    """RAII wrapper around a fit, for the tests and the benchmark."""

    def __init__(self, src, tgt, mix, layer_map, dtype, fit_bias=True, src_inv_freq=None,
                 tgt_inv_freq=None):
        self.tgt, self.mix, self.src = tgt, mix, src
        self.fit_bias = fit_bias
        self.handle = kvx_fit_create(src, tgt, mix, layer_map, dtype, fit_bias, src_inv_freq,
                                     tgt_inv_freq)

    def accumulate(self, src_k, src_v, tgt_k, tgt_v, tgt_tokens=None, row_ptr=None,
                   col_idx=None, weight=None, stream=None, src_stride=(0, 0, 0, 0),
                   tgt_stride=(0, 0, 0, 0)):
        """Source caches [Ls][B][Hs][T_s][Ds], native target caches
        [Lt][B][Ht][cap][Dt] (torch device tensors)."""
        batch, src_tokens = int(src_k.shape[1]), int(src_k.shape[3])
        io, keep = make_fit_io(batch, src_tokens, src_k, src_v, tgt_k, tgt_v,
                               int(tgt_k.shape[3]), tgt_tokens, row_ptr, col_idx, weight,
                               src_stride, tgt_stride)
        kvx_fit_accumulate(self.handle, io, stream)
        del keep

    def solve(self, lam, stream=None, noalloc=False):
        """Returns fp32 device tensors (w_k, w_v, b_k, b_v); ``noalloc``
        solves through kvx_fit_solve_noalloc."""
        import torch
        Lt = self.tgt.n_layers
        dout = self.tgt.n_kv_heads * self.tgt.head_dim
        din = self.mix * self.src.n_kv_heads * self.src.head_dim
        w_k = torch.empty((Lt, dout, din), dtype=torch.float32, device="cuda")
        w_v = torch.empty_like(w_k)
        b_k = torch.empty((Lt, dout), dtype=torch.float32, device="cuda")
        b_v = torch.empty_like(b_k)
        (kvx_fit_solve_noalloc if noalloc else kvx_fit_solve)(self.handle, lam, w_k, w_v, b_k,
                                                                b_v, stream)
        return w_k, w_v, b_k, b_v

    def reset(self, stream=None):
        kvx_fit_reset(self.handle, stream)

    @property
    def rows(self) -> int:
        return kvx_fit_rows(self.handle)

    def info(self) -> FitInfo:
        return kvx_fit_query(self.handle)

    def close(self):
        if self.handle:
            kvx_fit_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ---------------------------------------------------------------------------
# Decoding on a translated cache (include/kvx_attn.h)
# ---------------------------------------------------------------------------

def kvx_attn_create(model, n_heads: int, dtype: int, softcap: float = 0.0, scale: float = 0.0,
                    inv_freq=None, pair_axis: Optional[Sequence[int]] = None,
                    n_axes: Optional[int] = None) -> int:
    """Create the attention side of a target model; returns the handle.
    ``pair_axis``: position axis of each of the head_dim/2 rotary pairs (all
    axis 0 without it); ``n_axes`` defaults to the axes it names."""
    keep = []
    axes = None
    if pair_axis is not None:
        axes = _host_array([int(x) for x in pair_axis], C.c_uint8)
        if len(pair_axis) != int(model.head_dim) // 2:
            raise ValueError(f"pair_axis has {len(pair_axis)} entries, "
                             f"expected {int(model.head_dim) // 2}")
        if n_axes is None:
            n_axes = max(int(x) for x in pair_axis) + 1
    desc = AttnDesc(_model(model, inv_freq, keep), int(n_heads), int(dtype), float(scale),
                    float(softcap), 1 if n_axes is None else int(n_axes),
                    C.cast(axes, C.c_void_p).value if axes is not None else None)
    h = C.c_void_p()
    st = load().kvx_attn_create(C.byref(desc), C.byref(h))
    if st != KVX_OK:
        raise KvxError(st, "kvx_attn_create")
    return h.value


def _plain(what, t, dtype, size=None, last=None):
    """Refuses a tensor that the library would read as something else: it takes
    ``dtype`` elements one after another, ``size`` of them at least (``last``: in
    rows of so many)."""
    if not hasattr(t, "data_ptr"):
        return  # none, or an address, which the caller answers for
    if str(t.dtype) != "torch." + dtype:
        raise ValueError(f"{what} is {t.dtype}, expected torch.{dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    if size is not None and t.numel() < size:
        raise ValueError(f"{what} has {t.numel()} elements, expected {size}")
    if last is not None and (t.dim() == 0 or t.shape[-1] != last):
        raise ValueError(f"{what} has shape {tuple(t.shape)}, expected rows of {last}")


def _one_device(tensors):
    """Refuses tensors of different devices."""
    found = {str(t.device) for t in tensors if hasattr(t, "data_ptr")}
    if len(found) > 1:
        raise ValueError(f"tensors on different devices: {sorted(found)}")


def make_cache(k, v, block_table=None, stride=(0, 0, 0, 0), block_size: Optional[int] = None,
               num_blocks: Optional[int] = None, capacity: Optional[int] = None) -> Cache:
    """The kvx_cache struct of device tensors ``k``/``v``: contiguous
    [L][B][H][capacity][D], or with ``block_table`` ([B][max_blocks] int32)
    paged [L][num_blocks][H][block_size][D].  Other layouts: give ``stride``
    and the sizes that the shape does not show."""
    if hasattr(k, "data_ptr") and hasattr(v, "data_ptr"):
        if k.element_size() != v.element_size():
            raise ValueError(f"k is {k.dtype}, v is {v.dtype}")
        if not any(stride) and not (k.is_contiguous() and v.is_contiguous() and k.shape == v.shape):
            raise ValueError("without strides, k and v must be contiguous and of one shape")
    _plain("block_table", block_table, "int32")
    _one_device((k, v, block_table))
    if block_table is None:
        c = Cache(_ptr(k), _ptr(v), (C.c_int64 * 4)(*[int(x) for x in stride]),
                  int(k.shape[3] if capacity is None else capacity), None, 0, 0, 0)
    else:
        c = Cache(_ptr(k), _ptr(v), (C.c_int64 * 4)(*[int(x) for x in stride]), 0,
                  _ptr(block_table), int(k.shape[3] if block_size is None else block_size),
                  int(block_table.shape[1]),
                  int(k.shape[1] if num_blocks is None else num_blocks))
    c.tensors = (k, v, block_table)
    return c


def _row_stride(t):
    if t is None:
        return (C.c_int64 * 2)(0, 0)
    if t.stride(-1) != 1:
        raise ValueError("head_dim must be unit-stride")
    return (C.c_int64 * 2)(t.stride(0), t.stride(1))


def make_attn_io(cache: Cache, tokens, q=None, *, layer: int = 0, q_start=None, max_new: int = 1,
                 new_q=None, new_k=None, new_v=None, pos=None, window: int = 0, prefix=None,
                 out=None, lse=None, mass_in=None, mass=None) -> AttnIO:
    """Build the kvx_attn_io struct of one layer's append, forward and mass
    calls: ``q``, ``new_q``, ``new_k``, ``new_v``, ``out`` are [rows][heads][D]
    tensors (any row and head strides); ``mass`` [B][Hkv][mass_capacity].  The
    struct keeps its tensors alive."""
    first = next(t for t in (q, new_q, new_k) if t is not None)
    batch, rows = int(tokens.shape[0]), int(first.shape[0])
    k = getattr(cache, "tensors", (None,))[0]
    for name, t in (("q", q), ("new_q", new_q), ("new_k", new_k), ("new_v", new_v), ("out", out)):
        if t is None:
            continue
        like = q if name in ("new_q", "out") else new_k if name == "new_v" else None
        if t.dim() != 3 or t.shape[0] != rows or t.shape[2] != first.shape[2] or \
                (like is not None and t.shape != like.shape):
            raise ValueError(f"{name} has shape {tuple(t.shape)}")
        if t.element_size() != (k if hasattr(k, "element_size") else first).element_size():
            raise ValueError(f"{name} is {t.dtype}, the cache is not")
    _plain("tokens", tokens, "int32")
    _plain("q_start", q_start, "int32", batch + 1)
    _plain("pos", pos, "int32", last=rows)
    _plain("prefix", prefix, "int32", batch)
    _plain("lse", lse, "float32", None if q is None else rows * int(q.shape[1]))
    _plain("mass", mass, "float32")
    _plain("mass_in", mass_in, "float32", None if mass is None else mass.numel())
    _one_device((k, tokens, q, q_start, new_q, new_k, new_v, pos, prefix, out, lse, mass_in, mass))
    io = AttnIO(batch, int(layer), rows, int(max_new),
                _ptr(q_start), _ptr(tokens), cache, _ptr(new_q), _ptr(new_k), _ptr(new_v),
                _row_stride(new_q), _row_stride(new_k), _row_stride(new_v), _ptr(pos), _ptr(q),
                _row_stride(q), int(window), _ptr(prefix), _ptr(out), _row_stride(out), _ptr(lse),
                _ptr(mass_in), _ptr(mass), 0 if mass is None else int(mass.shape[-1]))
    io.tensors = (cache, tokens, q, q_start, new_q, new_k, new_v, pos, prefix, out, lse, mass_in,
               mass)
    return io


def make_evict_io(cache: Cache, tokens, mass, kept, keep: int, *, sink: int = 0, recent: int = 0,
                  mass_out=None, tokens_out=None, dst: Optional[Cache] = None) -> EvictIO:
    """Build the kvx_evict_io struct: ``mass`` [L][B][Hkv][mass_capacity],
    ``kept`` int32 [L][B][Hkv][keep]; ``dst`` None compacts in place."""
    _plain("tokens", tokens, "int32")
    _plain("mass", mass, "float32")
    _plain("mass_out", mass_out, "float32", mass.numel())
    _plain("kept", kept, "int32", mass.numel() // max(1, int(mass.shape[-1])) * int(keep))
    _plain("tokens_out", tokens_out, "int32", int(tokens.shape[0]))
    k = getattr(cache, "tensors", (None,))[0]
    to = None if dst is None else getattr(dst, "tensors", (None,))[0]
    if hasattr(to, "element_size") and hasattr(k, "element_size") and \
            to.element_size() != k.element_size():
        raise ValueError(f"dst is {to.dtype}, the cache {k.dtype}")
    _one_device((k, to, tokens, mass, mass_out, kept, tokens_out))
    io = EvictIO(int(tokens.shape[0]), _ptr(tokens), int(keep), int(sink), int(recent), cache,
                 Cache() if dst is None else dst, _ptr(mass), _ptr(mass_out),
                 int(mass.shape[-1]), _ptr(kept), _ptr(tokens_out))
    io.tensors = (cache, tokens, mass, kept, mass_out, tokens_out, dst)
    return io


def kvx_attn_append(attn: int, io: AttnIO, stream=None) -> int:
    st = load().kvx_attn_append(attn, C.byref(io), _stream_handle(stream))
    if st != KVX_OK:
        raise KvxError(st, "kvx_attn_append")
    return st


def kvx_attn_workspace_bytes(attn: int) -> int:
    n = C.c_size_t(0)
    st = load().kvx_attn_workspace_bytes(C.c_void_p(attn), C.byref(n))
    if st != KVX_OK:
        raise KvxError(st, "kvx_attn_workspace_bytes")
    return int(n.value)


def kvx_attn_forward(attn: int, io: AttnIO, workspace, stream=None) -> int:
    """``workspace``: a device tensor of at least kvx_attn_workspace_bytes."""
    if not (workspace.is_cuda and workspace.is_contiguous()):
        raise ValueError("the workspace must be a contiguous tensor on a GPU")
    st = load().kvx_attn_forward(attn, C.byref(io), workspace.data_ptr(),
                                 workspace.numel() * workspace.element_size(),
                                 _stream_handle(stream))
    if st != KVX_OK:
        raise KvxError(st, "kvx_attn_forward")
    return st


def kvx_attn_mass(attn: int, io: AttnIO, stream=None) -> int:
    st = load().kvx_attn_mass(attn, C.byref(io), _stream_handle(stream))
    if st != KVX_OK:
        raise KvxError(st, "kvx_attn_mass")
    return st


def kvx_attn_evict(attn: int, io: EvictIO, stream=None) -> int:
    st = load().kvx_attn_evict(attn, C.byref(io), _stream_handle(stream))
    if st != KVX_OK:
        raise KvxError(st, "kvx_attn_evict")
    return st


def kvx_attn_destroy(attn: Optional[int]) -> None:
    load().kvx_attn_destroy(C.c_void_p(attn) if attn else None)


class Attention:
    """RAII wrapper around the attention side of a target model.  The calls
    take structs of make_attn_io / make_evict_io, which a decoding loop builds
    once per layer."""

    def __init__(self, model, n_heads, dtype, softcap=0.0, scale=0.0, inv_freq=None,
                 pair_axis=None, n_axes=None):
        self.handle = None
        self.model, self.n_heads, self.dtype = model, int(n_heads), int(dtype)
        self.n_axes = n_axes if n_axes is not None else \
            1 if pair_axis is None else max(int(x) for x in pair_axis) + 1
        self.handle = kvx_attn_create(model, n_heads, dtype, softcap, scale, inv_freq, pair_axis,
                                      n_axes)

    def workspace(self, io=None):
        """A workspace for forward calls: any of this handle's, one at a time, so
        that ``io`` need not be given."""
        import torch
        return torch.empty(kvx_attn_workspace_bytes(self.handle), dtype=torch.uint8,
                           device="cuda")

    def _fits(self, io):
        """Whether a struct's tensors are this model's and on a GPU; asked once of a
        struct."""
        m, tensors = self.model, getattr(io, "tensors", None)
        if tensors is None:
            return  # built by hand, which the caller answers for
        heads, d, width = int(m.n_kv_heads), int(m.head_dim), 4 if self.dtype == KVX_F32 else 2
        caches = [c for c in (tensors[0], tensors[-1]) if isinstance(c, Cache)]
        given = [t for t in tensors if hasattr(t, "data_ptr")]
        for c in caches:
            k = getattr(c, "tensors", (None,))[0]
            if not hasattr(k, "data_ptr"):
                continue
            given.append(k)
            if k.element_size() != width:
                raise ValueError(f"the cache is {k.dtype}, the model's numbers have {width} bytes")
            if not any(c.stride) and (k.dim() != 5 or (k.shape[2], k.shape[4]) != (heads, d)):
                raise ValueError(f"the cache has shape {tuple(k.shape)}, the model {heads} KV "
                                 f"heads of {d}")
        if not all(t.is_cuda for t in given):
            raise ValueError("tensors must be on a GPU")
        if isinstance(io, EvictIO):
            sets = int(m.n_layers) * io.batch * heads
            if tensors[2].numel() < sets * int(tensors[2].shape[-1]):
                raise ValueError(f"mass has shape {tuple(tensors[2].shape)}")
        else:
            _, _, q, _, new_q, new_k, new_v, pos, _, out, _, _, mass = tensors
            for name, t, n in (("q", q, self.n_heads), ("new_q", new_q, self.n_heads),
                               ("new_k", new_k, heads), ("new_v", new_v, heads),
                               ("out", out, self.n_heads)):
                if t is not None and tuple(t.shape[1:]) != (n, d):
                    raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {n} heads of {d}")
            if hasattr(pos, "numel") and pos.numel() < self.n_axes * io.rows:
                raise ValueError(f"pos has shape {tuple(pos.shape)}, expected {self.n_axes} axes")
            if hasattr(mass, "numel") and mass.numel() < io.batch * heads * int(mass.shape[-1]):
                raise ValueError(f"mass has shape {tuple(mass.shape)}")
        io.fits = self

    def append(self, io, stream=None):
        if getattr(io, "fits", None) is not self:
            self._fits(io)
        kvx_attn_append(self.handle, io, stream)

    def forward(self, io, workspace, stream=None):
        if getattr(io, "fits", None) is not self:
            self._fits(io)
        kvx_attn_forward(self.handle, io, workspace, stream)

    def mass(self, io, stream=None):
        if getattr(io, "fits", None) is not self:
            self._fits(io)
        kvx_attn_mass(self.handle, io, stream)

    def evict(self, io, stream=None):
        if getattr(io, "fits", None) is not self:
            self._fits(io)
        kvx_attn_evict(self.handle, io, stream)

    def close(self):
        if self.handle:
            kvx_attn_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
