"""ctypes binding of liblocret.so (the C ABI of include/locret.h), same names, marshalling only.

PyTorch supplies device memory and streams; every step of the chunk path runs in the library's
HIP kernels.  Importing this module fails loudly if the library has not been built
(python -m paper_2410_01805_amd.build, or __graft_entry__.build()).
"""
from __future__ import annotations

import ctypes as C
import os
import struct

# PyTorch ships its own HIP runtime (soname libamdhip64.so.7).  It must be in the process before
# liblocret.so is opened so that the dynamic loader binds the library to that same runtime:
# two runtimes in one process do not share device allocations or streams.
import torch  # noqa: F401  (memory and streams come from here as well)

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "lib", "liblocret.so")

LOCRET_OK, LOCRET_EINVAL, LOCRET_ESHAPE, LOCRET_EALIGN, LOCRET_ESTATE, LOCRET_EHIP, LOCRET_ENOMEM, LOCRET_ELIMIT = 0, -1, -2, -3, -4, -5, -6, -7
LOCRET_F32, LOCRET_BF16 = 0, 1

EXPORTS = [
    "locret_workspace_bytes", "locret_create", "locret_set_weights", "locret_set_pinned_prefix", "locret_reset", "locret_prefill_chunk",
    "locret_score", "locret_decode_step", "locret_evict_compact", "locret_cache_len", "locret_tokens_seen", "locret_cache_view",
    "locret_destroy", "locret_strerror", "locret_profile_mode", "locret_profile_enable", "locret_profile_read",
    "locret_set_head_budgets", "locret_cache_lens", "locret_score_static", "locret_cache_view_q4",
    "locret_paged_workspace_bytes", "locret_paged_plan", "locret_rope_frequencies", "locret_paged_append", "locret_paged_decode",
    "locret_paged_prefill",
]
LOCRET_PROF_STAGES = 5
LOCRET_MAX_HEAD_BUDGETS = 64
PROF_STAGE_NAMES = ("append", "attention", "retaining_head", "select", "compact")


class locret_config(C.Structure):
    _fields_ = [
        ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("chunk_max", C.c_int32),
        ("budget", C.c_int32), ("d_hidden", C.c_int32), ("rh_kv_expand", C.c_int32), ("dtype", C.c_int32),
        ("rope_mode", C.c_int32), ("rope_theta", C.c_float), ("softmax_scale", C.c_float), ("kv_bits", C.c_int32),
    ]


class locret_paged_config(C.Structure):
    _fields_ = [
        ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("dtype", C.c_int32),
        ("page_size", C.c_int32), ("n_pages", C.c_int32), ("max_reqs", C.c_int32), ("max_pages", C.c_int32),
        ("window", C.c_int32), ("n_sink", C.c_int32), ("softmax_scale", C.c_float),
    ]


LOCRET_PAGED_MAX_REQS = 4096
LOCRET_ROPE_PLAIN, LOCRET_ROPE_LINEAR, LOCRET_ROPE_BANDS, LOCRET_ROPE_RAMP, LOCRET_ROPE_FACTORS = range(5)


class locret_rope_config(C.Structure):
    _fields_ = [
        ("scaling", C.c_int32), ("rotary_dim", C.c_int32), ("theta", C.c_double), ("factor", C.c_double),
        ("original", C.c_double), ("low", C.c_double), ("high", C.c_double), ("factors", C.POINTER(C.c_double)),
    ]


def _load() -> C.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build the HIP library first "
                          "(python -m paper_2410_01805_amd.build); there is no fallback path")
    lib = C.CDLL(LIB_PATH)
    vp, i32, f32p, i32p = C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p
    lib.locret_workspace_bytes.restype = C.c_size_t
    lib.locret_workspace_bytes.argtypes = [C.POINTER(locret_config)]
    lib.locret_create.restype = C.c_int
    lib.locret_create.argtypes = [C.POINTER(locret_config), vp, C.c_size_t, C.POINTER(vp)]
    lib.locret_set_weights.restype = C.c_int
    lib.locret_set_weights.argtypes = [vp, vp, vp, vp]
    lib.locret_reset.restype = C.c_int
    lib.locret_reset.argtypes = [vp]
    lib.locret_prefill_chunk.restype = C.c_int
    lib.locret_prefill_chunk.argtypes = [vp, vp, vp, vp, i32, i32, i32, f32p, vp, f32p, i32p, vp]
    lib.locret_score.restype = C.c_int
    lib.locret_score.argtypes = [vp, vp, vp, vp, i32, f32p, vp]
    lib.locret_score_static.restype = C.c_int
    lib.locret_score_static.argtypes = [vp, vp, vp, vp, i32, f32p, vp]
    lib.locret_decode_step.restype = C.c_int
    lib.locret_decode_step.argtypes = [vp, vp, vp, vp, i32, vp, f32p, vp]
    lib.locret_evict_compact.restype = C.c_int
    lib.locret_evict_compact.argtypes = [vp, f32p, vp, vp, i32, i32, i32p, vp]
    lib.locret_profile_mode.restype = C.c_int
    lib.locret_profile_mode.argtypes = [vp, i32]
    lib.locret_set_pinned_prefix.restype = C.c_int
    lib.locret_set_pinned_prefix.argtypes = [vp, i32]
    lib.locret_set_head_budgets.restype = C.c_int
    lib.locret_set_head_budgets.argtypes = [vp, C.POINTER(i32)]
    lib.locret_cache_lens.restype = C.c_int
    lib.locret_cache_lens.argtypes = [vp, C.POINTER(i32)]
    lib.locret_cache_len.restype = C.c_int32
    lib.locret_cache_len.argtypes = [vp]
    lib.locret_tokens_seen.restype = C.c_int64
    lib.locret_tokens_seen.argtypes = [vp]
    lib.locret_cache_view.restype = C.c_int
    lib.locret_cache_view.argtypes = [vp, C.POINTER(vp), C.POINTER(vp), C.POINTER(vp), C.POINTER(vp),
                                      C.POINTER(i32), C.POINTER(i32)]
    lib.locret_cache_view_q4.restype = C.c_int
    lib.locret_cache_view_q4.argtypes = [vp, C.POINTER(vp), C.POINTER(vp), C.POINTER(i32), C.POINTER(i32),
                                         C.POINTER(i32), C.POINTER(i32)]
    cfg = C.POINTER(locret_paged_config)
    lib.locret_paged_workspace_bytes.restype = C.c_size_t
    lib.locret_paged_workspace_bytes.argtypes = [cfg]
    lib.locret_paged_plan.restype = C.c_int
    lib.locret_paged_plan.argtypes = [cfg, i32] + [vp] * 7 + [i32] + [vp] * 4
    lib.locret_rope_frequencies.restype = C.c_int
    lib.locret_rope_frequencies.argtypes = [C.POINTER(locret_rope_config), C.POINTER(C.c_double), C.POINTER(C.c_float)]
    lib.locret_paged_append.restype = C.c_int
    lib.locret_paged_append.argtypes = [cfg, i32, vp, vp, vp, vp, vp, vp, vp, i32, i32, C.c_float, vp, vp,
                                        C.c_float, vp, vp, vp, vp]
    lib.locret_paged_decode.restype = C.c_int
    lib.locret_paged_decode.argtypes = [cfg, i32] + [vp] * 8 + [C.c_size_t, vp]
    lib.locret_paged_prefill.restype = C.c_int
    lib.locret_paged_prefill.argtypes = [cfg, i32, i32] + [vp] * 9 + [C.c_size_t, vp]
    lib.locret_profile_enable.restype = C.c_int
    lib.locret_profile_enable.argtypes = [vp, i32]
    lib.locret_profile_read.restype = C.c_int
    lib.locret_profile_read.argtypes = [vp, C.POINTER(C.c_double), C.POINTER(i32)]
    lib.locret_destroy.restype = None
    lib.locret_destroy.argtypes = [vp]
    lib.locret_strerror.restype = C.c_char_p
    lib.locret_strerror.argtypes = [C.c_int]
    return lib


lib = _load()


class LocretError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {locret_strerror(code)} ({code})")


def _check(code: int, where: str) -> None:
    if code != LOCRET_OK:
        raise LocretError(code, where)


def _ptr(t) -> int | None:
    """Device address of a torch tensor (None -> NULL); ints pass through."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    assert t.is_contiguous(), "tensors cross the boundary as dense row-major buffers"
    return t.data_ptr()


def _stream(stream) -> int | None:
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream or None
    if isinstance(stream, int):
        return stream or None
    return stream.cuda_stream or None


# ---- the C ABI, one Python function per entry point -------------------------------------------------
def locret_strerror(code: int) -> str:
    return lib.locret_strerror(code).decode()


def locret_workspace_bytes(cfg: locret_config) -> int:
    return lib.locret_workspace_bytes(C.byref(cfg) if cfg is not None else None)


def locret_create(cfg: locret_config, workspace, workspace_bytes: int | None = None) -> int:
    handle = C.c_void_p()
    nbytes = workspace_bytes if workspace_bytes is not None else (
        workspace.numel() * workspace.element_size() if workspace is not None and not isinstance(workspace, int) else 0)
    _check(lib.locret_create(C.byref(cfg) if cfg is not None else None, _ptr(workspace), nbytes, C.byref(handle)),
           "locret_create")
    return handle.value


def locret_set_weights(ctx, W1, W2, stream=None) -> None:
    _check(lib.locret_set_weights(ctx, _ptr(W1), _ptr(W2), _stream(stream)), "locret_set_weights")


def locret_reset(ctx) -> None:
    _check(lib.locret_reset(ctx), "locret_reset")


def locret_prefill_chunk(ctx, q, k, v, T, n_stab, evict, scores_in, attn_out, scores_out, kept_idx_out,
                         stream=None) -> None:
    _check(lib.locret_prefill_chunk(ctx, _ptr(q), _ptr(k), _ptr(v), T, n_stab, evict, _ptr(scores_in),
                                    _ptr(attn_out), _ptr(scores_out), _ptr(kept_idx_out), _stream(stream)),
           "locret_prefill_chunk")


def locret_profile_mode(ctx, mode: int) -> None:
    _check(lib.locret_profile_mode(ctx, mode), "locret_profile_mode")


def locret_set_pinned_prefix(ctx, n_pin: int) -> None:
    _check(lib.locret_set_pinned_prefix(ctx, n_pin), "locret_set_pinned_prefix")


def locret_set_head_budgets(ctx, budgets) -> None:
    """budgets: a sequence of n_kv_heads ints (host), or None for the config's single budget."""
    arr = None if budgets is None else (C.c_int32 * len(budgets))(*[int(b) for b in budgets])
    _check(lib.locret_set_head_budgets(ctx, arr), "locret_set_head_budgets")


def locret_cache_lens(ctx, n_kv_heads: int) -> list:
    arr = (C.c_int32 * n_kv_heads)()
    _check(lib.locret_cache_lens(ctx, arr), "locret_cache_lens")
    return list(arr)


def locret_decode_step(ctx, q, k, v, with_score, attn_out, scores_out=None, stream=None) -> None:
    _check(lib.locret_decode_step(ctx, _ptr(q), _ptr(k), _ptr(v), 1 if with_score else 0, _ptr(attn_out),
                                  _ptr(scores_out), _stream(stream)), "locret_decode_step")


def locret_score(ctx, q, k, v, T, scores, stream=None) -> None:
    _check(lib.locret_score(ctx, _ptr(q), _ptr(k), _ptr(v), T, _ptr(scores), _stream(stream)), "locret_score")


def locret_score_static(ctx, q, k, v, T, scores, stream=None) -> None:
    _check(lib.locret_score_static(ctx, _ptr(q), _ptr(k), _ptr(v), T, _ptr(scores), _stream(stream)),
           "locret_score_static")


def locret_evict_compact(ctx, chunk_scores, k_chunk, v_chunk, T, n_stab, kept_idx_out, stream=None) -> None:
    _check(lib.locret_evict_compact(ctx, _ptr(chunk_scores), _ptr(k_chunk), _ptr(v_chunk), T, n_stab,
                                    _ptr(kept_idx_out), _stream(stream)), "locret_evict_compact")


def locret_cache_len(ctx) -> int:
    return lib.locret_cache_len(ctx)


def locret_tokens_seen(ctx) -> int:
    return lib.locret_tokens_seen(ctx)


def locret_cache_view(ctx) -> dict:
    K, V, S, P = C.c_void_p(), C.c_void_p(), C.c_void_p(), C.c_void_p()
    n, stride = C.c_int32(), C.c_int32()
    _check(lib.locret_cache_view(ctx, C.byref(K), C.byref(V), C.byref(S), C.byref(P), C.byref(n), C.byref(stride)),
           "locret_cache_view")
    return dict(K=K.value, V=V.value, score=S.value, orig_pos=P.value, len=n.value, row_stride=stride.value)


def locret_cache_view_q4(ctx) -> dict:
    Kq, Vq = C.c_void_p(), C.c_void_p()
    n, stride, rb, rsb = C.c_int32(), C.c_int32(), C.c_int32(), C.c_int32()
    _check(lib.locret_cache_view_q4(ctx, C.byref(Kq), C.byref(Vq), C.byref(n), C.byref(stride), C.byref(rb), C.byref(rsb)),
           "locret_cache_view_q4")
    return dict(Kq=Kq.value, Vq=Vq.value, len=n.value, row_stride=stride.value, row_bytes=rb.value,
                row_stride_bytes=rsb.value)


def locret_profile_enable(ctx, max_calls: int) -> None:
    _check(lib.locret_profile_enable(ctx, max_calls), "locret_profile_enable")


def locret_profile_read(ctx):
    """(per-stage milliseconds summed over the recorded calls, number of calls)."""
    ms = (C.c_double * LOCRET_PROF_STAGES)()
    n = C.c_int32()
    _check(lib.locret_profile_read(ctx, ms, C.byref(n)), "locret_profile_read")
    return list(ms), n.value


def locret_destroy(ctx) -> None:
    lib.locret_destroy(ctx)


# ---- many requests on one pool of pages ------------------------------------------------------------------------------
# Tensors are checked against the configuration (type, density, device: LOCRET_EINVAL; size: LOCRET_ESHAPE), and the calls go to the device that
# holds them, on that device's current stream unless one is given.  Addresses (ints) pass through unchecked.  These calls take a few
# microseconds on the GPU, so they are written out plainly: some 6 us of host time a call, 15 with a helper per check and a device context.
_PAGED_DTYPE = {LOCRET_F32: torch.float32, LOCRET_BF16: torch.bfloat16}


def _paged_ptr(where, dev, t, dtype, numel):
    """Address of a dense tensor of at least `numel` elements on device `dev` (None -> NULL; ints pass through)."""
    if t is None or t.__class__ is int:
        return t
    if t.dtype is not dtype or t.get_device() != dev or not t.is_contiguous():
        raise LocretError(LOCRET_EINVAL, where)
    if t.numel() < numel:
        raise LocretError(LOCRET_ESHAPE, where)
    return t.data_ptr()


def _paged_device(where, *tensors) -> int:
    """Index of the device of the first tensor among a call's arguments; -1 (the current device) if all are addresses."""
    for t in tensors:
        if t is not None and t.__class__ is not int:
            dev = t.get_device()
            if dev < 0:
                raise LocretError(LOCRET_EINVAL, where)
            return dev
    return -1


# The current stream's handle without a Stream object, where torch offers it.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda dev: torch.cuda.current_stream(dev).cuda_stream)


def _paged_call(where, fn, dev, args, stream) -> None:
    current = torch.cuda.current_device()
    if dev < 0 or dev == current:
        if stream is None:
            stream = _raw_stream(current)
        elif stream.__class__ is not int:
            stream = stream.cuda_stream
        rc = fn(*args, stream or None)
        if rc:
            raise LocretError(rc, where)
    else:
        with torch.cuda.device(dev):
            _paged_call(where, fn, -1, args, stream)


def locret_paged_workspace_bytes(cfg: locret_paged_config) -> int:
    return lib.locret_paged_workspace_bytes(C.byref(cfg) if cfg is not None else None)


def locret_paged_plan(cfg, n_req, lens, n_new, lens_out, block_table, free_pages, n_free, n_free_out, max_tokens, cu_new, slots, positions,
                      stream=None) -> None:
    w, i32 = "locret_paged_plan", torch.int32
    dev = _paged_device(w, cu_new, free_pages, lens, n_new, lens_out, block_table, n_free, n_free_out, slots, positions)
    args = (C.byref(cfg), n_req, _paged_ptr(w, dev, lens, i32, n_req), _paged_ptr(w, dev, n_new, i32, n_req),
            _paged_ptr(w, dev, lens_out, i32, n_req), _paged_ptr(w, dev, block_table, i32, n_req * cfg.max_pages),
            _paged_ptr(w, dev, free_pages, i32, cfg.n_pages), _paged_ptr(w, dev, n_free, i32, 1), _paged_ptr(w, dev, n_free_out, i32, 1),
            max_tokens, _paged_ptr(w, dev, cu_new, i32, n_req + 1), _paged_ptr(w, dev, slots, i32, max_tokens),
            _paged_ptr(w, dev, positions, i32, max_tokens))
    _paged_call(w, lib.locret_paged_plan, dev, args, stream)


def locret_rope_frequencies(rotary_dim, theta, scaling=LOCRET_ROPE_PLAIN, factor=1.0, original=0.0, low=0.0, high=0.0, factors=None):
    """(frequencies in radians a position, a list of rotary_dim / 2 floats; amplitude)."""
    where = "locret_rope_frequencies"
    if factors is not None and len(factors) != rotary_dim // 2:
        raise LocretError(LOCRET_EINVAL, where)
    arr = None if factors is None else (C.c_double * len(factors))(*[float(x) for x in factors])
    cfg = locret_rope_config(scaling, rotary_dim, theta, factor, original, low, high, arr)
    freq, amplitude = (C.c_double * max(1, rotary_dim // 2))(), C.c_float()
    _check(lib.locret_rope_frequencies(C.byref(cfg), freq, C.byref(amplitude)), where)
    return list(freq), amplitude.value


_strides = struct.Struct("6q").pack                        # (0.1 us; an array of c_int64 takes 0.9)


def _paged_rows(where, dev, t, dtype, T, heads, d, st, i):
    """Address of q, k or v [T][heads][d] with any strides between tokens and heads, which go to st[i], st[i + 1]."""
    if t is None or t.__class__ is int:
        return t
    if t.dtype is not dtype or t.get_device() != dev:
        raise LocretError(LOCRET_EINVAL, where)
    shape = t.shape
    if len(shape) != 3:
        raise LocretError(LOCRET_ESHAPE, where)
    n, a, b = shape
    s0, s1, s2 = t.stride()
    if n < T or a != heads or b != d or s2 != 1:
        raise LocretError(LOCRET_ESHAPE, where)
    st[i] = s0
    st[i + 1] = s1
    return t.data_ptr()


def locret_paged_append(cfg, T, q, k, v, positions, slots, freq, rotary_dim, interleaved, amplitude, q_weight, k_weight, eps, q_out, K, V,
                        stream=None, strides=None) -> None:
    """q, k, v: [T][heads][head_dim] with any strides between tokens and heads (`strides` for addresses, see include/locret.h)."""
    w, f32 = "locret_paged_append", torch.float32
    h, m, d = cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim
    pool, dtype = cfg.n_pages * m * cfg.page_size * d, _PAGED_DTYPE.get(cfg.dtype)
    dev = _paged_device(w, q, K, k, v, positions, slots, freq, q_weight, k_weight, q_out, V)
    st = [h * d, d, m * d, d, m * d, d] if strides is None else list(strides)
    if len(st) != 6:
        raise LocretError(LOCRET_EINVAL, w)
    args = (C.byref(cfg), T, _paged_rows(w, dev, q, dtype, T, h, d, st, 0), _paged_rows(w, dev, k, dtype, T, m, d, st, 2),
            _paged_rows(w, dev, v, dtype, T, m, d, st, 4), _strides(*st), _paged_ptr(w, dev, positions, torch.int32, T),
            _paged_ptr(w, dev, slots, torch.int32, T), _paged_ptr(w, dev, freq, torch.float64, rotary_dim // 2), rotary_dim,
            1 if interleaved else 0, amplitude, _paged_ptr(w, dev, q_weight, f32, d), _paged_ptr(w, dev, k_weight, f32, d), eps,
            _paged_ptr(w, dev, q_out, dtype, T * h * d), _paged_ptr(w, dev, K, dtype, pool), _paged_ptr(w, dev, V, dtype, pool))
    _paged_call(w, lib.locret_paged_append, dev, args, stream)


def locret_paged_decode(cfg, n_req, q, K, V, block_table, lens, out, lse, workspace, stream=None, workspace_bytes=None) -> None:
    w, i32 = "locret_paged_decode", torch.int32
    h, d = cfg.n_q_heads, cfg.head_dim
    n, pool, dtype = n_req * h * d, cfg.n_pages * cfg.n_kv_heads * cfg.page_size * d, _PAGED_DTYPE.get(cfg.dtype)
    dev = _paged_device(w, q, K, V, block_table, lens, out, lse, workspace)
    if workspace_bytes is None:
        workspace_bytes = workspace.nbytes if torch.is_tensor(workspace) else 0
    args = (C.byref(cfg), n_req, _paged_ptr(w, dev, q, dtype, n), _paged_ptr(w, dev, K, dtype, pool), _paged_ptr(w, dev, V, dtype, pool),
            _paged_ptr(w, dev, block_table, i32, n_req * cfg.max_pages), _paged_ptr(w, dev, lens, i32, n_req), _paged_ptr(w, dev, out, dtype, n),
            _paged_ptr(w, dev, lse, torch.float32, n_req * h), _paged_ptr(w, dev, workspace, torch.uint8, 0), workspace_bytes)
    _paged_call(w, lib.locret_paged_decode, dev, args, stream)


def locret_paged_prefill(cfg, n_req, T, q, K, V, block_table, lens, cu_new, out, lse, workspace, stream=None, workspace_bytes=None) -> None:
    w, i32 = "locret_paged_prefill", torch.int32
    h, d = cfg.n_q_heads, cfg.head_dim
    n, pool, dtype = T * h * d, cfg.n_pages * cfg.n_kv_heads * cfg.page_size * d, _PAGED_DTYPE.get(cfg.dtype)
    dev = _paged_device(w, q, K, V, block_table, lens, cu_new, out, lse, workspace)
    if workspace_bytes is None:
        workspace_bytes = workspace.nbytes if torch.is_tensor(workspace) else 0
    args = (C.byref(cfg), n_req, T, _paged_ptr(w, dev, q, dtype, n), _paged_ptr(w, dev, K, dtype, pool), _paged_ptr(w, dev, V, dtype, pool),
            _paged_ptr(w, dev, block_table, i32, n_req * cfg.max_pages), _paged_ptr(w, dev, lens, i32, n_req),
            _paged_ptr(w, dev, cu_new, i32, n_req + 1), _paged_ptr(w, dev, out, dtype, n), _paged_ptr(w, dev, lse, torch.float32, T * h),
            _paged_ptr(w, dev, workspace, torch.uint8, 0), workspace_bytes)
    _paged_call(w, lib.locret_paged_prefill, dev, args, stream)


# ---- convenience: config from a synth.Workload, a context that owns its workspace tensor -----------------
def config_from_workload(w) -> locret_config:
    return locret_config(w.h, w.h_kv, w.d, w.B, w.b, w.d_R, w.rh_kv_expand,
                         LOCRET_BF16 if w.dtype == "bf16" else LOCRET_F32, 1 if w.rope else 0,
                         float(w.theta) if w.rope else 0.0, 0.0, getattr(w, "kv_bits", 0))


class LocretLayer:
    """Owns a workspace tensor and a context; methods forward to the C ABI (no arithmetic here)."""

    def __init__(self, cfg: locret_config, device="cuda:0"):
        import torch
        self.cfg = cfg
        self.device = torch.device(device)
        nbytes = locret_workspace_bytes(cfg)
        if nbytes == 0:
            raise LocretError(LOCRET_EINVAL, "locret_workspace_bytes")
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        self.ctx = locret_create(cfg, self.workspace)
        self.tdtype = torch.bfloat16 if cfg.dtype == LOCRET_BF16 else torch.float32

    def set_weights(self, W1, W2):
        locret_set_weights(self.ctx, W1, W2)

    def reset(self):
        locret_reset(self.ctx)

    def prefill_chunk(self, q, k, v, n_stab, evict=True, scores_in=None, want_scores=True, want_kept=True):
        import torch
        T = q.shape[0]
        out = torch.empty_like(q)
        sc = torch.empty((self.cfg.n_kv_heads, T), dtype=torch.float32, device=self.device) if want_scores else None
        kept = torch.full((self.cfg.n_kv_heads, self.cfg.budget), -1, dtype=torch.int32, device=self.device) \
            if (want_kept and evict) else None
        locret_prefill_chunk(self.ctx, q, k, v, T, n_stab, 1 if evict else 0, scores_in, out, sc, kept)
        return out, sc, kept

    def score(self, q, k, v):
        import torch
        T = q.shape[0]
        sc = torch.empty((self.cfg.n_kv_heads, T), dtype=torch.float32, device=self.device)
        locret_score(self.ctx, q, k, v, T, sc)
        return sc

    def set_pinned_prefix(self, n_pin: int) -> None:
        locret_set_pinned_prefix(self.ctx, n_pin)

    def set_head_budgets(self, budgets) -> None:
        if budgets is not None and len(budgets) != self.cfg.n_kv_heads:
            raise LocretError(LOCRET_EINVAL, "locret_set_head_budgets")
        locret_set_head_budgets(self.ctx, budgets)

    @property
    def cache_lens(self) -> list:
        return locret_cache_lens(self.ctx, self.cfg.n_kv_heads)

    def decode_step(self, q, k, v, with_score=False):
        """One generated token: q [1][h][d], k, v [1][h_kv][d] -> (attn_out [1][h][d], scores [h_kv] or None)."""
        import torch
        out = torch.empty_like(q)
        sc = torch.empty((self.cfg.n_kv_heads,), dtype=torch.float32, device=self.device) if with_score else None
        locret_decode_step(self.ctx, q, k, v, with_score, out, sc)
        return out, sc

    def evict_compact(self, scores, k, v, n_stab):
        import torch
        kept = torch.full((self.cfg.n_kv_heads, self.cfg.budget), -1, dtype=torch.int32, device=self.device)
        locret_evict_compact(self.ctx, scores, k, v, k.shape[0], n_stab, kept)
        return kept

    @property
    def cache_len(self) -> int:
        return locret_cache_len(self.ctx)

    def cache_tensors(self):
        """Copies of the live cache (K, V in storage dtype, score float32, orig_pos int32), each
        [h_kv][len][...], taken from the workspace through locret_cache_view (with head-wise budgets
        len is the longest head's: row m is meaningful up to cache_lens[m])."""
        import torch
        view = locret_cache_view(self.ctx)
        base = self.workspace.data_ptr()
        h_kv, d, n, stride = self.cfg.n_kv_heads, self.cfg.head_dim, view["len"], view["row_stride"]
        es = 2 if self.cfg.dtype == LOCRET_BF16 else 4

        def grab(addr, dtype, inner, esize):
            off = addr - base
            raw = self.workspace[off: off + h_kv * stride * inner * esize].view(dtype)
            return raw.view(h_kv, stride, inner)[:, :n].clone()
        K = grab(view["K"], self.tdtype, d, es) if view["K"] else None
        V = grab(view["V"], self.tdtype, d, es)
        S = grab(view["score"], torch.float32, 1, 4)[..., 0]
        P = grab(view["orig_pos"], torch.int32, 1, 4)[..., 0]
        if self.cfg.kv_bits:
            # packed rows instead of K, V: uint8 [h_kv][len][row_bytes] (padding bytes dropped)
            vq = locret_cache_view_q4(self.ctx)
            rb, rsb = vq["row_bytes"], vq["row_stride_bytes"]
            Kq = grab(vq["Kq"], torch.uint8, rsb, 1)[..., :rb].contiguous()
            Vq = grab(vq["Vq"], torch.uint8, rsb, 1)[..., :rb].contiguous()
            return Kq, Vq, S, P
        return K, V, S, P

    def close(self):
        if self.ctx:
            locret_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class PagedCache:
    """Owns one layer's pool of pages, its bookkeeping and a workspace; methods forward to the C ABI (no arithmetic here).

    A serving step: plan() gives the new tokens' places, append() brings their queries, keys and values there, decode() (one new token for each
    of the first n_req requests, row r of q is that of request r) or prefill() (any other step: chunks, requests that wait or are finished,
    whose packed tokens it finds by cu_new) attends.  `rope`: arguments of locret_rope_frequencies, None for no rotation."""

    def __init__(self, cfg: locret_paged_config, device="cuda:0", rope=None, interleaved=False):
        self.cfg, self.device = cfg, torch.device(device)
        nbytes = locret_paged_workspace_bytes(cfg)
        if nbytes == 0:
            raise LocretError(LOCRET_EINVAL, "locret_paged_workspace_bytes")
        self.tdtype = _PAGED_DTYPE[cfg.dtype]
        ints = dict(dtype=torch.int32, device=self.device)
        pool = (cfg.n_pages, cfg.n_kv_heads, cfg.page_size, cfg.head_dim)
        self.K, self.V = torch.empty(pool, dtype=self.tdtype, device=self.device), torch.empty(pool, dtype=self.tdtype, device=self.device)
        self.device = ints["device"] = self.K.device       # with its number, also where none was given
        self.block_table = torch.zeros((cfg.max_reqs, cfg.max_pages), **ints)
        self.lens = torch.zeros(cfg.max_reqs, **ints)
        self.free_pages = torch.arange(cfg.n_pages - 1, -1, -1, **ints)
        self.n_free = torch.full((1,), cfg.n_pages, **ints)
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        self.rotary_dim, self.interleaved, self.amplitude, self.freq = 0, interleaved, 1.0, None
        if rope is not None:
            freq, self.amplitude = locret_rope_frequencies(**rope)
            self.rotary_dim, self.freq = rope["rotary_dim"], torch.tensor(freq, dtype=torch.float64, device=self.device)

    def plan(self, n_new, max_tokens: int):
        """n_new int32 [n_req] on the device (-1: finished) -> (cu_new, slots, positions); lengths and pages are brought up to date."""
        n, ints = n_new.shape[0], dict(dtype=torch.int32, device=self.device)
        cu, slots, positions = torch.empty(n + 1, **ints), torch.empty(max_tokens, **ints), torch.empty(max_tokens, **ints)
        locret_paged_plan(self.cfg, n, self.lens, n_new, self.lens, self.block_table, self.free_pages, self.n_free, self.n_free, max_tokens,
                          cu, slots, positions)
        return cu, slots, positions

    def append(self, q, k, v, positions, slots, q_weight=None, k_weight=None, eps=1e-6):
        """q [T][h][d], k, v [T][h_kv][d] -> the normed and rotated queries."""
        out = torch.empty(q.shape, dtype=q.dtype, device=self.device)
        locret_paged_append(self.cfg, q.shape[0], q, k, v, positions, slots, self.freq, self.rotary_dim, self.interleaved, self.amplitude,
                            q_weight, k_weight, eps, out, self.K, self.V)
        return out

    def decode(self, q, want_lse=False):
        out = torch.empty_like(q)
        lse = torch.empty(q.shape[:2], dtype=torch.float32, device=self.device) if want_lse else None
        locret_paged_decode(self.cfg, q.shape[0], q, self.K, self.V, self.block_table, self.lens, out, lse, self.workspace)
        return (out, lse) if want_lse else out

    def prefill(self, q, cu_new, want_lse=False):
        out = torch.zeros_like(q)
        lse = torch.zeros(q.shape[:2], dtype=torch.float32, device=self.device) if want_lse else None
        locret_paged_prefill(self.cfg, cu_new.shape[0] - 1, q.shape[0], q, self.K, self.V, self.block_table, self.lens, cu_new, out, lse,
                             self.workspace)
        return (out, lse) if want_lse else out

    def adopt(self, layer: "LocretLayer", r: int) -> None:
        """The retained cache of `layer` (its heads equally long, rows not packed) becomes the next units of request r, which generation
        then continues: on an empty request, unit i sits at position i here as there.  Waits for the device: where the request's row of
        the block table is too short (LOCRET_ESHAPE) or too few pages are free (LOCRET_ENOMEM) the pool stays as it was."""
        c, n = layer.cfg, layer.cache_len
        if (c.n_kv_heads, c.head_dim, c.dtype) != (self.cfg.n_kv_heads, self.cfg.head_dim, self.cfg.dtype) or not 0 <= r < self.cfg.max_reqs:
            raise LocretError(LOCRET_ESHAPE, "adopt")
        if c.kv_bits or len(set(layer.cache_lens)) != 1 or layer.workspace.device != self.device:
            raise LocretError(LOCRET_ESTATE, "adopt")
        n_new = torch.zeros(r + 1, dtype=torch.int32, device=self.device)
        n_new[r] = n
        cu_new, slots, positions = self.plan(n_new, n)
        if cu_new[-1].item() != n:
            row = self.cfg.max_pages * self.cfg.page_size
            raise LocretError(LOCRET_ESHAPE if self.lens[r].item() + n > row else LOCRET_ENOMEM, "adopt")
        view = locret_cache_view(layer.ctx)
        row, d = view["row_stride"], c.head_dim
        locret_paged_append(self.cfg, n, None, view["K"], view["V"], positions, slots, self.freq, self.rotary_dim, self.interleaved, self.amplitude,
                            None, None, 0.0, None, self.K, self.V, strides=[0, 0, d, row * d, d, row * d])
