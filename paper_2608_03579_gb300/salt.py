"""ctypes binding of ``libsalt.so`` (the C ABI in ``include/salt.h``).

Argument marshalling only: every function below forwards to the C function
of the same name; all work runs in the library's CUDA kernels.  Tensors are
passed by ``data_ptr()``; streams are ``torch.cuda.Stream`` objects (or
None for the current stream).  A non-OK status raises ``SaltError``.  If
the library has not been built, importing this module raises ImportError:
there is no fallback.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsalt.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: build it with paper_2608_03579_gb300._build.build() "
                      "(nvcc, sm_103a); there is no CPU fallback")

_lib = ctypes.CDLL(LIB_PATH)

STATUS = {
    0: "SALT_OK", 1: "SALT_ERR_INVALID_ARG", 2: "SALT_ERR_OOM", 3: "SALT_ERR_NOT_PINNED_HOST",
    4: "SALT_ERR_DOMAIN_NOT_PINNED", 5: "SALT_ERR_SLOT_RANGE", 6: "SALT_ERR_RANK", 7: "SALT_ERR_LAYER_RANGE",
    8: "SALT_ERR_ALIGN", 9: "SALT_ERR_BAD_BLOB", 10: "SALT_ERR_DEVICE_IDS", 11: "SALT_ERR_TIMEOUT",
    12: "SALT_ERR_CUDA", 13: "SALT_ERR_SLOT_EMPTY", 14: "SALT_ERR_TOO_MANY_TOKENS", 15: "SALT_ERR_DOMAIN_RANGE",
    16: "SALT_ERR_STALE_SEGMENTS", 17: "SALT_ERR_NOT_BUILT", 18: "SALT_ERR_GAMMA_RANGE",
}
SALT_BLOB_HEADER_BYTES = 256
SALT_MAX_TOKENS = 16384
SALT_MAX_GROUP = 8
SALT_MAX_GAMMA_BINS = 16
SALT_MAX_RESIDUAL_RANK = 80
SALT_W_IN_OUT = 0
SALT_W_OUT_IN = 1


class SaltError(RuntimeError):
    def __init__(self, status: int, message: str = ""):
        self.status = status
        self.name = STATUS.get(status, f"status {status}")
        super().__init__(f"{self.name}: {message}" if message else self.name)


class salt_config(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("d_in", ctypes.POINTER(ctypes.c_int32)),
                ("d_out", ctypes.POINTER(ctypes.c_int32)), ("n_domains", ctypes.c_int32),
                ("rc_max", ctypes.c_int32), ("n_slots", ctypes.c_int32), ("r_max", ctypes.c_int32),
                ("max_tokens", ctypes.c_int32), ("device", ctypes.c_int32)]


class salt_align_pair(ctypes.Structure):
    _fields_ = [("At", ctypes.c_void_p), ("B", ctypes.c_void_p), ("At_c", ctypes.c_void_p),
                ("B_c", ctypes.c_void_p), ("r", ctypes.c_int32), ("rc", ctypes.c_int32),
                ("d_in", ctypes.c_int32), ("d_out", ctypes.c_int32), ("s", ctypes.c_float),
                ("s_c", ctypes.c_float)]


class salt_ctx_info(ctypes.Structure):
    _fields_ = [("arena_bytes", ctypes.c_int64), ("pool_bytes", ctypes.c_int64), ("slot_stride", ctypes.c_int64),
                ("apply_ctas", ctypes.c_int32), ("k_splits_max", ctypes.c_int32),
                ("apply_smem_bytes", ctypes.c_int32), ("block_tokens", ctypes.c_int32),
                ("block_users", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class salt_base_shape(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int32) for k in ("cta_group", "tile_cols", "k_splits", "shrink_ctas", "units", "clusters")]


class _kv_config(ctypes.Structure):
    _fields_ = ([(k, ctypes.c_int32) for k in ("n_layers", "n_pages", "n_kv_heads", "page_tokens", "head_dim")]
                + [(k, ctypes.c_void_p) for k in ("k", "v", "k_exp", "v_exp")])


class _rope_config(ctypes.Structure):
    _fields_ = ([(k, ctypes.c_int32) for k in ("head_dim", "rot_dim", "interleaved")] + [("inv_freq", ctypes.c_void_p)]
                + [(k, ctypes.c_float) for k in ("scale", "eps", "norm_offset")])


class _attn_config(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int32) for k in ("n_heads", "max_seqs", "max_tokens", "max_pages", "max_groups")]


class _attn_batch(ctypes.Structure):
    _fields_ = [("n_seqs", ctypes.c_int32), ("q_len", ctypes.c_void_p), ("kv_len", ctypes.c_void_p),
                ("page_ptr", ctypes.c_void_p), ("pages", ctypes.c_void_p), ("group", ctypes.c_void_p),
                ("n_groups", ctypes.c_int32), ("group_len", ctypes.c_void_p), ("group_page_ptr", ctypes.c_void_p),
                ("group_pages", ctypes.c_void_p)]


class _attn_shape(ctypes.Structure):
    _fields_ = ([(k, ctypes.c_int32) for k in ("wide_items", "wide_tiles", "wide_ctas", "narrow_items", "narrow_tiles",
                                               "narrow_ctas", "combined")] + [("workspace_bytes", ctypes.c_int64)])


_vp, _i32, _i64, _f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
_SIGS = {
    "salt_abi_version": (_i32, []),
    "salt_status_string": (ctypes.c_char_p, [ctypes.c_int]),
    "salt_ctx_create": (ctypes.c_int, [ctypes.POINTER(salt_config), ctypes.POINTER(_vp)]),
    "salt_ctx_destroy": (None, [_vp]),
    "salt_last_error": (ctypes.c_char_p, [_vp]),
    "salt_ctx_get_info": (ctypes.c_int, [_vp, ctypes.POINTER(salt_ctx_info)]),
    "salt_centroid_pin": (ctypes.c_int, [_vp, _i32, _i32, _vp, _vp, _f32]),
    "salt_residual_blob_bytes": (_i64, [ctypes.POINTER(salt_config), _i32]),
    "salt_residual_blob_pack": (ctypes.c_int, [ctypes.POINTER(salt_config), _i32, _f32, _vp, _vp, _vp, _i64]),
    "salt_residual_load": (ctypes.c_int, [_vp, _i32, _vp, _vp]),
    "salt_residual_load_batch": (ctypes.c_int, [_vp, _i32, _vp, _vp, _vp]),
    "salt_segments_create": (ctypes.c_int, [_vp, ctypes.POINTER(_vp)]),
    "salt_segments_destroy": (None, [_vp]),
    "salt_build_segments": (ctypes.c_int, [_vp, _vp, _vp, _vp, _i32, _vp]),
    "salt_segments_export": (ctypes.c_int, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp]),
    "salt_lora_apply": (ctypes.c_int, [_vp, _vp, _i32, _vp, _vp, _vp]),
    "salt_lora_apply_grouped": (ctypes.c_int, [_vp, _vp, _i32, _vp, _vp, _vp, _vp]),
    "salt_lora_apply_static": (ctypes.c_int, [_vp, _vp, _i32, _vp, _vp, _vp]),
    "salt_get_device_error": (ctypes.c_int, [_vp, _vp, ctypes.POINTER(ctypes.c_uint32)]),
    "salt_selftest_wait_timeout": (ctypes.c_int, [_vp, _vp]),
    "salt_host_alloc": (_vp, [_i64]),
    "salt_host_free": (None, [_vp]),
    "salt_residual_blob_concat": (ctypes.c_int, [ctypes.POINTER(salt_config), _i32, _vp, _vp, _f32, _i32, _vp, _vp,
                                                 _f32, _vp, _i64]),
    "salt_centroid_fold": (ctypes.c_int, [_vp, _i32, _i32, _f32, _vp, _i32, _vp]),
    "salt_build_segments_gamma": (ctypes.c_int, [_vp, _vp, _vp, _vp, _vp, _i32, _i32, _vp, _vp]),
    "salt_segments_export_gamma": (ctypes.c_int, [_vp, _vp, _vp, _vp]),
    "salt_align_loss": (ctypes.c_int, [_i32, ctypes.POINTER(salt_align_pair), _f32, _vp, _vp, _vp]),
    "salt_host_pipe_create": (ctypes.c_int, [_vp, _i32, _i64, ctypes.POINTER(_vp)]),
    "salt_host_pipe_destroy": (None, [_vp]),
    "salt_lora_apply_host": (ctypes.c_int, [_vp, _vp, _i32, _vp, _vp, _vp, _vp]),
    "salt_host_pipe_wait": (ctypes.c_int, [_vp, _vp]),
    "salt_guard_check": (ctypes.c_int, [_vp, _vp, ctypes.POINTER(ctypes.c_int32)]),
    "salt_lora_apply_with_base": (ctypes.c_int, [_vp, _vp, _i32, _vp, _vp, _i32, _vp, _vp]),
    "salt_base_get_shape": (ctypes.c_int, [_vp, _vp, _i32, ctypes.POINTER(salt_base_shape)]),
    "salt_fold_plan_create": (ctypes.c_int, [_vp, _i32, _i32, _vp, _vp, _i32, ctypes.POINTER(_vp)]),
    "salt_fold_plan_run": (ctypes.c_int, [_vp, _f32, _vp]),
    "salt_fold_plan_destroy": (None, [_vp]),
    "salt_kv_create": (ctypes.c_int, [_vp, ctypes.POINTER(_kv_config), ctypes.POINTER(_vp)]),
    "salt_kv_destroy": (None, [_vp]),
    "salt_kv_write": (ctypes.c_int, [_vp, _i32, _i32, _vp, _i64, _vp, _i64, _vp, _vp]),
    "salt_kv_read": (ctypes.c_int, [_vp, _i32, _i32, _vp, _vp, _i64, _vp, _i64, _vp]),
    "salt_rope_create": (ctypes.c_int, [_vp, ctypes.POINTER(_rope_config), ctypes.POINTER(_vp)]),
    "salt_rope_destroy": (None, [_vp]),
    "salt_rope_apply": (ctypes.c_int, [_vp, _i32, _vp, _i64, _i32, _vp, _i64, _i32, _vp, _vp, _vp, _vp, _i64, _vp, _i64, _vp]),
    "salt_rope_write": (ctypes.c_int, [_vp, _vp, _i32, _i32, _vp, _i64, _i32, _vp, _i64, _vp, _i64, _vp, _vp, _vp, _vp, _vp,
                                       _i64, _vp]),
    "salt_attn_create": (ctypes.c_int, [_vp, ctypes.POINTER(_attn_config), ctypes.POINTER(_vp)]),
    "salt_attn_destroy": (None, [_vp]),
    "salt_attn_build": (ctypes.c_int, [_vp, ctypes.POINTER(_attn_batch), _vp]),
    "salt_attn_get_shape": (ctypes.c_int, [_vp, ctypes.POINTER(_attn_shape)]),
    "salt_attn_run": (ctypes.c_int, [_vp, _i32, _vp, _i64, _f32, _vp, _i64, _vp, _vp]),
    "salt_attn_track": (ctypes.c_int, [_vp]),
    "salt_attn_weights": (ctypes.c_int, [_vp, _i32, _vp, _i64, _vp, _f32, _f32, _vp, _vp]),
    "salt_attn_evict": (ctypes.c_int, [_vp, _i32, _i32, _vp, _i32, _i32, _vp, _vp, _vp, _i64, _vp]),
    "salt_verify_drafts": (ctypes.c_int, [_vp, _i32, _i32, _i32, _vp, _vp, _vp, _i64, _vp, _i64, _vp, _vp, _vp, _vp,
                                          _vp]),
}
for _name, (_res, _args) in _SIGS.items():
    _f = getattr(_lib, _name)
    _f.restype = _res
    _f.argtypes = _args


def _check(status: int, ctx=None):
    if status != 0:
        msg = _lib.salt_last_error(ctx).decode() if ctx else ""
        raise SaltError(status, msg)


_raw_stream = None


def _current_stream() -> int:
    """The current stream's handle; by torch's own cheap accessor where it has
    one (a tenth of the time of torch.cuda.current_stream())."""
    global _raw_stream
    if _raw_stream is None:
        import torch
        get, device = getattr(torch._C, "_cuda_getCurrentRawStream", None), torch.cuda.current_device
        _raw_stream = (lambda: torch.cuda.current_stream().cuda_stream) if get is None else (lambda: get(device()))
    return _raw_stream()


def _stream(stream) -> int | None:
    if stream is None:
        return _current_stream()
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _ptr(a) -> int | None:
    if a is None:
        return None
    if isinstance(a, np.ndarray):
        assert a.flags.c_contiguous
        return a.ctypes.data
    if isinstance(a, int):
        return a
    assert a.is_contiguous()
    return a.data_ptr()


def make_config(d_in, d_out, n_domains=0, rc_max=0, n_slots=0, r_max=1, max_tokens=1, device=0):
    """A salt_config plus the arrays it points to (kept alive on the object)."""
    din = np.ascontiguousarray(d_in, dtype=np.int32)
    dout = np.ascontiguousarray(d_out, dtype=np.int32)
    c = salt_config(len(din), din.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)),
                    dout.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)), n_domains, rc_max, n_slots, r_max,
                    max_tokens, device)
    c._keep = (din, dout)
    return c


def salt_abi_version() -> int:
    return int(_lib.salt_abi_version())


def salt_status_string(status: int) -> str:
    return _lib.salt_status_string(status).decode()


def salt_ctx_create(d_in, d_out, n_domains, rc_max, n_slots, r_max, max_tokens, device=0) -> int:
    cfg = make_config(d_in, d_out, n_domains, rc_max, n_slots, r_max, max_tokens, device)
    out = _vp()
    _check(_lib.salt_ctx_create(ctypes.byref(cfg), ctypes.byref(out)))
    return out.value


def salt_ctx_destroy(ctx) -> None:
    _lib.salt_ctx_destroy(ctx)


def salt_last_error(ctx) -> str:
    return _lib.salt_last_error(ctx).decode()


def salt_ctx_get_info(ctx) -> dict:
    info = salt_ctx_info()
    _check(_lib.salt_ctx_get_info(ctx, ctypes.byref(info)), ctx)
    return {k: getattr(info, k) for (k, _) in salt_ctx_info._fields_ if k != "reserved"}


def salt_centroid_pin(ctx, domain: int, rc: int, At_c, B_c, s_c: float) -> None:
    _check(_lib.salt_centroid_pin(ctx, domain, rc, _ptr(At_c), _ptr(B_c), float(s_c)), ctx)


def salt_residual_blob_bytes(d_in, d_out, rank: int) -> int:
    return int(_lib.salt_residual_blob_bytes(ctypes.byref(make_config(d_in, d_out)), rank))


def salt_residual_blob_pack(d_in, d_out, rank: int, s_u: float, At_u, B_u, blob, blob_bytes: int) -> None:
    cfg = make_config(d_in, d_out)
    _check(_lib.salt_residual_blob_pack(ctypes.byref(cfg), rank, float(s_u), _ptr(At_u), _ptr(B_u),
                                        _ptr(blob), blob_bytes))


def salt_residual_blob_concat(d_in, d_out, rc: int, At_c, B_c, s_c: float, rank: int, At_u, B_u, s_u: float,
                              blob, blob_bytes: int) -> None:
    """Blob of rank rc + rank holding the scaled centroid and the residual as
    one ordinary adapter (the long-tail form)."""
    cfg = make_config(d_in, d_out)
    _check(_lib.salt_residual_blob_concat(ctypes.byref(cfg), rc, _ptr(At_c), _ptr(B_c), float(s_c), rank,
                                          _ptr(At_u), _ptr(B_u), float(s_u), _ptr(blob), blob_bytes))


def salt_centroid_fold(ctx, domain: int, layer: int, gamma: float, W, layout: int = SALT_W_IN_OUT,
                       stream=None) -> None:
    """W += gamma * s_c(domain) * A_c B_c in place (W a CUDA bf16 tensor)."""
    _check(_lib.salt_centroid_fold(ctx, domain, layer, float(gamma), _ptr(W), layout, _stream(stream)), ctx)


class FoldPlan:
    """A salt_fold_plan handle; keeps the weight tensors alive with it."""

    def __init__(self, ctx, handle, weights):
        self.ctx, self.handle, self._weights = ctx, handle, weights


def salt_fold_plan_create(ctx, domain: int, layers, weights, layout: int = SALT_W_IN_OUT) -> FoldPlan:
    """One launch that folds domain's centroid into every weight (CUDA bf16
    tensors) of `weights`, weights[i] being layer layers[i]'s."""
    n = len(layers)
    if len(weights) != n:
        raise ValueError("one weight per layer")
    ls = (ctypes.c_int32 * max(1, n))(*[int(l) for l in layers])
    ws = (_vp * max(1, n))(*[_ptr(w) for w in weights])
    h = _vp()
    _check(_lib.salt_fold_plan_create(ctx, int(domain), n, ls, ws, int(layout), ctypes.byref(h)), ctx)
    return FoldPlan(ctx, h, list(weights))


def salt_fold_plan_run(plan: FoldPlan, gamma: float, stream=None) -> None:
    _check(_lib.salt_fold_plan_run(plan.handle, float(gamma), _stream(stream)), plan.ctx)


def salt_fold_plan_destroy(plan: FoldPlan) -> None:
    if plan is not None and plan.handle:
        _lib.salt_fold_plan_destroy(plan.handle)
        plan.handle = None


def salt_align_pairs(pairs):
    """The C array of salt_align_pair for a sequence of dicts with At, B,
    At_c, B_c (CUDA bf16 tensors or device addresses), r, rc, d_in, d_out,
    s, s_c; reusable across calls while the tensors live."""
    arr = (salt_align_pair * max(1, len(pairs)))()
    for i, q in enumerate(pairs):
        arr[i] = salt_align_pair(_ptr(q["At"]), _ptr(q["B"]), _ptr(q["At_c"]), _ptr(q["B_c"]), int(q["r"]),
                                 int(q["rc"]), int(q["d_in"]), int(q["d_out"]), float(q["s"]), float(q["s_c"]))
    arr._n = len(pairs)
    return arr


def salt_align_loss(pairs, eps: float, loss, cosine=None, stream=None) -> None:
    """pairs: a sequence of dicts (see salt_align_pairs) or its prepared
    array.  loss / cosine: CUDA float32 tensors of len(pairs) (cosine may be
    None)."""
    arr = pairs if hasattr(pairs, "_n") else salt_align_pairs(pairs)
    _check(_lib.salt_align_loss(arr._n, arr, float(eps), _ptr(loss), _ptr(cosine), _stream(stream)))


class HostBuffer:
    """Huge-page-backed page-locked host memory from salt_host_alloc, viewed
    as a uint8 torch tensor (``.tensor``); freed by ``close()`` or on
    garbage collection."""

    def __init__(self, nbytes: int):
        import torch
        self.ptr = _lib.salt_host_alloc(int(nbytes))
        if not self.ptr:
            raise SaltError(2, f"salt_host_alloc({nbytes}) failed")
        self.nbytes = int(nbytes)
        arr = np.ctypeslib.as_array((ctypes.c_uint8 * self.nbytes).from_address(self.ptr))
        self.tensor = torch.from_numpy(arr)

    def close(self):
        if self.ptr:
            self.tensor = None
            _lib.salt_host_free(self.ptr)
            self.ptr = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def salt_host_alloc(nbytes: int) -> HostBuffer:
    return HostBuffer(nbytes)


def salt_host_free(buf) -> None:
    """Release a HostBuffer (or a raw pointer from the C call)."""
    if isinstance(buf, HostBuffer):
        buf.close()
    elif buf:
        _lib.salt_host_free(buf)


def salt_residual_load(ctx, slot: int, host_blob, stream=None) -> None:
    _check(_lib.salt_residual_load(ctx, slot, _ptr(host_blob), _stream(stream)), ctx)


def salt_residual_load_batch(ctx, slots, host_blobs, stream=None) -> None:
    """The loads of salt_residual_load for each (slot, blob) pair, in one call."""
    n = len(slots)
    if len(host_blobs) != n:
        raise ValueError("one blob per slot")
    sl = (_i32 * max(n, 1))(*[int(x) for x in slots])
    bl = (_vp * max(n, 1))(*[_ptr(b) for b in host_blobs])
    _check(_lib.salt_residual_load_batch(ctx, n, sl, bl, _stream(stream)), ctx)


def salt_segments_create(ctx) -> int:
    out = _vp()
    _check(_lib.salt_segments_create(ctx, ctypes.byref(out)), ctx)
    return out.value


def salt_segments_destroy(seg) -> None:
    _lib.salt_segments_destroy(seg)


def salt_build_segments(ctx, seg, domain_ids, slot_ids, n_tokens: int | None = None, stream=None) -> None:
    """ids: numpy / CPU tensors (host path) or CUDA int32 tensors (device path)."""
    if isinstance(domain_ids, np.ndarray):
        domain_ids = np.ascontiguousarray(domain_ids, dtype=np.int32)
        slot_ids = np.ascontiguousarray(slot_ids, dtype=np.int32)
    n = len(domain_ids) if n_tokens is None else n_tokens
    _check(_lib.salt_build_segments(ctx, seg, _ptr(domain_ids), _ptr(slot_ids), n, _stream(stream)), ctx)


def salt_build_segments_gamma(ctx, seg, domain_ids, gamma_bins, slot_ids, gamma, n_tokens: int | None = None,
                              stream=None) -> None:
    """salt_build_segments with per-token gamma bins; gamma: the bins' values."""
    if isinstance(domain_ids, np.ndarray):
        domain_ids = np.ascontiguousarray(domain_ids, dtype=np.int32)
        slot_ids = np.ascontiguousarray(slot_ids, dtype=np.int32)
    if isinstance(gamma_bins, np.ndarray):
        gamma_bins = np.ascontiguousarray(gamma_bins, dtype=np.int32)
    g = np.ascontiguousarray(gamma, dtype=np.float32)
    n = len(domain_ids) if n_tokens is None else n_tokens
    _check(_lib.salt_build_segments_gamma(ctx, seg, _ptr(domain_ids), _ptr(gamma_bins), _ptr(slot_ids), n,
                                          len(g), g.ctypes.data if len(g) else None, _stream(stream)), ctx)


def salt_segments_export_gamma(ctx, seg, max_tokens: int) -> dict:
    """The gamma bins of the domain runs and user runs of the last build."""
    counts = salt_segments_export(ctx, seg, max_tokens)["counts"]
    dg = np.zeros(max_tokens + 1, dtype=np.int32)
    ug = np.zeros(max_tokens + 1, dtype=np.int32)
    _check(_lib.salt_segments_export_gamma(ctx, seg, dg.ctypes.data, ug.ctypes.data), ctx)
    return {"dseg_gbin": dg[:int(counts[1])], "useg_gbin": ug[:int(counts[2])]}


def salt_segments_export(ctx, seg, max_tokens: int) -> dict:
    n = max_tokens + 1
    counts = np.zeros(4, dtype=np.int32)
    arrs = {k: np.zeros(n, dtype=np.int32) for k in
            ("perm", "dseg_ptr", "dseg_dom", "useg_ptr", "useg_dom", "useg_slot")}
    blocks = np.zeros(3 * n, dtype=np.int32)
    _check(_lib.salt_segments_export(ctx, seg, counts.ctypes.data, arrs["perm"].ctypes.data,
                                     arrs["dseg_ptr"].ctypes.data, arrs["dseg_dom"].ctypes.data,
                                     arrs["useg_ptr"].ctypes.data, arrs["useg_dom"].ctypes.data,
                                     arrs["useg_slot"].ctypes.data, blocks.ctypes.data), ctx)
    T, nd, nu, nb = (int(v) for v in counts)
    return {"perm": arrs["perm"][:T], "dseg_ptr": arrs["dseg_ptr"][:nd + 1], "dseg_dom": arrs["dseg_dom"][:nd],
            "useg_ptr": arrs["useg_ptr"][:nu + 1], "useg_dom": arrs["useg_dom"][:nu],
            "useg_slot": arrs["useg_slot"][:nu], "blocks": blocks[:3 * nb].reshape(nb, 3), "counts": counts}


def salt_lora_apply(ctx, seg, layer: int, x, y, stream=None) -> None:
    _check(_lib.salt_lora_apply(ctx, seg, layer, _ptr(x), _ptr(y), _stream(stream)), ctx)


def salt_lora_apply_with_base(ctx, seg, layer: int, x, W, layout: int, y, stream=None) -> None:
    """y = x W_base + the SALT delta (y written, not read)."""
    _check(_lib.salt_lora_apply_with_base(ctx, seg, layer, _ptr(x), _ptr(W), layout, _ptr(y), _stream(stream)), ctx)


def salt_base_get_shape(ctx, seg, layer: int) -> dict:
    """How salt_lora_apply_with_base would launch the layer's GEMM for the built batch."""
    s = salt_base_shape()
    _check(_lib.salt_base_get_shape(ctx, seg, layer, ctypes.byref(s)), ctx)
    return {k: getattr(s, k) for (k, _) in salt_base_shape._fields_}


def salt_lora_apply_static(ctx, seg, layer: int, x, y, stream=None) -> None:
    """salt_lora_apply without any device allocation behind it (static scratch)."""
    _check(_lib.salt_lora_apply_static(ctx, seg, layer, _ptr(x), _ptr(y), _stream(stream)), ctx)


def salt_lora_apply_grouped(ctx, seg, layers, xs, ys, stream=None) -> None:
    n = len(layers)
    la = (ctypes.c_int32 * n)(*layers)
    xa = (ctypes.c_void_p * n)(*[_ptr(t) for t in xs])
    ya = (ctypes.c_void_p * n)(*[_ptr(t) for t in ys])
    _check(_lib.salt_lora_apply_grouped(ctx, seg, n, la, xa, ya, _stream(stream)), ctx)


class HostPipe:
    """A salt_host_pipe handle with the context it belongs to (for error messages)."""

    def __init__(self, ctx, n_stages: int = 0, stage_bytes: int = 0):
        out = _vp()
        _check(_lib.salt_host_pipe_create(ctx, n_stages, stage_bytes, ctypes.byref(out)), ctx)
        self.ctx, self.ptr = ctx, out.value

    def close(self):
        if self.ptr:
            _lib.salt_host_pipe_destroy(self.ptr)
            self.ptr = None


def salt_host_pipe_create(ctx, n_stages: int = 0, stage_bytes: int = 0) -> HostPipe:
    return HostPipe(ctx, n_stages, stage_bytes)


def salt_host_pipe_destroy(pipe) -> None:
    pipe.close()


def salt_lora_apply_host(pipe, seg, layers, x_hosts, y_hosts, stream=None) -> None:
    """Grouped apply on page-locked host activations (copies in, apply, copies out)."""
    n = len(layers)
    la = (ctypes.c_int32 * n)(*layers)
    xa = (ctypes.c_void_p * n)(*[_ptr(t) for t in x_hosts])
    ya = (ctypes.c_void_p * n)(*[_ptr(t) for t in y_hosts])
    _check(_lib.salt_lora_apply_host(pipe.ptr, seg, n, la, xa, ya, _stream(stream)), pipe.ctx)


def salt_host_pipe_wait(pipe, stream=None) -> None:
    _check(_lib.salt_host_pipe_wait(pipe.ptr, _stream(stream)), pipe.ctx)


class KvCache:
    """A salt_kv handle on the caller's cache tensors (kept alive with it)."""

    def __init__(self, ctx, k, v, k_exp, v_exp):
        if k.dim() != 5 or tuple(v.shape) != tuple(k.shape):
            raise ValueError("k and v are [layers, pages, kv heads, page tokens, head dim]")
        if tuple(k_exp.shape) != tuple(k.shape[:4]) or tuple(v_exp.shape) != tuple(k.shape[:4]):
            raise ValueError("k_exp and v_exp are [layers, pages, kv heads, page tokens]")
        for t in (k, v, k_exp, v_exp):
            if t.element_size() != 1:
                raise TypeError("the cache's tensors hold bytes (uint8 or float8_e4m3fn)")
            _device_tensor(t)
        out = _vp()
        cfg = _kv_config(*(int(n) for n in k.shape), _ptr(k), _ptr(v), _ptr(k_exp), _ptr(v_exp))
        _check(_lib.salt_kv_create(ctx, ctypes.byref(cfg), ctypes.byref(out)), ctx)
        self.ctx, self.handle, self._tensors = ctx, out.value, (k, v, k_exp, v_exp)
        self.n_layers, self.n_pages, self.n_kv_heads, self.page_tokens, self.head_dim = (int(n) for n in k.shape)
        self.rows_shape = k.shape[:4]

    def close(self):
        if self.handle:
            _lib.salt_kv_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _device_tensor(t):
    if not t.is_cuda:
        raise TypeError("not a CUDA tensor")
    return t


_torch_bf16 = _torch_f32 = _torch_i32 = None


def _load_types():
    global _torch_bf16, _torch_f32, _torch_i32
    import torch
    _torch_bf16, _torch_f32, _torch_i32 = torch.bfloat16, torch.float32, torch.int32


def _head_rows(t, heads: int, dim: int):
    """(tokens, pointer, elements from row to row) of a CUDA bf16 tensor
    [tokens, heads, dim] whose heads are contiguous within a row."""
    if _torch_bf16 is None:
        _load_types()
    shape, s = t.shape, t.stride()
    if len(shape) != 3 or shape[1] != heads or shape[2] != dim or t.dtype is not _torch_bf16 or not t.is_cuda:
        raise ValueError(f"not a CUDA bf16 tensor [tokens, {heads}, {dim}]")
    if s[2] != 1 or (s[1] != dim and heads > 1):
        raise ValueError("the heads of a row are not contiguous")
    n = shape[0]
    return n, t.data_ptr(), s[0] if n > 1 else max(s[0], heads * dim)


def _int32s(t, n: int | None = None):
    """Pointer of a contiguous CUDA int32 tensor of n elements."""
    if _torch_i32 is None:
        _load_types()
    if t.dtype is not _torch_i32 or not t.is_cuda or not t.is_contiguous():
        raise ValueError("not a contiguous CUDA int32 tensor")
    if n is not None and t.numel() != n:
        raise ValueError(f"{t.numel()} entries, {n} expected")
    return t.data_ptr()


def salt_kv_create(ctx, k, v, k_exp, v_exp) -> KvCache:
    """A handle on cache memory: k, v [layers, pages, kv heads, page tokens,
    head dim] and k_exp, v_exp [layers, pages, kv heads, page tokens], CUDA
    tensors of bytes."""
    return KvCache(ctx, k, v, k_exp, v_exp)


def salt_kv_destroy(kv: KvCache) -> None:
    if kv is not None:
        kv.close()


def salt_kv_write(kv: KvCache, layer: int, k, v, slots, stream=None) -> None:
    """Quantise rows k, v (CUDA bf16 [tokens, kv heads, head dim], heads
    contiguous within a row) into slots (CUDA int32 [tokens], -1: skip)."""
    n, kp, ks = _head_rows(k, kv.n_kv_heads, kv.head_dim)
    m, vp, vs = _head_rows(v, kv.n_kv_heads, kv.head_dim)
    if m != n:
        raise ValueError("k and v have different numbers of tokens")
    _check(_lib.salt_kv_write(kv.handle, layer, n, kp, ks, vp, vs, _int32s(slots, n), _stream(stream)), kv.ctx)


def salt_kv_read(kv: KvCache, layer: int, slots, k, v, stream=None) -> None:
    """The cached rows of slots into k, v (CUDA bf16 [tokens, kv heads, head dim])."""
    n, kp, ks = _head_rows(k, kv.n_kv_heads, kv.head_dim)
    m, vp, vs = _head_rows(v, kv.n_kv_heads, kv.head_dim)
    if m != n:
        raise ValueError("k and v have different numbers of tokens")
    _check(_lib.salt_kv_read(kv.handle, layer, n, _int32s(slots, n), kp, ks, vp, vs, _stream(stream)), kv.ctx)


class Rope:
    """A salt_rope handle."""

    def __init__(self, ctx, head_dim, rot_dim, inv_freq, interleaved, scale, eps, norm_offset):
        freq = np.ascontiguousarray(inv_freq, dtype=np.float64)
        if freq.shape != (max(rot_dim, 0) // 2,):
            raise ValueError(f"{freq.size} frequencies for {rot_dim} rotated elements")
        out = _vp()
        cfg = _rope_config(head_dim, rot_dim, int(interleaved), freq.ctypes.data, scale, eps, norm_offset)
        _check(_lib.salt_rope_create(ctx, ctypes.byref(cfg), ctypes.byref(out)), ctx)
        self.ctx, self.handle, self.head_dim = ctx, out.value, head_dim

    def close(self):
        if self.handle:
            _lib.salt_rope_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def salt_rope_create(ctx, head_dim: int, rot_dim: int, inv_freq, interleaved: bool = False, scale: float = 1.0,
                     eps: float = 1e-6, norm_offset: float = 0.0) -> Rope:
    """Norms and rotation of heads; inv_freq: radians a position of each of
    the rot_dim / 2 pairs."""
    return Rope(ctx, int(head_dim), int(rot_dim), inv_freq, interleaved, scale, eps, norm_offset)


def salt_rope_destroy(rope: Rope) -> None:
    if rope is not None:
        rope.close()


def _norm_weights(w, dim: int):
    if w is None:
        return None
    if w.dtype is not _torch_bf16 or not w.is_cuda or w.numel() != dim or not w.is_contiguous():
        raise ValueError(f"norm weights are not a contiguous CUDA bf16 tensor of {dim}")
    return w.data_ptr()


def _heads_of(t, dim: int):
    """_head_rows of a tensor of any number of heads, and that number."""
    n, heads, d = t.shape
    s, h, e = t.stride()
    if d != dim or e != 1 or (h != dim and heads > 1) or t.dtype is not _torch_bf16 or not t.is_cuda:
        raise ValueError(f"not a CUDA bf16 tensor [tokens, heads, {dim}] whose heads are contiguous within a row")
    return n, t.data_ptr(), s if n > 1 else max(s, heads * dim), heads


def salt_rope_apply(rope: Rope, q, k, positions, q_out, k_out, q_norm=None, k_norm=None, stream=None) -> None:
    """Queries q and keys k (CUDA bf16 [tokens, heads, head dim], heads
    contiguous within a row) normalised and rotated into q_out and k_out
    (which may be q and k); positions CUDA int32 [tokens]."""
    D = rope.head_dim
    if _torch_bf16 is None:
        _load_types()
    n, qp, qs, H = _heads_of(q, D)
    nk, kp, ks, KV = _heads_of(k, D)
    no, qop, qos, Ho = _heads_of(q_out, D)
    nko, kop, kos, KVo = _heads_of(k_out, D)
    if not n == nk == no == nko or H != Ho or KV != KVo:
        raise ValueError("q, k and the outputs have different numbers of tokens or heads")
    st = _lib.salt_rope_apply(rope.handle, n, qp, qs, H, kp, ks, KV, _norm_weights(q_norm, D), _norm_weights(k_norm, D),
                              _int32s(positions, n), qop, qos, kop, kos, _stream(stream))
    if st:
        _check(st, rope.ctx)


def salt_rope_write(rope: Rope, kv: KvCache, layer: int, q, k, v, positions, slots, q_out, q_norm=None, k_norm=None,
                    stream=None) -> None:
    """The same for q, while k so treated and v as it is go into slots (CUDA
    int32 [tokens], -1: skip) of a layer of the cache."""
    D = rope.head_dim
    if _torch_bf16 is None:
        _load_types()
    n, qp, qs, H = _heads_of(q, D)
    no, qop, qos, Ho = _heads_of(q_out, D)
    nk, kp, ks, KV = _heads_of(k, D)
    nv, vp, vs, KVv = _heads_of(v, D)
    if not n == no == nk == nv or H != Ho or not KV == KVv == kv.n_kv_heads:
        raise ValueError("q, k, v and q_out have different numbers of tokens, or other heads than the cache")
    st = _lib.salt_rope_write(rope.handle, kv.handle, layer, n, qp, qs, H, kp, ks, vp, vs, _norm_weights(q_norm, D),
                              _norm_weights(k_norm, D), _int32s(positions, n), _int32s(slots, n), qop, qos, _stream(stream))
    if st:
        _check(st, rope.ctx)


class AttnPlan:
    """A salt_attn handle with the cache it reads."""

    def __init__(self, kv: KvCache, n_heads: int, max_seqs: int, max_tokens: int, max_pages: int, max_groups: int):
        out = _vp()
        cfg = _attn_config(n_heads, max_seqs, max_tokens, max_pages, max_groups)
        _check(_lib.salt_attn_create(kv.handle, ctypes.byref(cfg), ctypes.byref(out)), kv.ctx)
        self.kv, self.ctx, self.handle, self.n_heads = kv, kv.ctx, out.value, n_heads
        self.head_dim, self.n_tokens, self.n_seqs = kv.head_dim, 0, 0

    def close(self):
        if self.handle:
            _lib.salt_attn_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def salt_attn_create(kv: KvCache, n_heads: int, max_seqs: int, max_tokens: int, max_pages: int,
                     max_groups: int = 0) -> AttnPlan:
    return AttnPlan(kv, int(n_heads), int(max_seqs), int(max_tokens), int(max_pages), int(max_groups))


def salt_attn_destroy(plan: AttnPlan) -> None:
    if plan is not None:
        plan.close()


def salt_attn_batch(q_len, kv_len, page_ptr, pages, group=None, group_len=(), group_page_ptr=(0,), group_pages=()):
    """A salt_attn_batch of host sequences (with the arrays it points to)."""
    a = [np.ascontiguousarray(x, dtype=np.int32) for x in
         (q_len, kv_len, page_ptr, pages, [-1] * len(q_len) if group is None else group, group_len, group_page_ptr,
          group_pages)]
    n, g = len(a[0]), len(a[5])
    if len(a[1]) != n or len(a[2]) != n + 1 or len(a[4]) != n or len(a[6]) != g + 1:
        raise ValueError("a batch's arrays do not match")
    if a[2][-1] > len(a[3]) or a[6][-1] > len(a[7]):
        raise ValueError("a page list runs past its array")
    p = [x.ctypes.data for x in a]
    b = _attn_batch(n, p[0], p[1], p[2], p[3], p[4], g, p[5], p[6], p[7])
    b._keep, b._tokens = a, int(a[0].sum()) if n else 0
    return b


def salt_attn_build(plan: AttnPlan, batch, stream=None) -> None:
    """Plan a batch (salt_attn_batch)."""
    _check(_lib.salt_attn_build(plan.handle, ctypes.byref(batch), _stream(stream)), plan.ctx)
    plan.n_tokens, plan.n_seqs = batch._tokens, batch.n_seqs


def salt_attn_get_shape(plan: AttnPlan) -> dict:
    """How a run of the built batch is divided, and the plan's device memory."""
    s = _attn_shape()
    _check(_lib.salt_attn_get_shape(plan.handle, ctypes.byref(s)), plan.ctx)
    return {k: getattr(s, k) for (k, _) in _attn_shape._fields_}


def salt_attn_run(plan: AttnPlan, layer: int, q, out, scale: float, lse=None, stream=None) -> None:
    """Attention of the built batch: q, out CUDA bf16 [tokens, heads, head dim]
    (heads contiguous within a row), lse CUDA float32 [tokens, heads] or None."""
    n, qp, qs = _head_rows(q, plan.n_heads, plan.head_dim)
    m, op, os_ = _head_rows(out, plan.n_heads, plan.head_dim)
    if n < plan.n_tokens or m < plan.n_tokens:
        raise ValueError(f"q or out has fewer rows than the batch's {plan.n_tokens} query tokens")
    if lse is not None and (lse.numel() < plan.n_tokens * plan.n_heads or lse.dtype is not _torch_f32 or not lse.is_cuda):
        raise ValueError("lse is not a CUDA float32 tensor of the batch's rows")
    _check(_lib.salt_attn_run(plan.handle, layer, qp, qs, scale, op, os_, _ptr(lse), _stream(stream)), plan.ctx)


def salt_attn_track(plan: AttnPlan) -> None:
    """From its next build on the plan serves salt_attn_weights and salt_attn_evict."""
    _check(_lib.salt_attn_track(plan.handle), plan.ctx)


def _cache_floats(t, kv: KvCache, what: str) -> int:
    """Pointer of a contiguous CUDA float32 tensor [layers, pages, kv heads, page tokens]."""
    if _torch_f32 is None:
        _load_types()
    if t.dtype is not _torch_f32 or not t.is_cuda or not t.is_contiguous() or t.shape != kv.rows_shape:
        raise ValueError(f"{what} is not a contiguous CUDA float32 tensor {list(kv.rows_shape)}")
    return t.data_ptr()


def salt_attn_weights(plan: AttnPlan, layer: int, q, lse, scale: float, weights, decay: float = 1.0, stream=None) -> None:
    """Add the attention that the built batch's cached tokens of a layer get to
    weights (CUDA float32 [layers, pages, kv heads, page tokens]), after
    multiplying those by decay; q, lse and scale as in salt_attn_run."""
    n, qp, qs = _head_rows(q, plan.n_heads, plan.head_dim)
    if n < plan.n_tokens:
        raise ValueError(f"q has fewer rows than the batch's {plan.n_tokens} query tokens")
    if lse.numel() < plan.n_tokens * plan.n_heads or lse.dtype is not _torch_f32 or not lse.is_cuda or not lse.is_contiguous():
        raise ValueError("lse is not a contiguous CUDA float32 tensor of the batch's rows")
    _check(_lib.salt_attn_weights(plan.handle, layer, qp, qs, lse.data_ptr(), scale, decay, _cache_floats(weights, plan.kv, "weights"),
                                  _stream(stream)), plan.ctx)


def salt_attn_evict(plan: AttnPlan, layer: int, n_layers: int, keep, scores, kept, first: int = 0, recent: int = 0, weights=None,
                    stream=None) -> None:
    """Leave each request keep[b] (CUDA int32 [requests]) of its own tokens in
    n_layers layers: the last `recent`, the first `first`, of the others those of
    the largest scores (like weights, CUDA float32 [layers, pages, kv heads, page tokens]).  kept (CUDA int32
    [n_layers, requests, kv heads, places]) gets the places they had; weights, if given, move along."""
    n = plan.n_seqs
    if kept.dim() != 4 or tuple(kept.shape[:3]) != (n_layers, n, plan.kv.n_kv_heads):
        raise ValueError(f"kept is not [{n_layers}, {n}, {plan.kv.n_kv_heads}, places]")
    _check(_lib.salt_attn_evict(plan.handle, layer, n_layers, _int32s(keep, n), first, recent, _cache_floats(scores, plan.kv, "scores"),
                                None if weights is None else _cache_floats(weights, plan.kv, "weights"), _int32s(kept),
                                kept.shape[3], _stream(stream)), plan.ctx)


def _prob_rows(t, rows: int):
    """(pointer, elements from row to row, columns) of a CUDA float32 matrix of `rows` rows."""
    shape, s = t.shape, t.stride()
    if len(shape) != 2 or shape[0] != rows or t.dtype is not _torch_f32 or not t.is_cuda or (s[1] != 1 and shape[1] > 1):
        raise ValueError(f"not a CUDA float32 tensor of {rows} rows")
    return t.data_ptr(), s[0] if rows > 1 else max(s[0], shape[1]), shape[1]


def salt_verify_drafts(ctx, draft_ptr, draft_tokens, target_p, draft_p, accept_u, sample_u, accepted, next_token,
                       stream=None) -> None:
    """Accept drafted tokens and draw the next one.  CUDA tensors: draft_ptr
    int32 [requests + 1], draft_tokens int32 [drafts], target_p float32
    [drafts + requests, vocab], draft_p float32 [drafts, vocab], accept_u
    float32 [drafts], sample_u float32 [requests]; results accepted and
    next_token, int32 [requests].  ctx may be None (the current device)."""
    if _torch_f32 is None:
        _load_types()
    n, d = sample_u.numel(), draft_tokens.numel()
    tp, ts, vocab = _prob_rows(target_p, d + n)
    dp, ds, draft_vocab = _prob_rows(draft_p, d)
    if d and draft_vocab != vocab:
        raise ValueError("target_p and draft_p have different vocabularies")
    for t, m in ((accept_u, d), (sample_u, n)):
        if t.dtype is not _torch_f32 or not t.is_cuda or not t.is_contiguous() or t.numel() != m:
            raise ValueError(f"not a contiguous CUDA float32 tensor of {m} entries")
    _check(_lib.salt_verify_drafts(ctx, n, d, vocab, _int32s(draft_ptr, n + 1), _int32s(draft_tokens), tp, ts, dp, ds,
                                   accept_u.data_ptr(), sample_u.data_ptr(), _int32s(accepted, n),
                                   _int32s(next_token, n), _stream(stream)), ctx)


def salt_guard_check(ctx, seg=None) -> int:
    """Number of damaged guard bands around the library's device buffers (synchronous)."""
    n = ctypes.c_int32(0)
    _check(_lib.salt_guard_check(ctx, seg, ctypes.byref(n)), ctx)
    return int(n.value)


def salt_selftest_wait_timeout(ctx, stream=None) -> None:
    _check(_lib.salt_selftest_wait_timeout(ctx, _stream(stream)), ctx)


def salt_get_device_error(ctx, stream=None, raise_on_flags: bool = False) -> int:
    flags = ctypes.c_uint32(0)
    st = _lib.salt_get_device_error(ctx, _stream(stream), ctypes.byref(flags))
    if st not in (0, 10) or (raise_on_flags and st == 10):
        _check(st, ctx)
    return int(flags.value)
