"""ctypes binding of libhttm.so.  Argument marshalling only: every step of the path runs in
the HIP kernels behind the C ABI declared in include/httm.h.  torch is used for device memory
and the current stream, nothing else.  There is no CPU fallback: if the library is missing or
a call fails, an exception is raised."""
from __future__ import annotations

import ctypes as C
import os
import struct
from array import array

import numpy as np
import torch

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG_DIR, "libhttm.so")   # the library built in-tree; nothing else is ever loaded

VARIANT_HEADWISE, VARIANT_UNIFORM, VARIANT_NONE = 0, 1, 2
VARIANTS = {"headwise": VARIANT_HEADWISE, "uniform": VARIANT_UNIFORM, "none": VARIANT_NONE}
MAX_BLOCK = 4096
MAX_HEADS = 64


class HttmError(RuntimeError):
    pass


class Geom(C.Structure):
    _fields_ = [("S", C.c_int32), ("Hp", C.c_int32), ("Wp", C.c_int32), ("n_special", C.c_int32),
                ("H", C.c_int32), ("d_head", C.c_int32), ("b", C.c_int32), ("T", C.c_int32),
                ("rho_q", C.c_double), ("rho_kv", C.c_double), ("variant", C.c_int32),
                ("flags", C.c_int32), ("outlier_frac", C.c_double), ("dst_frac", C.c_double)]


class Sizes(C.Structure):
    _fields_ = [(n, C.c_int64) for n in
                ("N", "n_prefix", "n_blocks", "max_block", "M_q", "M_k", "workspace_bytes", "outlier_cap")]


class WorkspaceLayout(C.Structure):
    _fields_ = [(n, C.c_int64) for n in ("q_m", "k_m", "v_m", "o_m", "assign_q", "assign_k", "eps_q",
                                         "q_out", "o_out", "attn_split", "total")]


class NormRopeStruct(C.Structure):
    _fields_ = [("norm", C.c_int32), ("axes", C.c_int32), ("rot_dim", C.c_int32), ("pairing", C.c_int32), ("base", C.c_double),
                ("eps", C.c_float), ("k_scale", C.c_float), ("q_weight", C.c_void_p), ("q_bias", C.c_void_p),
                ("k_weight", C.c_void_p), ("k_bias", C.c_void_p)]


class RowsStruct(C.Structure):
    _fields_ = [("data", C.c_void_p), ("token_stride", C.c_int64), ("head_stride", C.c_int64)]


class PagedStruct(C.Structure):
    _fields_ = [("k_pages", C.c_void_p), ("v_pages", C.c_void_p), ("page_table", C.c_void_p), ("n_pages", C.c_int64),
                ("n_seqs", C.c_int32), ("table_stride", C.c_int32), ("page_size", C.c_int32), ("H_kv", C.c_int32)]


# The same three as bytes: small calls are bound by what stands in front of their launch.  us a call with a new NormRope or PagedCache, with
# Structures by reference / with these: norms with rotation 12.6 / 11.9, append 15.0 / 13.7, attention 12.3 / 11.8
_pack_norm_rope, _pack_rows, _pack_paged = (struct.Struct(f).pack for f in ("iiiidffPPPP", "Pqq", "PPPqiiii"))


_lib = None


def lib() -> C.CDLL:
    """Load libhttm.so (built in-tree by paper_2511_21317_amd.build) or raise."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise HttmError(f"{LIB_PATH} is missing: run `python -m paper_2511_21317_amd.build` "
                        "(or __graft_entry__.build()) first; there is no fallback path")
    L = C.CDLL(LIB_PATH)
    vp, i32p, i64p, f32p = C.c_void_p, C.c_void_p, C.POINTER(C.c_int64), C.c_void_p
    L.httm_version.restype = C.c_int
    L.httm_strerror.restype = C.c_char_p
    L.httm_strerror.argtypes = [C.c_int]
    L.httm_last_hip_error.restype = C.c_int
    L.httm_geom_sizes.argtypes = [C.POINTER(Geom), C.POINTER(Sizes)]
    L.httm_workspace_layout.argtypes = [C.POINTER(Geom), C.POINTER(WorkspaceLayout)]
    L.httm_geom_tables.argtypes = [C.POINTER(Geom)] + [vp] * 7
    L.httm_geom_block_forms.argtypes = [C.POINTER(Geom), vp, vp]
    L.httm_plan_create.argtypes = [C.POINTER(Geom), C.POINTER(vp)]
    L.httm_plan_clone.argtypes = [vp, C.POINTER(vp)]
    L.httm_plan_destroy.argtypes = [vp]
    L.httm_plan_query.argtypes = [vp, C.POINTER(Sizes)]
    L.httm_reorder.argtypes = [vp, vp, vp, C.c_int, vp]
    L.httm_match_merge.argtypes = [vp, vp, vp, vp, vp, vp, vp, i32p, i32p, f32p, f32p, vp]
    L.httm_reorder_match_merge.argtypes = [vp, vp, vp, vp, vp, vp, vp, i32p, i32p, f32p, f32p, vp]
    L.httm_attention.argtypes = [vp, vp, vp, vp, vp, vp, C.c_int, C.c_int, C.c_float, vp]
    L.httm_attention_scratch.argtypes = [vp, vp, vp, vp, vp, vp, C.c_int, C.c_int, C.c_float, vp, C.c_int64, vp]
    L.httm_attention_log2.argtypes = [vp, vp, vp, vp, vp, vp, C.c_int, C.c_int, vp]
    L.httm_attention_log2_scratch.argtypes = [vp, vp, vp, vp, vp, vp, C.c_int, C.c_int, vp, C.c_int64, vp]
    L.httm_attention_log2_static.argtypes = [vp, vp, vp, vp, vp, vp, C.c_int, C.c_int, vp]
    L.httm_attention_split_plan.argtypes = [i64p, i64p, C.c_int, C.c_int, vp, vp, C.c_int64, vp, C.c_int64]
    L.httm_attention_wide_plan.argtypes = [i64p, i64p, C.c_int, C.c_int, C.c_int64, vp, vp, C.c_int64]
    L.httm_attention_route.argtypes = [i64p, i64p, C.c_int, C.c_int, C.c_int64, vp, vp]
    L.httm_attention_scratch_bytes.argtypes = [C.c_int]
    L.httm_attention_scratch_bytes.restype = C.c_int64
    L.httm_unmerge.argtypes = [vp, vp, i32p, vp, C.c_int, vp]
    L.httm_layer_forward.argtypes = [vp, vp, vp, vp, vp, vp, C.c_size_t, vp]
    L.httm_reorder_match_merge_filtered.argtypes = [vp, vp, vp, vp, vp, vp, vp, i32p, i32p, f32p, vp, vp]
    L.httm_attention_outliers.argtypes = [vp, vp, vp, vp, vp, vp]
    L.httm_unmerge_filtered.argtypes = [vp, vp, vp, i32p, vp, vp]
    L.httm_outlier_stats.argtypes = [vp, C.POINTER(C.c_float), C.POINTER(C.c_int32), vp]
    L.httm_global_match.argtypes = [vp, C.c_int64, C.c_int, C.c_int, C.c_double, i32p, f32p, vp]
    i64, rows, norm_rope, paged = C.c_int64, vp, vp, vp     # (structs: bytes, or byref())
    L.httm_qk_norm_rope.argtypes = [norm_rope, rows, rows, rows, C.c_int, vp, i64, C.c_int, C.c_int, C.c_int, vp, vp, vp, vp]
    L.httm_cache_append.argtypes = [norm_rope, rows, rows, rows, C.c_int, vp, i64, i64, C.c_int, C.c_int, paged, vp, vp, vp, vp]
    L.httm_attention_cached_workspace.argtypes = [i64, C.c_int, C.c_int, C.c_int, i64]
    L.httm_attention_cached_workspace.restype = i64
    L.httm_attention_cached.argtypes = [rows, vp, vp, i64, paged, vp, vp, i64, C.c_int, C.c_int, C.c_float, C.c_int, vp, vp, i64, vp]
    for name in ("httm_qk_norm_rope", "httm_cache_append", "httm_attention_cached", "httm_geom_sizes", "httm_workspace_layout", "httm_geom_tables", "httm_geom_block_forms", "httm_plan_create", "httm_plan_clone",
                 "httm_plan_destroy", "httm_plan_query", "httm_reorder", "httm_match_merge",
                 "httm_reorder_match_merge",
                 "httm_attention", "httm_attention_scratch", "httm_attention_log2", "httm_attention_log2_scratch", "httm_attention_log2_static", "httm_attention_split_plan", "httm_attention_route", "httm_attention_wide_plan", "httm_unmerge", "httm_layer_forward",
                 "httm_reorder_match_merge_filtered", "httm_attention_outliers", "httm_unmerge_filtered",
                 "httm_outlier_stats", "httm_global_match"):
        getattr(L, name).restype = C.c_int
    _lib = L
    return L


def _check(rc: int, what: str):
    if rc != 0:
        L = lib()
        msg = L.httm_strerror(rc).decode()
        extra = f" (hipError_t {L.httm_last_hip_error()})" if rc == -4 else ""
        raise HttmError(f"{what} failed: {msg}{extra} [code {rc}]")


FLAG_ANCHOR_FIRST_FRAME = 1
FLAG_CHUNKED_BLOCKS = 2
FLAG_LOG2_KEYS = 4
LOG2_KEY_SCALE = 0.125 * 1.4426950408889634   # log2(e) / sqrt(64): the factor the scaled keys carry


def make_geom(S, Hp, Wp, b, T, rho_q, rho_kv=None, *, H=16, d_head=64, n_special=5,
              variant="headwise", anchor_first_frame=False, outlier_frac=0.0, chunked_blocks=False,
              dst_frac=0.0, log2_keys=False) -> Geom:
    if rho_kv is None:
        rho_kv = rho_q
    v = VARIANTS[variant] if isinstance(variant, str) else int(variant)
    flags = ((FLAG_ANCHOR_FIRST_FRAME if anchor_first_frame else 0) | (FLAG_CHUNKED_BLOCKS if chunked_blocks else 0)
             | (FLAG_LOG2_KEYS if log2_keys else 0))
    return Geom(S, Hp, Wp, n_special, H, d_head, b, T, float(rho_q), float(rho_kv), v, flags,
                float(outlier_frac), float(dst_frac))


def geom_sizes(g: Geom) -> Sizes:
    s = Sizes()
    _check(lib().httm_geom_sizes(C.byref(g), C.byref(s)), "httm_geom_sizes")
    return s


def workspace_layout(g: Geom) -> WorkspaceLayout:
    w = WorkspaceLayout()
    _check(lib().httm_workspace_layout(C.byref(g), C.byref(w)), "httm_workspace_layout")
    return w


def geom_tables(g: Geom) -> dict:
    """Host index tables of a geometry as int32 NumPy arrays (no GPU needed)."""
    s = geom_sizes(g)
    out = {"pi": np.empty(s.N, np.int32)}
    for name in ("block_start", "block_n", "block_kq", "block_kk", "block_offq", "block_offk"):
        out[name] = np.empty(s.n_blocks, np.int32)
    ptr = lambda a: a.ctypes.data_as(C.c_void_p)  # noqa: E731
    _check(lib().httm_geom_tables(C.byref(g), ptr(out["pi"]), ptr(out["block_start"]),
                                  ptr(out["block_n"]), ptr(out["block_kq"]), ptr(out["block_kk"]),
                                  ptr(out["block_offq"]), ptr(out["block_offk"])), "httm_geom_tables")
    return out


def geom_block_forms(g: Geom) -> dict:
    """The reorder inside every merging block in closed form (int32 NumPy arrays, no GPU needed)."""
    s = geom_sizes(g)
    out = {"block_src0": np.empty(s.n_blocks, np.int32), "block_dims": np.empty(s.n_blocks, np.int32)}
    ptr = lambda a: a.ctypes.data_as(C.c_void_p)  # noqa: E731
    _check(lib().httm_geom_block_forms(C.byref(g), ptr(out["block_src0"]), ptr(out["block_dims"])),
           "httm_geom_block_forms")
    return out


# A call costs the host several microseconds, as much as the GPU needs for a small scene, and most of that is
# marshalling: tensors are checked with one expression and passed as integers, the stream is asked for
# without making a Stream object.  us a call, before / now: a
# layer 14.5 / 10.3, an attention 10.8 / 7.5, a pass through the stages (8 calls) 63 / 41.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream() -> int:
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


def _stream_of(device: int) -> int:
    return _raw_stream(device) if _raw_stream is not None else torch.cuda.current_stream().cuda_stream


def _dev(t: torch.Tensor, dtype, shape=None) -> int:
    if t.is_cuda and t.dtype == dtype and t.is_contiguous() and (shape is None or t.shape == shape):
        return t.data_ptr()
    if not t.is_cuda:
        raise HttmError("tensor must live on the GPU")
    if t.dtype != dtype:
        raise HttmError(f"expected dtype {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise HttmError("tensor must be contiguous")
    raise HttmError(f"expected shape {tuple(shape)}, got {tuple(t.shape)}")


def _row_offsets(rows, n: int) -> array:
    """n row indices as int64; pass .buffer_info()[0] and keep the array until the call returns.  As in a C array
    with an initialiser, fewer are filled up with zeros (which no call accepts behind others) and more are refused."""
    try:
        a = array("q", rows) if type(rows) in (list, tuple) else array("q", [int(x) for x in rows])
    except TypeError:       # something else that int() takes
        a = array("q", [int(x) for x in rows])
    if len(a) > n:
        raise IndexError(f"{len(a)} row offsets, expected {n}")
    a.extend([0] * (n - len(a)))
    return a


class Plan:
    """Owns an httm_plan_t (device index tables of one geometry)."""

    def __init__(self, g: Geom, _clone_of=None):
        self.geom = g
        self._h = C.c_void_p()
        if _clone_of is None:
            _check(lib().httm_plan_create(C.byref(g), C.byref(self._h)), "httm_plan_create")
        else:
            _check(lib().httm_plan_clone(_clone_of._h, C.byref(self._h)), "httm_plan_clone")
        self.sizes = Sizes()
        _check(lib().httm_plan_query(self._h, C.byref(self.sizes)), "httm_plan_query")
        self.layout = workspace_layout(g)
        self._H, self._N = int(g.H), int(self.sizes.N)
        self._M_q, self._M_k = int(self.sizes.M_q), int(self.sizes.M_k)
        self._tok = (self._H, self._N, 64)                  # shapes of the tensors of a call
        self._mq, self._mk = (self._H, self._M_q, 64), (self._H, self._M_k, 64)
        self._per_tok, self._out = (self._H, self._N), (self._N, self._H * 64)

    def clone(self) -> "Plan":
        """A second plan of the same geometry with buffers of its own (for a second stream)."""
        return Plan(self.geom, _clone_of=self)

    def close(self):
        if self._h:
            lib().httm_plan_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # convenience
    @property
    def N(self): return self._N
    @property
    def M_q(self): return self._M_q
    @property
    def M_k(self): return self._M_k
    @property
    def H(self): return self._H
    @property
    def outlier_cap(self): return int(self.sizes.outlier_cap)
    @property
    def log2_keys(self): return bool(self.geom.flags & FLAG_LOG2_KEYS)


def reorder(plan: Plan, src: torch.Tensor, dst: torch.Tensor, direction: int = 0):
    shape = plan._tok
    _check(lib().httm_reorder(plan._h, _dev(src, torch.bfloat16, shape), _dev(dst, torch.bfloat16, shape),
                              int(direction), _stream()), "httm_reorder")
    return dst


def match_merge(plan: Plan, q_r, k_r, v_r, q_m, k_m, v_m, assign_q, assign_k, score_q=None, score_k=None):
    H, N = plan.H, plan.N
    bf, i32, f32 = torch.bfloat16, torch.int32, torch.float32
    _check(lib().httm_match_merge(
        plan._h, _dev(q_r, bf, plan._tok), _dev(k_r, bf, plan._tok), _dev(v_r, bf, plan._tok),
        _dev(q_m, bf, plan._mq), _dev(k_m, bf, plan._mk), _dev(v_m, bf, plan._mk),
        _dev(assign_q, i32, plan._per_tok), _dev(assign_k, i32, plan._per_tok),
        _dev(score_q, f32, plan._per_tok) if score_q is not None else None,
        _dev(score_k, f32, plan._per_tok) if score_k is not None else None, _stream()), "httm_match_merge")


def reorder_match_merge(plan: Plan, q, k, v, q_m, k_m, v_m, assign_q, assign_k, score_q=None, score_k=None):
    H, N = plan.H, plan.N
    bf, i32, f32 = torch.bfloat16, torch.int32, torch.float32
    _check(lib().httm_reorder_match_merge(
        plan._h, _dev(q, bf, plan._tok), _dev(k, bf, plan._tok), _dev(v, bf, plan._tok),
        _dev(q_m, bf, plan._mq), _dev(k_m, bf, plan._mk), _dev(v_m, bf, plan._mk),
        _dev(assign_q, i32, plan._per_tok), _dev(assign_k, i32, plan._per_tok),
        _dev(score_q, f32, plan._per_tok) if score_q is not None else None,
        _dev(score_k, f32, plan._per_tok) if score_k is not None else None, _stream()), "httm_reorder_match_merge")


def attention(q_m, k_m, v_m, o_m, q_offsets, k_offsets, scale: float = 0.125, scratch=None):
    """q_m/o_m: [sum M_q, 64] (or [H, M, 64]) bf16; offsets: sequences of H+1 row indices (host).
    scratch: a uint8 device tensor of at least attention_scratch_bytes(H) bytes, or None."""
    H = len(q_offsets) - 1
    q_off, k_off = _row_offsets(q_offsets, H + 1), _row_offsets(k_offsets, H + 1)
    qo, ko = q_off.buffer_info()[0], k_off.buffer_info()[0]
    bf = torch.bfloat16
    if scratch is None:
        _check(lib().httm_attention(_dev(q_m, bf), _dev(k_m, bf), _dev(v_m, bf), _dev(o_m, bf), qo, ko,
                                    H, 64, float(scale), _stream()), "httm_attention")
    else:
        _check(lib().httm_attention_scratch(_dev(q_m, bf), _dev(k_m, bf), _dev(v_m, bf), _dev(o_m, bf), qo, ko,
                                            H, 64, float(scale), _dev(scratch, torch.uint8), scratch.numel(),
                                            _stream()), "httm_attention_scratch")
    return o_m


def attention_split_plan(q_offsets, k_offsets, compute_units: int = 256) -> dict:
    """How stage 3 with scratch cuts a launch with these head lengths (host only, no GPU needed)."""
    H = len(q_offsets) - 1
    qo = (C.c_int64 * (H + 1))(*[int(x) for x in q_offsets])
    ko = (C.c_int64 * (H + 1))(*[int(x) for x in k_offsets])
    summary = np.zeros(8, np.int32)
    ptr = lambda a: a.ctypes.data_as(C.c_void_p)  # noqa: E731
    _check(lib().httm_attention_split_plan(qo, ko, H, int(compute_units), ptr(summary), None, 0, None, 0),
           "httm_attention_split_plan")
    names = ("n_tiles", "shares", "share_units", "span", "slots", "units", "kept_full", "split_ragged")
    out = {n: int(v) for n, v in zip(names, summary)}
    seg = np.zeros((out["slots"], 5), np.int32)
    tiles = np.zeros((out["n_tiles"], 4), np.int32)
    _check(lib().httm_attention_split_plan(qo, ko, H, int(compute_units), ptr(summary), ptr(seg), seg.shape[0],
                                           ptr(tiles), tiles.shape[0]), "httm_attention_split_plan")
    out["segments"], out["tiles"] = seg, tiles
    return out


ATTENTION_TILES = ("tiles256", "tiles128", "groups32", "groups64", "groups128", "groups128_wide", "groups256")


def attention_route(q_offsets, k_offsets, compute_units: int = 256, scratch_bytes: int | None = None) -> dict:
    """What stage 3 runs a launch with these head lengths in (host only): "tiles", a name per launch, and "rows",
    [launches, H, 2] first row inside the head and number of rows.  scratch_bytes: None = attention_scratch_bytes(H)."""
    H = len(q_offsets) - 1
    qo = (C.c_int64 * (H + 1))(*[int(x) for x in q_offsets])
    ko = (C.c_int64 * (H + 1))(*[int(x) for x in k_offsets])
    tiles, rows = np.zeros(2, np.int32), np.zeros((2, H, 2), np.int64)
    ptr = lambda a: a.ctypes.data_as(C.c_void_p)  # noqa: E731
    scratch = attention_scratch_bytes(H) if scratch_bytes is None else int(scratch_bytes)
    _check(lib().httm_attention_route(qo, ko, H, int(compute_units), scratch, ptr(tiles), ptr(rows)), "httm_attention_route")
    names = [ATTENTION_TILES[t] for t in tiles if t >= 0]
    return {"tiles": names, "rows": rows[:len(names)]}


def attention_wide_plan(q_offsets, k_offsets, compute_units: int = 256, scratch_bytes: int | None = None) -> dict | None:
    """How a launch with log2 keys runs in 512-row tiles (host only), None if it does not: "segments" are rows of share,
    head, first query row, first and last key tile, slot.  scratch_bytes: None = attention_scratch_bytes(H)."""
    H = len(q_offsets) - 1
    qo = (C.c_int64 * (H + 1))(*[int(x) for x in q_offsets])
    ko = (C.c_int64 * (H + 1))(*[int(x) for x in k_offsets])
    scratch = attention_scratch_bytes(H) if scratch_bytes is None else int(scratch_bytes)
    summary, seg = np.zeros(6, np.int32), np.zeros((2048, 6), np.int32)
    ptr = lambda a: a.ctypes.data_as(C.c_void_p)  # noqa: E731
    n = lib().httm_attention_wide_plan(qo, ko, H, int(compute_units), scratch, ptr(summary), ptr(seg), seg.shape[0])
    if n < 0:
        _check(n, "httm_attention_wide_plan")
    if not summary[0]:
        return None
    names = ("n_tiles", "shares", "slots", "kept_full", "split_ragged")
    return {**{k: int(v) for k, v in zip(names, summary[1:])}, "segments": seg[:n]}


def attention_scratch_bytes(H: int) -> int:
    return int(lib().httm_attention_scratch_bytes(int(H)))


def attention_log2(q_m, k_log2, v_m, o_m, q_offsets, k_offsets, scratch=None):
    """As attention(), for keys that carry the factor LOG2_KEY_SCALE (a plan with log2_keys).
    scratch: a uint8 device tensor of at least attention_scratch_bytes(H) bytes, or None."""
    H = len(q_offsets) - 1
    q_off, k_off = _row_offsets(q_offsets, H + 1), _row_offsets(k_offsets, H + 1)
    qo, ko = q_off.buffer_info()[0], k_off.buffer_info()[0]
    bf = torch.bfloat16
    if scratch is None:
        _check(lib().httm_attention_log2(_dev(q_m, bf), _dev(k_log2, bf), _dev(v_m, bf), _dev(o_m, bf), qo, ko,
                                         H, 64, _stream()), "httm_attention_log2")
    else:
        _check(lib().httm_attention_log2_scratch(_dev(q_m, bf), _dev(k_log2, bf), _dev(v_m, bf), _dev(o_m, bf),
                                                 qo, ko, H, 64, _dev(scratch, torch.uint8),
                                                 scratch.numel(), _stream()), "httm_attention_log2_scratch")
    return o_m


def attention_log2_static(q_m, k_log2, v_m, o_m, q_offsets, k_offsets):
    """attention_log2() with the library's own static scratch (httm_attention_log2_static): no
    allocation anywhere in the call."""
    H = len(q_offsets) - 1
    q_off, k_off = _row_offsets(q_offsets, H + 1), _row_offsets(k_offsets, H + 1)
    qo, ko = q_off.buffer_info()[0], k_off.buffer_info()[0]
    bf = torch.bfloat16
    _check(lib().httm_attention_log2_static(_dev(q_m, bf), _dev(k_log2, bf), _dev(v_m, bf), _dev(o_m, bf), qo, ko,
                                            H, 64, _stream()), "httm_attention_log2_static")
    return o_m


def unmerge(plan: Plan, o_m, assign_q, out, fuse_inverse_reorder: bool = True):
    H, N = plan.H, plan.N
    shape = (N, H * 64) if fuse_inverse_reorder else (H, N, 64)
    _check(lib().httm_unmerge(plan._h, _dev(o_m, torch.bfloat16, (H, plan.M_q, 64)),
                              _dev(assign_q, torch.int32, (H, N)), _dev(out, torch.bfloat16, shape),
                              1 if fuse_inverse_reorder else 0, _stream()), "httm_unmerge")
    return out


def layer_forward(plan: Plan, q, k, v, out, workspace):
    bf = torch.bfloat16
    if workspace.dtype != torch.uint8:
        raise HttmError("workspace must be a uint8 tensor")
    _check(lib().httm_layer_forward(plan._h, _dev(q, bf, plan._tok), _dev(k, bf, plan._tok),
                                    _dev(v, bf, plan._tok), _dev(out, bf, plan._out),
                                    _dev(workspace, torch.uint8), workspace.numel(), _stream()),
           "httm_layer_forward")
    return out


def workspace_views(plan: Plan, workspace: torch.Tensor) -> dict:
    """Typed views of the regions of the workspace of httm_layer_forward."""
    L, H, N = plan.layout, plan.H, plan.N
    def bf(off, rows):
        return workspace[off:off + H * rows * 128].view(torch.bfloat16).view(H, rows, 64)
    def i32(off):
        return workspace[off:off + H * N * 4].view(torch.int32).view(H, N)
    views = {"q_m": bf(L.q_m, plan.M_q), "k_m": bf(L.k_m, plan.M_k), "v_m": bf(L.v_m, plan.M_k),
             "o_m": bf(L.o_m, plan.M_q), "assign_q": i32(L.assign_q), "assign_k": i32(L.assign_k)}
    cap = plan.outlier_cap
    if cap:
        views["eps_q"] = workspace[L.eps_q:L.eps_q + H * N * 4].view(torch.float32).view(H, N)
        views["q_out"] = workspace[L.q_out:L.q_out + cap * 128].view(torch.bfloat16).view(cap, 64)
        views["o_out"] = workspace[L.o_out:L.o_out + cap * 128].view(torch.bfloat16).view(cap, 64)
    views["attn_split"] = workspace[L.attn_split:L.attn_split + attention_scratch_bytes(H)]   # stage 3's scratch
    return views


def reorder_match_merge_filtered(plan: Plan, q, k, v, q_m, k_m, v_m, assign_q, assign_k, eps_q, q_out):
    """Stage 2 with the adaptive outlier filter (plans with outlier_frac > 0)."""
    H, N = plan.H, plan.N
    bf, i32, f32 = torch.bfloat16, torch.int32, torch.float32
    _check(lib().httm_reorder_match_merge_filtered(
        plan._h, _dev(q, bf, plan._tok), _dev(k, bf, plan._tok), _dev(v, bf, plan._tok),
        _dev(q_m, bf, plan._mq), _dev(k_m, bf, plan._mk), _dev(v_m, bf, plan._mk),
        _dev(assign_q, i32, plan._per_tok), _dev(assign_k, i32, plan._per_tok), _dev(eps_q, f32, plan._per_tok),
        _dev(q_out, bf, (plan.outlier_cap, 64)), _stream()), "httm_reorder_match_merge_filtered")


def attention_outliers(plan: Plan, q_out, k_m, v_m, o_out):
    bf = torch.bfloat16
    cap = plan.outlier_cap
    _check(lib().httm_attention_outliers(plan._h, _dev(q_out, bf, (cap, 64)),
                                         _dev(k_m, bf, (plan.H, plan.M_k, 64)),
                                         _dev(v_m, bf, (plan.H, plan.M_k, 64)),
                                         _dev(o_out, bf, (cap, 64)), _stream()), "httm_attention_outliers")
    return o_out


def unmerge_filtered(plan: Plan, o_m, o_out, assign_q, out):
    H, N = plan.H, plan.N
    bf = torch.bfloat16
    _check(lib().httm_unmerge_filtered(plan._h, _dev(o_m, bf, plan._mq),
                                       _dev(o_out, bf, (plan.outlier_cap, 64)),
                                       _dev(assign_q, torch.int32, (H, N)), _dev(out, bf, (N, H * 64)),
                                       _stream()), "httm_unmerge_filtered")
    return out


def outlier_stats(plan: Plan):
    """(tau, outliers per head) of the last filtered stage 2 on this plan; waits for the stream."""
    tau = C.c_float()
    counts = (C.c_int32 * plan.H)()
    _check(lib().httm_outlier_stats(plan._h, C.byref(tau), counts, _stream()), "httm_outlier_stats")
    return float(tau.value), [int(c) for c in counts]


def global_match(x, dst_frac: float, best_dst, sim=None):
    """Un-blocked matching of x [H, N, 64] (Sec. 3.3's comparison point): best_dst / sim [H, N]."""
    H, N = int(x.shape[0]), int(x.shape[1])
    _check(lib().httm_global_match(_dev(x, torch.bfloat16, (H, N, 64)), N, H, 64, float(dst_frac),
                                   _dev(best_dst, torch.int32, (H, N)),
                                   _dev(sim, torch.float32, (H, N)) if sim is not None else None, _stream()),
           "httm_global_match")
    return best_dst


def alloc_workspace(plan: Plan) -> torch.Tensor:
    return torch.empty(int(plan.sizes.workspace_bytes), dtype=torch.uint8, device="cuda")


# ---- rows of a projection, paged cache, attention with a shared prefix ---------------------------------------

NORMS = {"none": 0, "rms": 1, "layer": 2}
PAIRINGS = {"halves": 0, "neighbours": 1}
_DTYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
MAX_SEQS = 4096


_device = getattr(torch._C, "_cuda_getDevice", None)      # (torch.cuda.current_device() without its checks: 0.8 us less)


def _here(t: torch.Tensor) -> int:
    """The current device, which a launch goes to; `t` (not None) must be there."""
    if not t.is_cuda:
        raise HttmError("tensor must live on the GPU")
    here = _device()
    if t.get_device() != here:
        _refuse(t, here)
    return here


def _refuse(t, here, dtype=None, shape=None):
    if t.is_cuda and t.get_device() != here:
        raise HttmError(f"tensor is on {t.device}, the current device is cuda:{here}")
    _dev(t, dtype, shape)


def _at(t: torch.Tensor, here: int, dtype, shape=None) -> int:
    """As _dev(), for a tensor on the current device."""
    if t is None:
        raise HttmError("a tensor is missing")
    if t.get_device() == here and t.dtype is dtype and t.is_contiguous() and (shape is None or t.shape == shape):
        return t.data_ptr()
    _refuse(t, here, dtype, shape)


_NO_ROWS = _pack_rows(0, 0, 0)


def _rows(t, here, shape, dtype):
    """A [N, H, 64] view whose channels are dense, as the C side takes it."""
    if t is None:
        return _NO_ROWS
    stride = t.stride()
    if t.get_device() != here or t.dtype is not dtype or t.shape != shape or stride[2] != 1:
        if t.get_device() != here:
            _refuse(t, here, dtype)
        if t.dtype != dtype:
            raise HttmError(f"expected dtype {dtype}, got {t.dtype}")
        if t.shape != shape:
            raise HttmError(f"expected shape {shape}, got {tuple(t.shape)}")
        raise HttmError("the 64 channels of a row must be contiguous")
    # (a stride along an axis of length 1 means nothing)
    return _pack_rows(t.data_ptr(), stride[0] if shape[0] > 1 else 0, stride[1] if shape[1] > 1 else 0)


class NormRope:
    """Norms of queries and keys and the rotation by position (httm_norm_rope_t).

    norm: "none", "rms" or "layer"; weights and biases: [64] fp32 tensors or None.
    axes: coordinates of a position, 0 (no rotation) to 3; rot_dim: channels that rotate, a multiple of 16 * axes;
    pairing: "halves" or "neighbours"; k_scale: factor on the keys (LOG2_KEY_SCALE for log2 keys)."""

    def __init__(self, norm="layer", eps=1e-6, axes=2, rot_dim=64, pairing="halves", base=100.0, q_weight=None, q_bias=None,
                 k_weight=None, k_bias=None, k_scale=1.0):
        self.affine = (q_weight, q_bias, k_weight, k_bias)      # kept alive
        self.device = None
        pointers = [0] * 4
        for i, t in enumerate(self.affine):
            if t is not None:
                if self.device is None:
                    self.device = _here(t)
                pointers[i] = _at(t, self.device, torch.float32, (64,))
        self.axes = int(axes)
        try:
            self.struct = _pack_norm_rope(NORMS[norm], self.axes, rot_dim, PAIRINGS[pairing], base, eps, k_scale, *pointers)
        except (KeyError, struct.error, OverflowError) as e:
            raise HttmError(f"no such norm, pairing or number: {e}") from None

    def check_device(self, here):
        if self.device is not None and self.device != here:
            raise HttmError(f"weights are on cuda:{self.device}, the current device is cuda:{here}")


class PagedCache:
    """Keys and values in pages (httm_paged_t): k_pages, v_pages [n_pages, H_kv, page_size, 64] bf16, page_table
    [n_seqs, pages of a sequence] int32."""

    def __init__(self, k_pages, v_pages, page_table):
        if k_pages is None or page_table is None:
            raise HttmError("a tensor is missing")
        shape, table_shape = k_pages.shape, page_table.shape
        if len(shape) != 4 or shape[3] != 64 or len(table_shape) != 2:
            raise HttmError("expected k_pages [n_pages, H_kv, page_size, 64] and page_table [n_seqs, pages]")
        here = _here(k_pages)
        self.device = here
        self.k_pages, self.v_pages, self.page_table = k_pages, v_pages, page_table
        self.n_seqs, self.H_kv, self.page_size = table_shape[0], shape[1], shape[2]
        self.struct = _pack_paged(_at(k_pages, here, torch.bfloat16), _at(v_pages, here, torch.bfloat16, shape),
                                  _at(page_table, here, torch.int32), shape[0], table_shape[0], table_shape[1], shape[2], shape[1])

    def check_device(self, here):
        if self.device != here:
            raise HttmError(f"the cache is on cuda:{self.device}, the current device is cuda:{here}")


def _rows_type(t) -> int:
    if t is None:
        raise HttmError("a tensor is missing")
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise HttmError(f"rows must be bf16, fp16 or fp32, got {t.dtype}")
    return code


def qk_norm_rope(nr: NormRope, q, k, v, pos, q_out, k_out, v_out):
    """Rows of a projection -> the layer's tensors: q [N, H_q, 64], k, v [N, H_kv, 64] (any token and head strides, bf16, fp16 or
    fp32) -> q_out [H_q, N, 64], k_out, v_out [H_kv, N, 64] bf16.  pos: [N, axes] int32 (None without axes).
    Any of q, k, v may be None, with its output."""
    first = q if q is not None else k if k is not None else v
    if first is None or first.dim() != 3:
        raise HttmError("expected q [N, H_q, 64], k or v [N, H_kv, 64]")
    if (q is None) != (q_out is None) or (k is None) != (k_out is None) or (v is None) != (v_out is None):
        raise HttmError("every tensor needs its output, and every output its tensor")
    code, dtype, here = _rows_type(first), first.dtype, _here(first)
    N, H_q, _ = first.shape
    kv = k if k is not None else v
    H_kv = H_q if kv is first or kv is None or kv.dim() != 3 else kv.shape[1]
    q_shape, kv_shape, bf = (N, H_q, 64), (N, H_kv, 64), torch.bfloat16
    rows = _rows(q, here, q_shape, dtype), _rows(k, here, kv_shape, dtype), _rows(v, here, kv_shape, dtype)
    p = None
    if nr.axes > 0 and (q is not None or k is not None):
        if pos is None:
            raise HttmError("positions are needed for a rotation")
        p = _at(pos, here, torch.int32, (N, nr.axes))
    nr.check_device(here)
    rc = lib().httm_qk_norm_rope(nr.struct, *rows, code, p, N, H_q, H_kv, 64,
                                 None if q is None else _at(q_out, here, bf, (H_q, N, 64)),
                                 None if k is None else _at(k_out, here, bf, (H_kv, N, 64)),
                                 None if v is None else _at(v_out, here, bf, (H_kv, N, 64)), _stream_of(here))
    if rc:
        _check(rc, "httm_qk_norm_rope")
    return q_out, k_out, v_out


def cache_append(nr: NormRope, q, k, v, pos, cache: PagedCache, offsets, seq_lens, q_out, first_pos: int = 0):
    """New tokens of the sequences of a batch into the cache: q [n, H_q, 64] (or None, with q_out), k, v [n, H_kv, 64]; offsets
    [n_seqs + 1], seq_lens [n_seqs] (with the new tokens) int32 on the GPU; q_out [n, H_q, 64] bf16.
    pos: [n, axes] int32, or None with one axis: first_pos + a token's row in its sequence."""
    code, dtype, here = _rows_type(k), k.dtype, _here(k)
    n, H_kv = k.shape[0] if k.dim() == 3 else 0, cache.H_kv
    H_q = q.shape[1] if q is not None and q.dim() == 3 else H_kv
    if v is None:
        raise HttmError("keys need values")
    if (q is None) != (q_out is None):
        raise HttmError("q needs q_out, and q_out needs q")
    shape = (n, H_kv, 64)
    rows = _rows(q, here, (n, H_q, 64), dtype), _rows(k, here, shape, dtype), _rows(v, here, shape, dtype)
    out = None if q_out is None else _at(q_out, here, torch.bfloat16, (n, H_q, 64))
    p = _at(pos, here, torch.int32, (n, nr.axes)) if pos is not None and nr.axes > 0 else None
    if not 0 <= first_pos < 1 << 31:      # (ctypes would take it modulo 2^64)
        raise HttmError(f"first_pos must be from 0 to 2^31 - 1, got {first_pos}")
    nr.check_device(here)
    cache.check_device(here)
    rc = lib().httm_cache_append(nr.struct, *rows, code, p, first_pos, n, H_q, 64, cache.struct,
                                 _at(offsets, here, torch.int32, (cache.n_seqs + 1,)), _at(seq_lens, here, torch.int32, (cache.n_seqs,)),
                                 out, _stream_of(here))
    if rc:
        _check(rc, "httm_cache_append")
    return q_out


def attention_cached_workspace(n_tokens: int, n_seqs: int, H_q: int, H_kv: int, P: int) -> int:
    """Bytes of workspace of attention_cached()."""
    sizes = n_tokens, n_seqs, H_q, H_kv, P
    if min(sizes) < 0 or max(sizes) >= 1 << 31:      # (ctypes would take them modulo 2^32 or 2^64)
        raise HttmError(f"sizes must be from 0 to 2^31 - 1, got {sizes}")
    n = int(lib().httm_attention_cached_workspace(int(n_tokens), int(n_seqs), int(H_q), int(H_kv), int(P)))
    if n < 0:
        _check(n, "httm_attention_cached_workspace")
    return n


def attention_cached(q, k_prefix, v_prefix, cache: PagedCache, offsets, seq_lens, out, scale: float = 0.125, causal: bool = False,
                     workspace=None):
    """Attention of a batch's tokens q [n, H_q, 64] (any strides) to the prefix [H_kv, P, 64] (or None) that all sequences
    share and to their own rows in the cache.  offsets, seq_lens as for cache_append; out [n, H_q * 64] bf16.
    workspace: a uint8 tensor of at least attention_cached_workspace(...) bytes."""
    bf = torch.bfloat16
    if q is None or q.dim() != 3:
        raise HttmError(f"expected q [n, H_q, 64], got {None if q is None else tuple(q.shape)}")
    here = _here(q)
    n, H_q, _ = q.shape
    P, kp, vp = 0, None, None
    if (k_prefix is None) != (v_prefix is None):
        raise HttmError("a prefix has keys and values")
    if k_prefix is not None:
        if k_prefix.dim() != 3:
            raise HttmError(f"expected a prefix [{cache.H_kv}, P, 64], got {tuple(k_prefix.shape)}")
        P = k_prefix.shape[1]
        shape = (cache.H_kv, P, 64)
        kp, vp = _at(k_prefix, here, bf, shape), _at(v_prefix, here, bf, shape)
    if workspace is None:
        raise HttmError("a workspace of attention_cached_workspace() bytes is needed")
    cache.check_device(here)
    rc = lib().httm_attention_cached(_rows(q, here, (n, H_q, 64), bf), kp, vp, P, cache.struct,
                                     _at(offsets, here, torch.int32, (cache.n_seqs + 1,)), _at(seq_lens, here, torch.int32, (cache.n_seqs,)),
                                     n, H_q, 64, scale, 1 if causal else 0, _at(out, here, bf, (n, H_q * 64)),
                                     _at(workspace, here, torch.uint8), workspace.numel(), _stream_of(here))
    if rc:
        _check(rc, "httm_attention_cached")
    return out
