"""ctypes binding of libcr.so with the C ABI's names (argument marshalling only).

Every function takes torch tensors that already live on the GPU (device memory and
the current stream come from PyTorch) and passes their raw pointers to the library.
Integer buffers use torch's signed dtypes of the same width; the library reads them
as the unsigned types of the header. Nothing here computes any step of the path, and
there is no fallback: without the built library every call raises.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import Optional, Sequence

import torch

from .build import LIB

CR_OK, CR_EINVAL, CR_ESIZE, CR_EHIP = 0, -1, -2, -3
CR_ERR_KEY_RANGE, CR_ERR_DEST_RANGE, CR_ERR_SPEC, CR_ERR_KEYMAP_FULL = 1, 2, 4, 8
CR_NO_KEY = 0xFFFFFFFF
CR_EMPTY_SLOT = 0xFFFFFFFF
CR_ROUTE_SINGLE = 0x80000000
CR_MAX_R, CR_MAX_W, CR_MAX_CANDS, CR_MAX_J = 1024, 512, 256, 65535
CR_ADMIT_SCRATCH_BYTES = 64 << 20

EXPORTS = ("cr_count_rates", "cr_count_slice_workspace_bytes", "cr_count_slice", "cr_admit_workspace_bytes",
           "cr_admit", "cr_admit_noalloc", "cr_plan_sizes", "cr_workspace_bytes", "cr_place_lpt", "cr_place_hash", "cr_route",
           "cr_route_live", "cr_plan_churn", "cr_keymap_bytes", "cr_keymap_workspace_bytes", "cr_keymap_build",
           "cr_keymap_lookup", "cr_keymap_scatter", "cr_replay_workspace_bytes", "cr_lru_state_bytes",
           "cr_lru_reset", "cr_replay", "cr_replay_partition", "cr_replay_lru", "cr_replay_set_group_min_records",
           "cr_pages_workspace_bytes", "cr_pages_extend", "cr_pages_fork", "cr_pages_free", "cr_pages_compact",
           "cr_pages_copy", "cr_kv_append", "cr_attn_prompt_workspace_bytes", "cr_attn_prompt",
           "cr_attn_shared_workspace_bytes", "cr_attn_shared", "cr_kvq_extend", "cr_kvq_fork", "cr_kvq_free", "cr_kvq_compact",
           "cr_kvq_copy", "cr_kvq_append", "cr_kvq_read", "cr_kvq_attn_workspace_bytes", "cr_kvq_attn", "cr_rotary", "cr_version")
CR_WINDOW_SUM = 0xFFFFFFFFFFFFFFFF
CR_PLAN_BUFFERS = 16
CR_GROUP_MULTI, CR_GROUP_COLD = 0xFFFE, 0xFFFF

_u32, _u64, _P = ctypes.c_uint32, ctypes.c_uint64, ctypes.c_void_p


CR_PLAN_FULL, CR_PLAN_AFFINITY, CR_PLAN_REPLICATED, CR_PLAN_FLAT = 0, 1, 2, 3
PLAN_VARIANTS = {"full": CR_PLAN_FULL, "affinity": CR_PLAN_AFFINITY, "replicated": CR_PLAN_REPLICATED,
                 "flat": CR_PLAN_FLAT}


class CrPlanSpec(ctypes.Structure):
    _fields_ = [("window", _u32), ("W", _u32), ("n_window", _u64), ("q_num", _u64), ("q_den", _u64),
                ("variant", _u32), ("place_seed", _u32)]


class CrPlanSet(ctypes.Structure):
    _fields_ = [("num_plans", _u32), ("cands", _u32), ("R", _u32), ("max_W", _u32), ("num_keys", _u32),
                ("num_windows", _u32), ("specs", _P), ("order", _P), ("order_count", _P), ("n_order", _P),
                ("num_admitted", _P), ("cold", _P), ("clamped", _P), ("member_off", _P), ("members", _P),
                ("load", _P), ("key_index", _P), ("route", _P), ("window_rank", _P), ("group_dest", _P),
                ("group_rank", _P), ("group_multi", _P)]


CR_BF16, CR_F16 = 0, 1
CR_E4M3, CR_E5M2, CR_MAX_BLOCK_TOKENS = 0, 1, 128
CR_ROTARY_HALF, CR_ROTARY_PAIRS = 0, 1
CR_NO_PAGE = 0xFFFFFFFF
CR_ERR_SEQ, CR_ERR_PAGE, CR_ERR_PAGES_OUT = 16, 32, 64

_i64, _f32 = ctypes.c_int64, ctypes.c_float


class CrRows(ctypes.Structure):
    _fields_ = [("p", _P), ("token_stride", _i64), ("head_stride", _i64)]


class CrKvCache(ctypes.Structure):
    _fields_ = [("dtype", _u32), ("heads", _u32), ("dim", _u32), ("page_tokens", _u32), ("num_pages", _u32),
                ("layers", _u32), ("k", _P), ("v", _P), ("layer_stride", _i64), ("page_stride", _i64),
                ("head_stride", _i64), ("token_stride", _i64), ("refs", _P)]


class CrAttnPromptArgs(ctypes.Structure):
    _fields_ = [("dtype", _u32), ("heads_q", _u32), ("heads_kv", _u32), ("dim", _u32), ("batch", _u32), ("causal", _u32),
                ("total_q", _u32), ("total_k", _u32), ("scale", _f32), ("q", CrRows), ("k", CrRows), ("v", CrRows),
                ("out", CrRows), ("lse", _P), ("q_off", _P), ("k_off", _P)]


class CrAttnSharedArgs(ctypes.Structure):
    _fields_ = [("heads_q", _u32), ("layer", _u32), ("batch", _u32), ("groups", _u32), ("total_q", _u32),
                ("prefix_width", _u32), ("own_width", _u32), ("scale", _f32), ("q", CrRows), ("out", CrRows), ("lse", _P),
                ("q_off", _P), ("group_off", _P), ("prefix_table", _P), ("prefix_len", _P), ("own_table", _P),
                ("own_len", _P)]


class CrKvqCache(ctypes.Structure):
    _fields_ = [("dtype", _u32), ("code", _u32), ("heads", _u32), ("dim", _u32), ("page_tokens", _u32), ("block_tokens", _u32),
                ("num_pages", _u32), ("layers", _u32), ("k", _P), ("v", _P), ("layer_stride", _i64), ("page_stride", _i64),
                ("head_stride", _i64), ("token_stride", _i64), ("scale", _P), ("refs", _P)]


class CrKvqTokens(ctypes.Structure):
    _fields_ = [("layer", _u32), ("total", _u32), ("n", _u32), ("width", _u32), ("k", CrRows), ("v", CrRows), ("off", _P), ("length", _P),
                ("table", _P)]


class CrRotaryArgs(ctypes.Structure):
    _fields_ = [("dtype", _u32), ("heads_q", _u32), ("heads_k", _u32), ("dim", _u32), ("rotated", _u32), ("layout", _u32),
                ("total", _u32), ("magnitude", _f32), ("q", CrRows), ("k", CrRows), ("q_out", CrRows), ("k_out", CrRows),
                ("positions", _P), ("freq", _P)]


# The arguments laid out in one step (a ctypes structure takes ten times as long to fill); the calls take either.
ROWS = struct.Struct("@Pqq")
PROMPT_ARGS = struct.Struct("@8If" + "Pqq" * 4 + "PPP")
SHARED_ARGS = struct.Struct("@7If" + "Pqq" * 2 + "PPPPPPP")
ROTARY_ARGS = struct.Struct("@7If" + "Pqq" * 4 + "PP")
TOKENS_ARGS = struct.Struct("@4I" + "Pqq" * 2 + "PPP")
assert [x.size for x in (ROWS, PROMPT_ARGS, SHARED_ARGS, ROTARY_ARGS, TOKENS_ARGS)] == \
    [ctypes.sizeof(x) for x in (CrRows, CrAttnPromptArgs, CrAttnSharedArgs, CrRotaryArgs, CrKvqTokens)]


class CrError(RuntimeError):
    pass


_lib = None


def load(path: Optional[str] = None):
    """Load libcr.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    p = path or LIB
    if not os.path.exists(p):
        raise CrError(f"{p} is missing: build it with paper_2608_19677_amd/build.py (no fallback exists)")
    L = ctypes.CDLL(p)
    L.cr_count_rates.argtypes = [_P, _u64, _P, _u32, _u32, _P, _P, _P]
    L.cr_replay_set_group_min_records.argtypes = [_u64]
    L.cr_replay_set_group_min_records.restype = None
    L.cr_count_slice_workspace_bytes.argtypes = [_u64, _u32]
    L.cr_count_slice_workspace_bytes.restype = ctypes.c_size_t
    L.cr_count_slice.argtypes = [_P, _u64, _u32, _P, _P, _P, ctypes.c_size_t, _P]
    L.cr_plan_sizes.argtypes = [_u32, _u32, _u32, _u32, _u32, _u32, ctypes.POINTER(ctypes.c_size_t)]
    L.cr_plan_sizes.restype = None
    L.cr_workspace_bytes.argtypes = [_u32, _u32, _u32, _u64]
    L.cr_workspace_bytes.restype = ctypes.c_size_t
    L.cr_lru_state_bytes.argtypes = [_u32, _u32, _u32]
    L.cr_lru_state_bytes.restype = ctypes.c_size_t
    L.cr_lru_reset.argtypes = [_P, _u32, _u32, _u32, _P]
    L.cr_admit_workspace_bytes.argtypes = [_u32, _u32, _u32]
    L.cr_admit_workspace_bytes.restype = ctypes.c_size_t
    L.cr_admit.argtypes = [_P, ctypes.POINTER(CrPlanSet), _P, ctypes.c_size_t, _P, _P]
    L.cr_admit_noalloc.argtypes = [_P, ctypes.POINTER(CrPlanSet), _P, _P]
    L.cr_place_lpt.argtypes = [_P, ctypes.POINTER(CrPlanSet), _P]
    L.cr_place_hash.argtypes = [_P, ctypes.POINTER(CrPlanSet), _P]
    L.cr_route.argtypes = [_P, _u64, _u64, _u64, _P, _P, _u32, ctypes.POINTER(CrPlanSet), _P, _P, _P]
    L.cr_keymap_bytes.argtypes = [_u32]
    L.cr_keymap_bytes.restype = ctypes.c_size_t
    L.cr_keymap_workspace_bytes.argtypes = [_u64]
    L.cr_keymap_workspace_bytes.restype = ctypes.c_size_t
    L.cr_keymap_build.argtypes = [_P, _u64, _u32, _P, ctypes.c_size_t, _P, ctypes.c_size_t, _P, _P, _P]
    L.cr_keymap_lookup.argtypes = [_P, ctypes.c_size_t, _u32, _P, _u64, _P, _P]
    L.cr_keymap_scatter.argtypes = [_P, ctypes.c_size_t, _u32, _P, _P, _u64, _P, _u32, _P]
    L.cr_route_live.argtypes = [_P, _u64, _u64, _u64, _P, _P, _u32, ctypes.POINTER(CrPlanSet), _P, _P, _P]
    L.cr_plan_churn.argtypes = [ctypes.POINTER(CrPlanSet), _P, _u32, _P, _P, _P]
    L.cr_replay_workspace_bytes.argtypes = [_u64, _u32, _u32]
    L.cr_replay_workspace_bytes.restype = ctypes.c_size_t
    L.cr_replay.argtypes = [_P, _P, _P, _u32, _P, _u64, _P, _u32, _u32, _u32, ctypes.POINTER(_u32), _u32, _P, _P,
                            _P, _P, ctypes.c_size_t, _P, _P]
    L.cr_replay_partition.argtypes = [_P, _P, _P, _u64, _P, _u32, _u32, _u32, ctypes.POINTER(_u32), _P,
                                      ctypes.c_size_t, _P, _P]
    L.cr_replay_lru.argtypes = [_P, _u32, _u64, _u32, _u32, _u32, ctypes.POINTER(_u32), _u32, _P, _P, _P, _P,
                                ctypes.c_size_t, _P, _P]
    cache, size = ctypes.POINTER(CrKvCache), ctypes.c_size_t
    L.cr_pages_workspace_bytes.argtypes = [_u32, _u32]
    L.cr_pages_extend.argtypes = [cache, _P, _P, _u32, _P, _u32, _P, size, _P, _P]
    L.cr_pages_fork.argtypes = [cache, _P, _u32, _u32, _P, _P, _u32, _P, _u32, _P, size, _P, _P]
    L.cr_pages_free.argtypes = [cache, _P, _u32, _P, _u32, _P, _P]
    L.cr_pages_compact.argtypes = [cache, _P, _P, _u32, _u32, _P, _P, _P, size, _P, _P]
    L.cr_pages_copy.argtypes = [cache, _P, _P, _u32, _P, _P]
    L.cr_kv_append.argtypes = [cache, _u32, _P, _P, _u32, _P, _P, _u32, _P, _u32, _P, _P]
    L.cr_attn_prompt_workspace_bytes.argtypes = [_P]
    L.cr_attn_prompt.argtypes = [_P, _P, size, _P, _P]
    L.cr_attn_shared_workspace_bytes.argtypes = [cache, _P]
    L.cr_attn_shared.argtypes = [cache, _P, _P, size, _P, _P]
    coded = ctypes.POINTER(CrKvqCache)
    for f in ("extend", "fork", "free", "compact", "copy"):
        getattr(L, "cr_kvq_" + f).argtypes = [coded] + getattr(L, "cr_pages_" + f).argtypes[1:]
    L.cr_kvq_append.argtypes = L.cr_kvq_read.argtypes = [coded, _P, _P, _P]
    L.cr_kvq_attn_workspace_bytes.argtypes = [coded, _P]
    L.cr_kvq_attn.argtypes = [coded, _P, _P, size, _P, _P]
    L.cr_rotary.argtypes = [_P, _P]
    for f in ("cr_pages_workspace_bytes", "cr_attn_prompt_workspace_bytes", "cr_attn_shared_workspace_bytes", "cr_kvq_attn_workspace_bytes"):
        getattr(L, f).restype = size
    L.cr_version.restype = ctypes.c_char_p
    for f in ("cr_count_rates", "cr_count_slice", "cr_lru_reset", "cr_admit", "cr_admit_noalloc", "cr_place_lpt", "cr_place_hash", "cr_route", "cr_route_live", "cr_plan_churn",
              "cr_keymap_build", "cr_keymap_lookup", "cr_keymap_scatter", "cr_replay",
              "cr_replay_partition", "cr_replay_lru", "cr_pages_extend", "cr_pages_fork", "cr_pages_free",
              "cr_pages_compact", "cr_pages_copy", "cr_kv_append", "cr_attn_prompt", "cr_attn_shared", "cr_kvq_extend",
              "cr_kvq_fork", "cr_kvq_free", "cr_kvq_compact", "cr_kvq_copy", "cr_kvq_append", "cr_kvq_read", "cr_kvq_attn", "cr_rotary"):
        getattr(L, f).restype = ctypes.c_int32
    _lib = L
    return L


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_cuda:
        raise CrError("libcr takes device tensors")
    if not t.is_contiguous():
        raise CrError("libcr takes contiguous tensors")
    return t.data_ptr()


# The current stream's handle without a Stream object around it (4 us less per call), where torch has it.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _stream(stream) -> Optional[int]:
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is not None:
        return _raw_stream(_device())
    return torch.cuda.current_stream().cuda_stream


def _check(rc: int, name: str):
    if rc != CR_OK:
        raise CrError(f"{name} returned {rc}")


def cr_version() -> str:
    return load().cr_version().decode()


def cr_count_rates(keys, off, J: int, num_keys: int, counts, err, stream=None, n: Optional[int] = None):
    n = keys.numel() if n is None else n
    _check(load().cr_count_rates(_ptr(keys), n, _ptr(off), J, num_keys, _ptr(counts), _ptr(err), _stream(stream)),
           "cr_count_rates")


def cr_count_slice_workspace_bytes(n: int, num_keys: int) -> int:
    return int(load().cr_count_slice_workspace_bytes(n, num_keys))


def cr_count_slice(keys, num_keys: int, counts, err, ws, stream=None, n: Optional[int] = None):
    n = keys.numel() if n is None else n
    _check(load().cr_count_slice(_ptr(keys), n, num_keys, _ptr(counts), _ptr(err), _ptr(ws), _nbytes(ws),
                                 _stream(stream)), "cr_count_slice")


def cr_plan_sizes(num_plans: int, cands: int, R: int, max_W: int, num_keys: int, num_windows: int):
    out = (ctypes.c_size_t * CR_PLAN_BUFFERS)()
    load().cr_plan_sizes(num_plans, cands, R, max_W, num_keys, num_windows, out)
    return [int(x) for x in out]


def cr_workspace_bytes(num_keys: int, R: int, P: int, max_n: int) -> int:
    return int(load().cr_workspace_bytes(num_keys, R, P, max_n))


def cr_lru_state_bytes(P: int, R: int, max_W: int) -> int:
    return int(load().cr_lru_state_bytes(P, R, max_W))


def cr_lru_reset(lru_state, P: int, R: int, max_W: int, stream=None):
    _check(load().cr_lru_reset(_ptr(lru_state), P, R, max_W, _stream(stream)), "cr_lru_reset")


def cr_admit_workspace_bytes(num_windows: int, R: int, max_W: int) -> int:
    return int(load().cr_admit_workspace_bytes(num_windows, R, max_W))


def cr_admit(counts, plans: CrPlanSet, ws, err, stream=None):
    _check(load().cr_admit(_ptr(counts), ctypes.byref(plans), _ptr(ws), ws.numel() * ws.element_size(), _ptr(err),
                           _stream(stream)), "cr_admit")


def cr_admit_noalloc(counts, plans: CrPlanSet, err, stream=None):
    _check(load().cr_admit_noalloc(_ptr(counts), ctypes.byref(plans), _ptr(err), _stream(stream)), "cr_admit_noalloc")


def cr_place_lpt(counts, plans: CrPlanSet, stream=None):
    _check(load().cr_place_lpt(_ptr(counts), ctypes.byref(plans), _stream(stream)), "cr_place_lpt")


def cr_place_hash(counts, plans: CrPlanSet, stream=None):
    _check(load().cr_place_hash(_ptr(counts), ctypes.byref(plans), _stream(stream)), "cr_place_hash")


def cr_route(keys, first_index: int, seed: int, off, gmap, J: int, plans: CrPlanSet, dest, err, stream=None,
             n: Optional[int] = None):
    n = keys.numel() if n is None else n
    _check(load().cr_route(_ptr(keys), n, first_index, seed, _ptr(off), _ptr(gmap), J, ctypes.byref(plans),
                           _ptr(dest), _ptr(err), _stream(stream)), "cr_route")


def cr_keymap_bytes(capacity: int) -> int:
    return int(load().cr_keymap_bytes(capacity))


def cr_keymap_workspace_bytes(n: int) -> int:
    return int(load().cr_keymap_workspace_bytes(n))


def _nbytes(t) -> int:
    return t.numel() * t.element_size()


def cr_keymap_build(ids, capacity: int, table, ws, num_keys, err, stream=None, n: Optional[int] = None):
    n = ids.numel() if n is None else n
    _check(load().cr_keymap_build(_ptr(ids), n, capacity, _ptr(table), _nbytes(table), _ptr(ws), _nbytes(ws),
                                  _ptr(num_keys), _ptr(err), _stream(stream)), "cr_keymap_build")


def cr_keymap_lookup(table, capacity: int, ids, dense, stream=None, n: Optional[int] = None):
    n = ids.numel() if n is None else n
    _check(load().cr_keymap_lookup(_ptr(table), _nbytes(table), capacity, _ptr(ids), n, _ptr(dense), _stream(stream)),
           "cr_keymap_lookup")


def cr_keymap_scatter(table, capacity: int, ids, values, out, stream=None):
    _check(load().cr_keymap_scatter(_ptr(table), _nbytes(table), capacity, _ptr(ids), _ptr(values), ids.numel(),
                                    _ptr(out), out.numel(), _stream(stream)), "cr_keymap_scatter")


def cr_route_live(keys, first_index: int, seed: int, off, gmap, J: int, plans: CrPlanSet, dest, err, stream=None,
                  n: Optional[int] = None):
    n = keys.numel() if n is None else n
    _check(load().cr_route_live(_ptr(keys), n, first_index, seed, _ptr(off), _ptr(gmap), J, ctypes.byref(plans),
                                _ptr(dest), _ptr(err), _stream(stream)), "cr_route_live")


def cr_plan_churn(plans: CrPlanSet, pairs, out, err, stream=None):
    """pairs: int32 [num_pairs, 2] plan indices; out: int64 [num_pairs, 4]."""
    num_pairs = pairs.shape[0]
    _check(load().cr_plan_churn(ctypes.byref(plans), _ptr(pairs), num_pairs, _ptr(out), _ptr(err), _stream(stream)),
           "cr_plan_churn")


def cr_replay_workspace_bytes(n: int, P: int, R: int) -> int:
    return int(load().cr_replay_workspace_bytes(n, P, R))


GROUP_MIN_RECORDS_DEFAULT = 1 << 25


def cr_replay_set_group_min_records(min_records: int) -> None:
    load().cr_replay_set_group_min_records(min_records)


def cr_replay(keys, suffix, prefix_len, num_keys: int, dest, off, J: int, P: int, R: int, W: Sequence[int],
              max_W: int, lru_in, lru_out, stats, ws, err, stream=None, n: Optional[int] = None):
    n = keys.numel() if n is None else n
    Wa = (_u32 * len(W))(*[int(x) for x in W])
    _check(load().cr_replay(_ptr(keys), _ptr(suffix), _ptr(prefix_len), num_keys, _ptr(dest), n, _ptr(off), J, P, R,
                            Wa, max_W, _ptr(lru_in), _ptr(lru_out), _ptr(stats), _ptr(ws),
                            ws.numel() * ws.element_size(), _ptr(err), _stream(stream)), "cr_replay")


def cr_replay_partition(keys, suffix, dest, off, J: int, P: int, R: int, W: Sequence[int], ws, err, stream=None,
                        n: Optional[int] = None):
    n = keys.numel() if n is None else n
    Wa = (_u32 * len(W))(*[int(x) for x in W])
    _check(load().cr_replay_partition(_ptr(keys), _ptr(suffix), _ptr(dest), n, _ptr(off), J, P, R, Wa, _ptr(ws),
                                      ws.numel() * ws.element_size(), _ptr(err), _stream(stream)),
           "cr_replay_partition")


def cr_replay_lru(prefix_len, num_keys: int, n: int, J: int, P: int, R: int, W: Sequence[int], max_W: int, lru_in,
                  lru_out, stats, ws, err, stream=None):
    Wa = (_u32 * len(W))(*[int(x) for x in W])
    _check(load().cr_replay_lru(_ptr(prefix_len), num_keys, n, J, P, R, Wa, max_W, _ptr(lru_in), _ptr(lru_out),
                                _ptr(stats), _ptr(ws), ws.numel() * ws.element_size(), _ptr(err), _stream(stream)),
           "cr_replay_lru")


def cr_pages_workspace_bytes(num_pages: int, n: int) -> int:
    return int(load().cr_pages_workspace_bytes(num_pages, n))


def _table_width(t) -> int:
    return 0 if t is None else t.shape[-1]


def cr_pages_extend(cache: CrKvCache, len_old, len_new, table, ws, err, stream=None):
    """len_old (or None), len_new: int32 [n]; table: int32 [n, width]."""
    _check(load().cr_pages_extend(ctypes.byref(cache), _ptr(len_old), _ptr(len_new), len_new.numel(), _ptr(table),
                                  _table_width(table), _ptr(ws), _nbytes(ws), _ptr(err), _stream(stream)),
           "cr_pages_extend")


def cr_pages_fork(cache: CrKvCache, table, parent, length, child, ws, err, stream=None):
    """table: int32 [rows, width]; parent, length: int32 [n]; child: int32 [n, child_width]."""
    _check(load().cr_pages_fork(ctypes.byref(cache), _ptr(table), table.shape[0], _table_width(table), _ptr(parent),
                                _ptr(length), parent.numel(), _ptr(child), _table_width(child), _ptr(ws), _nbytes(ws),
                                _ptr(err), _stream(stream)), "cr_pages_fork")


def cr_pages_free(cache: CrKvCache, table, length, err, stream=None):
    _check(load().cr_pages_free(ctypes.byref(cache), _ptr(table), _table_width(table), _ptr(length), length.numel(),
                                _ptr(err), _stream(stream)), "cr_pages_free")


def cr_pages_compact(cache: CrKvCache, table, length, table_out, refs_out, ws, err, stream=None):
    """table, table_out: int32 [rows, width] (or None); length: int32 [rows]."""
    rows = 0 if table is None else table.shape[0]
    _check(load().cr_pages_compact(ctypes.byref(cache), _ptr(table), _ptr(length), rows, _table_width(table),
                                   _ptr(table_out), _ptr(refs_out), _ptr(ws), _nbytes(ws), _ptr(err), _stream(stream)),
           "cr_pages_compact")


def cr_pages_copy(cache: CrKvCache, src, dst, err, stream=None):
    _check(load().cr_pages_copy(ctypes.byref(cache), _ptr(src), _ptr(dst), src.numel(), _ptr(err), _stream(stream)),
           "cr_pages_copy")


def _ref(s):
    """A structure, or its packed bytes."""
    return s if type(s) is bytes else ctypes.byref(s)


def cr_kv_append(cache: CrKvCache, layer: int, k: CrRows, v: CrRows, total: int, off, length, table, err, stream=None):
    _check(load().cr_kv_append(ctypes.byref(cache), layer, _ref(k), _ref(v), total, _ptr(off), _ptr(length),
                               length.numel(), _ptr(table), _table_width(table), _ptr(err), _stream(stream)), "cr_kv_append")


def cr_attn_prompt_workspace_bytes(args: CrAttnPromptArgs) -> int:
    return int(load().cr_attn_prompt_workspace_bytes(_ref(args)))


def cr_attn_prompt(args: CrAttnPromptArgs, ws, err, stream=None):
    _check(load().cr_attn_prompt(_ref(args), _ptr(ws), 0 if ws is None else _nbytes(ws), _ptr(err), _stream(stream)),
           "cr_attn_prompt")


def cr_attn_shared_workspace_bytes(cache: CrKvCache, args: CrAttnSharedArgs) -> int:
    return int(load().cr_attn_shared_workspace_bytes(ctypes.byref(cache), _ref(args)))


def cr_attn_shared(cache: CrKvCache, args: CrAttnSharedArgs, ws, err, stream=None):
    _check(load().cr_attn_shared(ctypes.byref(cache), _ref(args), _ptr(ws), 0 if ws is None else _nbytes(ws),
                                 _ptr(err), _stream(stream)), "cr_attn_shared")


def cr_kvq_extend(cache: CrKvqCache, len_old, len_new, table, ws, err, stream=None):
    _check(load().cr_kvq_extend(ctypes.byref(cache), _ptr(len_old), _ptr(len_new), len_new.numel(), _ptr(table),
                                _table_width(table), _ptr(ws), _nbytes(ws), _ptr(err), _stream(stream)), "cr_kvq_extend")


def cr_kvq_fork(cache: CrKvqCache, table, parent, length, child, ws, err, stream=None):
    _check(load().cr_kvq_fork(ctypes.byref(cache), _ptr(table), table.shape[0], _table_width(table), _ptr(parent),
                              _ptr(length), parent.numel(), _ptr(child), _table_width(child), _ptr(ws), _nbytes(ws),
                              _ptr(err), _stream(stream)), "cr_kvq_fork")


def cr_kvq_free(cache: CrKvqCache, table, length, err, stream=None):
    _check(load().cr_kvq_free(ctypes.byref(cache), _ptr(table), _table_width(table), _ptr(length), length.numel(), _ptr(err),
                              _stream(stream)), "cr_kvq_free")


def cr_kvq_compact(cache: CrKvqCache, table, length, table_out, refs_out, ws, err, stream=None):
    """table, table_out: int32 [rows, width] (or None); length: int32 [rows]."""
    rows = 0 if table is None else table.shape[0]
    _check(load().cr_kvq_compact(ctypes.byref(cache), _ptr(table), _ptr(length), rows, _table_width(table),
                                 _ptr(table_out), _ptr(refs_out), _ptr(ws), _nbytes(ws), _ptr(err), _stream(stream)),
           "cr_kvq_compact")


def cr_kvq_copy(cache: CrKvqCache, src, dst, err, stream=None):
    _check(load().cr_kvq_copy(ctypes.byref(cache), _ptr(src), _ptr(dst), src.numel(), _ptr(err), _stream(stream)), "cr_kvq_copy")


def cr_kvq_append(cache: CrKvqCache, tokens: CrKvqTokens, err, stream=None):
    _check(load().cr_kvq_append(ctypes.byref(cache), _ref(tokens), _ptr(err), _stream(stream)), "cr_kvq_append")


def cr_kvq_read(cache: CrKvqCache, tokens: CrKvqTokens, err, stream=None):
    _check(load().cr_kvq_read(ctypes.byref(cache), _ref(tokens), _ptr(err), _stream(stream)), "cr_kvq_read")


def cr_kvq_attn_workspace_bytes(cache: CrKvqCache, args: CrAttnSharedArgs) -> int:
    return int(load().cr_kvq_attn_workspace_bytes(ctypes.byref(cache), _ref(args)))


def cr_kvq_attn(cache: CrKvqCache, args: CrAttnSharedArgs, ws, err, stream=None):
    _check(load().cr_kvq_attn(ctypes.byref(cache), _ref(args), _ptr(ws), 0 if ws is None else _nbytes(ws), _ptr(err),
                              _stream(stream)), "cr_kvq_attn")


def cr_rotary(args: CrRotaryArgs, stream=None):
    _check(load().cr_rotary(_ref(args), _stream(stream)), "cr_rotary")


class PlanSet:
    """Device buffers of a cr_plan_set (NP = NG * cands plans over num_windows rows).
    ``group_tables`` also allocates the optional group dispatch tables that let cr_route
    serve every candidate of a request from one row (candidates of a group must share
    their counting window)."""

    def __init__(self, specs, cands: int, R: int, max_W: int, num_keys: int, num_windows: int, device,
                 group_tables: bool = False):
        self.num_plans = len(specs)
        self.cands, self.R, self.max_W, self.num_keys, self.num_windows = cands, R, max_W, num_keys, num_windows
        cmax = R * max_W
        self.cmax = cmax
        NP, NW = self.num_plans, num_windows
        raw = (CrPlanSpec * NP)(*[CrPlanSpec(*s) for s in specs])
        host = torch.frombuffer(bytearray(bytes(raw)), dtype=torch.uint8)
        self.specs = host.to(device)
        i32 = dict(dtype=torch.int32, device=device)
        self.order = torch.empty((NW, cmax), **i32)
        self.order_count = torch.empty((NW, cmax), **i32)
        self.n_order = torch.empty(NW, **i32)
        self.num_admitted = torch.empty(NP, **i32)
        self.cold = torch.empty(NP, dtype=torch.int64, device=device)
        self.clamped = torch.empty(NP, **i32)
        self.member_off = torch.empty((NP, cmax + 1), **i32)
        self.members = torch.empty((NP, cmax), dtype=torch.int16, device=device)
        self.load = torch.empty((NP, R), dtype=torch.float64, device=device)
        self.key_index = torch.empty((NP, (num_keys + 63) // 64, 2), dtype=torch.int64, device=device)
        self.route = torch.empty((NP, cmax), **i32)
        self.window_rank = self.group_dest = self.group_rank = self.group_multi = None
        if group_tables:
            NG = NP // cands
            self.window_rank = torch.empty((NW, num_keys), **i32)
            self.group_dest = torch.empty((NG, cmax, group_row(cands)), dtype=torch.int16, device=device)
            self.group_rank = torch.empty((NG, R, group_row(cands)), dtype=torch.int16, device=device)
            self.group_multi = torch.empty((NG, cmax, group_row(cands)), **i32)
        self.c = CrPlanSet(NP, cands, R, max_W, num_keys, NW, _ptr(self.specs), _ptr(self.order),
                           _ptr(self.order_count), _ptr(self.n_order),
                           _ptr(self.num_admitted), _ptr(self.cold), _ptr(self.clamped), _ptr(self.member_off),
                           _ptr(self.members), _ptr(self.load), _ptr(self.key_index), _ptr(self.route),
                           _ptr(self.window_rank), _ptr(self.group_dest), _ptr(self.group_rank),
                           _ptr(self.group_multi))


def group_row(cands: int) -> int:
    """Entries per group_dest row: cands rounded up to a multiple of 8."""
    return (cands + 7) // 8 * 8


def group_table_bytes(NG: int, cands: int, R: int, max_W: int, num_keys: int, num_windows: int) -> int:
    """Bytes of the four group dispatch tables."""
    return (num_windows * num_keys * 4 + NG * R * max_W * group_row(cands) * 6
            + NG * R * group_row(cands) * 2)
