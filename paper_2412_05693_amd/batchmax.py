"""Thin ctypes binding of ``libbatchmax.so`` (include/batchmax.h).

The functions named ``bm_*`` mirror the C ABI one to one: they marshal
arguments (integers, pointers as Python ints, ctypes structs) and raise
``BatchMaxError`` on a non-OK status.  Every step of the path runs in the HIP
kernels behind the library; nothing here computes.

``PDAttention`` is a convenience owner of the cache tensors (torch allocates the
device memory; the library never does) that checks dtype, device, shape and
contiguity before handing raw pointers and the current HIP stream to the ABI.

Importing this module loads the library and fails loudly if it is missing:
there is no fallback path.
"""
from __future__ import annotations

import ctypes
import math
import os
import warnings

HERE = os.path.dirname(os.path.abspath(__file__))
# BATCHMAX_LIB selects another build of the same library (the host-sanitizer
# build of build.py --sanitize, for CPU tests); the default is the in-tree one
LIB_PATH = os.environ.get("BATCHMAX_LIB") or os.path.join(HERE, "libbatchmax.so")

BM_OK, BM_ERR_INVALID_ARG, BM_ERR_UNSUPPORTED, BM_ERR_CAPACITY, BM_ERR_ORDER, BM_ERR_HIP = range(6)
BM_F32, BM_BF16 = 0, 1
BM_RANK_AVE, BM_RANK_SUM, BM_RANK_RECENT, BM_RANK_TOVA = 0, 1, 2, 3
RANK_RULES = {"ave": BM_RANK_AVE, "sum": BM_RANK_SUM, "recent": BM_RANK_RECENT,
              "tova": BM_RANK_TOVA}
STATUS_NAMES = {0: "BM_OK", 1: "BM_ERR_INVALID_ARG", 2: "BM_ERR_UNSUPPORTED",
                3: "BM_ERR_CAPACITY", 4: "BM_ERR_ORDER", 5: "BM_ERR_HIP"}


class BatchMaxError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {message}")
        self.status = status


class bm_dims(ctypes.Structure):
    _fields_ = [("b", ctypes.c_int32), ("s", ctypes.c_int32), ("kv_max", ctypes.c_int32),
                ("block", ctypes.c_int32), ("max_gen", ctypes.c_int32),
                ("n_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("sm_scale", ctypes.c_float)]


class bm_synth(ctypes.Structure):
    _fields_ = [("b", ctypes.c_int32), ("n_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32), ("seed", ctypes.c_uint32),
                ("layer", ctypes.c_int32), ("s", ctypes.c_int32), ("hh_threshold", ctypes.c_uint32),
                ("hh_scale", ctypes.c_float), ("n_sinks", ctypes.c_int32),
                ("sink_scale", ctypes.c_float), ("value_scale", ctypes.c_float)]


class bm_cache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("score", ctypes.c_void_p),
                ("pos", ctypes.c_void_p), ("len", ctypes.c_void_p), ("work", ctypes.c_void_p),
                ("work_bytes", ctypes.c_size_t)]


class bm_kv4_cache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p), ("score", ctypes.c_void_p), ("pos", ctypes.c_void_p),
                ("len", ctypes.c_void_p), ("work", ctypes.c_void_p),
                ("work_bytes", ctypes.c_size_t)]


class bm_win_cache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("work", ctypes.c_void_p),
                ("work_bytes", ctypes.c_size_t)]


BM_DRAFT_MAX = 64       # nodes of a tree of drafted tokens
BM_KV4_GROUP = 32       # elements that share one scale of a 4-bit row
_INT32_MAX = 0x7FFFFFFF # ctypes passes an integer modulo 2^32: the library would not see one beyond


def _load() -> ctypes.CDLL:
    # torch ships its own HIP runtime under the same soname as ROCm's; load it
    # first so this library binds to that single runtime instead of a second copy
    import torch  # noqa: F401

    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is not built; run `python -m paper_2412_05693_amd.build` "
            "(there is no non-HIP fallback)")
    lib = ctypes.CDLL(LIB_PATH)
    P, I32, SZ = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    dims_p, cache_p = ctypes.POINTER(bm_dims), ctypes.POINTER(bm_cache)
    kv4_p = ctypes.POINTER(bm_kv4_cache)
    win_p = ctypes.POINTER(bm_win_cache)
    sig = {
        "bm_abi_version": (ctypes.c_int, []),
        "bm_last_error": (ctypes.c_char_p, []),
        "bm_cache_slots": (I32, [dims_p]),
        "bm_workspace_bytes": (SZ, [dims_p]),
        "bm_prefill_positions_per_workgroup": (I32, [dims_p]),
        "bm_validate_dims": (ctypes.c_int, [dims_p]),
        "bm_init": (ctypes.c_int, [dims_p, cache_p, P, ctypes.POINTER(P)]),
        "bm_init_static_workspace": (ctypes.c_int, [dims_p, cache_p, P, ctypes.POINTER(P)]),
        "bm_resume": (ctypes.c_int, [dims_p, cache_p, I32, I32, ctypes.POINTER(P)]),
        "bm_prefill_block": (ctypes.c_int, [P, I32, I32, P, P, P, P, I32, P]),
        "bm_prefill_block_cut": (ctypes.c_int, [P, I32, I32, P, P, P, P, I32, P]),
        "bm_evict_compact": (ctypes.c_int, [P, I32, P]),
        "bm_set_decode_removal": (ctypes.c_int, [P, I32]),
        "bm_set_rank_rule": (ctypes.c_int, [P, I32]),
        "bm_set_decode_bound": (ctypes.c_int, [P, I32]),
        "bm_set_score_accumulation": (ctypes.c_int, [P, I32]),
        "bm_set_left_padding": (ctypes.c_int, [P, P]),
        "bm_set_split_event": (ctypes.c_int, [P, P]),
        "bm_decode_step": (ctypes.c_int, [P, I32, P, P, P, P, I32, P]),
        "bm_kv4_slots": (I32, [dims_p]),
        "bm_kv4_workspace_bytes": (SZ, [dims_p]),
        "bm_kv4_init": (ctypes.c_int, [dims_p, kv4_p, P, ctypes.POINTER(P)]),
        "bm_kv4_resume": (ctypes.c_int, [dims_p, kv4_p, I32, I32, ctypes.POINTER(P)]),
        "bm_kv4_write": (ctypes.c_int, [dims_p, kv4_p, I32, I32, P, P, I32, P]),
        "bm_kv4_read": (ctypes.c_int, [dims_p, kv4_p, I32, I32, P, P, I32, P]),
        "bm_win_workspace_bytes": (SZ, [dims_p]),
        "bm_win_validate": (ctypes.c_int, [dims_p, I32]),
        "bm_win_init": (ctypes.c_int, [dims_p, I32, win_p, ctypes.POINTER(P)]),
        "bm_win_resume": (ctypes.c_int, [dims_p, I32, win_p, I32, ctypes.POINTER(P)]),
        "bm_draft_workspace_bytes": (SZ, [dims_p, I32]),
        "bm_draft_attend": (ctypes.c_int, [P, I32, P, P, P, P, P, I32, P, P, SZ, P]),
        "bm_draft_accept": (ctypes.c_int, [P, I32, I32, P, P, P, P, P, I32, P, P]),
        "bm_ctx_len": (I32, [P]),
        "bm_ctx_next_pos": (I32, [P]),
        "bm_destroy": (None, [P]),
        "bm_synth_qkv": (ctypes.c_int, [ctypes.POINTER(bm_synth), I32, I32, P, P, P, I32, P]),
        "bm_philox4x32_10": (ctypes.c_int, [P, P, ctypes.c_int64, P]),
        "bm_probe_stream_read": (ctypes.c_int, [P, SZ, P, I32, I32, P]),
        "bm_probe_mfma": (ctypes.c_int, [I32, P, I32, P]),
        "bm_prefill_timeline": (ctypes.c_int, [P, I32]),
        "bm_prefill_tile_workgroups": (I32, [P, I32, P, P, I32]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    return lib


_lib = _load()
EXPORTED = ("bm_abi_version", "bm_last_error", "bm_cache_slots", "bm_workspace_bytes",
            "bm_prefill_positions_per_workgroup",
            "bm_validate_dims", "bm_init", "bm_init_static_workspace", "bm_resume", "bm_prefill_block",
            "bm_prefill_block_cut", "bm_evict_compact",
            "bm_set_decode_removal", "bm_set_rank_rule", "bm_set_decode_bound",
            "bm_set_score_accumulation", "bm_set_left_padding", "bm_set_split_event",
            "bm_decode_step", "bm_ctx_len", "bm_ctx_next_pos", "bm_destroy", "bm_synth_qkv",
            "bm_kv4_slots", "bm_kv4_workspace_bytes", "bm_kv4_init", "bm_kv4_resume", "bm_kv4_write", "bm_kv4_read",
            "bm_win_workspace_bytes", "bm_win_validate", "bm_win_init", "bm_win_resume",
            "bm_draft_workspace_bytes", "bm_draft_attend", "bm_draft_accept",
            "bm_philox4x32_10", "bm_probe_stream_read", "bm_probe_mfma",
            "bm_prefill_timeline", "bm_prefill_tile_workgroups")


def _check(status: int) -> None:
    if status != BM_OK:
        raise BatchMaxError(status, _lib.bm_last_error().decode())


# ---------------------------------------------------------------------------
# one-to-one ABI wrappers
# ---------------------------------------------------------------------------
def bm_abi_version() -> int:
    return _lib.bm_abi_version()


def bm_last_error() -> str:
    return _lib.bm_last_error().decode()


def bm_cache_slots(dims: bm_dims) -> int:
    return _lib.bm_cache_slots(ctypes.byref(dims))


def bm_workspace_bytes(dims: bm_dims) -> int:
    return _lib.bm_workspace_bytes(ctypes.byref(dims))


def bm_prefill_positions_per_workgroup(dims: bm_dims) -> int:
    return _lib.bm_prefill_positions_per_workgroup(ctypes.byref(dims))


def bm_validate_dims(dims: bm_dims) -> None:
    _check(_lib.bm_validate_dims(ctypes.byref(dims)))


def bm_init(dims: bm_dims, cache: bm_cache, stream: int) -> int:
    out = ctypes.c_void_p()
    _check(_lib.bm_init(ctypes.byref(dims), ctypes.byref(cache), stream, ctypes.byref(out)))
    return out.value


def bm_init_static_workspace(dims: bm_dims, cache: bm_cache, stream: int) -> int:
    out = ctypes.c_void_p()
    _check(_lib.bm_init_static_workspace(ctypes.byref(dims), ctypes.byref(cache), stream,
                                         ctypes.byref(out)))
    return out.value


def bm_resume(dims: bm_dims, cache: bm_cache, length: int, next_pos: int) -> int:
    out = ctypes.c_void_p()
    _check(_lib.bm_resume(ctypes.byref(dims), ctypes.byref(cache), length, next_pos,
                          ctypes.byref(out)))
    return out.value


def bm_prefill_block(ctx: int, t0: int, n_tok: int, q: int, k: int, v: int, o: int,
                     seq_ld: int, stream: int) -> None:
    _check(_lib.bm_prefill_block(ctx, t0, n_tok, q, k, v, o, seq_ld, stream))


def bm_prefill_block_cut(ctx: int, t0: int, n_tok: int, q: int, k: int, v: int, o: int,
                         seq_ld: int, stream: int) -> None:
    _check(_lib.bm_prefill_block_cut(ctx, t0, n_tok, q, k, v, o, seq_ld, stream))


def bm_evict_compact(ctx: int, curr_id: int, stream: int) -> None:
    _check(_lib.bm_evict_compact(ctx, curr_id, stream))


def bm_set_decode_removal(ctx: int, p: int) -> None:
    _check(_lib.bm_set_decode_removal(ctx, p))


def bm_set_rank_rule(ctx: int, rule: int) -> None:
    _check(_lib.bm_set_rank_rule(ctx, rule))


def bm_set_decode_bound(ctx: int, bound: int) -> None:
    _check(_lib.bm_set_decode_bound(ctx, bound))


def bm_set_score_accumulation(ctx: int, on: int) -> None:
    _check(_lib.bm_set_score_accumulation(ctx, on))


def bm_set_left_padding(ctx: int, pad_ptr: int) -> None:
    _check(_lib.bm_set_left_padding(ctx, pad_ptr))


def bm_set_split_event(ctx: int, event: int) -> None:
    _check(_lib.bm_set_split_event(ctx, event))


def bm_decode_step(ctx: int, pos: int, q: int, k: int, v: int, o: int, seq_ld: int,
                   stream: int) -> None:
    _check(_lib.bm_decode_step(ctx, pos, q, k, v, o, seq_ld, stream))


def bm_kv4_slots(dims: bm_dims) -> int:
    return _lib.bm_kv4_slots(ctypes.byref(dims))


def bm_kv4_workspace_bytes(dims: bm_dims) -> int:
    return _lib.bm_kv4_workspace_bytes(ctypes.byref(dims))


def bm_kv4_init(dims: bm_dims, cache: bm_kv4_cache, stream: int) -> int:
    out = ctypes.c_void_p()
    _check(_lib.bm_kv4_init(ctypes.byref(dims), ctypes.byref(cache), stream, ctypes.byref(out)))
    return out.value


def bm_kv4_resume(dims: bm_dims, cache: bm_kv4_cache, length: int, next_pos: int) -> int:
    out = ctypes.c_void_p()
    _check(_lib.bm_kv4_resume(ctypes.byref(dims), ctypes.byref(cache), length, next_pos,
                              ctypes.byref(out)))
    return out.value


def bm_kv4_write(dims: bm_dims, cache: bm_kv4_cache, slot0: int, n: int, k: int, v: int,
                 seq_ld: int, stream: int) -> None:
    _check(_lib.bm_kv4_write(ctypes.byref(dims), ctypes.byref(cache), slot0, n, k, v, seq_ld, stream))


def bm_kv4_read(dims: bm_dims, cache: bm_kv4_cache, slot0: int, n: int, k: int, v: int,
                seq_ld: int, stream: int) -> None:
    _check(_lib.bm_kv4_read(ctypes.byref(dims), ctypes.byref(cache), slot0, n, k, v, seq_ld, stream))


def bm_win_workspace_bytes(dims: bm_dims) -> int:
    return _lib.bm_win_workspace_bytes(ctypes.byref(dims))


def bm_win_validate(dims: bm_dims, sinks: int) -> None:
    _check(_lib.bm_win_validate(ctypes.byref(dims), sinks))


def bm_win_init(dims: bm_dims, sinks: int, cache: bm_win_cache) -> int:
    out = ctypes.c_void_p()
    _check(_lib.bm_win_init(ctypes.byref(dims), sinks, ctypes.byref(cache), ctypes.byref(out)))
    return out.value


def bm_win_resume(dims: bm_dims, sinks: int, cache: bm_win_cache, next_pos: int) -> int:
    out = ctypes.c_void_p()
    _check(_lib.bm_win_resume(ctypes.byref(dims), sinks, ctypes.byref(cache), next_pos,
                              ctypes.byref(out)))
    return out.value


def bm_draft_workspace_bytes(dims: bm_dims, n: int) -> int:
    return _lib.bm_draft_workspace_bytes(ctypes.byref(dims), n)


def bm_draft_attend(ctx: int, n: int, parent: int, q: int, k: int, v: int, o: int, seq_ld: int,
                    lse: int, work: int, work_bytes: int, stream: int) -> None:
    _check(_lib.bm_draft_attend(ctx, n, parent, q, k, v, o, seq_ld, lse, work, work_bytes, stream))


def bm_draft_accept(ctx: int, n: int, m: int, path: int, count: int, q: int, k: int, v: int,
                    seq_ld: int, lse: int, stream: int) -> None:
    _check(_lib.bm_draft_accept(ctx, n, m, path, count, q, k, v, seq_ld, lse, stream))


def bm_ctx_len(ctx: int) -> int:
    return _lib.bm_ctx_len(ctx)


def bm_ctx_next_pos(ctx: int) -> int:
    return _lib.bm_ctx_next_pos(ctx)


def bm_destroy(ctx: int) -> None:
    _lib.bm_destroy(ctx)


def bm_synth_qkv(params: bm_synth, t0: int, n_rows: int, q: int, k: int, v: int, seq_ld: int,
                 stream: int) -> None:
    _check(_lib.bm_synth_qkv(ctypes.byref(params), t0, n_rows, q, k, v, seq_ld, stream))


def bm_philox4x32_10(inp: int, out: int, n: int, stream: int) -> None:
    _check(_lib.bm_philox4x32_10(inp, out, n, stream))


def bm_probe_stream_read(src: int, nbytes: int, sink: int, blocks: int, nontemporal: bool,
                         stream: int) -> None:
    _check(_lib.bm_probe_stream_read(src, nbytes, sink, blocks, 1 if nontemporal else 0, stream))


def bm_probe_mfma(iters: int, sink: int, blocks: int, stream: int) -> None:
    _check(_lib.bm_probe_mfma(iters, sink, blocks, stream))


TIMELINE_FIELDS = 16
TIMELINE_MAX_RECORDS = 65536


def bm_prefill_timeline(n_records: int):
    """The last prefill launch's per-workgroup timeline records (a library
    built with BM_PREFILL_TIMELINE): uint64 array [n_records, 16]."""
    import numpy as np

    out = np.zeros((n_records, TIMELINE_FIELDS), dtype=np.uint64)
    _check(_lib.bm_prefill_timeline(out.ctypes.data_as(ctypes.c_void_p), n_records))
    return out


def bm_prefill_tile_workgroups(ctx: int, n_tok: int, q: int, o: int, seq_ld: int) -> int:
    return _lib.bm_prefill_tile_workgroups(ctx, n_tok, q, o, seq_ld)


def make_dims(*, b, s, kv_max, block, max_gen, n_heads, n_kv_heads, head_dim, dtype,
              sm_scale=0.0) -> bm_dims:
    dt = {"f32": BM_F32, "bf16": BM_BF16}.get(dtype, dtype)
    return bm_dims(b, s, kv_max, block, max_gen, n_heads, n_kv_heads, head_dim, dt, sm_scale)


# ---------------------------------------------------------------------------
# tensor-owning convenience wrapper
# ---------------------------------------------------------------------------
# Pad arrays that acceptances have grown, by device and address: how often, and the K plane of
# the cache that the last time was for.  An array that grows for one cache is no other cache's.
_grown_pads: dict = {}


class PDAttention:
    """Owns one layer's bounded cache (torch tensors on a GPU) and drives the ABI.

    Tensors passed to the calls have the sequence as dimension 2:
    q, o ``[b, n_heads, T, d]`` and k, v ``[b, n_kv_heads, T, d]``, contiguous,
    of the configured dtype, on the cache's device.  ``row`` selects the first
    row of the block (prefill) or the step's row (decode) inside them.
    """

    def __init__(self, *, b, s, kv_max, block, max_gen, n_heads, n_kv_heads, head_dim,
                 dtype="bf16", sm_scale=0.0, device="cuda", init=True, buffers=None,
                 static_workspace=False):
        """``static_workspace``: no workspace tensor; contexts come from
        bm_init_static_workspace and use the library's static device array.

        ``buffers``: the caller's own k, v, score (float32), pos, len (int32) and work,
        contiguous on the device.  A tensor of another type whose elements are at least as
        large is raw storage (a warning says so): the object's attribute is then a view
        of its first bytes in the type that the library reads."""
        import torch

        self.torch = torch
        self.dims = make_dims(b=b, s=s, kv_max=kv_max, block=block, max_gen=max_gen,
                              n_heads=n_heads, n_kv_heads=n_kv_heads, head_dim=head_dim,
                              dtype=dtype, sm_scale=sm_scale)
        self.cap = self._validate()
        self.tdtype = torch.float32 if self.dims.dtype == BM_F32 else torch.bfloat16
        dev = torch.device(device)
        if dev.type == "cuda" and dev.index is None:
            dev = torch.device("cuda", torch.cuda.current_device())
        self.device = dev
        self.group = n_heads // n_kv_heads
        U = b * n_kv_heads
        self.work_bytes = self._workspace_bytes(self.dims)
        self.static_workspace = static_workspace
        if static_workspace and buffers is not None:
            raise ValueError("static_workspace takes no caller buffers")
        want = self._buffers()
        if buffers is None:
            for nm, (shape, dt) in want.items():
                # (positions start defined: resume() may count entries that a caller never wrote)
                make = torch.zeros if nm == "pos" else torch.empty
                setattr(self, nm, make(shape, dtype=dt, device=self.device))
            self.work = (None if static_workspace else
                         torch.empty(self.work_bytes, dtype=torch.uint8, device=self.device))
        else:
            # caller-provided views (for example slices of one arena), checked
            for nm, x in zip((*want, "work"), buffers, strict=True):
                setattr(self, nm, x)
            for nm, (shp, dt) in want.items():
                x = getattr(self, nm)
                if (tuple(x.shape) != shp or not x.is_contiguous() or x.device != self.device
                        or not self._takes(x.dtype, dt)):
                    raise ValueError(f"buffer {nm}: need a contiguous {shp} tensor of {dt} on {self.device}")
                if x.dtype != dt:
                    warnings.warn(f"buffer {nm}: {x.dtype} taken as raw storage of {dt}", stacklevel=2)
                    raw = x.detach().view(-1).view(torch.uint8)
                    setattr(self, nm, raw[:x.numel() * dt.itemsize].view(dt).view(shp))
            if not self.work.is_contiguous() or self.work.device != self.device:
                raise ValueError(f"buffer work: need a contiguous tensor on {self.device}")
            if self.work.numel() * self.work.element_size() < self.work_bytes:
                raise ValueError("work buffer is smaller than bm_workspace_bytes")
        self.cache = self._cache()
        self.units = U
        # for every call's checks and stream: the current stream of a device index as an
        # integer, without the stream object that torch.cuda.current_stream makes
        self._raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        self._dev_index = self.device.index if self.device.type == "cuda" else None
        self._bhd = (b, n_heads, n_kv_heads, head_dim)
        self._row_bytes = head_dim * (4 if self.dims.dtype == BM_F32 else 2)
        self.ctx = None
        self._pads, self._pads_grown = None, 0
        self._draft_works = []      # the buffer of trees, once there is one (a stack's layers share the list)
        # schedule settings (bm_set_*): kept here and applied again to every new
        # context, so they survive reset() and resume()
        self._settings = {}
        if init:
            self.reset()

    # -- the cache ----------------------------------------------------------------
    def _validate(self) -> int:
        """Check the dimensions; returns the slots a unit has."""
        bm_validate_dims(self.dims)
        return bm_cache_slots(self.dims)

    def _buffers(self) -> dict:
        """Shape and element type of every tensor of the cache, in the order of ``buffers``."""
        t, d = self.torch, self.dims
        unit = (d.b, d.n_kv_heads)
        row = (*unit, self.cap, d.head_dim)
        return {"k": (row, self.tdtype), "v": (row, self.tdtype),
                "score": (row[:3], t.float32), "pos": (row[:3], t.int32), "len": (unit, t.int32)}

    def _work_ptr(self):
        return (0, 0) if self.work is None else (self.work.data_ptr(), self.work_bytes)

    def _cache(self):
        return bm_cache(self.k.data_ptr(), self.v.data_ptr(), self.score.data_ptr(),
                        self.pos.data_ptr(), self.len.data_ptr(), *self._work_ptr())

    @staticmethod
    def _takes(given, want) -> bool:
        """Whether a caller's tensor of type ``given`` can stand for one of type ``want``."""
        return given.itemsize >= want.itemsize

    _workspace_bytes = staticmethod(bm_workspace_bytes)

    def _new_context(self) -> int:
        init = bm_init_static_workspace if self.static_workspace else bm_init
        return init(self.dims, self.cache, self._stream())

    def _resumed_context(self, length, next_pos) -> int:
        return bm_resume(self.dims, self.cache, length, next_pos)

    # -- helpers ----------------------------------------------------------------
    def _stream(self) -> int:
        if self._raw_stream is not None and self._dev_index is not None:
            return self._raw_stream(self._dev_index)
        return self.torch.cuda.current_stream(self.device).cuda_stream

    def _args_ok(self, q, k, v, o) -> bool:
        """Whether q, k, v and o are what a call takes, checked with as few torch
        calls as possible: the host side of a call is as long as a small step's
        kernel (15 us a decode step with the checks one by one, 7 us like this).
        On False the caller's own checks name what is wrong."""
        s = q.shape
        if len(s) != 4:
            return False
        b, H, Hk, d = self._bhd
        hq, hk, dt, dev = (b, H, s[2], d), (b, Hk, s[2], d), self.tdtype, self._dev_index
        return (s == hq and o.shape == hq and k.shape == hk and v.shape == hk
                and q.dtype is dt and k.dtype is dt and v.dtype is dt and o.dtype is dt
                and q.get_device() == dev and k.get_device() == dev and v.get_device() == dev
                and o.get_device() == dev and q.is_contiguous() and k.is_contiguous()
                and v.is_contiguous() and o.is_contiguous())

    def _row_ptrs(self, q, k, v, o, row):
        off = row * self._row_bytes
        return q.data_ptr() + off, k.data_ptr() + off, v.data_ptr() + off, o.data_ptr() + off

    def _check_tensor(self, x, heads, name):
        t = self.torch
        if x.device != self.device or x.dtype != self.tdtype or not x.is_contiguous():
            raise ValueError(f"{name}: need a contiguous {self.tdtype} tensor on {self.device}")
        if x.dim() != 4 or x.shape[0] != self.dims.b or x.shape[1] != heads or \
                x.shape[3] != self.dims.head_dim:
            raise ValueError(f"{name}: shape {tuple(x.shape)} is not [b, {heads}, T, d]")
        return x

    def _row_ptr(self, x, row):
        if not 0 <= row < x.shape[2]:
            raise ValueError(f"row {row} outside the tensor's {x.shape[2]} rows")
        return x.data_ptr() + row * x.shape[3] * x.element_size()

    # -- schedule ---------------------------------------------------------------
    _SETTERS = {"removal": bm_set_decode_removal, "rule": bm_set_rank_rule,
                "bound": bm_set_decode_bound, "accumulate": bm_set_score_accumulation,
                "pad": bm_set_left_padding, "split": bm_set_split_event}

    def _apply_settings(self) -> None:
        for key, val in self._settings.items():
            self._SETTERS[key](self.ctx, val)

    def _set(self, key, val) -> None:
        if self.ctx is not None:
            self._SETTERS[key](self.ctx, val)   # raises before anything is stored
        self._settings[key] = val

    def _replace_context(self, new) -> None:
        # (the new one was made first: a refusal leaves the old one in place)
        old, self.ctx = self.ctx, new
        if old is not None:
            bm_destroy(old)
        self._apply_settings()
        self._pads_grown = self._grown()[0]

    def reset(self) -> None:
        self._replace_context(self._new_context())

    def resume(self, length: int, next_pos: int) -> None:
        if self.static_workspace:
            raise ValueError("resume needs a caller-allocated workspace")
        self._replace_context(self._resumed_context(length, next_pos))

    def _block_args(self, t0, n_tok, q, k, v, o, row):
        row = t0 if row is None else row
        if t0 == 0 and self._pads is not None:
            self._pads_grown = self._grown()[0]         # (a new prompt takes the pads as they are)
        if self._args_ok(q, k, v, o) and 0 <= row < q.shape[2] and row + n_tok <= q.shape[2]:
            return (self.ctx, t0, n_tok, *self._row_ptrs(q, k, v, o, row), q.shape[2],
                    self._stream())
        H, Hk = self.dims.n_heads, self.dims.n_kv_heads
        for x, hh, nm in ((q, H, "q"), (k, Hk, "k"), (v, Hk, "v"), (o, H, "o")):
            self._check_tensor(x, hh, nm)
            if row + n_tok > x.shape[2]:
                raise ValueError(f"{nm}: rows [{row}, {row + n_tok}) exceed {x.shape[2]}")
        T = q.shape[2]
        if not (k.shape[2] == v.shape[2] == o.shape[2] == T):
            raise ValueError("q, k, v and o need the same number of rows")
        return (self.ctx, t0, n_tok, self._row_ptr(q, row), self._row_ptr(k, row),
                self._row_ptr(v, row), self._row_ptr(o, row), T, self._stream())

    def prefill_block(self, t0, n_tok, q, k, v, o, row=None) -> None:
        bm_prefill_block(*self._block_args(t0, n_tok, q, k, v, o, row))

    def prefill_block_cut(self, t0, n_tok, q, k, v, o, row=None) -> None:
        """prefill_block then evict_compact(t0 + n_tok - 1), fused where possible."""
        bm_prefill_block_cut(*self._block_args(t0, n_tok, q, k, v, o, row))

    def evict_compact(self, curr_id) -> None:
        bm_evict_compact(self.ctx, curr_id, self._stream())

    # settings persist across reset() and resume()
    def set_decode_removal(self, p: int) -> None:
        """0: one removal per decode step after appending (default); p > 0:
        Algorithm 1's decoding loop, p removals when a step starts full."""
        self._set("removal", p)

    def set_rank_rule(self, rule) -> None:
        """"ave" (default, Sec. 3.2), "sum", "recent" or "tova" (or a BM_RANK_* value)."""
        self._set("rule", RANK_RULES.get(rule, rule))

    def set_decode_bound(self, bound: int) -> None:
        self._set("bound", bound)

    def set_score_accumulation(self, on: bool) -> None:
        self._set("accumulate", 1 if on else 0)

    def set_left_padding(self, pads) -> None:
        """Left pad tokens per sample: a contiguous int32 tensor of b values on
        the device (kept referenced here), or None for no padding."""
        if pads is None:
            self._pads = None
            self._set("pad", None)
            return
        t = self.torch
        if pads.dtype != t.int32 or pads.device != self.device or not pads.is_contiguous() or \
                tuple(pads.shape) != (self.dims.b,):
            raise ValueError(f"pads: need a contiguous int32 [{self.dims.b}] tensor on {self.device}")
        self._set("pad", pads.data_ptr())
        self._pads = pads
        self._pads_grown = self._grown()[0]

    def _grown(self) -> tuple:
        """How often the pad array has grown, and for which cache last."""
        if self._pads is None:
            return 0, None
        return _grown_pads.get((self._dev_index, self._pads.data_ptr()), (0, None))

    def _own_pads(self) -> int:
        """How often the pad array has grown; refuses one that grew for another cache."""
        times, cache = self._grown()
        if times != self._pads_grown and cache != self.k.data_ptr():
            raise ValueError("the left padding has grown with another cache's accepted tokens: each cache "
                             "(layer) needs a tensor of its own")
        return times

    def set_split_event(self, event) -> None:
        """Record ``event`` (a torch.cuda.Event, or None to stop) between each
        later prefill block's attention kernel and its fold/cut launches, so the
        two can be timed separately on one stream.  The event is recorded once
        here on the current stream so that it exists."""
        if event is None:
            self._split = None
            self._set("split", None)
            return
        event.record(self.torch.cuda.current_stream(self.device))
        self._split = event
        self._set("split", event.cuda_event)

    def decode_step(self, pos, q, k, v, o, row=0) -> None:
        if self._args_ok(q, k, v, o) and 0 <= row < q.shape[2]:
            bm_decode_step(self.ctx, pos, *self._row_ptrs(q, k, v, o, row), q.shape[2],
                           self._stream())
            return
        H, Hk = self.dims.n_heads, self.dims.n_kv_heads
        for x, hh, nm in ((q, H, "q"), (k, Hk, "k"), (v, Hk, "v"), (o, H, "o")):
            self._check_tensor(x, hh, nm)
        T = q.shape[2]
        if not (k.shape[2] == v.shape[2] == o.shape[2] == T):
            raise ValueError("q, k, v and o need the same number of rows")
        bm_decode_step(self.ctx, pos, self._row_ptr(q, row), self._row_ptr(k, row),
                       self._row_ptr(v, row), self._row_ptr(o, row), T, self._stream())

    # -- drafted tokens (include/bm_draft.h) -----------------------------------------
    def _ints(self, x, shape, name):
        if x.dtype is not self.torch.int32 or x.get_device() != self._dev_index or x.shape != shape or \
                not x.is_contiguous():
            raise ValueError(f"{name}: need a contiguous int32 {list(shape)} tensor on {self.device}")
        return x.data_ptr()

    def _lse_ptr(self, lse, n):
        if lse is None:
            return None
        shape = (*self._bhd[:2], n)
        if lse.dtype is not self.torch.float32 or lse.get_device() != self._dev_index or lse.shape != shape or \
                not lse.is_contiguous():
            raise ValueError(f"lse: need a contiguous float32 {list(shape)} tensor on {self.device}")
        return lse.data_ptr()

    def _tree_rows(self, n, q, k, v, o, row):
        """Pointers of rows row .. row + n - 1 of q, k, v (and o)."""
        if not (self._args_ok(q, k, v, o) and 0 <= row and row + n <= q.shape[2]):
            H, Hk = self.dims.n_heads, self.dims.n_kv_heads
            for x, hh, nm in ((q, H, "q"), (k, Hk, "k"), (v, Hk, "v"), (o, H, "o")):
                self._check_tensor(x, hh, nm)
                if x.shape[2] != q.shape[2]:
                    raise ValueError("q, k, v and o need the same number of rows")
            raise ValueError(f"rows [{row}, {row + n}) exceed {q.shape[2]}")
        if self.torch.cuda.current_device() != self._dev_index:
            # the library launches on the current device: a stream of another one would not do
            raise ValueError(f"make {self.device} the current device")
        return self._row_ptrs(q, k, v, o, row)

    def draft_work_bytes(self, n=BM_DRAFT_MAX) -> int:
        """Bytes of scratch of a tree of n nodes (``draft_attend``'s work)."""
        return bm_draft_workspace_bytes(self.dims, n)

    @property
    def _draft_work(self):
        return self._draft_works[-1] if self._draft_works else None

    def _draft_scratch(self, work):
        """Pointer and bytes of the caller's scratch, or of this object's own."""
        if work is None:
            work = self._draft_work
            if work is None:
                # (once, for the largest tree: a buffer that stays is what captured graphs need)
                work = self.torch.empty(self.draft_work_bytes(), dtype=self.torch.uint8, device=self.device)
                self._draft_works.append(work)
        elif work.device != self.device or not work.is_contiguous():
            raise ValueError(f"work: need a contiguous tensor on {self.device}")
        return work.data_ptr(), work.numel() * work.element_size()

    def draft_attend(self, parent, q, k, v, o, lse=None, row=0, work=None) -> None:
        """The attention of a tree's n nodes over the cache, their ancestors and themselves:
        rows row .. row + n - 1 of q, k, v into o.  ``parent`` int32 ``[b, n]`` (-1: a root);
        ``lse`` float32 ``[b, n_heads, n]`` or None takes their log-sum-exps.  The cache
        is left as it is (one above the decode bound is cut to it).  ``work``: scratch of at
        least ``draft_work_bytes(n)`` bytes whose contents need not survive the call, so that
        caches whose calls run one after another can share it; without it the object (a
        ``PDStack``: its layers together) makes one of ``draft_work_bytes()`` at its first
        tree and keeps it."""
        n = parent.shape[-1]
        tree = self._ints(parent, (self.dims.b, n), "parent")
        rows = self._tree_rows(n, q, k, v, o, row)
        self._own_pads()
        bm_draft_attend(self.ctx, n, tree, *rows, q.shape[2], self._lse_ptr(lse, n),
                        *self._draft_scratch(work), self._stream())

    def draft_accept(self, path, q, k, v, lse=None, count=None, row=0, n=None) -> None:
        """Append the m tokens ``path`` (int32 ``[b, m]``: node numbers, a root and then each
        one's child) of the tree of n nodes (by default all rows from ``row`` on; ``lse``, if
        given, has n columns) and advance by m.  ``lse``: as draft_attend left it.  ``count``
        int32 ``[b]``: sample j takes only the first count[j]; the samples' left padding has to
        be set, and that tensor grows by m - count: caches (layers) must not share it (a draft
        over another cache with the same tensor is then refused, until its padding is set
        anew or it begins again)."""
        if n is None:
            n = lse.shape[-1] if lse is not None else q.shape[2] - row
        m = path.shape[-1]
        tree = self._ints(path, (self.dims.b, m), "path")
        taken = None if count is None else self._ints(count, (self.dims.b,), "count")
        rows = self._tree_rows(n, q, k, v, q, row)
        times = self._own_pads()
        bm_draft_accept(self.ctx, n, m, tree, taken, *rows[:3], q.shape[2], self._lse_ptr(lse, n),
                        self._stream())
        if count is not None:
            self._pads_grown = times + 1
            _grown_pads[self._dev_index, self._pads.data_ptr()] = times + 1, self.k.data_ptr()

    def run_prefill(self, q, k, v, o, fused_cut=False) -> None:
        """Algorithm 1 prefill under the block loop: every block, then a cut
        (with ``fused_cut`` through prefill_block_cut)."""
        s, B = self.dims.s, self.dims.block
        for t0 in range(0, s, B):
            n = min(B, s - t0)
            if fused_cut:
                self.prefill_block_cut(t0, n, q, k, v, o)
            else:
                self.prefill_block(t0, n, q, k, v, o)
                self.evict_compact(t0 + n - 1)

    def run_decode(self, q, k, v, o, steps=None, first_row=None) -> None:
        """Decode steps at positions s, s+1, ... using rows first_row.. (default s)."""
        s = self.dims.s
        steps = self.dims.max_gen if steps is None else steps
        r0 = s if first_row is None else first_row
        for t in range(steps):
            self.decode_step(s + t, q, k, v, o, row=r0 + t)

    def capture_decode(self, q, k, v, o, steps=None, first_row=None):
        """Record run_decode's launches into one HIP graph (the decode loop of
        Algorithm 1 without host work between steps) and return it.

        Call it where the decode would start (right after the prefill).  Nothing
        runs during the capture; the context then describes the state after the
        decode steps.  Every position, length and pointer is fixed inside the
        graph, so ``graph.replay()`` is valid whenever the device state equals
        the one at capture time, e.g. after the same prefill has run again.  The
        decode path enqueues kernels only (no memset nodes)."""
        t = self.torch
        g = t.cuda.CUDAGraph()
        side = t.cuda.Stream(device=self.device)          # default priority
        side.wait_stream(t.cuda.current_stream(self.device))
        with t.cuda.graph(g, stream=side):
            self.run_decode(q, k, v, o, steps, first_row)
        t.cuda.current_stream(self.device).wait_stream(side)
        return g

    @property
    def length(self) -> int:
        return bm_ctx_len(self.ctx)

    @property
    def next_pos(self) -> int:
        return bm_ctx_next_pos(self.ctx)

    def close(self) -> None:
        if self.ctx is not None:
            bm_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class PDAttentionKV4(PDAttention):
    """PDAttention over a cache held in 4 bits (include/bm_kv4.h), every call included:
    a call's own K and V rows are attended to as given and stored in 4 bits,
    earlier entries as they read back.

    ``k``, ``v`` hold the codes, uint8 ``[b, n_kv_heads, slots, d / 2]``, ``k_scale``, ``v_scale``
    the scale bytes, uint8 ``[b, n_kv_heads, slots, d / 32]``, in the library's own order of
    bytes within a unit.  ``buffers``: those four, then score (float32), pos, len (int32) and work.
    ``write_rows`` and ``read_rows`` convert rows of the configured dtype to and from slots.
    """

    def __init__(self, *, static_workspace=False, **kw):
        if static_workspace:
            raise ValueError("a 4-bit cache needs a caller-allocated workspace")
        super().__init__(**kw)

    def _buffers(self) -> dict:
        t, d = self.torch, self.dims
        plain = super()._buffers()
        slots = (d.b, d.n_kv_heads, bm_kv4_slots(d))
        code, scale = (*slots, d.head_dim // 2), (*slots, d.head_dim // BM_KV4_GROUP)
        return {"k": (code, t.uint8), "v": (code, t.uint8), "k_scale": (scale, t.uint8),
                "v_scale": (scale, t.uint8), **{x: plain[x] for x in ("score", "pos", "len")}}

    def _cache(self):
        return bm_kv4_cache(self.k.data_ptr(), self.v.data_ptr(), self.k_scale.data_ptr(),
                            self.v_scale.data_ptr(), self.score.data_ptr(), self.pos.data_ptr(),
                            self.len.data_ptr(), *self._work_ptr())

    @staticmethod
    def _takes(given, want) -> bool:
        # codes, scores and positions of another type would be read as other values
        return given == want

    _workspace_bytes = staticmethod(bm_kv4_workspace_bytes)

    def _stream(self) -> int:
        # the library launches on the current device: a stream of another one would not do
        if self._dev_index is not None and self.torch.cuda.current_device() != self._dev_index:
            raise ValueError(f"make {self.device} the current device")
        return super()._stream()

    def _new_context(self) -> int:
        return bm_kv4_init(self.dims, self.cache, self._stream())

    def _resumed_context(self, length, next_pos) -> int:
        if not (-_INT32_MAX <= length <= _INT32_MAX and -_INT32_MAX <= next_pos <= _INT32_MAX):
            raise ValueError(f"length {length}, next_pos {next_pos}: beyond 32 bits")
        return bm_kv4_resume(self.dims, self.cache, length, next_pos)

    def _rows(self, k, v):
        """Rows of k and v, checked with few torch calls; what is wrong is named on failure."""
        s, d = k.shape, self.dims
        if (len(s) == 4 and s == v.shape and s == (d.b, d.n_kv_heads, s[2], d.head_dim)
                and k.dtype is self.tdtype and v.dtype is self.tdtype
                and k.get_device() == self._dev_index and v.get_device() == self._dev_index
                and k.is_contiguous() and v.is_contiguous()):
            return s[2]
        for x, nm in ((k, "k"), (v, "v")):
            self._check_tensor(x, d.n_kv_heads, nm)
        if k.shape[2] != v.shape[2]:
            raise ValueError("k and v need the same number of rows")
        return k.shape[2]

    def write_rows(self, slot0, k, v) -> None:
        """Store every row of k, v ``[b, n_kv_heads, n, d]`` in slots slot0 .. slot0 + n - 1 of
        its unit; scores, positions and lengths are left as they are."""
        n = self._rows(k, v)
        if not -_INT32_MAX <= slot0 <= _INT32_MAX:
            raise ValueError(f"slot0 {slot0}: beyond 32 bits")
        bm_kv4_write(self.dims, self.cache, slot0, n, k.data_ptr(), v.data_ptr(), n, self._stream())

    def read_rows(self, slot0, n, k=None, v=None):
        """Slots slot0 .. slot0 + n - 1 of every unit as k, v ``[b, n_kv_heads, n, d]`` of the
        configured dtype (new tensors unless given), which are returned."""
        t, d = self.torch, self.dims
        if k is None:
            k = t.empty((d.b, d.n_kv_heads, n, d.head_dim), dtype=self.tdtype, device=self.device)
        if v is None:
            v = t.empty_like(k)
        if self._rows(k, v) != n:
            raise ValueError(f"k and v need {n} rows")
        if not -_INT32_MAX <= slot0 <= _INT32_MAX:
            raise ValueError(f"slot0 {slot0}: beyond 32 bits")
        bm_kv4_read(self.dims, self.cache, slot0, n, k.data_ptr(), v.data_ptr(), n, self._stream())
        return k, v


class WindowAttention(PDAttention):
    """Attention with a sliding window and sinks over a cache of window + sinks rows a unit
    (include/bm_window.h): a token sees the last ``window`` tokens, its own included, and the
    first ``sinks`` of its sample.  ``prefill_block`` takes up to ``block`` tokens (by default
    all of the prompt), ``decode_step`` one; drafted tokens as over a bounded cache.

    ``k``, ``v``: ``[b, n_kv_heads, window + sinks, d]``; token j < sinks lies in slot j, any other
    one in slot sinks + (j - sinks) mod window, j counted from the sample's first real token.
    ``buffers``: those two and work."""

    def __init__(self, *, window, sinks=0, b, s, max_gen, block=None, static_workspace=False, **kw):
        if static_workspace:
            raise ValueError("a window cache needs a caller-allocated workspace")
        if not (1 <= window <= _INT32_MAX and 0 <= sinks <= _INT32_MAX):
            raise ValueError(f"window {window} must be positive, sinks {sinks} not negative")
        self.window, self.sinks = window, sinks
        super().__init__(b=b, s=s, kv_max=window + sinks, block=s if block is None else block,
                         max_gen=max_gen, **kw)

    def _validate(self):
        bm_win_validate(self.dims, self.sinks)
        return self.dims.kv_max

    def _buffers(self) -> dict:
        d = self.dims
        row = (d.b, d.n_kv_heads, self.cap, d.head_dim)
        return {"k": (row, self.tdtype), "v": (row, self.tdtype)}

    def _cache(self):
        return bm_win_cache(self.k.data_ptr(), self.v.data_ptr(), *self._work_ptr())

    @staticmethod
    def _takes(given, want) -> bool:
        # rows of another type would be read as other values
        return given == want

    _workspace_bytes = staticmethod(bm_win_workspace_bytes)

    def _stream(self) -> int:
        # the library launches on the current device: a stream of another one would not do
        if self._dev_index is not None and self.torch.cuda.current_device() != self._dev_index:
            raise ValueError(f"make {self.device} the current device")
        return super()._stream()

    def _new_context(self) -> int:
        return bm_win_init(self.dims, self.sinks, self.cache)

    def resume(self, next_pos: int, s: int | None = None) -> None:
        """A context over the rows of the tokens before ``next_pos`` as they lie in k and v.  ``s``:
        another prompt length, for a turn behind generated tokens: after ``resume(p, s=p + n)``
        with p = ``next_pos``, n more tokens go through ``prefill_block`` (at most ``block`` a call)
        and steps follow from p + n on.  (``reset`` keeps it; ``resume(0, s=..)`` begins anew
        with another.)"""
        s = self.dims.s if s is None else s
        if not (-_INT32_MAX <= next_pos <= _INT32_MAX and -_INT32_MAX <= s <= _INT32_MAX):
            raise ValueError(f"next_pos {next_pos}, s {s}: beyond 32 bits")
        old, self.dims.s = self.dims.s, s
        try:
            new = bm_win_resume(self.dims, self.sinks, self.cache, next_pos)
        except BatchMaxError:
            self.dims.s = old
            raise
        self._replace_context(new)


# ---------------------------------------------------------------------------
# synthetic inputs of the layer stack (bm_synth.h)
# ---------------------------------------------------------------------------
def synth_params(*, b, n_heads, n_kv_heads, head_dim, dtype, seed, layer, s, hh_frac=0.02,
                 hh_scale=4.0, n_sinks=0, sink_scale=6.0, heavy=True) -> bm_synth:
    """Generator parameters: value_scale = float32(sqrt(3) / sqrt(d) / 65536) and
    hh_threshold = round(hh_frac * 2^32) (0 when there are no heavy hitters)."""
    dt = {"f32": BM_F32, "bf16": BM_BF16}.get(dtype, dtype)
    thr = int(round(hh_frac * 2.0 ** 32)) if heavy else 0
    vs = ctypes.c_float(math.sqrt(3.0) / math.sqrt(head_dim) / 65536.0).value
    return bm_synth(b, n_heads, n_kv_heads, head_dim, dt, seed, layer, s, thr, hh_scale, n_sinks,
                    sink_scale, vs)


def synth_qkv(params: bm_synth, t0: int, q, k, v) -> None:
    """Fill every row of q [b, H, T, d], k/v [b, Hk, T, d] (torch, contiguous, on one
    GPU) with the stream's rows for positions t0 .. t0+T-1, on the current stream."""
    import torch

    tdt = torch.float32 if params.dtype == BM_F32 else torch.bfloat16
    T = q.shape[2]
    for x, hh, nm in ((q, params.n_heads, "q"), (k, params.n_kv_heads, "k"), (v, params.n_kv_heads, "v")):
        if x.dtype != tdt or not x.is_contiguous() or x.device.type != "cuda" or \
                tuple(x.shape) != (params.b, hh, T, params.head_dim):
            raise ValueError(f"{nm}: need a contiguous {tdt} [b, {hh}, {T}, d] tensor on the GPU")
    stream = torch.cuda.current_stream(q.device).cuda_stream
    bm_synth_qkv(params, t0, T, q.data_ptr(), k.data_ptr(), v.data_ptr(), T, stream)


# ---------------------------------------------------------------------------
# a stack of layers: one bounded cache per layer in a single device arena
# ---------------------------------------------------------------------------
def _align(n: int, a: int = 256) -> int:
    return (n + a - 1) // a * a


def _row_planes(cap, head_dim, dtype, kv_bits) -> tuple:
    """Slots of a unit in the planes of K (and of V), and the bytes of a slot in each: K's
    rows and, held in 4 bits, their scales."""
    if kv_bits == 16:
        return cap, (head_dim * (4 if dtype in ("f32", BM_F32) else 2),)
    if kv_bits == 4:
        return _align(cap, 64), (head_dim // 2, head_dim // BM_KV4_GROUP)
    raise ValueError("kv_bits is 16 (rows of the element type) or 4")


def stack_layer_bytes(*, b, kv_max, block, n_kv_heads, head_dim, dtype, kv_bits=16) -> int:
    """Device bytes of one layer's cache (K, V and their scales, score, pos, len),
    256-byte aligned."""
    cap = kv_max + block
    units = b * n_kv_heads
    slots, planes = _row_planes(cap, head_dim, dtype, kv_bits)
    return (sum(2 * _align(units * slots * x) for x in planes) + 2 * _align(units * cap * 4)
            + _align(units * 4))


class PDStack:
    """``n_layers`` independent bounded caches (the attention layers of one
    model, each with its own scores and evictions) carved from one device
    arena, sharing one workspace (its contents never outlive a call) and, once
    a layer has drafted tokens, one buffer of ``draft_work_bytes()`` for them
    besides the arena.  Layer ``l`` is driven through ``self.layers[l]``, a
    ``PDAttention`` (``kv_bits`` 4: a ``PDAttentionKV4``)."""

    def __init__(self, *, n_layers, b, s, kv_max, block, max_gen, n_heads, n_kv_heads, head_dim,
                 dtype="bf16", sm_scale=0.0, device="cuda", kv_bits=16):
        import torch

        dims = make_dims(b=b, s=s, kv_max=kv_max, block=block, max_gen=max_gen, n_heads=n_heads,
                         n_kv_heads=n_kv_heads, head_dim=head_dim, dtype=dtype, sm_scale=sm_scale)
        bm_validate_dims(dims)
        dev = torch.device(device)
        if dev.type == "cuda" and dev.index is None:
            dev = torch.device("cuda", torch.cuda.current_device())
        tdt = torch.float32 if dims.dtype == BM_F32 else torch.bfloat16
        cap = kv_max + block
        per_layer = stack_layer_bytes(b=b, kv_max=kv_max, block=block, n_kv_heads=n_kv_heads,
                                      head_dim=head_dim, dtype=dims.dtype, kv_bits=kv_bits)
        layer_type = PDAttentionKV4 if kv_bits == 4 else PDAttention
        work_bytes = layer_type._workspace_bytes(dims)
        self.arena_bytes = n_layers * per_layer + _align(work_bytes)
        self.arena = torch.empty(self.arena_bytes, dtype=torch.uint8, device=dev)
        work = self.arena[n_layers * per_layer:n_layers * per_layer + work_bytes]
        rows = b * n_kv_heads * cap
        self.layers = []
        for layer in range(n_layers):
            off = layer * per_layer

            def take(nbytes, dt, shape):
                nonlocal off
                x = self.arena[off:off + nbytes].view(dt).view(shape)
                off += _align(nbytes)
                return x

            kv = []
            slots, planes = _row_planes(cap, head_dim, dims.dtype, kv_bits)
            for row in planes:
                dt = torch.uint8 if kv_bits == 4 else tdt
                shape, size = (b, n_kv_heads, slots, row // dt.itemsize), b * n_kv_heads * slots * row
                kv += [take(size, dt, shape), take(size, dt, shape)]
            sc = take(rows * 4, torch.float32, (b, n_kv_heads, cap))
            ps = take(rows * 4, torch.int32, (b, n_kv_heads, cap))
            ln = take(b * n_kv_heads * 4, torch.int32, (b, n_kv_heads))
            self.layers.append(layer_type(b=b, s=s, kv_max=kv_max, block=block, max_gen=max_gen,
                                          n_heads=n_heads, n_kv_heads=n_kv_heads,
                                          head_dim=head_dim, dtype=dtype, sm_scale=sm_scale,
                                          device=dev, init=False,
                                          buffers=(*kv, sc, ps, ln, work)))
            # (scratch of drafted tokens' trees, made at the first one)
            self.layers[-1]._draft_works = self.layers[0]._draft_works
        self.n_layers = n_layers
        self.device = dev

    def reset(self) -> None:
        for layer in self.layers:
            layer.reset()

    def close(self) -> None:
        for layer in self.layers:
            layer.close()


def stack_bytes(*, b, n_layers, s, kv_max, block, max_gen, n_heads, n_kv_heads, head_dim,
                dtype, kv_bits=16, drafts=False) -> int:
    """Device bytes a P&D run of the layer stack needs at batch b: every layer's
    bounded cache, the shared workspace (with ``drafts`` also that of drafted
    tokens), and the reusable input/output buffers of one prefill block and one
    decode row."""
    es = 4 if dtype in ("f32", BM_F32) else 2
    dims = make_dims(b=b, s=s, kv_max=kv_max, block=block, max_gen=max_gen, n_heads=n_heads,
                     n_kv_heads=n_kv_heads, head_dim=head_dim, dtype=dtype)
    caches = n_layers * stack_layer_bytes(b=b, kv_max=kv_max, block=block, n_kv_heads=n_kv_heads,
                                          head_dim=head_dim, dtype=dtype, kv_bits=kv_bits)
    work = _align(bm_kv4_workspace_bytes(dims) if kv_bits == 4 else bm_workspace_bytes(dims))
    if drafts:
        work += _align(bm_draft_workspace_bytes(dims, BM_DRAFT_MAX))
    rows = block + 1
    io = rows * b * (2 * n_heads + 2 * n_kv_heads) * head_dim * es
    return caches + work + io


def full_cache_bytes_per_sample(*, n_layers, s, n_kv_heads, head_dim, dtype) -> int:
    """K and V of every prompt position of every layer: the memory a
    decoding-only compression scheme holds before its first decode step."""
    es = 4 if dtype in ("f32", BM_F32) else 2
    return n_layers * n_kv_heads * s * head_dim * es * 2


def plan_stack_batch(budget_bytes: int, **shape) -> int:
    """Largest b with stack_bytes(b, **shape) <= budget_bytes (0 if none)."""
    lo, hi = 0, 1
    while stack_bytes(b=hi, **shape) <= budget_bytes:
        lo, hi = hi, hi * 2
    while hi - lo > 1:
        mid = (lo + hi) // 2
        if stack_bytes(b=mid, **shape) <= budget_bytes:
            lo = mid
        else:
            hi = mid
    return lo


# ---------------------------------------------------------------------------
# algorithmic work (used by the benchmark's roofline figures)
# ---------------------------------------------------------------------------
def prefill_flops_padded(*, pads, n_kv_heads, group, head_dim, s, kv_max, block) -> int:
    """prefill_flops with left padding (Sec. 3): only real queries and the real
    keys they see count.  Pads are removed before any real entry, so after a
    cut the cache holds min(real so far, kv_max) real entries."""
    total = 0
    for p in (int(x) for x in pads):
        real = pad = 0                     # entries in the cache
        for t0 in range(0, s, block):
            t1 = min(s, t0 + block)
            r0 = max(p, t0)                # first real row of the block
            n = max(0, t1 - r0)
            total += n * real + n * (n + 1) // 2
            real += n
            pad += (t1 - t0) - n
            excess = real + pad - kv_max
            if excess > 0:
                drop = min(pad, excess)
                pad -= drop
                real -= excess - drop
    return total * 4 * head_dim * group * n_kv_heads


def prefill_flops(*, b, n_kv_heads, group, head_dim, s, kv_max, block) -> int:
    """QK^T + PV flops the method must do: 4 d G per visible (query, key) pair."""
    total = 0
    length = 0
    for t0 in range(0, s, block):
        n = min(block, s - t0)
        # row r of the block sees length + r + 1 entries
        total += n * length + n * (n + 1) // 2
        length = min(kv_max, length + n)
    return 4 * head_dim * group * total * b * n_kv_heads


def decode_cache_lengths(*, s, kv_max, n_decode, p=0, bound=None) -> list:
    """Cached entries each decode step's attention reads (before its own pair),
    under the removal schedule chosen with ``bm_set_decode_removal`` and the
    decode bound of ``bm_set_decode_bound`` (default kv_max): the prompt leaves
    min(s, kv_max); with p = 0 a cache above the bound is cut to it, and a step
    appends then removes one when over the bound; with p > 0 a step that starts
    at or above the bound first drops to bound - p."""
    kd = kv_max if bound is None else bound
    n = min(s, kv_max)
    out = []
    for _ in range(n_decode):
        if p > 0 and n >= kd:
            n = kd - p
        elif p == 0 and n > kd:
            n = kd
        out.append(n)
        n = min(n + 1, kd)
    return out


MAX_DECODE_LEN = 4097   # entries one step of the scoring decode kernel attends to


def decode_bytes_outputs_only(*, b, n_kv_heads, group, head_dim, n, elem_bytes) -> int:
    """HBM bytes of one outputs-only decode step over n cached entries (the
    split path past MAX_DECODE_LEN): read n K and V rows, q, the new k and v;
    write o and append the new K, V row, score and position."""
    d, G, es = head_dim, group, elem_bytes
    per_unit = 2 * n * d * es + (G + 2) * d * es + G * d * es + 2 * d * es + 8
    return per_unit * b * n_kv_heads


def decode_bytes_per_step(*, b, n_kv_heads, group, head_dim, kv_max, elem_bytes) -> int:
    """HBM bytes one decode step must move per the fused design: read the K̄
    cached K and V rows, scores and positions; write K̄ scores, one K/V row,
    one score and position; read q (G rows), k and v of the step; write o."""
    d, G, es = head_dim, group, elem_bytes
    per_unit = (2 * kv_max * d * es          # cached K and V
                + kv_max * 4 * 2             # scores read and written
                + kv_max * 4                 # positions
                + (G + 2) * d * es           # q, new k, new v
                + G * d * es                 # o
                + 2 * d * es + 8)            # evicted slot overwrite (K, V, score, pos)
    return per_unit * b * n_kv_heads
