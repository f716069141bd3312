"""Binding of liblocks.so (ctypes; calls that a serving loop makes per layer and step: natively, csrc/calls.cpp).  Names mirror
include/locks.h; tensors are torch CUDA tensors."""
from __future__ import annotations

import ctypes as C
import importlib.util
import os
import sys
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "liblocks.so")
_CALLS_PATH = os.path.join(_HERE, "_calls.so")

F32, BF16 = 0, 1
FMT_F32, FMT_I4, FMT_I8, FMT_BF16 = 0, 1, 2, 3

SYMBOLS = ["locks_summary_bytes", "locks_workspace_bytes", "locks_create", "locks_destroy",
           "locks_build_summaries", "locks_select", "locks_sparse_attend", "locks_decode_step",
           "locks_decode_step_host", "locks_poll_status", "locks_last_launch_count", "locks_strerror",
           "locks_profile_begin", "locks_profile_end", "locks_profile_read", "locks_sparse_attend_noalloc",
           "locks_set_scan_partition", "locks_selftest_wait_timeout", "locks_last_scan_partition",
           "locks_host_cache_clear", "locks_select_exact", "locks_selection_quality",
           "locks_select_rival", "locks_fake_quantize_pages", "locks_scan",
           "locks_select_scored", "locks_merge_selection", "locks_merge_attention",
           "locks_build_summaries_layers", "locks_rope", "locks_append_rows", "locks_kvq_append", "locks_kvq_attend",
           "locks_kvq_build_summaries"]


PARTITION_AUTO, PARTITION_STRIDED, PARTITION_BALANCED = 0, 1, 2   # LOCKS_PARTITION_* of include/locks.h
SCORER_SUMMARY, SCORER_CENTROID, SCORER_MOMENT, SCORER_ENVELOPE = 0, 1, 2, 3   # LOCKS_SCORER_*


class LocksError(RuntimeError):
    pass


class Config(C.Structure):
    _fields_ = [("head_dim", C.c_int32), ("page_size", C.c_int32), ("num_q_heads", C.c_int32),
                ("num_kv_heads", C.c_int32), ("rank", C.c_int32), ("summary_fmt", C.c_int32),
                ("kv_dtype", C.c_int32), ("q_dtype", C.c_int32), ("max_batch", C.c_int32),
                ("max_pages_per_seq", C.c_int32), ("budget_tokens", C.c_int32), ("sm_scale", C.c_float),
                ("combine", C.c_int32)]


class KV(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("stride_block", C.c_int64), ("stride_head", C.c_int64),
                ("stride_token", C.c_int64), ("num_blocks", C.c_int32), ("block_table", C.c_void_p),
                ("seq_lens", C.c_void_p)]


KVQ_INT, KVQ_FLOAT = 0, 1   # LOCKS_KVQ_*


class KVQ(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("stride_block", C.c_int64), ("stride_head", C.c_int64),
                ("stride_token", C.c_int64), ("num_blocks", C.c_int32), ("fmt", C.c_int32), ("k_scale", C.c_void_p),
                ("v_scale", C.c_void_p), ("k_tail", C.c_void_p), ("v_tail", C.c_void_p), ("block_table", C.c_void_p),
                ("seq_lens", C.c_void_p), ("tail_pages", C.c_int32)]


class Rows(C.Structure):
    _fields_ = [("p", C.c_void_p), ("stride_token", C.c_int64), ("stride_head", C.c_int64)]


class Rotary(C.Structure):
    _fields_ = [("inv_freq", C.c_float * 64), ("axis", C.c_uint8 * 64), ("rot_dim", C.c_int32), ("num_axes", C.c_int32),
                ("interleaved", C.c_int32)]


_lib = None
_calls_module = None


def library_path() -> str:
    return _LIB_PATH


def lib():
    """Load liblocks.so (built in-tree by paper_2607_24555_b200.build).  Raises if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise LocksError(f"{_LIB_PATH} is missing: run `python -m paper_2607_24555_b200.build` "
                             "(there is no CPU or PyTorch fallback)")
        L = C.CDLL(_LIB_PATH)
        vp, i32p = C.c_void_p, C.c_void_p
        L.locks_summary_bytes.restype = C.c_size_t
        L.locks_summary_bytes.argtypes = [C.POINTER(Config)]
        L.locks_workspace_bytes.restype = C.c_size_t
        L.locks_workspace_bytes.argtypes = [C.POINTER(Config)]
        L.locks_create.argtypes = [C.POINTER(Config), vp, C.c_size_t, C.POINTER(vp)]
        L.locks_destroy.argtypes = [vp]
        L.locks_build_summaries.argtypes = [vp, C.POINTER(KV), C.c_int, i32p, i32p, vp, vp]
        L.locks_select.argtypes = [vp, vp, vp, C.POINTER(KV), C.c_int, i32p, i32p, vp, vp, vp]
        L.locks_build_summaries_layers.argtypes = [vp, C.POINTER(KV), vp, vp, C.c_int, C.c_int, i32p, i32p, vp]
        L.locks_build_summaries_layers.restype = C.c_int
        L.locks_sparse_attend.argtypes = [vp, vp, C.POINTER(KV), C.c_int, i32p, i32p, vp, vp, vp]
        L.locks_decode_step.argtypes = [vp, vp, vp, vp, C.POINTER(KV), vp, C.c_int, vp, i32p, i32p, vp]
        L.locks_decode_step_host.argtypes = [vp, vp, vp, vp, C.POINTER(KV), vp, C.c_int, vp, i32p, i32p, vp]
        L.locks_poll_status.argtypes = [vp, C.POINTER(C.c_int32), vp]
        L.locks_last_launch_count.argtypes = [vp]
        L.locks_profile_begin.argtypes = [vp, C.c_int]
        L.locks_profile_end.argtypes = [vp, C.POINTER(C.c_float), C.POINTER(C.c_int)]
        L.locks_profile_read.argtypes = [vp, C.POINTER(C.c_float), vp]
        L.locks_profile_read.restype = C.c_int
        L.locks_profile_begin.restype = C.c_int
        L.locks_profile_end.restype = C.c_int
        L.locks_sparse_attend_noalloc.argtypes = [C.POINTER(Config), vp, C.POINTER(KV), C.c_int, i32p, i32p, vp, vp, vp]
        L.locks_sparse_attend_noalloc.restype = C.c_int
        L.locks_set_scan_partition.argtypes = [vp, C.c_int]
        L.locks_selftest_wait_timeout.argtypes = [vp, C.c_int, vp]
        L.locks_selftest_wait_timeout.restype = C.c_int
        L.locks_set_scan_partition.restype = C.c_int
        L.locks_last_scan_partition.argtypes = [vp]
        L.locks_last_scan_partition.restype = C.c_int
        L.locks_host_cache_clear.argtypes = [vp]
        L.locks_host_cache_clear.restype = C.c_int
        L.locks_select_rival.argtypes = [vp, C.c_int, vp, vp, C.POINTER(KV), C.c_int, i32p, i32p, vp, vp, vp]
        L.locks_select_rival.restype = C.c_int
        L.locks_fake_quantize_pages.argtypes = [vp, C.POINTER(KV), C.c_int, i32p, i32p, C.c_int, vp]
        L.locks_fake_quantize_pages.restype = C.c_int
        L.locks_scan.argtypes = [vp, vp, vp, C.POINTER(KV), C.c_int, vp, vp, vp]
        L.locks_select_scored.argtypes = [vp, vp, vp, C.c_int, C.POINTER(KV), C.c_int, i32p, i32p, vp, vp]
        L.locks_merge_selection.argtypes = [vp, vp, i32p, C.c_int, C.c_int, i32p, i32p, vp]
        L.locks_merge_attention.argtypes = [vp, vp, vp, C.c_int, C.c_int, vp, vp, vp]
        for fn in ("locks_scan", "locks_select_scored", "locks_merge_selection", "locks_merge_attention"):
            getattr(L, fn).restype = C.c_int
        L.locks_select_exact.argtypes = [vp, vp, C.POINTER(KV), C.c_int, i32p, i32p, vp, vp, vp]
        L.locks_select_exact.restype = C.c_int
        L.locks_selection_quality.argtypes = [vp, vp, C.POINTER(KV), C.c_int, i32p, i32p, i32p, i32p, i32p, C.c_int, vp, vp]
        L.locks_selection_quality.restype = C.c_int
        rows, rotary, kvq = C.POINTER(Rows), C.POINTER(Rotary), C.POINTER(KVQ)
        L.locks_rope.argtypes = [vp, rotary, vp, C.c_int, rows, rows, rows, rows, vp]
        L.locks_append_rows.argtypes = [vp, rotary, vp, vp, C.c_int, rows, rows, rows, rows, C.POINTER(KV), C.c_int, vp]
        L.locks_kvq_append.argtypes = [vp, rotary, vp, vp, C.c_int, rows, rows, rows, rows, kvq, C.c_int, vp]
        L.locks_kvq_attend.argtypes = [vp, vp, vp, C.c_int, kvq, C.c_int, vp, vp, vp, vp, vp]
        L.locks_kvq_build_summaries.argtypes = [vp, kvq, C.c_int, vp, vp, vp, vp]
        for fn in ("locks_rope", "locks_append_rows", "locks_kvq_append", "locks_kvq_attend", "locks_kvq_build_summaries"):
            getattr(L, fn).restype = C.c_int
        L.locks_strerror.restype = C.c_char_p
        L.locks_strerror.argtypes = [C.c_int]
        for fn in ("locks_create", "locks_destroy", "locks_build_summaries", "locks_select", "locks_sparse_attend",
                   "locks_decode_step", "locks_decode_step_host", "locks_poll_status", "locks_last_launch_count"):
            getattr(L, fn).restype = C.c_int
        _lib = L
    return _lib


def calls_path() -> str:
    return _CALLS_PATH


def calls_stamp() -> str:
    """What _calls.so was compiled for, which it has as a string in it: it takes torch's tensors by their C++ classes."""
    return f"locks calls: torch {torch.__version__}, python {sys.version_info[0]}.{sys.version_info[1]}."


def calls():
    """The native marshalling module (_calls.so, built in-tree beside the library), bound to the library's functions.  Loaded when a call
    first takes it."""
    global _calls_module
    if _calls_module is None:
        path = calls_path()
        if not os.path.exists(path):
            raise LocksError(f"{path} is missing: run `python -m paper_2607_24555_b200.build`")
        with open(path, "rb") as f:
            if calls_stamp().encode() not in f.read():
                raise LocksError(f"{path} was built for another torch or Python than torch {torch.__version__}: run `python -m paper_2607_24555_b200.build`")
        spec = importlib.util.spec_from_file_location(__package__ + "._calls", path)
        m = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(m)
        L = lib()
        m.bind(LocksError, *[C.cast(getattr(L, f), C.c_void_p).value for f in
                             ("locks_rope", "locks_append_rows", "locks_kvq_append", "locks_kvq_attend", "locks_kvq_build_summaries", "locks_strerror")])
        _calls_module = m
    return _calls_module


def locks_strerror(code: int) -> str:
    return lib().locks_strerror(code).decode()


def locks_summary_bytes(cfg: Config) -> int:
    return int(lib().locks_summary_bytes(C.byref(cfg)))


def locks_workspace_bytes(cfg: Config) -> int:
    return int(lib().locks_workspace_bytes(C.byref(cfg)))


def _check(rc: int, what: str):
    if rc != 0:
        raise LocksError(f"{what} failed: {locks_strerror(rc)} ({rc})")


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _stream(stream) -> int:
    if stream is None:
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


COMBINE_SHARE_AVG, COMBINE_GROUP_MAX, COMBINE_GROUP_MASS, COMBINE_PER_HEAD = 0, 1, 2, 3   # LOCKS_COMBINE_* of include/locks.h


def make_config(Hq, Hkv, rank, fmt, dtype, max_batch, max_pages, budget, sm_scale=None, d=128, B=16,
                combine=COMBINE_SHARE_AVG) -> Config:
    if sm_scale is None:
        sm_scale = d ** -0.5
    dt = BF16 if dtype in ("bf16", torch.bfloat16) else F32
    f = {"i4": FMT_I4, "f32": FMT_F32, "i8": FMT_I8, "bf16": FMT_BF16}[fmt]
    return Config(d, B, Hq, Hkv, rank, f, dt, dt, max_batch, max_pages, budget, sm_scale, combine)


def make_rotary(inv_freq, axis=None, interleaved=False) -> Rotary:
    """Rotary description (locks_rotary): frequency and position axis of each rotated pair of a head's dimensions.

    inv_freq: rot_dim / 2 numbers; axis: as many axis indexes (None: one axis)."""
    n = len(inv_freq)
    if not 0 < n <= 64 or (axis is not None and len(axis) != n):
        raise LocksError("make_rotary: at most 64 frequencies, and an axis for each")
    r = Rotary()
    for i in range(n):
        r.inv_freq[i] = float(inv_freq[i])
        a = 0 if axis is None else int(axis[i])
        if not 0 <= a < 4:
            raise LocksError("make_rotary: axes are 0 .. 3")
        r.axis[i] = a
    r.rot_dim, r.num_axes, r.interleaved = 2 * n, 1 if axis is None else max(int(a) for a in axis) + 1, int(bool(interleaved))
    return r


def _need(ok, what):
    if not ok:
        raise LocksError(what)


@dataclass
class KVQView:
    """A paged cache in 8 bits.  k, v: [block, head, token, dim] int8 or float8_e4m3fn tensors (views of any layout whose dims are
    contiguous); k_scale, v_scale: [block, head] fp32; k_tail, v_tail: [max_batch, head, page_size, dim] fp32, or with twice as many tokens:
    then a sequence may be shortened by a page (see include/locks.h)."""
    k: torch.Tensor
    v: torch.Tensor
    k_scale: torch.Tensor
    v_scale: torch.Tensor
    k_tail: torch.Tensor
    v_tail: torch.Tensor
    block_table: torch.Tensor   # [max_batch, max_pages] int32, device
    seq_lens: torch.Tensor      # [max_batch] int32, device

    def __post_init__(self):
        k, v, f32, i32 = self.k, self.v, torch.float32, torch.int32
        _need(k.dim() == 4 and k.shape == v.shape and k.stride() == v.stride() and k.stride(3) == 1, "KVQView: k and v are [block, head, token, dim], dims contiguous, laid out alike")
        _need(k.dtype == v.dtype and k.dtype in (torch.int8, torch.float8_e4m3fn), "KVQView: codes are int8 or float8_e4m3fn")
        for t in (self.k_scale, self.v_scale):
            _need(t.dtype == f32 and t.shape == k.shape[:2] and t.is_contiguous(), "KVQView: scales are contiguous fp32 [block, head]")
        for t in (self.k_tail, self.v_tail):
            _need(t.dtype == f32 and t.dim() == 4 and t.shape[1] == k.shape[1] and t.shape[2] in (k.shape[2], 2 * k.shape[2]) and t.shape[3] == k.shape[3] and t.is_contiguous(),
                  "KVQView: tails are contiguous fp32 [max_batch, head, page_size or twice that, dim]")
        _need(self.k_tail.shape[2] == self.v_tail.shape[2], "KVQView: tails of one size")
        _need(self.block_table.dtype == i32 and self.block_table.dim() == 2 and self.block_table.is_contiguous(), "KVQView: block_table is contiguous int32 [max_batch, max_pages]")
        _need(self.seq_lens.dtype == i32 and self.seq_lens.dim() == 1 and self.seq_lens.is_contiguous(), "KVQView: seq_lens is contiguous int32 [max_batch]")
        _need(all(t.device == k.device for t in (v, self.k_scale, self.v_scale, self.k_tail, self.v_tail, self.block_table, self.seq_lens)), "KVQView: tensors on different devices")

    def struct(self) -> KVQ:
        sb, sh, st, _ = self.k.stride()
        return KVQ(self.k.data_ptr(), self.v.data_ptr(), sb, sh, st, self.k.shape[0], KVQ_INT if self.k.dtype == torch.int8 else KVQ_FLOAT,
                   self.k_scale.data_ptr(), self.v_scale.data_ptr(), self.k_tail.data_ptr(), self.v_tail.data_ptr(),
                   self.block_table.data_ptr(), self.seq_lens.data_ptr(), self.tail_pages)

    @property
    def tail_pages(self) -> int:
        return self.k_tail.shape[2] // self.k.shape[2]

    def kv_view(self) -> "KVView":
        """For locks_select, locks_scan, locks_select_scored and locks_selection_quality, which read the block table and the lengths only;
        calls that read the cache refuse it (codes are half as long as the rows that they would take)."""
        return TableView(self.k, self.v, self.k.stride()[:3], self.k.shape[0], self.block_table, self.seq_lens)


def new_kvq_cache(num_blocks, max_batch, Hkv, page_size, block_table, seq_lens, fmt="int8", layout="HND", tail_pages=1) -> KVQView:
    """An empty 8-bit cache on the table's device; layout "HND" [block, head, token, dim] or "NHD" [block, token, head, dim] in memory.
    tail_pages=2: sequences may be shortened by a page (drafted tokens that are refused; see include/locks.h)."""
    dev, d = block_table.device, 128
    dt = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}[fmt]

    def codes():
        if layout == "NHD":
            return torch.zeros(num_blocks, page_size, Hkv, d, dtype=torch.uint8, device=dev).view(dt).transpose(1, 2)
        return torch.zeros(num_blocks, Hkv, page_size, d, dtype=torch.uint8, device=dev).view(dt)

    def f32(*shape):
        return torch.zeros(*shape, dtype=torch.float32, device=dev)

    return KVQView(codes(), codes(), f32(num_blocks, Hkv), f32(num_blocks, Hkv), f32(max_batch, Hkv, tail_pages * page_size, d),
                   f32(max_batch, Hkv, tail_pages * page_size, d), block_table, seq_lens)


@dataclass
class KVView:
    """A paged cache: torch tensors plus element strides (block, head, token)."""
    k: torch.Tensor
    v: torch.Tensor
    strides: tuple
    num_blocks: int
    block_table: torch.Tensor   # [max_batch, max_pages] int32, device
    seq_lens: torch.Tensor      # [max_batch] int32, device

    def struct(self) -> KV:
        sb, sh, st = self.strides
        return KV(self.k.data_ptr(), self.v.data_ptr(), sb, sh, st, self.num_blocks, self.block_table.data_ptr(),
                  self.seq_lens.data_ptr())

    def tables(self) -> KV:
        """For calls that read no keys and values."""
        return KVView.struct(self)


class TableView(KVView):
    """Block table and lengths of a cache that is kept in another form."""

    def struct(self) -> KV:
        raise LocksError("an 8-bit cache's view has its block table and lengths only: this call reads keys or values")


class Context:
    """Owns a locks_ctx and its torch-allocated workspace.  Methods mirror the C entry points."""

    def __init__(self, cfg: Config, device="cuda:0"):
        self.cfg = cfg
        self.device = torch.device(device)
        if self.device.type == "cuda" and self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        L = lib()
        nbytes = locks_workspace_bytes(cfg)
        if nbytes == 0:
            raise LocksError("invalid or unsupported configuration")
        self.summary_bytes = locks_summary_bytes(cfg)
        self.k = -(-cfg.budget_tokens // cfg.page_size)
        with torch.cuda.device(self.device):
            self.workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
            base = (self.workspace.data_ptr() + 255) // 256 * 256
            h = C.c_void_p()
            _check(L.locks_create(C.byref(cfg), base, nbytes, C.byref(h)), "locks_create")
        self.handle = h

    def __getattr__(self, name):   # the native call layer, made by the first call that takes it
        if name not in ("_calls", "_call"):
            raise AttributeError(f"{type(self).__name__!r} object has no attribute {name!r}")
        if not self.__dict__.get("handle"):
            raise LocksError("the context is closed")
        cfg, m = self.cfg, calls()
        self._call = m.context(self.handle.value, cfg.num_q_heads, cfg.num_kv_heads, cfg.max_batch, cfg.max_pages_per_seq, cfg.page_size, self.k,
                               self.device.index, cfg.combine == COMBINE_PER_HEAD, self.summary_bytes, cfg.q_dtype == BF16)
        self._calls = m
        return self.__dict__[name]

    def close(self):
        if self.__dict__.get("handle"):
            if "_call" in self.__dict__:
                self._calls.close(self._call)
            lib().locks_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def new_summaries(self, num_blocks: int) -> torch.Tensor:
        return torch.zeros(num_blocks, self.cfg.num_kv_heads, self.summary_bytes, dtype=torch.uint8, device=self.device)

    def locks_build_summaries(self, kv: KVView, batch, summaries, page_begin=None, page_end=None, stream=None):
        s = kv.struct()
        _check(lib().locks_build_summaries(self.handle, C.byref(s), batch, _ptr(page_begin), _ptr(page_end),
                                           _ptr(summaries), _stream(stream)), "locks_build_summaries")

    def locks_build_summaries_layers(self, kv: KVView, k_layers, summaries_layers, batch, page_begin=None, page_end=None,
                                     stream=None):
        """k_layers / summaries_layers: lists of tensors (one per layer).  Returns the two device pointer arrays, which
        the caller keeps alive until the launch has run."""
        import torch
        dev = summaries_layers[0].device
        kp = torch.tensor([t.data_ptr() for t in k_layers], dtype=torch.int64, device=dev)
        sp = torch.tensor([t.data_ptr() for t in summaries_layers], dtype=torch.int64, device=dev)
        s = kv.struct()
        _check(lib().locks_build_summaries_layers(self.handle, C.byref(s), _ptr(kp), _ptr(sp), len(k_layers), batch,
                                                  _ptr(page_begin), _ptr(page_end), _stream(stream)),
               "locks_build_summaries_layers")
        return kp, sp

    def locks_fake_quantize_pages(self, kv: KVView, batch, bits, page_begin=None, page_end=None, stream=None):
        s = kv.struct()
        _check(lib().locks_fake_quantize_pages(self.handle, C.byref(s), batch, _ptr(page_begin), _ptr(page_end), int(bits),
                                               _stream(stream)), "locks_fake_quantize_pages")

    def locks_scan(self, q, summaries, kv: KVView, batch, head_logz, page_logmass=None, stream=None):
        s = kv.tables()
        _check(lib().locks_scan(self.handle, _ptr(q), _ptr(summaries), C.byref(s), batch, _ptr(page_logmass), _ptr(head_logz),
                                _stream(stream)), "locks_scan")

    def locks_select_scored(self, head_logz_parts, kv: KVView, batch, page_ids, page_count, page_logshare=None,
                            page_logmass=None, stream=None):
        s = kv.tables()
        _check(lib().locks_select_scored(self.handle, _ptr(page_logmass), _ptr(head_logz_parts), int(head_logz_parts.shape[0]),
                                         C.byref(s), batch, _ptr(page_ids), _ptr(page_count), _ptr(page_logshare),
                                         _stream(stream)), "locks_select_scored")

    def locks_merge_selection(self, cand_key, cand_page, batch, page_ids, page_count, stream=None):
        _check(lib().locks_merge_selection(self.handle, _ptr(cand_key), _ptr(cand_page), int(cand_key.shape[0]), batch,
                                           _ptr(page_ids), _ptr(page_count), _stream(stream)), "locks_merge_selection")

    def locks_merge_attention(self, part_out, part_lse, batch, out, lse=None, stream=None):
        _check(lib().locks_merge_attention(self.handle, _ptr(part_out), _ptr(part_lse), int(part_out.shape[0]), batch,
                                           _ptr(out), _ptr(lse), _stream(stream)), "locks_merge_attention")

    def locks_select(self, q, summaries, kv: KVView, batch, page_ids, page_count, page_logmass=None,
                     page_logshare=None, stream=None):
        s = kv.tables()
        _check(lib().locks_select(self.handle, _ptr(q), _ptr(summaries), C.byref(s), batch, _ptr(page_ids),
                                  _ptr(page_count), _ptr(page_logmass), _ptr(page_logshare), _stream(stream)),
               "locks_select")

    def locks_select_exact(self, q, kv: KVView, batch, page_ids, page_count, page_logmass=None, page_logshare=None,
                           stream=None):
        s = kv.struct()
        _check(lib().locks_select_exact(self.handle, _ptr(q), C.byref(s), batch, _ptr(page_ids), _ptr(page_count),
                                        _ptr(page_logmass), _ptr(page_logshare), _stream(stream)), "locks_select_exact")

    def locks_select_rival(self, scorer, q, summaries, kv: KVView, batch, page_ids, page_count, page_score=None,
                           page_logshare=None, stream=None):
        s = kv.struct()
        _check(lib().locks_select_rival(self.handle, int(scorer), _ptr(q), _ptr(summaries), C.byref(s), batch,
                                        _ptr(page_ids), _ptr(page_count), _ptr(page_score), _ptr(page_logshare),
                                        _stream(stream)), "locks_select_rival")

    def locks_selection_quality(self, exact_logmass, kv: KVView, batch, page_ids, page_count, ref_ids, ref_count,
                                quality, marked_pages=None, stream=None):
        s = kv.tables()
        n_marked = 0 if marked_pages is None else int(marked_pages.shape[-1])
        _check(lib().locks_selection_quality(self.handle, _ptr(exact_logmass), C.byref(s), batch, _ptr(page_ids),
                                             _ptr(page_count), _ptr(ref_ids), _ptr(ref_count), _ptr(marked_pages),
                                             n_marked, _ptr(quality), _stream(stream)), "locks_selection_quality")

    def locks_sparse_attend(self, q, kv: KVView, batch, page_ids, page_count, out, lse=None, stream=None):
        s = kv.struct()
        _check(lib().locks_sparse_attend(self.handle, _ptr(q), C.byref(s), batch, _ptr(page_ids), _ptr(page_count),
                                         _ptr(out), _ptr(lse), _stream(stream)), "locks_sparse_attend")

    def locks_decode_step(self, q, k_new, v_new, kv: KVView, summaries, batch, out, page_ids=None, page_count=None,
                          stream=None):
        s = kv.struct()
        _check(lib().locks_decode_step(self.handle, _ptr(q), _ptr(k_new), _ptr(v_new), C.byref(s), _ptr(summaries),
                                       batch, _ptr(out), _ptr(page_ids), _ptr(page_count), _stream(stream)),
               "locks_decode_step")

    def locks_decode_step_host(self, q_host, k_new_host, v_new_host, kv: KVView, summaries, batch, out_host,
                               page_ids_host=None, page_count_host=None, stream=None):
        s = kv.struct()
        _check(lib().locks_decode_step_host(self.handle, _ptr(q_host), _ptr(k_new_host), _ptr(v_new_host), C.byref(s),
                                            _ptr(summaries), batch, _ptr(out_host), _ptr(page_ids_host),
                                            _ptr(page_count_host), _stream(stream)), "locks_decode_step_host")

    # ---- rotary positions, appends and the 8-bit cache: checked (type, shape, strides, device) and marshalled natively, in csrc/calls.cpp
    def locks_rope(self, rotary, positions, q, q_out, k=None, k_out=None, stream=None):
        """Rotate q [tokens, Hq, 128] into q_out and k [tokens, Hkv, 128] into k_out (either pair may be None; in place: pass a
        tensor twice).  positions: int32 [axes, tokens], or [tokens] with one axis."""
        self._calls.rope(self._call, rotary, positions, q, q_out, k, k_out, stream)

    def locks_append_rows(self, k_new, v_new, kv: KVView, batch, rotary=None, positions=None, q=None, q_out=None, cu_tokens=None,
                          stream=None):
        """Append k_new, v_new [tokens, Hkv, 128] (keys rotated, if there is a rotary description) to the cache and rotate q into
        q_out.  kv.seq_lens counts the new tokens already; cu_tokens: see include/locks.h."""
        self._calls.append_rows(self._call, k_new, v_new, kv, batch, rotary, positions, q, q_out, cu_tokens, stream)

    def locks_kvq_append(self, k_new, v_new, kvq: KVQView, batch, rotary=None, positions=None, q=None, q_out=None, cu_tokens=None,
                         stream=None):
        """locks_append_rows for the 8-bit cache: complete pages as codes, the unfinished one in the tails."""
        self._calls.kvq_append(self._call, k_new, v_new, kvq, batch, rotary, positions, q, q_out, cu_tokens, stream)

    def locks_kvq_attend(self, q, kvq: KVQView, batch, out, lse=None, page_ids=None, page_count=None, cu_tokens=None, stream=None):
        """Attention of q [tokens, Hq, 128] over the 8-bit cache into out; one token per request (all pages, or page_ids and
        page_count of locks_select), or with cu_tokens several, each seeing what is before it."""
        self._calls.kvq_attend(self._call, q, kvq, batch, out, lse, page_ids, page_count, cu_tokens, stream)

    def locks_kvq_build_summaries(self, kvq: KVQView, batch, summaries, page_begin=None, page_end=None, stream=None):
        """locks_build_summaries from the codes of the 8-bit cache."""
        self._calls.kvq_build_summaries(self._call, kvq, batch, summaries, page_begin, page_end, stream)

    def locks_poll_status(self, stream=None) -> int:
        st = C.c_int32(0)
        _check(lib().locks_poll_status(self.handle, C.byref(st), _stream(stream)), "locks_poll_status")
        return int(st.value)

    def locks_selftest_wait_timeout(self, limit_ms: int, stream=None):
        _check(lib().locks_selftest_wait_timeout(self.handle, int(limit_ms), _stream(stream)), "locks_selftest_wait_timeout")

    def locks_set_scan_partition(self, mode: int):
        _check(lib().locks_set_scan_partition(self.handle, int(mode)), "locks_set_scan_partition")

    def locks_last_scan_partition(self) -> int:
        return int(lib().locks_last_scan_partition(self.handle))

    def locks_host_cache_clear(self):
        _check(lib().locks_host_cache_clear(self.handle), "locks_host_cache_clear")

    def locks_profile_begin(self, max_steps: int):
        _check(lib().locks_profile_begin(self.handle, max_steps), "locks_profile_begin")

    def locks_profile_end(self):
        ms = (C.c_float * 3)()
        n = C.c_int(0)
        _check(lib().locks_profile_end(self.handle, ms, C.byref(n)), "locks_profile_end")
        return {"scan": ms[0], "select": ms[1], "attend": ms[2]}, int(n.value)

    def locks_profile_read(self, stream=None):
        ms = (C.c_float * 3)()
        _check(lib().locks_profile_read(self.handle, ms, _stream(stream)), "locks_profile_read")
        return {"scan": ms[0], "select": ms[1], "attend": ms[2]}

    def locks_last_launch_count(self) -> int:
        return int(lib().locks_last_launch_count(self.handle))


def locks_sparse_attend_noalloc(cfg: Config, q, kv: KVView, batch, page_ids, page_count, out, lse=None, stream=None):
    """Sparse attention without a context or workspace, for callers that cannot allocate device memory
    (see include/locks.h).  Raises LocksError with the library's message if the problem exceeds the
    built-in scratch."""
    s = kv.struct()
    _check(lib().locks_sparse_attend_noalloc(C.byref(cfg), _ptr(q), C.byref(s), batch, _ptr(page_ids), _ptr(page_count),
                                             _ptr(out), _ptr(lse), _stream(stream)), "locks_sparse_attend_noalloc")
