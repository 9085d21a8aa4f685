"""ctypes binding of ``include/ngram_spec.h``: same names, argument marshalling only."""
from __future__ import annotations

import ctypes as C
import os
import re

import torch

from .build import LIB, build_library

FLAG_DEDUP, FLAG_MODEL_FILL, FLAG_KEY_NEXT_TOKEN, FLAG_PARTIAL_TAIL = 1, 2, 4, 8
STATUS_TOKEN_RANGE, STATUS_CAPACITY, STATUS_TIMEOUT, STATUS_GROUPS, STATUS_INDEX = 1, 2, 4, 8, 16
SPEC_F32, SPEC_BF16, SPEC_E4M3 = 0, 1, 2

_HEADER = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "include", "ngram_spec.h")
_lib = None


def flag_reserve(n: int) -> int:
    """Draft flag bits that reserve ``n`` rows for the model strategy (SPEC_FLAG_RESERVE)."""
    return (int(n) & 0xFF) << 8


class SpecError(RuntimeError):
    pass


class _KVCacheStruct(C.Structure):
    _fields_ = [("d_k", C.c_void_p), ("d_v", C.c_void_p), ("d_k_exp", C.c_void_p), ("d_v_exp", C.c_void_p), ("d_table", C.c_void_p),
                ("dtype", C.c_int), ("n_pages", C.c_int), ("max_pages", C.c_int), ("page", C.c_int), ("heads", C.c_int),
                ("head_dim", C.c_int)]


class _RopeStruct(C.Structure):
    _fields_ = [("d_freq", C.c_void_p), ("rot", C.c_int), ("interleaved", C.c_int), ("factor", C.c_float)]


def declared_symbols() -> list[str]:
    """Function names declared in the public header."""
    text = re.sub(r"/\*.*?\*/", "", open(_HEADER).read(), flags=re.S)
    return sorted(set(re.findall(r"\b([a-z_][a-z0-9_]*)\s*\(", text)) - {"defined"})


def load_library(build: bool = True) -> C.CDLL:
    """Load (building first if needed) the CUDA library.  Fails loudly if it cannot be loaded."""
    global _lib
    if _lib is not None:
        return _lib
    if build:
        build_library()
    if not os.path.exists(LIB):
        raise SpecError(f"{LIB} is missing: build it with `python -m paper_2411_03786_b200.build`")
    lib = C.CDLL(LIB)
    vp, ip, i32p, fp = C.c_void_p, C.POINTER(C.c_int), C.c_void_p, C.c_void_p
    lib.spec_init.argtypes = [C.POINTER(vp), vp, vp, C.c_int, C.c_int, C.c_int, C.c_int, vp]
    lib.spec_destroy.argtypes = [vp]
    lib.spec_get_status.argtypes = [vp, ip, vp]
    lib.spec_last_error.argtypes = [vp]
    lib.spec_last_error.restype = C.c_char_p
    lib.build_model_ngram_tables.argtypes = [vp, vp, C.c_int, C.c_int, i32p, fp, i32p, vp]
    lib.build_model_unigram.argtypes = [vp, C.c_int, i32p, fp, vp]
    lib.spec_set_model_table.argtypes = [vp, i32p, C.c_int, i32p, C.c_int]
    lib.draft_context_ngrams.argtypes = [vp, i32p, i32p, C.c_int, C.c_int, ip, C.c_int, C.c_int, C.c_int, C.c_int,
                                         C.c_int, i32p, i32p, i32p, i32p, vp]
    lib.verify_lmhead_argmax.argtypes = [vp, vp, C.c_int, i32p, fp, vp]
    lib.accept_and_commit.argtypes = [vp, i32p, i32p, i32p, C.c_int, C.c_int, C.c_int, i32p, i32p, C.c_int, i32p,
                                      i32p, i32p, vp]
    lib.verify_accept_commit.argtypes = [vp, vp, i32p, i32p, C.c_int, C.c_int, C.c_int, i32p, i32p, i32p, C.c_int, i32p,
                                         i32p, i32p, vp]
    lib.verify_lmhead_keys.argtypes = [vp, vp, C.c_int, C.c_int, vp, vp]
    lib.spec_unpack_keys.argtypes = [vp, C.c_int, C.c_int, i32p, fp, vp]
    lib.spec_accumulate_stats.argtypes = [vp, i32p, i32p, i32p, C.c_int, C.c_int, C.c_int, vp, vp]
    lib.spec_debug_logits.argtypes = [vp, vp, C.c_int, fp, vp]
    lib.spec_quantize_rows_fp8.argtypes = [vp, vp, C.c_int, vp, fp, vp]
    lib.spec_quantize_head_fp8.argtypes = [vp, vp, fp, vp]
    lib.spec_set_head_fp8.argtypes = [vp, vp, fp]
    lib.verify_lmhead_argmax_fp8.argtypes = [vp, vp, C.c_int, vp, fp, i32p, fp, vp]
    lib.verify_lmhead_argmax_noalloc.argtypes = [vp, C.c_int, C.c_int, vp, C.c_int, i32p, fp, C.c_int, vp]
    lib.build_model_ngram_table_rows.argtypes = [vp, vp, C.c_int, C.c_int, C.c_int, i32p, fp, vp]
    lib.spec_extend_model_table.argtypes = [vp, i32p, C.c_int, C.c_int, i32p, vp]
    lib.spec_debug_expire_wait.argtypes = [vp, C.c_ulonglong, C.c_int, vp]
    lib.spec_debug_wait_limit.argtypes = [vp, C.c_ulonglong]
    lib.spec_context_index_bytes.argtypes = [C.c_int, C.c_int, C.c_int]
    lib.spec_context_index_bytes.restype = C.c_size_t
    lib.spec_context_index_build.argtypes = [vp, vp, i32p, i32p, C.c_int, C.c_int, ip, C.c_int, C.c_int, C.c_int, vp]
    lib.draft_context_ngrams_indexed.argtypes = [vp, vp, i32p, i32p, C.c_int, C.c_int, ip, C.c_int, C.c_int, C.c_int, C.c_int,
                                                 C.c_int, i32p, i32p, i32p, i32p, vp]
    lib.accept_and_commit_indexed.argtypes = [vp, vp, i32p, i32p, i32p, C.c_int, C.c_int, C.c_int, i32p, i32p, C.c_int, i32p,
                                              i32p, i32p, vp]
    i, ll, cachep, ropep = C.c_int, C.c_longlong, C.POINTER(_KVCacheStruct), C.POINTER(_RopeStruct)
    rows = [vp, ll, ll]
    lib.spec_rope_rows.argtypes = [vp, ropep, vp, i, ll, ll, vp, vp, i, ll, ll, vp, i, i32p, i, vp]
    lib.spec_cache_write.argtypes = [vp, cachep, *rows, *rows, i, i, i, i32p, i32p, i32p, ropep, vp]
    lib.spec_cache_read.argtypes = [vp, cachep, i, i, i32p, i32p, vp, vp, vp]
    lib.spec_score_bytes.argtypes = [vp, i, i]
    lib.spec_score_bytes.restype = C.c_size_t
    lib.score_tokens.argtypes = [vp, vp, i, i32p, i, fp, fp, i32p, fp, vp, C.c_size_t, vp]
    lib.spec_tree_mask.argtypes = [vp, i32p, i, i, i32p, i32p, i32p, vp]
    lib.spec_tree_attention_bytes.argtypes = [vp, cachep, i, i, i]
    lib.spec_tree_attention_bytes.restype = C.c_size_t
    lib.spec_tree_attention.argtypes = [vp, cachep, *rows, *rows, *rows, i, i, i, i32p, i32p, i32p, C.c_float, vp, fp, vp, C.c_size_t, vp]
    lib.spec_launch_count.argtypes = [vp]
    lib.spec_launch_count.restype = C.c_longlong
    _lib = lib
    return lib


def _ptr(t, dtype=None):
    if t is None:
        return None
    # pinned host memory is mapped into the device address space (unified addressing): small outputs may
    # live there so that a kernel's result reaches the host without a separate copy
    assert (t.is_cuda or t.is_pinned()) and t.is_contiguous(), "tensors must be contiguous CUDA (or pinned host) tensors"
    if dtype is not None:
        assert t.dtype == dtype, f"expected {dtype}, got {t.dtype}"
    return C.c_void_p(t.data_ptr())


def _stream():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def _new(like: torch.Tensor) -> torch.Tensor:
    return torch.empty_like(like, memory_format=torch.contiguous_format)


def _need(ok: bool, what: str):
    if not ok:
        raise SpecError(what)


def _rows(t: torch.Tensor, name: str):
    """Pointer, token stride and head stride of ``t[..., heads, D]`` (see _strides)."""
    if not t.is_cuda or t.dtype is not torch.bfloat16:
        raise SpecError(f"{name}: expected a bfloat16 CUDA tensor")
    st = t.stride()  # (the two usual forms without a call)
    if len(st) == 4 and st[3] == 1 and st[0] == st[1] * t.shape[1]:
        return t.data_ptr(), st[1], st[2]
    if len(st) == 3 and st[2] == 1:
        return t.data_ptr(), st[0], st[1]
    return t.data_ptr(), *_strides(t, name)


def _strides(t: torch.Tensor, name: str):
    """Token and head stride of ``t[..., heads, D]`` whose head vectors are contiguous and whose tokens are all one stride
    apart.  The stride of a dimension of one means nothing: with one node to a sequence the sequences are the tokens."""
    if t.dim() < 3:
        raise SpecError(f"{name}: expected [..., heads, head_dim]")
    *lead, head, one = t.stride()
    if one != 1:
        raise SpecError(f"{name}: head vectors must be contiguous")
    tok = lead[-1]
    if len(lead) > 2 or (len(lead) == 2 and lead[0] != tok * t.shape[1]):
        after = None  # where the next dimension has to go on
        for n, st in zip(reversed(t.shape[:-2]), reversed(lead)):
            if n == 0:
                break
            if n > 1:
                if after is None:
                    tok = after = st
                elif st != after:
                    raise SpecError(f"{name}: tokens must be one stride apart (sequences N tokens)")
                after *= n
    return tok, head


def _i32(t: torch.Tensor | None, name: str, shape):
    if t is None:
        return None
    if not t.is_cuda or t.dtype is not torch.int32 or t.shape != shape or not t.is_contiguous():
        raise SpecError(f"{name}: expected a contiguous int32 CUDA tensor of shape {tuple(shape)}")
    return t.data_ptr()


def _out(t: torch.Tensor, shape, dtype: torch.dtype, what: str):
    # (pinned host memory will do, as in _ptr)
    if t is None or not (t.is_cuda or t.is_pinned()) or t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
        raise SpecError(f"{what}: expected a contiguous {dtype} CUDA (or pinned host) tensor of shape {tuple(shape)}")


def _scratch(work: torch.Tensor, what: str):
    """Pointer and bytes of a caller's workspace."""
    if not work.is_cuda or not work.is_contiguous():
        raise SpecError(f"{what}: work must be a contiguous CUDA tensor")
    return work.data_ptr(), work.numel() * work.element_size()


class KVCache:
    """A paged key/value cache in the caller's tensors (see ``spec_kv_cache`` in the header).

    ``k``, ``v`` are ``[n_pages, heads, page, head_dim]``, bfloat16 or uint8 (E4M3 codes); ``table[S, max_pages]`` int32
    holds each sequence's pages; an E4M3 cache has ``k_exp``, ``v_exp`` ``[n_pages, heads, page]`` uint8.  A program that writes
    codes itself marks a vector with a NaN by scale byte 255: attention does not look for E4M3's own NaN codes.
    """

    def __init__(self, k: torch.Tensor, v: torch.Tensor, table: torch.Tensor, k_exp: torch.Tensor | None = None, v_exp: torch.Tensor | None = None):
        _need(k.dim() == 4 and k.shape == v.shape and k.dtype == v.dtype and k.dtype in (torch.bfloat16, torch.uint8),
              "KVCache: k and v must be [n_pages, heads, page, head_dim], both bfloat16 or both uint8")
        _need((k.dtype == torch.uint8) == (k_exp is not None) == (v_exp is not None), "KVCache: k_exp and v_exp belong to uint8 codes")
        _need(table.dim() == 2 and table.dtype == torch.int32, "KVCache: table must be int32 [S, max_pages]")
        for t in (k_exp, v_exp):
            _need(t is None or (t.dtype == torch.uint8 and t.shape == k.shape[:3]), "KVCache: scales must be uint8 [n_pages, heads, page]")
        for t in (k, v, table, k_exp, v_exp):
            _need(t is None or (t.is_cuda and t.is_contiguous()), "KVCache: tensors must be contiguous CUDA tensors")
        self.k, self.v, self.table, self.k_exp, self.v_exp = k, v, table, k_exp, v_exp
        self.n_pages, self.heads, self.page, self.head_dim = (int(x) for x in k.shape)
        self.sequences = int(table.shape[0])
        ptr = lambda t: None if t is None else t.data_ptr()
        self._struct = _KVCacheStruct(ptr(k), ptr(v), ptr(k_exp), ptr(v_exp), ptr(table), SPEC_BF16 if k.dtype == torch.bfloat16 else SPEC_E4M3,
                                      self.n_pages, int(table.shape[1]), self.page, self.heads, self.head_dim)
        self._ref = C.byref(self._struct)

    @classmethod
    def empty(cls, n_pages: int, heads: int, page: int, head_dim: int, table: torch.Tensor, quantised: bool = False) -> "KVCache":
        shape = (n_pages, heads, page, head_dim)
        k, v = (torch.empty(shape, dtype=torch.uint8 if quantised else torch.bfloat16, device=table.device) for _ in range(2))
        ke, ve = (torch.empty(shape[:3], dtype=torch.uint8, device=table.device) if quantised else None for _ in range(2))
        return cls(k, v, table, ke, ve)


class Rope:
    """Rotary positions: ``freq[rot / 2]`` float32 radians per position (see ``spec_rope`` in the header)."""

    def __init__(self, freq: torch.Tensor, interleaved: bool = False, scale: float = 1.0):
        _need(freq.is_cuda and freq.dtype == torch.float32 and freq.dim() == 1 and freq.is_contiguous(), "Rope: freq must be a contiguous float32 CUDA vector")
        self.freq = freq
        self._struct = _RopeStruct(freq.data_ptr(), 2 * int(freq.shape[0]), int(interleaved), float(scale))
        self._ref = C.byref(self._struct)


class SpecContext:
    """One model head on one GPU.  Methods mirror the C entry points and launch on torch's current stream."""

    def __init__(self, embed: torch.Tensor, unembed: torch.Tensor):
        self._lib = load_library()
        self._h = C.c_void_p()
        if not torch.cuda.is_available():
            raise SpecError("no CUDA device: this library has no CPU path")
        assert embed.shape == unembed.shape and embed.dtype == unembed.dtype
        dtype = {torch.float32: SPEC_F32, torch.bfloat16: SPEC_BF16}[embed.dtype]
        self.V, self.d = int(embed.shape[0]), int(embed.shape[1])
        self._keep = [embed, unembed]
        self._device = embed.device.index or 0
        self._work_bytes = {}  # scratch of a tree_attention call, by its sizes
        rc = self._lib.spec_init(C.byref(self._h), _ptr(embed), _ptr(unembed), dtype, self.V, self.d,
                                 embed.device.index or 0, _stream())
        if rc != 0:
            raise SpecError(f"spec_init failed ({rc}): {self._lib.spec_last_error(None).decode()}")

    def _check(self, rc: int, what: str):
        if rc != 0:
            raise SpecError(f"{what} failed ({rc}): {self._lib.spec_last_error(self._h).decode()}")

    def _raw_stream(self) -> int:
        """torch's current stream on the context's device (torch.cuda.current_stream() makes an object of it: 3 us)."""
        return torch._C._cuda_getCurrentRawStream(self._device)

    def close(self):
        if self._h:
            torch.cuda.synchronize()
            self._lib.spec_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def get_status(self) -> int:
        bits = C.c_int(0)
        self._check(self._lib.spec_get_status(self._h, C.byref(bits), _stream()), "spec_get_status")
        return bits.value

    def launch_count(self) -> int:
        return int(self._lib.spec_launch_count(self._h))

    def build_model_ngram_tables(self, k_tab: int, rows: torch.Tensor | None = None, w_ext: int = 0,
                                 with_values: bool = False):
        dev = self._keep[0].device
        tab = torch.empty((self.V, k_tab), dtype=torch.int32, device=dev)
        val = torch.empty((self.V, k_tab), dtype=torch.float32, device=dev) if with_values else None
        ext = torch.empty((self.V, k_tab, w_ext), dtype=torch.int32, device=dev) if w_ext > 0 else None
        self._check(self._lib.build_model_ngram_tables(self._h, _ptr(rows, torch.bfloat16), k_tab, w_ext, _ptr(tab),
                                                       _ptr(val), _ptr(ext), _stream()), "build_model_ngram_tables")
        self._keep_table = (tab, ext, rows)
        return tab, val, ext

    def build_model_ngram_table_rows(self, k_tab: int, row_begin: int, row_count: int, tab: torch.Tensor,
                                     val: torch.Tensor | None = None, rows: torch.Tensor | None = None):
        """Writes rows ``[row_begin, row_begin + row_count)`` of the whole ``tab[V, k_tab]`` (one rank's slice)."""
        assert tuple(tab.shape) == (self.V, k_tab)
        self._check(self._lib.build_model_ngram_table_rows(self._h, _ptr(rows, torch.bfloat16), int(row_begin), int(row_count),
                                                           k_tab, _ptr(tab, torch.int32), _ptr(val, torch.float32), _stream()),
                    "build_model_ngram_table_rows")
        return tab

    def extend_model_table(self, tab: torch.Tensor, w_ext: int):
        """Extension ``ext[V, k_tab, w_ext]`` of a complete table; adopts both for drafting."""
        k_tab = int(tab.shape[1])
        ext = torch.empty((self.V, k_tab, w_ext), dtype=torch.int32, device=tab.device)
        self._check(self._lib.spec_extend_model_table(self._h, _ptr(tab, torch.int32), k_tab, int(w_ext), _ptr(ext), _stream()),
                    "spec_extend_model_table")
        self._keep_table = (tab, ext, None)
        return ext

    def debug_expire_wait(self, limit_ns: int = 20000, mark_verify_incomplete: bool = False):
        self._check(self._lib.spec_debug_expire_wait(self._h, int(limit_ns), int(mark_verify_incomplete), _stream()),
                    "spec_debug_expire_wait")

    def debug_wait_limit(self, limit_ns: int = 2_000_000_000):
        self._check(self._lib.spec_debug_wait_limit(self._h, int(limit_ns)), "spec_debug_wait_limit")

    def build_model_unigram(self, k_uni: int):
        """Returns ``(ids[k_uni] by ascending distance, dist2[V])``."""
        dev = self._keep[0].device
        idx = torch.empty(max(k_uni, 1), dtype=torch.int32, device=dev)
        dist2 = torch.empty(self.V, dtype=torch.float32, device=dev)
        self._check(self._lib.build_model_unigram(self._h, k_uni, _ptr(idx), _ptr(dist2), _stream()), "build_model_unigram")
        return idx[:k_uni], dist2

    def set_model_table(self, tab: torch.Tensor, ext: torch.Tensor | None = None):
        k_tab = int(tab.shape[1])
        w_ext = int(ext.shape[2]) if ext is not None else 0
        self._check(self._lib.spec_set_model_table(self._h, _ptr(tab, torch.int32), k_tab, _ptr(ext, torch.int32), w_ext),
                    "spec_set_model_table")
        self._keep_table = (tab, ext, None)

    def draft_context_ngrams(self, hist: torch.Tensor, lens: torch.Tensor, qs, topk: int, B: int, w: int,
                             flags: int = FLAG_DEDUP | FLAG_MODEL_FILL, out=None):
        S, cap = int(hist.shape[0]), int(hist.shape[1])
        dev = hist.device
        if out is None:
            out = (torch.empty((S, B, w), dtype=torch.int32, device=dev), torch.empty(S, dtype=torch.int32, device=dev),
                   torch.empty((S, B), dtype=torch.int32, device=dev), torch.empty((S, B), dtype=torch.int32, device=dev))
        drafts, nd, src, counts = out
        qs_arr = (C.c_int * max(1, len(qs)))(*[int(q) for q in qs])
        self._check(self._lib.draft_context_ngrams(self._h, _ptr(hist, torch.int32), _ptr(lens, torch.int32), S, cap,
                                                   qs_arr, len(qs), topk, B, w, flags, _ptr(drafts), _ptr(nd),
                                                   _ptr(src), _ptr(counts), _stream()), "draft_context_ngrams")
        return drafts, nd, src, counts

    def context_index_build(self, hist: torch.Tensor, lens: torch.Tensor, qs, w: int, flags: int = 0, index: torch.Tensor | None = None):
        """Builds (and registers) the incremental context index of the current histories; returns the index buffer."""
        S, cap = int(hist.shape[0]), int(hist.shape[1])
        need = int(self._lib.spec_context_index_bytes(S, cap, len(qs)))
        if index is None:
            index = torch.empty(need, dtype=torch.uint8, device=hist.device)
        assert index.numel() >= need
        qs_arr = (C.c_int * max(1, len(qs)))(*[int(q) for q in qs])
        self._check(self._lib.spec_context_index_build(self._h, _ptr(index), _ptr(hist, torch.int32), _ptr(lens, torch.int32), S, cap,
                                                       qs_arr, len(qs), w, flags, _stream()), "spec_context_index_build")
        self._keep_index = index
        return index

    def draft_context_ngrams_indexed(self, index: torch.Tensor, hist: torch.Tensor, lens: torch.Tensor, qs, topk: int, B: int, w: int,
                                     flags: int = FLAG_DEDUP | FLAG_MODEL_FILL, out=None):
        S, cap = int(hist.shape[0]), int(hist.shape[1])
        dev = hist.device
        if out is None:
            out = (torch.empty((S, B, w), dtype=torch.int32, device=dev), torch.empty(S, dtype=torch.int32, device=dev),
                   torch.empty((S, B), dtype=torch.int32, device=dev), torch.empty((S, B), dtype=torch.int32, device=dev))
        drafts, nd, src, counts = out
        qs_arr = (C.c_int * max(1, len(qs)))(*[int(q) for q in qs])
        self._check(self._lib.draft_context_ngrams_indexed(self._h, _ptr(index), _ptr(hist, torch.int32), _ptr(lens, torch.int32), S, cap,
                                                           qs_arr, len(qs), topk, B, w, flags, _ptr(drafts), _ptr(nd),
                                                           _ptr(src), _ptr(counts), _stream()), "draft_context_ngrams_indexed")
        return drafts, nd, src, counts

    def accept_and_commit_indexed(self, index: torch.Tensor, drafts, n_drafts, argmax, hist, lens, out=None):
        S, B, w = (int(x) for x in drafts.shape)
        cap = int(hist.shape[1])
        dev = hist.device
        if out is None:
            out = (torch.empty(S, dtype=torch.int32, device=dev), torch.empty(S, dtype=torch.int32, device=dev),
                   torch.empty((S, w + 1), dtype=torch.int32, device=dev))
        acc, best, com = out
        self._check(self._lib.accept_and_commit_indexed(self._h, _ptr(index), _ptr(drafts, torch.int32), _ptr(n_drafts, torch.int32),
                                                        _ptr(argmax, torch.int32), S, B, w, _ptr(hist, torch.int32),
                                                        _ptr(lens, torch.int32), cap, _ptr(acc), _ptr(best), _ptr(com),
                                                        _stream()), "accept_and_commit_indexed")
        return acc, best, com

    def verify_lmhead_argmax(self, hidden: torch.Tensor, out=None, with_max: bool = False):
        M = int(hidden.shape[0])
        if out is None:
            out = (torch.empty(M, dtype=torch.int32, device=hidden.device),
                   torch.empty(M, dtype=torch.float32, device=hidden.device) if with_max else None)
        am, mx = out
        self._check(self._lib.verify_lmhead_argmax(self._h, _ptr(hidden, torch.bfloat16), M, _ptr(am), _ptr(mx),
                                                   _stream()), "verify_lmhead_argmax")
        return am, mx

    def accept_and_commit(self, drafts, n_drafts, argmax, hist, lens, out=None):
        S, B, w = (int(x) for x in drafts.shape)
        cap = int(hist.shape[1])
        dev = hist.device
        if out is None:
            out = (torch.empty(S, dtype=torch.int32, device=dev), torch.empty(S, dtype=torch.int32, device=dev),
                   torch.empty((S, w + 1), dtype=torch.int32, device=dev))
        acc, best, com = out
        self._check(self._lib.accept_and_commit(self._h, _ptr(drafts, torch.int32), _ptr(n_drafts, torch.int32),
                                                _ptr(argmax, torch.int32), S, B, w, _ptr(hist, torch.int32),
                                                _ptr(lens, torch.int32), cap, _ptr(acc), _ptr(best), _ptr(com),
                                                _stream()), "accept_and_commit")
        return acc, best, com

    def verify_accept_commit(self, hidden, drafts, n_drafts, hist, lens, argmax=None, out=None):
        """Fused verify + accept: returns ``(argmax[S, B, w+1], acc_len, best_row, committed)``."""
        S, B, w = (int(x) for x in drafts.shape)
        cap = int(hist.shape[1])
        dev = hist.device
        if argmax is None:
            argmax = torch.empty(S * B * (w + 1), dtype=torch.int32, device=dev)
        if out is None:
            out = (torch.empty(S, dtype=torch.int32, device=dev), torch.empty(S, dtype=torch.int32, device=dev),
                   torch.empty((S, w + 1), dtype=torch.int32, device=dev))
        acc, best, com = out
        self._check(self._lib.verify_accept_commit(self._h, _ptr(hidden, torch.bfloat16), _ptr(drafts, torch.int32),
                                                   _ptr(n_drafts, torch.int32), S, B, w, _ptr(argmax, torch.int32),
                                                   _ptr(hist, torch.int32), _ptr(lens, torch.int32), cap, _ptr(acc),
                                                   _ptr(best), _ptr(com), _stream()), "verify_accept_commit")
        return argmax.view(S, B, w + 1), acc, best, com

    def verify_lmhead_keys(self, hidden: torch.Tensor, vocab_offset: int, keys: torch.Tensor | None = None):
        """Per-row (logit, global id) keys of this context's vocabulary shard, as sortable int64."""
        M = int(hidden.shape[0])
        if keys is None:
            keys = torch.empty(M, dtype=torch.int64, device=hidden.device)
        self._check(self._lib.verify_lmhead_keys(self._h, _ptr(hidden, torch.bfloat16), M, int(vocab_offset),
                                                 _ptr(keys, torch.int64), _stream()), "verify_lmhead_keys")
        return keys

    def accumulate_stats(self, acc_len, best_row, src, w: int, stats: torch.Tensor | None = None):
        """Adds one step to the ablation histograms ([w+1] | [B] | [5] | [5] int64)."""
        S, B = int(src.shape[0]), int(src.shape[1])
        if stats is None:
            stats = torch.zeros((w + 1) + B + 10, dtype=torch.int64, device=src.device)
        self._check(self._lib.spec_accumulate_stats(self._h, _ptr(acc_len, torch.int32), _ptr(best_row, torch.int32),
                                                    _ptr(src, torch.int32), S, B, w, _ptr(stats, torch.int64), _stream()),
                    "spec_accumulate_stats")
        return stats

    def quantize_rows_fp8(self, rows: torch.Tensor, out=None):
        """Per-row E4M3 quantisation of a bf16 matrix: ``(codes uint8 [n, d], scale float32 [n])``."""
        n = int(rows.shape[0])
        if out is None:
            out = (torch.empty((n, self.d), dtype=torch.uint8, device=rows.device),
                   torch.empty(n, dtype=torch.float32, device=rows.device))
        codes, scale = out
        self._check(self._lib.spec_quantize_rows_fp8(self._h, _ptr(rows, torch.bfloat16), n, _ptr(codes, torch.uint8),
                                                     _ptr(scale, torch.float32), _stream()), "spec_quantize_rows_fp8")
        return codes, scale

    def quantize_head_fp8(self):
        """Builds (and adopts) the 8-bit copy of the unembedding: ``(codes uint8 [V, d], scale float32 [V])``."""
        dev = self._keep[0].device
        wq = torch.empty((self.V, self.d), dtype=torch.uint8, device=dev)
        ws = torch.empty(self.V, dtype=torch.float32, device=dev)
        self._check(self._lib.spec_quantize_head_fp8(self._h, _ptr(wq), _ptr(ws), _stream()), "spec_quantize_head_fp8")
        self._keep_fp8 = (wq, ws)
        return wq, ws

    def set_head_fp8(self, wq: torch.Tensor, ws: torch.Tensor):
        self._check(self._lib.spec_set_head_fp8(self._h, _ptr(wq, torch.uint8), _ptr(ws, torch.float32)), "spec_set_head_fp8")
        self._keep_fp8 = (wq, ws)

    def verify_lmhead_argmax_fp8(self, hidden: torch.Tensor | None, scratch=None, out=None, with_max: bool = False):
        """``scratch = (codes uint8 [M, d], scale float32 [M])`` receives the quantised hidden states; with
        ``hidden=None`` it already holds them."""
        M = int(hidden.shape[0]) if hidden is not None else int(scratch[0].shape[0])
        dev = hidden.device if hidden is not None else scratch[0].device
        if scratch is None:
            scratch = (torch.empty((M, self.d), dtype=torch.uint8, device=dev), torch.empty(M, dtype=torch.float32, device=dev))
        if out is None:
            out = (torch.empty(M, dtype=torch.int32, device=dev),
                   torch.empty(M, dtype=torch.float32, device=dev) if with_max else None)
        am, mx = out
        self._check(self._lib.verify_lmhead_argmax_fp8(self._h, _ptr(hidden, torch.bfloat16), M, _ptr(scratch[0], torch.uint8),
                                                       _ptr(scratch[1], torch.float32), _ptr(am), _ptr(mx), _stream()),
                    "verify_lmhead_argmax_fp8")
        return am, mx

    def score_tokens(self, hidden: torch.Tensor, tokens: torch.Tensor, n_alt: int = 0, out=None, work: torch.Tensor | None = None):
        """Log probability of ``tokens[M]`` after ``hidden[M, d]``, entropy, and the ``n_alt`` likeliest tokens.

        Returns ``(logp[M], entropy[M], alt_ids[M, n_alt] or None, alt_logp[M, n_alt] or None)``; an alternative that does not
        exist (logits of NaN or -inf are none) has id -1 and -inf.
        """
        M = hidden.shape[0]
        _need(hidden.dim() == 2 and hidden.shape[1] == self.d and hidden.dtype == torch.bfloat16 and hidden.is_cuda and hidden.is_contiguous(),
              "score_tokens: hidden must be contiguous bfloat16 [M, d]")
        if out is None:
            logp = torch.empty_like(tokens, dtype=torch.float32)
            idx = tokens.new_empty((M, n_alt)) if n_alt > 0 else None
            out = (logp, torch.empty_like(logp), idx, None if idx is None else torch.empty_like(idx, dtype=torch.float32))
        else:
            _need(len(out) == 4, "score_tokens: out must be (logp, entropy, alt_ids, alt_logp)")
            for y, shape, dtype, name in zip(out[: 4 if n_alt else 2], ((M,), (M,), (M, n_alt), (M, n_alt)), (torch.float32, torch.float32, torch.int32, torch.float32),
                                             ("logp", "entropy", "alt_ids", "alt_logp")):
                _out(y, shape, dtype, f"score_tokens: {name}")
            if not n_alt:
                out = (out[0], out[1], None, None)
        if work is None:
            need = max(16, self._lib.spec_score_bytes(self._h, M, n_alt))
            work = hidden.new_empty(need, dtype=torch.uint8)
            scratch = work.data_ptr(), need
        else:
            scratch = _scratch(work, "score_tokens")
        ptr = lambda y: None if y is None else y.data_ptr()
        self._check(self._lib.score_tokens(self._h, hidden.data_ptr(), M, _i32(tokens, "tokens", (M,)), n_alt, ptr(out[0]), ptr(out[1]), ptr(out[2]),
                                           ptr(out[3]), *scratch, self._raw_stream()), "score_tokens")
        return out

    def rope_rows(self, rope: Rope, q: torch.Tensor, k: torch.Tensor | None, pos: torch.Tensor, out=None):
        """Rotates ``q[T, Hq, D]`` and ``k[T, Hk, D]`` (or ``[S, N, heads, D]``; ``k`` may be None) at ``pos`` [T] (or [S, N]).

        Returns contiguous ``(q_out, k_out)``, or writes to ``out``, whose tensors may be ``q`` and ``k`` themselves.
        """
        shape = q.shape
        _need(k is None or (k.shape[-1] == shape[-1] and k.shape[:-2] == shape[:-2]), "rope_rows: q and k must have the same tokens and head size")
        if out is None:
            out = (_new(q), None if k is None else _new(k))
        else:
            _need(len(out) == 2, "rope_rows: out must be (q_out, k_out)")
            for x, y, name in zip((q, k), out, ("q_out", "k_out")):
                if x is not None:
                    _out(y, x.shape, torch.bfloat16, f"rope_rows: {name}")
        qp, qt, qh = _rows(q, "q")
        kp, kt, kh = (None, 0, 0) if k is None else _rows(k, "k")
        self._check(self._lib.spec_rope_rows(self._h, rope._ref, qp, shape[-2], qt, qh, out[0].data_ptr(), kp, 0 if k is None else k.shape[-2],
                                             kt, kh, None if k is None else out[1].data_ptr(), shape[-1], _i32(pos, "pos", shape[:-2]), pos.numel(),
                                             self._raw_stream()), "spec_rope_rows")
        return out

    def cache_write(self, cache: KVCache, k: torch.Tensor, v: torch.Tensor, start: torch.Tensor, count: torch.Tensor | None = None,
                    nodes: torch.Tensor | None = None, rope: Rope | None = None):
        """Writes ``k``, ``v`` ``[S, N, heads, D]`` to positions ``start[s] + i``, ``i < count[s]`` (all N): node ``nodes[s, i]`` or ``i``."""
        _need(k.dim() == 4 and k.shape == v.shape, "cache_write: k and v must be [S, N, heads, head_dim]")
        S, N, heads, D = k.shape
        _need(heads == cache.heads and D == cache.head_dim and S == cache.sequences, "cache_write: k and v must have the cache's heads, head_dim and sequences")
        n = N if nodes is None else nodes.shape[1]
        self._check(self._lib.spec_cache_write(self._h, cache._ref, *_rows(k, "k"), *_rows(v, "v"), S, N, n, _i32(nodes, "nodes", (S, n)),
                                               _i32(start, "start", (S,)), _i32(count, "count", (S,)), None if rope is None else rope._ref,
                                               self._raw_stream()), "spec_cache_write")

    def cache_read(self, cache: KVCache, start: torch.Tensor, n: int, count: torch.Tensor | None = None, out=None):
        """Positions ``start[s] + i``, ``i < count[s]`` (``n``), as bfloat16 ``(k, v)`` ``[S, n, heads, D]``; zeros beyond."""
        S = cache.sequences
        if out is None:
            k = torch.empty((S, n, cache.heads, cache.head_dim), dtype=torch.bfloat16, device=cache.k.device)
            out = (k, torch.empty_like(k))
        else:
            _need(len(out) == 2, "cache_read: out must be (k, v)")
            for t, name in zip(out, "kv"):
                _out(t, (S, n, cache.heads, cache.head_dim), torch.bfloat16, f"cache_read: {name}")
        self._check(self._lib.spec_cache_read(self._h, cache._ref, S, n, _i32(start, "start", (S,)), _i32(count, "count", (S,)),
                                              out[0].data_ptr(), out[1].data_ptr(), self._raw_stream()), "spec_cache_read")
        return out

    def tree_mask(self, parent: torch.Tensor, n_nodes: torch.Tensor | None = None):
        """Mask words ``[S, N, ceil(N / 32)]`` and depths ``[S, N]`` (int32) of the forests ``parent[S, N]`` (-1 = root)."""
        S, N = int(parent.shape[0]), int(parent.shape[1])
        mask = torch.empty((S, N, (N + 31) // 32), dtype=torch.int32, device=parent.device)
        depth = torch.empty((S, N), dtype=torch.int32, device=parent.device)
        self._check(self._lib.spec_tree_mask(self._h, _i32(parent, "parent", (S, N)), S, N, _i32(n_nodes, "n_nodes", (S,)), mask.data_ptr(),
                                             depth.data_ptr(), self._raw_stream()), "spec_tree_mask")
        return mask, depth

    def tree_attention(self, cache: KVCache, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, mask: torch.Tensor, lens: torch.Tensor,
                       n_nodes: torch.Tensor | None = None, scale: float | None = None, with_lse: bool = False, out=None,
                       work: torch.Tensor | None = None):
        """Attention of the block ``q[S, N, Hq, D]``, ``k``, ``v`` ``[S, N, heads, D]`` over the cache and its own ancestors (``mask``).

        Returns ``(out[S, N, Hq, D] bfloat16, lse[S, N, Hq] float32 or None)``; ``scale`` defaults to ``D ** -0.5``.
        """
        S, N, Hq, D = q.shape
        _need(k.shape == v.shape and k.shape == (S, N, cache.heads, cache.head_dim) and D == cache.head_dim and S == cache.sequences,
              "tree_attention: q must be [S, N, Hq, head_dim], k and v [S, N, heads, head_dim] of the cache")
        if out is None:
            out = (_new(q), q.new_empty((S, N, Hq), dtype=torch.float32) if with_lse else None)
        else:
            _need(len(out) == 2, "tree_attention: out must be (out, lse or None)")
            _out(out[0], q.shape, torch.bfloat16, "tree_attention: out")
            if out[1] is not None:
                _out(out[1], q.shape[:3], torch.float32, "tree_attention: lse")
        if work is None:
            key = (S, N, Hq, cache.heads, D)
            need = self._work_bytes.get(key)
            if need is None:
                need = self._lib.spec_tree_attention_bytes(self._h, cache._ref, S, N, Hq)
                if need:  # (0: something else is refused, which is not a property of the sizes)
                    self._work_bytes[key] = need
            need = max(need, 16)
            work = q.new_empty(need, dtype=torch.uint8)
            scratch = work.data_ptr(), need
        else:
            scratch = _scratch(work, "tree_attention")
        self._check(self._lib.spec_tree_attention(self._h, cache._ref, *_rows(q, "q"), *_rows(k, "k"), *_rows(v, "v"), S, N, Hq,
                                                  _i32(mask, "mask", (S, N, (N + 31) // 32)), _i32(lens, "lens", (S,)),
                                                  _i32(n_nodes, "n_nodes", (S,)), D ** -0.5 if scale is None else scale,
                                                  out[0].data_ptr(), None if out[1] is None else out[1].data_ptr(), *scratch,
                                                  self._raw_stream()), "spec_tree_attention")
        return out

    def debug_logits(self, rows: torch.Tensor) -> torch.Tensor:
        m = int(rows.shape[0])
        out = torch.empty((m, self.V), dtype=torch.float32, device=rows.device)
        self._check(self._lib.spec_debug_logits(self._h, _ptr(rows, torch.bfloat16), m, _ptr(out), _stream()),
                    "spec_debug_logits")
        return out


def verify_lmhead_argmax_noalloc(unembed: torch.Tensor, hidden: torch.Tensor, out):
    """Context-free verification for callers that must not allocate device memory.

    ``out = (argmax int32 [M], max float32 [M] or None)`` must be preallocated by the caller: this
    wrapper allocates nothing either.  See ``verify_lmhead_argmax_noalloc`` in the header for the
    row limit and the rule that calls must not overlap on the GPU.
    """
    lib = load_library()
    am, mx = out
    V, d = int(unembed.shape[0]), int(unembed.shape[1])
    rc = lib.verify_lmhead_argmax_noalloc(_ptr(unembed, torch.bfloat16), V, d, _ptr(hidden, torch.bfloat16),
                                          int(hidden.shape[0]), _ptr(am, torch.int32), _ptr(mx), unembed.device.index or 0,
                                          _stream())
    if rc != 0:
        raise SpecError(f"verify_lmhead_argmax_noalloc failed ({rc}): {lib.spec_last_error(None).decode()}")
    return am, mx


def unpack_keys(keys: torch.Tensor, V_total: int, with_max: bool = False):
    """Token ids (and winning logits) from merged shard keys."""
    lib = load_library()
    M = int(keys.shape[0])
    am = torch.empty(M, dtype=torch.int32, device=keys.device)
    mx = torch.empty(M, dtype=torch.float32, device=keys.device) if with_max else None
    rc = lib.spec_unpack_keys(_ptr(keys, torch.int64), M, int(V_total), _ptr(am), _ptr(mx), _stream())
    if rc != 0:
        raise SpecError(f"spec_unpack_keys failed ({rc}): {lib.spec_last_error(None).decode()}")
    return am, mx
