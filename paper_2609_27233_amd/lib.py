"""Thin binding of ``libspanmerge.so`` (argument marshalling only): the
structures and the raw C entries through ctypes, the calls themselves through
the extension module ``_binding``.

Every function mirrors one C entry point of ``include/spanmerge.h`` and takes
torch tensors that already live on the GPU; the work itself runs in the HIP
kernels.  There is no CPU fallback: loading fails loudly when the library
has not been built.
"""
from __future__ import annotations

import ctypes as C
import importlib
import os
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libspanmerge.so")

SM_F32, SM_BF16, SM_E4M3 = 0, 1, 2
SM_OK, SM_EINVAL, SM_ERANGE, SM_ENOMEM, SM_EHIP = 0, 1, 2, 3, 4
ERR_EINVAL, ERR_ERANGE, ERR_ENOMEM = 1, 2, 4
MAX_REQUESTS = 1024
MAX_TOP = 64
ROPE_LAYOUTS = {"half": 0, "interleaved": 1}
ROPE_SCALINGS = {None: 0, "linear": 1, "bands": 2, "ramp": 3}
NORM_KINDS = {"rms": 0, "layer": 1}

_P, _I, _L, _F, _Z = C.c_void_p, C.c_int, C.c_int64, C.c_float, C.c_size_t

EXPORTED = ("sm_status_string", "sm_merge_workspace_bytes", "sm_merge_spans",
            "sm_merge_token_table", "sm_merge_spans_tabled",
            "sm_pack_spans", "sm_kv_rollback", "sm_kv_append",
            "sm_decode_workspace_bytes", "sm_decode_attention", "sm_decode_step", "sm_decode_merge_step",
            "sm_decode_step_noalloc_max_bytes", "sm_decode_step_noalloc", "sm_set_commit_wait_limit",
            "sm_decode_shared_workspace_bytes", "sm_decode_attention_shared",
            "sm_prefill_attention", "sm_rules_build_workspace_bytes", "sm_rules_build",
            "sm_rules_lookup", "sm_match_prompt_workspace_bytes", "sm_match_prompt",
            "sm_match_decode", "sm_gather_surrogates", "sm_span_dedupe_workspace_bytes", "sm_span_dedupe",
            "sm_kv_project_workspace_bytes", "sm_kv_project", "sm_kv_append_projected",
            "sm_kv_reserve", "sm_rotary", "sm_kv_write_rotary", "sm_kv_read", "sm_block_norm",
            "sm_token_logprobs_workspace_bytes", "sm_token_logprobs", "sm_sample_workspace_bytes", "sm_sample_tokens")


class MergeParams(C.Structure):
    _fields_ = [("d", _I), ("h", _I), ("ln_eps", _F), ("Q", _P), ("W_kv", _P),
                ("b_kv", _P), ("g_kv", _P), ("beta_kv", _P), ("W_o", _P),
                ("b_o", _P), ("g_o", _P), ("beta_o", _P)]


class PagedCacheDesc(C.Structure):
    _fields_ = [("dtype", _I), ("num_kv_heads", _I), ("head_dim", _I),
                ("block_size", _I), ("num_blocks", _I), ("max_seqs", _I),
                ("max_blocks_per_seq", _I), ("k_pool", _P), ("v_pool", _P),
                ("block_table", _P), ("lengths", _P), ("free_stack", _P),
                ("free_top", _P), ("err", _P)]


class RuleTableDesc(C.Structure):
    _fields_ = [("capacity", _I), ("keys", _P), ("ids", _P), ("err", _P)]


class KVProjParams(C.Structure):
    _fields_ = [("d", _I), ("W_k", _P), ("W_v", _P), ("rope_theta", _F), ("rms_eps", _F)]


class RopeParams(C.Structure):
    _fields_ = [("rot_dim", _I), ("layout", _I), ("scaling", _I), ("theta", _F), ("attn_scale", _F), ("factor", _F),
                ("low", _F), ("high", _F), ("context", _F)]


class NormParams(C.Structure):
    _fields_ = [("kind", _I), ("eps", _F), ("gain", _P), ("bias", _P)]


class SpanMergeError(RuntimeError):
    pass


_lib = None
_fast = None      # the extension module, once load() has run


def load(path: str = LIB_PATH):
    """Load the HIP library (raises if it is missing: no fallback)."""
    global _lib, _fast
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise SpanMergeError(
            f"{path} is missing; build it with `python -m paper_2609_27233_amd.build`")
    L = C.CDLL(path)
    L.sm_status_string.argtypes = [_I]
    L.sm_status_string.restype = C.c_char_p
    L.sm_merge_workspace_bytes.argtypes = [_I, _I, _I, _I]
    L.sm_merge_workspace_bytes.restype = _Z
    L.sm_merge_spans.argtypes = [_P, _L, _P, _I, _P, _I, C.POINTER(MergeParams), _I,
                                 _P, _P, _Z, _P, _P]
    L.sm_merge_spans.restype = _I
    L.sm_merge_token_table.argtypes = [_P, _L, C.POINTER(MergeParams), _I, _P, _P, _P]
    L.sm_merge_token_table.restype = _I
    L.sm_merge_spans_tabled.argtypes = [_P, _L, _P, _I, _P, _I, C.POINTER(MergeParams), _I,
                                        _P, _P, _Z, _P, _P]
    L.sm_merge_spans_tabled.restype = _I
    L.sm_pack_spans.argtypes = [_I, _P, _I, _I, _P, _P, _P, _P, _P, _P, _P, _P, _L,
                                _P, _I, _I, _P, _P, _P]
    L.sm_pack_spans.restype = _I
    L.sm_kv_rollback.argtypes = [C.POINTER(PagedCacheDesc), _P, _P, _I, _P]
    L.sm_kv_rollback.restype = _I
    L.sm_kv_append.argtypes = [C.POINTER(PagedCacheDesc), _P, _P, _I, _I, _P, _P, _P]
    L.sm_kv_append.restype = _I
    L.sm_decode_workspace_bytes.argtypes = [_I, _I, _I, _I]
    L.sm_decode_workspace_bytes.restype = _Z
    L.sm_decode_attention.argtypes = [C.POINTER(PagedCacheDesc), _P, _I, _P, _I, _F,
                                      _I, _P, _P, _Z, _P]
    L.sm_decode_attention.restype = _I
    L.sm_decode_shared_workspace_bytes.argtypes = [_I, _I, _I, _I, _I]
    L.sm_decode_shared_workspace_bytes.restype = _Z
    L.sm_decode_attention_shared.argtypes = [C.POINTER(PagedCacheDesc), _P, _I, _P, _P, _I, _P, _I, _F, _I, _I, _P, _P, _Z, _P]
    L.sm_decode_attention_shared.restype = _I
    L.sm_decode_step.argtypes = [C.POINTER(PagedCacheDesc), _P, _I, _P, _P, _P, _I, _F,
                                 _I, _P, _P, _Z, _P]
    L.sm_decode_step.restype = _I
    L.sm_decode_merge_step.argtypes = [C.POINTER(PagedCacheDesc), _P, _P, _I, _P, _P, _P, _I, _F,
                                       _I, _P, _P, _Z, _P]
    L.sm_decode_merge_step.restype = _I
    L.sm_decode_step_noalloc_max_bytes.argtypes = []
    L.sm_decode_step_noalloc_max_bytes.restype = _Z
    L.sm_decode_step_noalloc.argtypes = [C.POINTER(PagedCacheDesc), _P, _I, _P, _P, _P, _I, _F, _I, _P, _P]
    L.sm_decode_step_noalloc.restype = _I
    L.sm_set_commit_wait_limit.argtypes = [_I]
    L.sm_set_commit_wait_limit.restype = None
    L.sm_prefill_attention.argtypes = [C.POINTER(PagedCacheDesc), _P, _I, _P, _I, _P, _I, _F, _I, _P, _P]
    L.sm_prefill_attention.restype = _I
    L.sm_rules_build_workspace_bytes.argtypes = [_I]
    L.sm_rules_build_workspace_bytes.restype = _Z
    L.sm_rules_build.argtypes = [_P, _I, C.POINTER(RuleTableDesc), _P, _Z, _P]
    L.sm_rules_build.restype = _I
    L.sm_rules_lookup.argtypes = [C.POINTER(RuleTableDesc), _P, _I, _P, _P]
    L.sm_rules_lookup.restype = _I
    L.sm_match_prompt_workspace_bytes.argtypes = [_I, _I]
    L.sm_match_prompt_workspace_bytes.restype = _Z
    L.sm_match_prompt.argtypes = [C.POINTER(RuleTableDesc), _P, _P, _I, _I, _P, _P, _P, _P, _P, _Z, _P]
    L.sm_match_prompt.restype = _I
    L.sm_match_decode.argtypes = [C.POINTER(RuleTableDesc), _P, _I, _P, _P, _I, _P, _P,
                                  C.POINTER(PagedCacheDesc), _P]
    L.sm_match_decode.restype = _I
    L.sm_gather_surrogates.argtypes = [_P, _L, _P, _L, _P, _P, _I, _I, _I, _P, _P, _P]
    L.sm_gather_surrogates.restype = _I
    L.sm_span_dedupe_workspace_bytes.argtypes = [_I, _I]
    L.sm_span_dedupe_workspace_bytes.restype = _Z
    L.sm_span_dedupe.argtypes = [_P, _P, _P, _I, _I, _P, _I, _P, _P, _P, _P, _P, _P, _Z, _P, _P]
    L.sm_span_dedupe.restype = _I
    L.sm_kv_project_workspace_bytes.argtypes = [_I, _I, _I, _I]
    L.sm_kv_project_workspace_bytes.restype = _Z
    L.sm_kv_project.argtypes = [C.POINTER(PagedCacheDesc), _P, _I, _P, C.POINTER(KVProjParams), _P, _P, _P, _Z, _P]
    L.sm_kv_project.restype = _I
    L.sm_kv_append_projected.argtypes = [C.POINTER(PagedCacheDesc), _P, _I, _P, C.POINTER(KVProjParams), _P, _Z, _P]
    L.sm_kv_append_projected.restype = _I
    L.sm_kv_reserve.argtypes = [C.POINTER(PagedCacheDesc), _P, _P, _P, _I, _I, _P, _P, _P, _P]
    L.sm_kv_reserve.restype = _I
    L.sm_rotary.argtypes = [_P, _L, _P, _I, _I, _I, C.POINTER(RopeParams), _I, _I, _P, _L, _P]
    L.sm_rotary.restype = _I
    L.sm_kv_write_rotary.argtypes = [C.POINTER(PagedCacheDesc), _P, _P, _I, _P, _L, _I, _P, _L, _P, _L,
                                     C.POINTER(RopeParams), _P, _L, _P]
    L.sm_kv_write_rotary.restype = _I
    L.sm_kv_read.argtypes = [C.POINTER(PagedCacheDesc), _P, _P, _P, _I, _I, _P, _L, _P, _L, _P]
    L.sm_kv_read.restype = _I
    L.sm_block_norm.argtypes = [_P, _L, _P, _L, _I, _I, C.POINTER(NormParams), _P, _L, _F, C.POINTER(NormParams), _I,
                                _P, _L, _P, _L, _P]
    L.sm_block_norm.restype = _I
    L.sm_token_logprobs_workspace_bytes.argtypes = [_I, _I, _I]
    L.sm_token_logprobs_workspace_bytes.restype = _Z
    L.sm_token_logprobs.argtypes = [_P, _L, _I, _I, _I, _F, _P, _P, _P, _I, _P, _P, _P, _Z, _P, _P]
    L.sm_token_logprobs.restype = _I
    L.sm_sample_workspace_bytes.argtypes = [_I, _I]
    L.sm_sample_workspace_bytes.restype = _Z
    L.sm_sample_tokens.argtypes = [_P, _L, _I, _I, _I, _P, _P, _P, _P, _P, _P, _P, _P, _Z, _P, _P]
    L.sm_sample_tokens.restype = _I
    try:
        fast = importlib.import_module("._binding", __package__)
    except ImportError as e:
        raise SpanMergeError(f"the extension module is missing ({e}); build it with "
                             "`python -m paper_2609_27233_amd.build`") from e
    fast.setup((SpanMergeError, C.ArgumentError, PagedCacheDesc, RuleTableDesc, _I, _L, _F, _Z, _P))
    fast.torch_types(torch.int32, torch.float32, torch.bfloat16, torch.Tensor, torch.nn.Parameter,
                     getattr(torch.Tensor, "__dlpack_c_exchange_api__", None))
    fast.open(path)
    _fast = fast
    _lib = L
    return L


def _calls():
    """The extension module's entries (loads the library on first use)."""
    if _fast is None:
        load()
    return _fast


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_cuda:
        raise SpanMergeError("expected a GPU tensor")
    if not t.is_contiguous():
        raise SpanMergeError("expected a contiguous tensor")
    return t.data_ptr()


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _stream(stream=None):
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


def _check(st: int, what: str):
    if st != SM_OK:
        msg = load().sm_status_string(st).decode()
        raise SpanMergeError(f"{what}: {msg} (status {st})")


def dtype_code(dt: torch.dtype) -> int:
    if dt == torch.bfloat16:
        return SM_BF16
    if dt == torch.float32:
        return SM_F32
    raise SpanMergeError(f"unsupported dtype {dt}")


# --------------------------------------------------------------------------
# merge_spans

def merge_workspace_bytes(total_rows: int, num_spans: int, d: int, dtype: torch.dtype) -> int:
    return load().sm_merge_workspace_bytes(total_rows, num_spans, d, dtype_code(dtype))


def merge_spans(emb, row_idx, span_offsets, params: dict, h: int, out, ws, err,
                ln_eps: float = 1e-5, total_rows: Optional[int] = None, stream=None):
    """z_s = M_phi(emb[row_idx[span s]]) for every span; writes ``out``."""
    S = span_offsets.numel() - 1
    R = row_idx.numel() if total_rows is None else total_rows
    p = _merge_params(emb.shape[1], h, params, ln_eps)
    st = _calls().sm_merge_spans(emb, emb.shape[0], row_idx, R, span_offsets, S, p, dtype_code(emb.dtype), out, ws,
                                 ws.nbytes, err, _stream(stream))
    _check(st, "sm_merge_spans")


def _merge_params(d: int, h: int, params: dict, ln_eps: float):
    return _calls().merge_params(d, h, ln_eps, *(params[k] for k in
                                 ("Q", "W_kv", "b_kv", "g_kv", "beta_kv", "W_o", "b_o", "g_o", "beta_o")))


def merge_token_table(emb, params: dict, h: int, table, err, ln_eps: float = 1e-5, stream=None):
    """table[v] = GELU(Linear_kv(emb[v])) for every row of ``emb``."""
    p = _merge_params(emb.shape[1], h, params, ln_eps)
    st = _calls().sm_merge_token_table(emb, emb.shape[0], p, dtype_code(emb.dtype), table, err, _stream(stream))
    _check(st, "sm_merge_token_table")


def merge_spans_tabled(table, row_idx, span_offsets, params: dict, h: int, out, ws, err,
                       ln_eps: float = 1e-5, total_rows: Optional[int] = None, stream=None):
    """The surrogates of merge_spans, the first stage read from ``table``
    (rows = token ids)."""
    S = span_offsets.numel() - 1
    R = row_idx.numel() if total_rows is None else total_rows
    p = _merge_params(table.shape[1], h, params, ln_eps)
    st = _calls().sm_merge_spans_tabled(table, table.shape[0], row_idx, R, span_offsets, S, p,
                                        dtype_code(table.dtype), out, ws, ws.nbytes, err, _stream(stream))
    _check(st, "sm_merge_spans_tabled")


# --------------------------------------------------------------------------
# pack_spans

def pack_spans(seq_offsets, span_start, span_len, seq_span_offsets, pi,
               packed_offsets, packed_src, err, total_tokens: int,
               token_ids=None, emb=None, surrogates=None, packed=None, stream=None):
    B = seq_offsets.numel() - 1
    S = span_start.numel()
    d = emb.shape[1] if emb is not None else 0
    dt = dtype_code(emb.dtype) if emb is not None else SM_BF16
    st = _calls().sm_pack_spans(B, seq_offsets, total_tokens, S, span_start, span_len, seq_span_offsets, pi,
                                packed_offsets, packed_src, token_ids, emb, emb.shape[0] if emb is not None else 0,
                                surrogates, d, dt, packed, err, _stream(stream))
    _check(st, "sm_pack_spans")


# --------------------------------------------------------------------------
# paged cache

class PagedCache:
    """Device buffers of one paged KV cache (allocated with torch) and the
    descriptor the C calls take.  Pools: K [NB, Hkv, bs, D], V [NB, Hkv, D, bs].
    ``tables``: another cache of the same sizes, a layer's neighbour, whose
    block table, lengths, free stack and error word this one shares; only the
    pools are its own.  kv_reserve (or kv_rollback) moves the shared lengths
    once for all layers and kv_write_rotary fills each layer's pages; the calls
    that append to one cache (kv_append, decode_step and their like) would
    move them once a layer.

    dtype torch.float8_e4m3fn: pages in 8 bits, with an exponent byte for each
    entry and head (k_exp, v_exp [NB, Hkv, bs]: feature = value * 2^(byte - 127)).
    kv_write_rotary fills them; decode_attention, decode_attention_shared,
    prefill_attention and kv_read read them; rows, queries and results (row_dtype) are bf16."""

    def __init__(self, *, dtype: torch.dtype, num_kv_heads: int, head_dim: int,
                 block_size: int, num_blocks: int, max_seqs: int,
                 max_blocks_per_seq: int, device="cuda", free_order=None,
                 tables: Optional["PagedCache"] = None):
        self.dtype = dtype
        self.H, self.D, self.bs = num_kv_heads, head_dim, block_size
        self.num_blocks, self.max_seqs, self.max_blocks = num_blocks, max_seqs, max_blocks_per_seq
        self.row_dtype, self.k_exp, self.v_exp = dtype, None, None
        shapes = (num_blocks, num_kv_heads, block_size, head_dim), (num_blocks, num_kv_heads, head_dim, block_size)
        if dtype == torch.float8_e4m3fn:
            self.row_dtype = torch.bfloat16
            (self.k_pool, self.k_exp), (self.v_pool, self.v_exp) = (self._eight_bits(s, block_size, device) for s in shapes)
        else:
            self.k_pool, self.v_pool = (torch.zeros(s, dtype=dtype, device=device) for s in shapes)
        if tables is not None:
            if ((tables.bs, tables.num_blocks, tables.max_seqs, tables.max_blocks) !=
                    (block_size, num_blocks, max_seqs, max_blocks_per_seq) or free_order is not None
                    or tables.k_pool.device != self.k_pool.device):
                raise SpanMergeError("caches that share their tables have the same blocks, sequences and device")
            self.block_table, self.lengths = tables.block_table, tables.lengths
            self.free_stack, self.free_top, self.err = tables.free_stack, tables.free_top, tables.err
        else:
            self.block_table = torch.full((max_seqs, max_blocks_per_seq), -1, dtype=torch.int32, device=device)
            self.lengths = torch.zeros(max_seqs, dtype=torch.int32, device=device)
            order = (torch.arange(num_blocks, dtype=torch.int32) if free_order is None
                     else torch.as_tensor(free_order, dtype=torch.int32))
            # the top of the stack (last element) is handed out first
            self.free_stack = order.flip(0).contiguous().to(device)
            self.free_top = torch.tensor([num_blocks], dtype=torch.int32, device=device)
            self.err = torch.zeros(1, dtype=torch.int32, device=device)
        self.desc = PagedCacheDesc(SM_E4M3 if self.k_exp is not None else dtype_code(dtype), num_kv_heads, head_dim, block_size,
                                   num_blocks, max_seqs, max_blocks_per_seq,
                                   _ptr(self.k_pool), _ptr(self.v_pool), _ptr(self.block_table),
                                   _ptr(self.lengths), _ptr(self.free_stack), _ptr(self.free_top),
                                   _ptr(self.err))

    @staticmethod
    def _eight_bits(shape, bs: int, device):
        """A pool of e4m3 values and, behind them in the same memory, its exponent bytes."""
        values = shape[0] * shape[1] * shape[2] * shape[3]
        buf = torch.zeros(values + shape[0] * shape[1] * bs, dtype=torch.uint8, device=device)
        return buf[:values].view(torch.float8_e4m3fn).view(shape), buf[values:].view(shape[0], shape[1], bs)

    def error_bits(self) -> int:
        return int(self.err.item())

    def clear_error(self):
        self.err.zero_()


def kv_rollback(cache: PagedCache, seq_ids, k, stream=None):
    st = _calls().sm_kv_rollback(cache.desc, seq_ids, k, seq_ids.numel(), _stream(stream))
    _check(st, "sm_kv_rollback")


def kv_append(cache: PagedCache, seq_ids, row_offsets, K, V, total_rows: Optional[int] = None,
              stream=None):
    R = K.shape[0] if total_rows is None else total_rows
    st = _calls().sm_kv_append(cache.desc, seq_ids, row_offsets, seq_ids.numel(), R, K, V, _stream(stream))
    _check(st, "sm_kv_append")


def decode_workspace_bytes(n: int, num_q_heads: int, head_dim: int, max_len: int) -> int:
    return load().sm_decode_workspace_bytes(n, num_q_heads, head_dim, max_len)


def _row_types(cache: PagedCache, q, out):
    """Queries and results of 8-bit pages are bf16 (other pages': their own type)."""
    if cache.k_exp is not None and not q.dtype == out.dtype == cache.row_dtype:
        raise SpanMergeError(f"q, out: expected {cache.row_dtype}, got {q.dtype} and {out.dtype}")


def decode_attention(cache: PagedCache, seq_ids, q, out, ws, max_len: int,
                     scale: Optional[float] = None, stream=None):
    n, Hq, D = q.shape
    _row_types(cache, q, out)
    sc = D ** -0.5 if scale is None else scale
    st = _calls().sm_decode_attention(cache.desc, seq_ids, n, q, Hq, sc, max_len, out, ws, ws.nbytes, _stream(stream))
    _check(st, "sm_decode_attention")


def decode_shared_workspace_bytes(n: int, num_q_heads: int, head_dim: int, max_len: int, max_prefix: int) -> int:
    return load().sm_decode_shared_workspace_bytes(n, num_q_heads, head_dim, max_len, max_prefix)


def decode_attention_shared(cache: PagedCache, seq_ids, prefix_ids, group_offsets, q, out, ws, max_len: int, max_prefix: int,
                            scale: Optional[float] = None, stream=None):
    """decode_attention of requests behind shared entries: the requests
    group_offsets[p] .. group_offsets[p + 1] - 1 attend over the entries of
    sequence prefix_ids[p] (-1: none), then over their own.  q, out [n, Hq, D]
    bf16; max_len and max_prefix bound the sequences' and the prefixes' lengths.
    For single tokens: a prompt's rows attend to a prefix through a sequence
    that holds a copy of its entries (prefill_attention sees one sequence)."""
    b = _calls()
    n, Hq, D = _shape(q, 3, "q")
    for t, name in ((q, "q"), (out, "out")):
        b.row_stride(t, torch.bfloat16, name, n, Hq, cache.D)
    groups = prefix_ids.numel()
    b.need(seq_ids, n, "seq_ids")
    b.need(group_offsets, groups + 1, "group_offsets")
    handle, dev = _here(stream)
    _cache_here(cache, dev)
    sc = D ** -0.5 if scale is None else scale
    st = b.sm_decode_attention_shared(cache.desc, seq_ids, n, prefix_ids, group_offsets, groups, q, Hq, sc, max_len, max_prefix,
                                      out, ws, ws.nbytes, handle, dev)
    _check(st, "sm_decode_attention_shared")


def decode_step(cache: PagedCache, seq_ids, K, V, q, out, ws, max_len: int,
                scale: Optional[float] = None, stream=None):
    """Append one K/V row per sequence and attend, in one launch: the same
    as kv_append(cache, seq_ids, arange(n + 1), K, V) then decode_attention."""
    n, Hq, D = q.shape
    sc = D ** -0.5 if scale is None else scale
    st = _calls().sm_decode_step(cache.desc, seq_ids, n, K, V, q, Hq, sc, max_len, out, ws, ws.nbytes,
                                 _stream(stream))
    _check(st, "sm_decode_step")


def decode_merge_step(cache: PagedCache, seq_ids, crop, K, V, q, out, ws, max_len: int,
                      scale: Optional[float] = None, stream=None):
    """The decode step at which spans complete: drop crop[i] cached entries
    of each request, append its row and attend, in one launch (the same as
    kv_rollback(cache, seq_ids, crop) then decode_step, made whole or not at
    all)."""
    n, Hq, D = q.shape
    sc = D ** -0.5 if scale is None else scale
    st = _calls().sm_decode_merge_step(cache.desc, seq_ids, crop, n, K, V, q, Hq, sc, max_len, out, ws, ws.nbytes,
                                       _stream(stream))
    _check(st, "sm_decode_merge_step")


def decode_step_noalloc(cache: PagedCache, seq_ids, K, V, q, out, max_len: int,
                        scale: Optional[float] = None, stream=None):
    """decode_step with the library's own per-device scratch array as its
    workspace (no allocation in the call; calls on one device must not
    overlap)."""
    n, Hq, D = q.shape
    sc = D ** -0.5 if scale is None else scale
    st = _calls().sm_decode_step_noalloc(cache.desc, seq_ids, n, K, V, q, Hq, sc, max_len, out, _stream(stream))
    _check(st, "sm_decode_step_noalloc")


def prefill_attention(cache: PagedCache, seq_ids, q_offsets, q, out, max_rows: int,
                      scale: Optional[float] = None, stream=None):
    """Causal attention of each request's last m_i cached positions:
    q, out [rows, Hq, D] bf16; q_offsets [n + 1] int32 row ranges."""
    rows, Hq, D = q.shape
    _row_types(cache, q, out)
    sc = D ** -0.5 if scale is None else scale
    st = _calls().sm_prefill_attention(cache.desc, seq_ids, seq_ids.numel(), q_offsets, rows, q, Hq, sc, max_rows,
                                       out, _stream(stream))
    _check(st, "sm_prefill_attention")


# --------------------------------------------------------------------------
# merge rules

class RuleTable:
    """Device buffers of the rule hash table (allocated with torch) and its
    descriptor.  capacity: a power of two >= 4/3 x the number of rules."""

    def __init__(self, capacity: int, device="cuda"):
        self.capacity = capacity
        self.keys = torch.full((capacity, 4), -1, dtype=torch.int32, device=device)
        self.ids = torch.full((capacity,), -1, dtype=torch.int32, device=device)
        self.err = torch.zeros(1, dtype=torch.int32, device=device)
        self.desc = RuleTableDesc(capacity, _ptr(self.keys), _ptr(self.ids), _ptr(self.err))

    @staticmethod
    def capacity_for(count: int) -> int:
        c = 16
        while 3 * c < 4 * count:
            c *= 2
        return c

    def error_bits(self) -> int:
        return int(self.err.item())

    def clear_error(self):
        self.err.zero_()


def rules_build(table: RuleTable, rules, ws=None, stream=None):
    """rules: [count, 4] int32 on the GPU (n >= 2 ids, then -1)."""
    need = load().sm_rules_build_workspace_bytes(table.capacity)
    if ws is None:
        ws = torch.empty(need, dtype=torch.uint8, device=rules.device)
    st = _calls().sm_rules_build(rules, rules.shape[0], table.desc, ws, ws.nbytes, _stream(stream))
    _check(st, "sm_rules_build")


def rules_lookup(table: RuleTable, grams, ids, stream=None):
    st = _calls().sm_rules_lookup(table.desc, grams, grams.shape[0], ids, _stream(stream))
    _check(st, "sm_rules_lookup")


def match_prompt_workspace_bytes(B: int, total_tokens: int) -> int:
    return load().sm_match_prompt_workspace_bytes(B, total_tokens)


def match_prompt(table: RuleTable, token_ids, seq_offsets, span_start, span_len, span_rule,
                 seq_span_offsets, ws, stream=None):
    B = seq_offsets.numel() - 1
    st = _calls().sm_match_prompt(table.desc, token_ids, seq_offsets, B, token_ids.numel(), span_start, span_len,
                                  span_rule, seq_span_offsets, ws, ws.nbytes, _stream(stream))
    _check(st, "sm_match_prompt")


def match_decode(table: RuleTable, state, seq_ids, new_tokens, k_out, rule_out,
                 cache: Optional[PagedCache] = None, stream=None):
    """state [max_seqs, 4] int32 (zeroed when a sequence starts generating)."""
    st = _calls().sm_match_decode(table.desc, state, state.shape[0], seq_ids, new_tokens, seq_ids.numel(), k_out,
                                  rule_out, None if cache is None else cache.desc, _stream(stream))
    _check(st, "sm_match_decode")


# --------------------------------------------------------------------------
# surrogate lookup and span dedupe

def gather_surrogates(lut, rule_ids, out, err, emb=None, token_ids=None, stream=None):
    """out[i] = lut[rule_ids[i]] if rule_ids[i] >= 0 else emb[token_ids[i]]."""
    n, d = out.shape
    st = _calls().sm_gather_surrogates(emb, 0 if emb is None else emb.shape[0], lut, lut.shape[0], token_ids,
                                       rule_ids, n, d, dtype_code(out.dtype), out, err, _stream(stream))
    _check(st, "sm_gather_surrogates")


def span_dedupe(span_rule, span_start, span_len, num_rules, token_ids, uniq_span, span_slot, uniq_row_idx,
                uniq_span_offsets, num_uniq, err, ws=None, stream=None):
    S = span_rule.numel()
    need = load().sm_span_dedupe_workspace_bytes(S, num_rules)
    if ws is None:
        ws = torch.empty(need, dtype=torch.uint8, device=span_rule.device)
    st = _calls().sm_span_dedupe(span_rule, span_start, span_len, S, num_rules, token_ids, token_ids.numel(),
                                 uniq_span, span_slot, uniq_row_idx, uniq_span_offsets, num_uniq, ws, ws.nbytes, err,
                                 _stream(stream))
    _check(st, "sm_span_dedupe")


# --------------------------------------------------------------------------
# K/V state of an input row at its compressed position

def _proj_params(W_k, W_v, rope_theta, rms_eps):
    return _calls().kv_proj_params(W_k.shape[1], W_k, W_v, rope_theta, rms_eps)


def kv_project_workspace_bytes(n: int, d: int, num_kv_heads: int, head_dim: int) -> int:
    return load().sm_kv_project_workspace_bytes(n, d, num_kv_heads, head_dim)


def kv_project(cache: PagedCache, seq_ids, x, W_k, W_v, K, V, ws=None, rope_theta=500000.0, rms_eps=1e-5,
               stream=None):
    """K, V [n, Hkv, D] bf16 of the rows x [n, d] at positions lengths[seq_ids]."""
    n = seq_ids.numel()
    if ws is None:
        ws = torch.empty(kv_project_workspace_bytes(n, x.shape[1], cache.H, cache.D), dtype=torch.uint8,
                         device=x.device)
    p = _proj_params(W_k, W_v, rope_theta, rms_eps)
    st = _calls().sm_kv_project(cache.desc, seq_ids, n, x, p, K, V, ws, ws.nbytes, _stream(stream))
    _check(st, "sm_kv_project")


def kv_append_projected(cache: PagedCache, seq_ids, x, W_k, W_v, ws=None, rope_theta=500000.0, rms_eps=1e-5,
                        stream=None):
    n = seq_ids.numel()
    if ws is None:
        ws = torch.empty(kv_project_workspace_bytes(n, x.shape[1], cache.H, cache.D), dtype=torch.uint8,
                         device=x.device)
    p = _proj_params(W_k, W_v, rope_theta, rms_eps)
    st = _calls().sm_kv_append_projected(cache.desc, seq_ids, n, x, p, ws, ws.nbytes, _stream(stream))
    _check(st, "sm_kv_append_projected")


# --------------------------------------------------------------------------
# rows of a backbone's layers: reserved, normed, turned, written, scored
#
# These calls look at their tensors before anything is enqueued: a wrong
# type, size or device raises SpanMergeError.

def _here(stream):
    """(handle of the stream, index of the current device, which its tensors have to be on as well)"""
    dev = _device()
    if stream is None:
        return (_raw_stream(dev) if _raw_stream is not None else _stream()), dev
    if stream.device_index != dev:
        raise SpanMergeError(f"expected a stream of the current device cuda:{dev}")
    return stream.cuda_stream, dev


def _cache_here(cache: PagedCache, dev: int):
    if cache.k_pool.get_device() != dev:
        raise SpanMergeError(f"expected a cache on the current device cuda:{dev}")


def _shape(t, dims: int, name: str):
    s = t.shape
    if len(s) != dims:
        raise SpanMergeError(f"{name}: expected {dims} dimensions, got {len(s)}")
    return s


def _columns(t, rows: int, name: str) -> int:
    """k of a [rows, k] tensor ([rows]: 1), which may have more rows."""
    s = t.shape
    if len(s) not in (1, 2) or s[0] < rows:
        raise SpanMergeError(f"{name}: expected {rows} rows of alternatives, got {tuple(s)}")
    return s[1] if len(s) == 2 else 1


def _rows(t):
    """Rows with a stride, which row_stride has looked at, for a call."""
    return None if t is None else (t,)


def kv_reserve(cache: PagedCache, seq_ids, rows, row_offsets, pos, slots, crop=None, stream=None):
    """Drop crop[i] entries of each listed sequence, then take room for rows[i]
    more: block tables and lengths, and for each row its position and slot.
    pos and slots (their size is the room for rows) get 0 and -1 past the last."""
    b = _calls()
    n, most, need = seq_ids.numel(), pos.numel(), b.need
    need(rows, n, "rows")
    need(row_offsets, n + 1, "row_offsets")
    need(slots, most, "slots")
    if crop is not None:
        need(crop, n, "crop")
    handle, dev = _here(stream)
    _cache_here(cache, dev)
    st = b.sm_kv_reserve(cache.desc, seq_ids, crop, rows, n, most, row_offsets, pos, slots, handle, dev)
    _check(st, "sm_kv_reserve")


def rope_params(rot_dim: int, theta: float = 500000.0, layout: str = "half", scaling: Optional[str] = None,
                factor: float = 1.0, low: float = 1.0, high: float = 4.0, context: float = 8192,
                attn_scale: float = 1.0) -> bytes:
    """A rotation for rotary and kv_write_rotary; layout "half" or
    "interleaved", scaling None, "linear", "bands" or "ramp"."""
    if layout not in ROPE_LAYOUTS or scaling not in ROPE_SCALINGS:
        raise SpanMergeError(f"unknown rotary layout or scaling: {layout!r}, {scaling!r}")
    return bytes(RopeParams(rot_dim, ROPE_LAYOUTS[layout], ROPE_SCALINGS[scaling], theta, attn_scale, factor, low, high,
                            context))


def rotary(x, pos, rope: bytes, out, transpose: bool = False, stream=None):
    """out[r, h] = x[r, h] turned by pos[r]; x, out [rows, heads, D], each row
    contiguous; out may be x.  transpose: the gradient of that with respect to x."""
    b = _calls()
    (rows, heads, D), dt = _shape(x, 3, "x"), x.dtype
    sx, so = b.row_stride(x, dt, "x", rows, heads, D), b.row_stride(out, dt, "out", rows, heads, D)
    b.need(pos, rows, "pos")
    handle, dev = _here(stream)
    st = b.sm_rotary((x,), sx, pos, rows, heads, D, rope, int(transpose), dtype_code(dt), (out,), so, handle, dev)
    _check(st, "sm_rotary")


def kv_write_rotary(cache: PagedCache, pos, slots, q, k, v, rope: bytes, q_out, stream=None):
    """q_out = q turned by pos; K (turned) and V rows into the slots of the
    cache's pages (-1: not written).  q, q_out [rows, Hq, D] or both None; k, v
    [rows, Hkv, D]; each row contiguous, so the three may be views of one buffer."""
    b = _calls()
    row_stride, dt, H, D = b.row_stride, cache.row_dtype, cache.H, cache.D
    rows = _shape(k, 3, "k")[0]
    sk, sv = row_stride(k, dt, "k", rows, H, D), row_stride(v, dt, "v", rows, H, D)
    b.need(pos, rows, "pos")
    b.need(slots, rows, "slots")
    hq = sq = so = 0
    if (q is None) != (q_out is None):
        raise SpanMergeError("q and q_out go together")
    if q is not None:
        hq = _shape(q, 3, "q")[1]
        sq, so = row_stride(q, dt, "q", rows, hq, D), row_stride(q_out, dt, "q_out", rows, hq, D)
    handle, dev = _here(stream)
    _cache_here(cache, dev)
    st = b.sm_kv_write_rotary(cache.desc, pos, slots, rows, _rows(q), sq, hq, (k,), sk, (v,), sv, rope, _rows(q_out), so,
                              handle, dev)
    _check(st, "sm_kv_write_rotary")


def kv_read(cache: PagedCache, seq_ids, row_offsets, K, V, start=None, stream=None):
    """Entries start[i], start[i] + 1, ... (None: from 0) of each listed sequence
    as rows row_offsets[i] .. row_offsets[i + 1] - 1 of K and V [rows, Hkv, D]
    (the cache's row_dtype; each row contiguous; either may be None)."""
    b = _calls()
    n, out = seq_ids.numel(), K if K is not None else V
    if out is None:
        raise SpanMergeError("kv_read: neither K nor V")
    rows = _shape(out, 3, "K" if K is not None else "V")[0]
    sk = 0 if K is None else b.row_stride(K, cache.row_dtype, "K", rows, cache.H, cache.D)
    sv = 0 if V is None else b.row_stride(V, cache.row_dtype, "V", rows, cache.H, cache.D)
    b.need(row_offsets, n + 1, "row_offsets")
    if start is not None:
        b.need(start, n, "start")
    handle, dev = _here(stream)
    _cache_here(cache, dev)
    st = b.sm_kv_read(cache.desc, seq_ids, start, row_offsets, n, rows, _rows(K), sk, _rows(V), sv, handle, dev)
    _check(st, "sm_kv_read")


class Norm:
    """A norm for block_norm: its kind ("rms" or "layer"), epsilon and [d]
    tensors (None: 1, 0), which it keeps."""

    def __init__(self, kind: str = "rms", gain=None, bias=None, eps: float = 1e-5):
        if kind not in NORM_KINDS:
            raise SpanMergeError(f"unknown norm: {kind!r}")
        self.kind, self.eps, self.gain, self.bias = NORM_KINDS[kind], eps, gain, bias
        self.last = (None, None)

    def look(self, b, dtype, d: int, dev: int, name: str) -> bytes:
        """The structure for a call over rows of d values (its fields may have
        other values since the last one, its tensors new memory: a module that
        was moved)."""
        fields = (self.kind, self.eps, b.parameter(self.gain, dtype, d, dev, name), b.parameter(self.bias, dtype, d, dev, name))
        last, packed = self.last
        if fields != last:
            packed = bytes(NormParams(*fields))
            self.last = (fields, packed)
        return packed


def norm_params(kind: str = "rms", gain=None, bias=None, eps: float = 1e-5) -> Norm:
    return Norm(kind, gain, bias, eps)


def block_norm(h, y, h_out, n_out, post: Optional[Norm] = None, gate=None, scale: float = 1.0,
               pre: Optional[Norm] = None, stream=None):
    """h_out = h + scale * gate * post(y), n_out = pre(h_out) of the unrounded
    sum; [rows, d] with contiguous rows.  y None: h alone; gate [d] or
    [rows, d]; h_out or n_out may be None, or an input itself."""
    b = _calls()
    row_stride, (rows, d), dt = b.row_stride, _shape(h, 2, "h"), h.dtype
    sh = row_stride(h, dt, "h", rows, d)
    sy = 0 if y is None else row_stride(y, dt, "y", rows, d)
    sho = 0 if h_out is None else row_stride(h_out, dt, "h_out", rows, d)
    sno = 0 if n_out is None else row_stride(n_out, dt, "n_out", rows, d)
    sg = 0
    if gate is not None:
        if gate.dim() == 1:
            row_stride(gate.unsqueeze(0), dt, "gate", 1, d)
        else:
            sg = row_stride(gate, dt, "gate", rows, d)
    handle, dev = _here(stream)
    po = None if post is None else post.look(b, dt, d, dev, "post")
    pr = None if pre is None else pre.look(b, dt, d, dev, "pre")
    st = b.sm_block_norm((h,), sh, _rows(y), sy, rows, d, po, _rows(gate), sg, scale, pr, dtype_code(dt), _rows(h_out), sho,
                         _rows(n_out), sno, handle, dev)
    _check(st, "sm_block_norm")


def token_logprobs_workspace_bytes(rows: int, vocab: int, k: int) -> int:
    return load().sm_token_logprobs_workspace_bytes(rows, vocab, k)


def token_logprobs(logits, tokens, logprob, entropy, top_ids, top_logprobs, ws, scale: float = 1.0, err=None, stream=None):
    """Log probability of tokens[r], entropy and the k = top_ids.shape[1]
    largest logits of each row of logits [rows, vocab] (contiguous rows);
    scale = 1 / temperature.  top_ids and top_logprobs are [rows, k] (or [rows]:
    one alternative).  Each output may be None."""
    b = _calls()
    (rows, vocab), dt, need = _shape(logits, 2, "logits"), logits.dtype, b.need
    sl = b.row_stride(logits, dt, "logits", rows, vocab)
    k = 0
    if tokens is not None:
        need(tokens, rows, "tokens")
    if logprob is not None:
        need(logprob, rows, "logprob")
    if entropy is not None:
        need(entropy, rows, "entropy")
    if top_ids is not None:
        k = _columns(top_ids, rows, "top_ids")
        if top_logprobs is not None and _columns(top_logprobs, rows, "top_logprobs") != k:
            raise SpanMergeError(f"top_logprobs: expected {k} columns, as top_ids has, got {tuple(top_logprobs.shape)}")
    elif top_logprobs is not None and top_logprobs.numel():
        raise SpanMergeError("top_logprobs without top_ids")
    if err is not None:
        need(err, 1, "err")
    handle, dev = _here(stream)
    st = b.sm_token_logprobs((logits,), sl, rows, vocab, dtype_code(dt), scale, tokens, logprob, entropy, k, top_ids,
                             top_logprobs, ws, ws.nbytes, err, handle, dev)
    _check(st, "sm_token_logprobs")


def sample_workspace_bytes(rows: int, vocab: int) -> int:
    return load().sm_sample_workspace_bytes(rows, vocab)


def sample_tokens(logits, u, tokens, ws, temperature=None, top_k=None, top_p=None, min_p=None, logprob=None, err=None,
                  stream=None):
    """tokens[r] drawn from the row logits[r] by the random number u[r]: weights
    exp(logits / temperature), of which top_k, then min_p, then top_p keep the
    likeliest (each [rows], or None: 1 and no filter; a temperature of 0 takes
    the likeliest token).  logprob: log of the token's share of what is kept."""
    b = _calls()
    (rows, vocab), dt, need = _shape(logits, 2, "logits"), logits.dtype, b.need
    sl = b.row_stride(logits, dt, "logits", rows, vocab)
    need(u, rows, "u")
    need(tokens, rows, "tokens")
    for t, name in ((temperature, "temperature"), (top_k, "top_k"), (top_p, "top_p"), (min_p, "min_p"), (logprob, "logprob")):
        if t is not None:
            need(t, rows, name)
    if err is not None:
        need(err, 1, "err")
    handle, dev = _here(stream)
    st = b.sm_sample_tokens((logits,), sl, rows, vocab, dtype_code(dt), u, temperature, top_k, top_p, min_p, tokens, logprob, ws,
                            ws.nbytes, err, handle, dev)
    _check(st, "sm_sample_tokens")
