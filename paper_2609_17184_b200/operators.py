"""The operators between the linear maps of a serving step (see include/loopspec.h): argument marshalling only.

Tensors of one call live on one device, which need not be the current one; work goes to that device's current stream.  Shapes, types
and strides are checked here and in the library before anything is launched.  The smallest calls take a few microseconds on the device, so the
checks ask each tensor as little as they can."""
import ctypes as C

import torch

from .binding import LoopSpecError, PagedKv, lib

_I32, _F32, _F64 = torch.int32, torch.float32, torch.float64
_DTYPE = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_append_kv = lib.loopspec_op_append_kv
_prefix_attention = lib.loopspec_op_prefix_attention
_prefix_scratch = lib.loopspec_prefix_attention_scratch_bytes
_sample = lib.loopspec_op_sample
_device = torch._C._cuda_getDevice
_stream = torch._C._cuda_getCurrentRawStream


def _bad(what):
    raise LoopSpecError(-1, what)


def _vec(t, what, dtype, n, dev):
    """The address of a contiguous vector of n elements on device dev (None: null)."""
    if t is None:
        return None
    if t.dtype is not dtype or t.dim() != 1 or t.numel() != n or t.get_device() != dev or not t.is_contiguous():
        _bad(f"{what}: a contiguous vector of {n} {dtype} elements on cuda:{dev} is needed")
    return t.data_ptr()


def _table(t, dev):
    """A page table's address, row stride and width."""
    if t.dtype is not _I32 or t.dim() != 2 or t.get_device() != dev:
        _bad(f"page_table: [sequences, pages] int32 on cuda:{dev} is needed")
    (rows, width), (ld, step) = t.shape, t.stride()
    if (step != 1 and width > 1) or (ld < width and rows > 1):
        _bad("page_table: contiguous rows that do not overlap are needed")
    return t.data_ptr(), ld if ld > width else width, width


def _paged(k, v, dev):
    """The cache's description: [page][head][slot][d] views of one shape and one set of strides."""
    shape, st, dt = k.shape, k.stride(), k.dtype
    if dt is not torch.bfloat16 and dt is not torch.float16 or v.dtype is not dt or len(shape) != 4 or k.get_device() != dev or v.get_device() != dev:
        _bad(f"k_cache, v_cache: [pages, heads, page_size, head_dim] bf16 or fp16 on cuda:{dev} are needed")
    if v.shape != shape or v.stride() != st or st[3] != 1 and shape[3] > 1:
        _bad("k_cache, v_cache: one shape and one set of strides are needed, the last dimension contiguous")
    return PagedKv(k.data_ptr(), v.data_ptr(), st[0], st[1], st[2], shape[0], shape[2], shape[1], shape[3], _DTYPE[dt])


def _heads(t, what, dtype, shape, dev):
    """The row stride of [rows, heads, d] with contiguous heads."""
    st = t.stride()
    if t.dtype is not dtype or tuple(t.shape) != shape or t.get_device() != dev or t.numel() and (st[2] != 1 and shape[2] > 1 or st[1] != shape[2] and shape[1] > 1):
        _bad(f"{what}: {list(shape)} {dtype} on cuda:{dev} with contiguous heads is needed")
    return st[0]


def _call(fn, dev, what, *args):
    """The call on the device's current stream, the last argument of every entry point."""
    if dev == _device():
        rc = fn(*args, _stream(dev))
    else:
        with torch.cuda.device(dev):
            rc = fn(*args, _stream(dev))
    if rc:
        raise LoopSpecError(rc, what)


def append_kv(qkv, k_cache, v_cache, page_table, cached, cu_rows, n_q_heads, inv_freq=None, q_norm=None, k_norm=None, eps=1e-6, pos_offset=None,
              out=None, flag=None):
    """Append the rows of a QKV projection to a paged cache; returns the queries [T, n_q_heads, d] in the cache's type.

    qkv [T, (n_q + 2 n_kv) d] fp32 / bf16 / fp16; k_cache, v_cache [pages, n_kv, page_size, d] bf16 / fp16 (views of any strides); page_table
    [B, W], cached [B], cu_rows [B + 1] and pos_offset [B] int32; inv_freq [rot / 2] fp64 or None (no rotation); q_norm, k_norm [d] fp32 gains
    or None (no norm).  Rows behind cu_rows[B] are left as they are in `out` and not appended.  flag: int32 tensor of one element that
    bits are or-ed into when a page lies outside the cache (such rows are not appended)."""
    dev = qkv.get_device()
    code = _DTYPE.get(qkv.dtype)
    if code is None or dev < 0 or qkv.dim() != 2:
        _bad("qkv: [rows, (n_q_heads + 2 n_kv_heads) head_dim] fp32, bf16 or fp16 on a CUDA device is needed")
    kv = _paged(k_cache, v_cache, dev)
    table, table_ld, width = _table(page_table, dev)
    (T, row), (ld, step) = qkv.shape, qkv.stride()
    d, B = kv.head_dim, page_table.size(0)
    if row != (n_q_heads + 2 * kv.n_kv_heads) * d or step != 1 and row > 1 and T:
        _bad("qkv: contiguous rows of (n_q_heads + 2 n_kv_heads) * head_dim elements are needed")
    if out is None:
        out = torch.empty((T, n_q_heads, d), dtype=k_cache.dtype, device=qkv.device)
    half = 0 if inv_freq is None else inv_freq.numel()
    _call(_append_kv, dev, "append_kv", qkv.data_ptr(), code, ld, T, n_q_heads, C.byref(kv), table, table_ld, width, _vec(cached, "cached", _I32, B, dev),
          _vec(cu_rows, "cu_rows", _I32, B + 1, dev), B, _vec(pos_offset, "pos_offset", _I32, B, dev), _vec(inv_freq, "inv_freq", _F64, half, dev), 2 * half,
          _vec(q_norm, "q_norm", _F32, d, dev), _vec(k_norm, "k_norm", _F32, d, dev), eps, out.data_ptr(),
          _heads(out, "out", k_cache.dtype, (T, n_q_heads, d), dev), _vec(flag, "flag", _I32, 1, dev))
    return out


def prefix_attention_scratch_bytes(T, n_seqs, n_q_heads, n_kv_heads, head_dim, prefix_len):
    return _prefix_scratch(T, n_seqs, n_q_heads, n_kv_heads, head_dim, prefix_len)


def prefix_attention(q, k_cache, v_cache, prefix_pages, prefix_len, page_table, lens, cu_rows, scale=None, out=None, lse=None, scratch=None, flag=None):
    """Attention of a batch whose sequences share a prefix; returns (out [T, n_q, d], lse fp32 [T, n_q]).

    q [T, n_q, d] in the cache's type; k_cache, v_cache [pages, n_kv, page_size, d] bf16 / fp16 (views of any strides), d 64 or 128; prefix_pages
    int32 [>= ceil(prefix_len / page_size)] (None without a prefix); page_table [B, W], lens [B], cu_rows [B + 1] int32: the sequences' own pages, how
    many own positions they hold (the new rows included) and where their rows begin.  Row j of n sees the prefix and the own positions below lens - (n
    - 1 - j).  scale: None = 1 / sqrt(d).  Rows behind cu_rows[B] are left as they are.  scratch: uint8, 256-byte aligned,
    prefix_attention_scratch_bytes (allocated here if None).  flag: int32 tensor of one element that bits are or-ed into when a page lies outside the cache
    (1), lengths or row counts are not what they should be (2) or a bounded wait ran out (4)."""
    dev = q.get_device()
    if dev < 0 or q.dim() != 3:
        _bad("q: [rows, n_q_heads, head_dim] on a CUDA device is needed")
    kv = _paged(k_cache, v_cache, dev)
    table, table_ld, width = _table(page_table, dev)
    shape = T, nq, d = tuple(q.shape)
    B = page_table.size(0)
    if d != kv.head_dim:
        _bad("q: the cache's head_dim is needed")
    q_ld = _heads(q, "q", k_cache.dtype, shape, dev)
    where = q.device
    if out is None:
        out = torch.empty(shape, dtype=q.dtype, device=where)
    if lse is None:
        lse = torch.empty((T, nq), dtype=_F32, device=where)
    elif lse.dtype is not _F32 or tuple(lse.shape) != (T, nq) or lse.get_device() != dev or not lse.is_contiguous():
        _bad("lse: [rows, n_q_heads] fp32, contiguous, is needed")
    pages = None
    if prefix_len > 0:
        if prefix_pages is None or prefix_pages.numel() * kv.page_size < prefix_len:
            _bad("prefix_pages: ceil(prefix_len / page_size) entries are needed")
        pages = _vec(prefix_pages, "prefix_pages", _I32, prefix_pages.numel(), dev)
    need = _prefix_scratch(T, B, nq, kv.n_kv_heads, d, prefix_len)
    if need == 0:
        _bad("prefix_attention: head_dim 64 or 128, n_q_heads a multiple of the key heads, at most 2048 sequences")
    if scratch is None:
        scratch = torch.empty(need, dtype=torch.uint8, device=where)
    elif scratch.dtype is not torch.uint8 or scratch.get_device() != dev or not scratch.is_contiguous():
        _bad("scratch: contiguous uint8 on q's device is needed")
    _call(_prefix_attention, dev, "prefix_attention", q.data_ptr(), q_ld, T, nq, C.byref(kv), pages, prefix_len, table, table_ld, width,
          _vec(lens, "lens", _I32, B, dev), _vec(cu_rows, "cu_rows", _I32, B + 1, dev), B, 0.0 if scale is None else scale, out.data_ptr(),
          _heads(out, "out", q.dtype, shape, dev), lse.data_ptr(), _vec(flag, "flag", _I32, 1, dev), scratch.data_ptr(), scratch.numel())
    return out, lse


def sample(logits, uniforms, temperature=None, top_k=None, top_p=None, min_p=None, out=None, probs=None):
    """One token per row of logits [rows, V] (fp32 / bf16 / fp16, V <= 262144) from given uniform numbers fp32 [rows]; returns (tokens int32 [rows],
    their probabilities fp32 [rows]).

    temperature, top_p, min_p fp32 [rows] and top_k int32 [rows], or None (1, off, off, off): the filters apply in the order top-k, top-p
    (of what top-k kept), min-p; a temperature of 0 is the first of the largest logits.  -inf and NaN are masked out; a row of nothing else gets
    token -1."""
    dev = logits.get_device()
    code = _DTYPE.get(logits.dtype)
    if code is None or dev < 0 or logits.dim() != 2:
        _bad("logits: [rows, vocabulary] fp32, bf16 or fp16 on a CUDA device is needed")
    (rows, V), (ld, step) = logits.shape, logits.stride()
    if step != 1 and V > 1 and rows:
        _bad("logits: contiguous rows are needed")
    if out is None:
        out = torch.empty(rows, dtype=_I32, device=logits.device)
    if probs is None:
        probs = torch.empty(rows, dtype=_F32, device=logits.device)
    _call(_sample, dev, "sample", logits.data_ptr(), code, ld, rows, V, _vec(uniforms, "uniforms", _F32, rows, dev),
          _vec(temperature, "temperature", _F32, rows, dev), _vec(top_k, "top_k", _I32, rows, dev), _vec(top_p, "top_p", _F32, rows, dev),
          _vec(min_p, "min_p", _F32, rows, dev), _vec(out, "out", _I32, rows, dev), _vec(probs, "probs", _F32, rows, dev))
    return out, probs
