"""The operators between the linear maps of a serving step (see include/loopspec.h): argument marshalling only.

Tensors of one call live on one device, which need not be the current one; work goes to that device's current stream.  Shapes, types
and strides are checked here and in the library before anything is launched."""
import ctypes as C

import torch

from .binding import LoopSpecError, PagedKv, lib

_DTYPE = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


def _bad(what):
    raise LoopSpecError(-1, what)


def _need(t, what, dtype, ndim, dev):
    """A tensor of this type and rank on the call's device, its last dimension contiguous."""
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or t.dim() != ndim or t.device != dev:
        _bad(f"{what}: a {ndim}-dimensional {dtype} tensor on {dev} is needed")
    if t.stride(-1) != 1 and t.size(-1) > 1 and t.numel():
        _bad(f"{what}: the last dimension has to be contiguous")


def _vec(t, what, dtype, n, dev):
    """The address of a contiguous vector of n elements (None: null)."""
    if t is None:
        return None
    _need(t, what, dtype, 1, dev)
    if t.size(0) != n:
        _bad(f"{what}: {n} elements are needed")
    return t.data_ptr()


def _table(t, dev):
    """A page table's address, row stride and width."""
    _need(t, "page_table", torch.int32, 2, dev)
    rows, width = t.shape
    if rows > 1 and t.stride(0) < width:
        _bad("page_table: rows that do not overlap are needed")
    return t.data_ptr(), max(t.stride(0), width), width


def _paged(k, v, dev):
    """The cache's description: [page][head][slot][d] views of one shape and one set of strides."""
    if not isinstance(k, torch.Tensor) or k.dtype not in (torch.bfloat16, torch.float16):
        _bad("k_cache: bf16 or fp16 is needed")
    _need(k, "k_cache", k.dtype, 4, dev)
    _need(v, "v_cache", k.dtype, 4, dev)
    sk, pages = k.stride(), k.shape
    if v.shape != pages or v.stride() != sk:
        _bad("k_cache and v_cache: one shape and one set of strides are needed")
    return PagedKv(k.data_ptr(), v.data_ptr(), sk[0], sk[1], sk[2], pages[0], pages[2], pages[1], pages[3], _DTYPE[k.dtype])


def _call(fn, dev, what, *args):
    """The call on the device's current stream, the last argument of every entry point."""
    i = dev.index
    if i == torch.cuda.current_device():
        rc = fn(*args, torch._C._cuda_getCurrentRawStream(i))
    else:
        with torch.cuda.device(i):
            rc = fn(*args, torch._C._cuda_getCurrentRawStream(i))
    if rc:
        raise LoopSpecError(rc, what)


def append_kv(qkv, k_cache, v_cache, page_table, cached, cu_rows, n_q_heads, inv_freq=None, q_norm=None, k_norm=None, eps=1e-6, pos_offset=None,
              out=None, flag=None):
    """Append the rows of a QKV projection to a paged cache; returns the queries [T, n_q_heads, d] in the cache's type.

    qkv [T, (n_q + 2 n_kv) d] fp32 / bf16 / fp16; k_cache, v_cache [pages, n_kv, page_size, d] bf16 / fp16 (views of any strides); page_table
    [B, W], cached [B], cu_rows [B + 1] and pos_offset [B] int32; inv_freq [rot / 2] fp64 or None (no rotation); q_norm, k_norm [d] fp32 gains
    or None (no norm).  Rows behind cu_rows[B] are left as they are in `out` and not appended.  flag: int32 tensor of one element that
    bits are or-ed into when a page lies outside the cache (such rows are not appended)."""
    dev = qkv.device
    if qkv.dtype not in _DTYPE or dev.type != "cuda":
        _bad("qkv: a CUDA tensor of fp32, bf16 or fp16 is needed")
    _need(qkv, "qkv", qkv.dtype, 2, dev)
    kv = _paged(k_cache, v_cache, dev)
    table = _table(page_table, dev)
    T, d = qkv.size(0), kv.head_dim
    B = page_table.size(0)
    if qkv.size(1) != (n_q_heads + 2 * kv.n_kv_heads) * d:
        _bad("qkv: rows of (n_q_heads + 2 n_kv_heads) * head_dim elements are needed")
    if out is None:
        out = torch.empty((T, n_q_heads, d), dtype=k_cache.dtype, device=dev)
    else:
        _need(out, "out", k_cache.dtype, 3, dev)
        if out.shape != (T, n_q_heads, d) or (out.stride(1) != d and n_q_heads > 1 and T):
            _bad("out: [T, n_q_heads, head_dim] with contiguous heads is needed")
    rot = 0
    if inv_freq is not None:
        rot = 2 * inv_freq.numel()
    _call(lib.loopspec_op_append_kv, dev, "append_kv", qkv.data_ptr(), _DTYPE[qkv.dtype], qkv.stride(0), T, n_q_heads, C.byref(kv),
          *table, _vec(cached, "cached", torch.int32, B, dev),
          _vec(cu_rows, "cu_rows", torch.int32, B + 1, dev), B, _vec(pos_offset, "pos_offset", torch.int32, B, dev),
          _vec(inv_freq, "inv_freq", torch.float64, rot // 2, dev), rot, _vec(q_norm, "q_norm", torch.float32, d, dev),
          _vec(k_norm, "k_norm", torch.float32, d, dev), eps, out.data_ptr(), out.stride(0), _vec(flag, "flag", torch.int32, 1, dev))
    return out


def prefix_attention_scratch_bytes(T, n_seqs, n_q_heads, n_kv_heads, head_dim, prefix_len):
    return lib.loopspec_prefix_attention_scratch_bytes(T, n_seqs, n_q_heads, n_kv_heads, head_dim, prefix_len)


def prefix_attention(q, k_cache, v_cache, prefix_pages, prefix_len, page_table, lens, cu_rows, scale=None, out=None, lse=None, scratch=None, flag=None):
    """Attention of a batch whose sequences share a prefix; returns (out [T, n_q, d], lse fp32 [T, n_q]).

    q [T, n_q, d] in the cache's type; k_cache, v_cache [pages, n_kv, page_size, d] bf16 / fp16 (views of any strides), d 64 or 128; prefix_pages
    int32 [>= ceil(prefix_len / page_size)] (None without a prefix); page_table [B, W], lens [B], cu_rows [B + 1] int32: the sequences' own pages, how
    many own positions they hold (the new rows included) and where their rows begin.  Row j of n sees the prefix and the own positions below lens - (n
    - 1 - j).  scale: None = 1 / sqrt(d).  Rows behind cu_rows[B] are left as they are.  scratch: uint8, 256-byte aligned,
    prefix_attention_scratch_bytes (allocated here if None).  flag: int32 tensor of one element that bits are or-ed into when a page lies outside the cache
    (1), lengths or row counts are not what they should be (2) or a bounded wait ran out (4)."""
    dev = q.device
    if dev.type != "cuda":
        _bad("q: a CUDA tensor is needed")
    kv = _paged(k_cache, v_cache, dev)
    _need(q, "q", k_cache.dtype, 3, dev)
    table = _table(page_table, dev)
    T, nq, d = q.shape
    B = page_table.size(0)
    if d != kv.head_dim or (q.stride(1) != d and nq > 1 and T):
        _bad("q: [T, n_q_heads, head_dim] with contiguous heads is needed")
    if out is None:
        out = torch.empty((T, nq, d), dtype=q.dtype, device=dev)
    else:
        _need(out, "out", q.dtype, 3, dev)
        if out.shape != q.shape or (out.stride(1) != d and nq > 1 and T):
            _bad("out: [T, n_q_heads, head_dim] with contiguous heads is needed")
    if lse is None:
        lse = torch.empty((T, nq), dtype=torch.float32, device=dev)
    else:
        _need(lse, "lse", torch.float32, 2, dev)
        if lse.shape != (T, nq) or not lse.is_contiguous():
            _bad("lse: [T, n_q_heads], contiguous, is needed")
    pages = None
    if prefix_len > 0:
        _need(prefix_pages, "prefix_pages", torch.int32, 1, dev)
        if prefix_pages.size(0) * kv.page_size < prefix_len:
            _bad("prefix_pages: ceil(prefix_len / page_size) entries are needed")
        pages = prefix_pages.data_ptr()
    need = prefix_attention_scratch_bytes(T, B, nq, kv.n_kv_heads, d, prefix_len)
    if need == 0:
        _bad("prefix_attention: head_dim 64 or 128, n_q_heads a multiple of the key heads, at most 2048 sequences")
    if scratch is None:
        scratch = torch.empty(need, dtype=torch.uint8, device=dev)
    else:
        _need(scratch, "scratch", torch.uint8, 1, dev)
    _call(lib.loopspec_op_prefix_attention, dev, "prefix_attention", q.data_ptr(), q.stride(0), T, nq, C.byref(kv), pages, prefix_len, *table,
          _vec(lens, "lens", torch.int32, B, dev), _vec(cu_rows, "cu_rows", torch.int32, B + 1, dev), B, 0.0 if scale is None else scale, out.data_ptr(),
          out.stride(0), lse.data_ptr(), _vec(flag, "flag", torch.int32, 1, dev), scratch.data_ptr(), scratch.numel())
    return out, lse


def sample(logits, uniforms, temperature=None, top_k=None, top_p=None, min_p=None, out=None, probs=None):
    """One token per row of logits [rows, V] (fp32 / bf16 / fp16, V <= 262144) from given uniform numbers fp32 [rows]; returns (tokens int32 [rows],
    their probabilities fp32 [rows]).

    temperature, top_p, min_p fp32 [rows] and top_k int32 [rows], or None (1, off, off, off): the filters apply in the order top-k, top-p
    (of what top-k kept), min-p; a temperature of 0 is the first of the largest logits.  -inf and NaN are masked out; a row of nothing else gets
    token -1."""
    dev = logits.device
    if logits.dtype not in _DTYPE or dev.type != "cuda":
        _bad("logits: a CUDA tensor of fp32, bf16 or fp16 is needed")
    _need(logits, "logits", logits.dtype, 2, dev)
    rows, V = logits.shape
    if out is None:
        out = torch.empty(rows, dtype=torch.int32, device=dev)
    if probs is None:
        probs = torch.empty(rows, dtype=torch.float32, device=dev)
    _call(lib.loopspec_op_sample, dev, "sample", logits.data_ptr(), _DTYPE[logits.dtype], logits.stride(0), rows, V,
          _vec(uniforms, "uniforms", torch.float32, rows, dev), _vec(temperature, "temperature", torch.float32, rows, dev),
          _vec(top_k, "top_k", torch.int32, rows, dev), _vec(top_p, "top_p", torch.float32, rows, dev), _vec(min_p, "min_p", torch.float32, rows, dev),
          _vec(out, "out", torch.int32, rows, dev), _vec(probs, "probs", torch.float32, rows, dev))
    return out, probs
