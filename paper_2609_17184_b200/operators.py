"""The operators between the linear maps of a serving step (see include/loopspec.h): argument marshalling only.

Tensors of one call live on one device, which need not be the current one; work goes to that device's current stream.  Shapes, types
and strides are checked - in csrc/marshal.cpp, which asks the tensors, and in the library - before anything is launched; what is refused raises LoopSpecError."""
import importlib.util
import os

from . import build as _build
from .binding import LoopSpecError, lib

_marshal = None  # the compiled marshalling, from the first call on: what needs no tensors needs no torch


def _load():
    global _marshal
    import torch
    where = os.path.dirname(torch.__file__)
    path = _build.marshal_path(where)
    if _build.marshal_needs_build(where):
        try:
            _build.build_marshal(where)
        except Exception as e:  # (one that was made for this torch and Python serves on)
            if not os.path.exists(path):
                raise ImportError(f"{os.path.basename(path)} is missing and could not be built: {e}") from e
    spec = importlib.util.spec_from_file_location(__package__ + "._marshal", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    module.set_error(LoopSpecError)
    _marshal = module
    return module


def append_kv(qkv, k_cache, v_cache, page_table, cached, cu_rows, n_q_heads, inv_freq=None, q_norm=None, k_norm=None, eps=1e-6, pos_offset=None,
              out=None, flag=None):
    """Append the rows of a QKV projection to a paged cache; returns the queries [T, n_q_heads, d] in the cache's type.

    qkv [T, (n_q + 2 n_kv) d] fp32 / bf16 / fp16; k_cache, v_cache [pages, n_kv, page_size, d] bf16 / fp16 (views of any strides); page_table
    [B, W], cached [B], cu_rows [B + 1] and pos_offset [B] int32; inv_freq [rot / 2] fp64 or None (no rotation); q_norm, k_norm [d] fp32 gains
    or None (no norm).  Rows behind cu_rows[B] are left as they are in `out` and not appended.  flag: int32 tensor of one element that
    bits are or-ed into when a page lies outside the cache (1; such rows are not appended) or row counts do not ascend within [0, T] (2; rows that they give
    to no sequence are not appended, and nothing is written in front of cached[b])."""
    return (_marshal or _load()).append_kv(qkv, k_cache, v_cache, page_table, cached, cu_rows, n_q_heads, inv_freq, q_norm, k_norm, eps, pos_offset, out, flag)


def prefix_attention_scratch_bytes(T, n_seqs, n_q_heads, n_kv_heads, head_dim, prefix_len):
    return lib.loopspec_prefix_attention_scratch_bytes(T, n_seqs, n_q_heads, n_kv_heads, head_dim, prefix_len)


def prefix_attention(q, k_cache, v_cache, prefix_pages, prefix_len, page_table, lens, cu_rows, scale=None, out=None, lse=None, scratch=None, flag=None):
    """Attention of a batch whose sequences share a prefix; returns (out [T, n_q, d], lse fp32 [T, n_q]).

    q [T, n_q, d] in the cache's type; k_cache, v_cache [pages, n_kv, page_size, d] bf16 / fp16 (views of any strides), d 64 or 128; prefix_pages
    int32 [>= ceil(prefix_len / page_size)] (None without a prefix); page_table [B, W], lens [B], cu_rows [B + 1] int32: the sequences' own pages, how
    many own positions they hold (the new rows included) and where their rows begin.  Row j of n sees the prefix and the own positions below lens - (n
    - 1 - j).  scale: None = 1 / sqrt(d).  Rows behind cu_rows[B] are left as they are.  scratch: uint8, 256-byte aligned,
    prefix_attention_scratch_bytes (allocated here if None).  flag: int32 tensor of one element that bits are or-ed into when a page lies outside the cache
    (1), lengths or row counts are not what they should be (2) or a bounded wait ran out (4: the rows that waited are NaN, with a flag or without)."""
    return (_marshal or _load()).prefix_attention(q, k_cache, v_cache, prefix_pages, prefix_len, page_table, lens, cu_rows, scale, out, lse, scratch, flag)


def sample(logits, uniforms, temperature=None, top_k=None, top_p=None, min_p=None, out=None, probs=None):
    """One token per row of logits [rows, V] (fp32 / bf16 / fp16, V <= 262144) from given uniform numbers fp32 [rows]; returns (tokens int32 [rows],
    their probabilities fp32 [rows]).

    temperature, top_p, min_p fp32 [rows] and top_k int32 [rows], or None (1, off, off, off): the filters apply in the order top-k, top-p
    (of what top-k kept), min-p; a temperature of 0 is the first of the largest logits.  -inf and NaN are masked out, and so is a token below 2^-(S + 1) of the
    largest weight, S = min(48, 61 - ceil(log2 V)); a row of nothing else gets token -1."""
    return (_marshal or _load()).sample(logits, uniforms, temperature, top_k, top_p, min_p, out, probs)
