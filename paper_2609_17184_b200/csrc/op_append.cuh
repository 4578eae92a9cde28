// Appending new tokens to a paged cache, straight from the rows of a QKV projection: y = x / sqrt(mean(x^2) + eps) * gain per head of
// queries and keys (optional), rotation of the pairs (i, i + rot/2) by index * inv_freq[i] (optional), queries to q, keys and values to
// the pages of their sequence.  Every element is read once and written once; bound by that traffic for prompts and by the launch for
// decoded tokens.
//
// A lane holds four pairs of a head - elements 4c .. 4c + 3 of either half of the rotated part (or of the unrotated rest) - for every head
// it serves: the angles are the token's, so their sine and cosine are computed once and not per head.  d / 8 lanes make a head.
// Angles: index * inv_freq is taken in 64 bits and reduced to a part of a turn before it is rounded, so positions of any size keep
// the precision of near ones (in 32 bits the angle of position 10^6 is off by 0.03).  Norms and rotations are fp32, rounded once.
#pragma once
#include "op_common.cuh"

namespace ls {

constexpr int APP_WARPS = 4;

struct AppendParams {
  const void* qkv;  // [T][ld]: nq heads of queries, n_kv of keys, n_kv of values
  long long ld, q_ld;
  void* q;          // [T][q_ld]
  PagedKv kv;
  const int* page_table;  // [B][table_ld]
  const int* cached;      // [B]
  const int* cu_rows;     // [B + 1]
  const int* pos_offset;  // [B] or null
  const double* inv_freq; // [rot / 2]
  const float *q_norm, *k_norm;
  float eps;
  long long table_ld;    // elements from a row of the table to the next
  int table_w;
  int T, B, nq, rot;
  int* err;
};

template <typename T>
__device__ __forceinline__ void app_load4(const T* p, float (&v)[4]) {
  if constexpr (sizeof(T) == 4) {
    const float4 w = __ldcs(reinterpret_cast<const float4*>(p));
    v[0] = w.x, v[1] = w.y, v[2] = w.z, v[3] = w.w;
  } else {
    const uint2 w = __ldcs(reinterpret_cast<const uint2*>(p));
    const T* e = reinterpret_cast<const T*>(&w);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = to_f32<T>(e[i]);
  }
}

// LH: lanes per head (a power of two >= d / 8)
template <typename TI, typename TO, int LH>
__global__ void __launch_bounds__(APP_WARPS * 32) append_kernel(const __grid_constant__ AppendParams p) {
  constexpr int HPW = 32 / LH;  // heads a warp works on at once
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, row = blockIdx.x;
  const int d = p.kv.d, n_heads = p.nq + 2 * p.kv.n_kv;
  const int c = lane & (LH - 1), step = gridDim.y * APP_WARPS * HPW;
  int h = (blockIdx.y * APP_WARPS + warp) * HPW + lane / LH;
  const bool live = c < d / 8, turns = 8 * c < p.rot;
  // this lane's elements: i0 .. i0 + 3 and i1 .. i1 + 3 of a head
  const int c0 = turns ? 4 * c : p.rot + 4 * (c - p.rot / 8), i0 = live ? c0 : 0, i1 = live ? i0 + (turns ? p.rot : d - p.rot) / 2 : 0;
  const TI* x = static_cast<const TI*>(p.qkv) + (long long)row * p.ld;
  float a[4], b[4];
  if (h < n_heads) app_load4(x + h * d + i0, a), app_load4(x + h * d + i1, b);  // (requested ahead of the look-ups)

  const int seq = seq_of_row(p.cu_rows, p.B, row, lane);
  if (seq < 0 || row >= __ldg(p.cu_rows + seq + 1)) return;  // behind the last sequence: left as it was
  const long long pos = (long long)__ldg(p.cached + seq) + (row - __ldg(p.cu_rows + seq));
  const long long pg = pos >> p.kv.page_shift;
  int page = -1;
  if (pos >= 0 && pg < p.table_w) page = __ldg(p.page_table + seq * p.table_ld + pg);
  const bool ok = page >= 0 && page < p.kv.n_pages;
  if (!ok && p.err && threadIdx.x == 0 && blockIdx.y == 0) atomicOr(p.err, OP_BAD_PAGE);
  const long long slot = pos & ((1ll << p.kv.page_shift) - 1);
  const long long at = (long long)page * p.kv.page_stride + slot * p.kv.slot_stride;

  float cs[4] = {1.f, 1.f, 1.f, 1.f}, sn[4] = {0.f, 0.f, 0.f, 0.f};
  if (live && turns) {
    const double index = (double)(pos + (p.pos_offset ? __ldg(p.pos_offset + seq) : 0));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      double t = index * __ldg(p.inv_freq + i0 + i) * 0.15915494309189533577;  // 1 / (2 pi): turns
      t -= rint(t);
      sincospif(2.f * (float)t, &sn[i], &cs[i]);
    }
  }
  float gq[8], gk[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    gq[i] = p.q_norm ? __ldg(p.q_norm + i0 + i) : 1.f, gq[4 + i] = p.q_norm ? __ldg(p.q_norm + i1 + i) : 1.f;
    gk[i] = p.k_norm ? __ldg(p.k_norm + i0 + i) : 1.f, gk[4 + i] = p.k_norm ? __ldg(p.k_norm + i1 + i) : 1.f;
  }
  const float inv_d = 1.f / (float)d;
  // (the trip count is the warp's: its lanes shuffle together)
  for (int h0 = (blockIdx.y * APP_WARPS + warp) * HPW; h0 < n_heads; h0 += step, h += step) {
    float na[4], nb[4];
    const bool more = h + step < n_heads;
    if (more) app_load4(x + (h + step) * d + i0, na), app_load4(x + (h + step) * d + i1, nb);
    const bool is_q = h < p.nq, is_k = !is_q && h < p.nq + p.kv.n_kv, is_v = !is_q && !is_k;
    const bool norm = is_q ? p.q_norm != nullptr : is_k && p.k_norm != nullptr;
    float ss = 0.f;
    if (live && h < n_heads)
#pragma unroll
      for (int i = 0; i < 4; ++i) ss += a[i] * a[i] + b[i] * b[i];
#pragma unroll
    for (int o = LH / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    if (live && h < n_heads) {
      if (norm) {
        const float r = 1.f / sqrtf(ss * inv_d + p.eps);
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = a[i] * r * (is_q ? gq[i] : gk[i]), b[i] = b[i] * r * (is_q ? gq[4 + i] : gk[4 + i]);
      }
      if (turns && !is_v) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float u = a[i], w = b[i];
          a[i] = u * cs[i] - w * sn[i], b[i] = w * cs[i] + u * sn[i];
        }
      }
      TO* dst = nullptr;
      if (is_q) dst = static_cast<TO*>(p.q) + (long long)row * p.q_ld + h * d;
      else if (ok) dst = static_cast<TO*>(is_k ? p.kv.k : p.kv.v) + at + (long long)(h - p.nq - (is_k ? 0 : p.kv.n_kv)) * p.kv.head_stride;
      if (dst) {
        *reinterpret_cast<uint2*>(dst + i0) = make_uint2(pack2<TO>(a[0], a[1]), pack2<TO>(a[2], a[3]));
        *reinterpret_cast<uint2*>(dst + i1) = make_uint2(pack2<TO>(b[0], b[1]), pack2<TO>(b[2], b[3]));
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = na[i], b[i] = nb[i];
  }
}

}  // namespace ls
