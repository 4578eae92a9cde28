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

// four elements as they come
template <typename T>
struct AppRaw {
  uint2 w;
  __device__ __forceinline__ void load(const T* p) { w = __ldcs(reinterpret_cast<const uint2*>(p)); }
  __device__ __forceinline__ void store(void* p) const { *static_cast<uint2*>(p) = w; }
  __device__ __forceinline__ void get(float (&v)[4]) const {
    const T* e = reinterpret_cast<const T*>(&w);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = to_f32<T>(e[i]);
  }
};
template <>
struct AppRaw<float> {
  float4 w;
  __device__ __forceinline__ void load(const float* p) { w = __ldcs(reinterpret_cast<const float4*>(p)); }
  __device__ __forceinline__ void store(void* p) const { *static_cast<float4*>(p) = w; }
  __device__ __forceinline__ void get(float (&v)[4]) const { v[0] = w.x, v[1] = w.y, v[2] = w.z, v[3] = w.w; }
};

// Where a row's keys and values go, and its angles: a chain of four reads, one sine and cosine per pair of this lane
struct AppRow {
  bool in, ok;      // belongs to a sequence; its page is one of the cache
  long long at;     // elements from the cache's start to the row's slot
  float cs[4], sn[4];
};
__device__ __forceinline__ AppRow app_row(const AppendParams& p, int row, int lane, bool turns, int i0) {
  AppRow r;
  const int seq = seq_of_row(p.cu_rows, p.B, row, lane);
  // (counts that do not ascend may give any answer: a row is behind the sequence's first, so nothing that is cached is written again)
  const int at = max(seq, 0), first = __ldg(p.cu_rows + at);
  r.in = seq >= 0 && first >= 0 && first <= row && row < __ldg(p.cu_rows + at + 1);
  if (!r.in) return r;
  const long long pos = (long long)__ldg(p.cached + seq) + (row - first);
  const long long pg = pos >> p.kv.page_shift;
  int page = -1;
  if (pos >= 0 && pg < p.table_w) page = __ldg(p.page_table + seq * p.table_ld + pg);
  r.ok = page >= 0 && page < p.kv.n_pages;
  if (!r.ok && p.err && lane == 0) atomicOr(p.err, OP_BAD_PAGE);
  const long long slot = pos & ((1ll << p.kv.page_shift) - 1);
  r.at = (long long)page * p.kv.page_stride + slot * p.kv.slot_stride;
#pragma unroll
  for (int i = 0; i < 4; ++i) r.cs[i] = 1.f, r.sn[i] = 0.f;
  if (turns) {
    const double index = (double)(pos + (p.pos_offset ? __ldg(p.pos_offset + seq) : 0));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      double t = index * __ldg(p.inv_freq + i0 + i) * 0.15915494309189533577;  // 1 / (2 pi): turns
      t -= rint(t);
      sincospif(2.f * (float)t, &r.sn[i], &r.cs[i]);
    }
  }
  return r;
}

// Whether the row counts ascend within [0, T]: the first CTA asks, for all
__device__ __forceinline__ void app_check_counts(const AppendParams& p) {
  if (!p.err || blockIdx.x || blockIdx.y) return;
  bool bad = false;
  for (int i = threadIdx.x; i <= p.B; i += APP_WARPS * 32) {
    const int c = __ldg(p.cu_rows + i);
    bad |= c < 0 || c > p.T || (i && c < __ldg(p.cu_rows + i - 1));
  }
  if (bad) atomicOr(p.err, OP_BAD_ROWS);
}

// Both kernels below do a head's arithmetic in the same order, so a token's query and key are the same bits in calls of any number of rows.  A lane's
// squares are two chains, of its even and of its odd elements:
__device__ __forceinline__ float app_squares(float a, float b, float c, float d) { return fmaf(d, d, fmaf(c, c, fmaf(b, b, __fmul_rn(a, a)))); }

// Few rows: a row's heads over the warps of one CTA or several, for what counts is the way to the last store.
// LH: lanes per head (a power of two >= d / 8)
template <typename TI, typename TO, int LH>
__global__ void __launch_bounds__(APP_WARPS * 32) append_kernel(const __grid_constant__ AppendParams p) {
  constexpr int HPW = 32 / LH;                  // heads a warp works on at once
  constexpr int AHEAD = sizeof(TI) == 4 ? 2 : 3;  // such turns in flight: the look-ups below are a chain of four reads, and a row is over after a few turns
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int row = blockIdx.x;
  const int d = p.kv.d, n_heads = p.nq + 2 * p.kv.n_kv;
  const int c = lane & (LH - 1), step = gridDim.y * APP_WARPS * HPW;
  const int h_warp = (blockIdx.y * APP_WARPS + warp) * HPW, h_lane = lane / LH;
  const bool live = c < d / 8, turns = 8 * c < p.rot;
  // this lane's elements: i0 .. i0 + 3 and i1 .. i1 + 3 of a head
  const int c0 = turns ? 4 * c : p.rot + 4 * (c - p.rot / 8), i0 = live ? c0 : 0, i1 = live ? i0 + (turns ? p.rot : d - p.rot) / 2 : 0;
  const TI* x = static_cast<const TI*>(p.qkv) + (long long)row * p.ld;
  AppRaw<TI> ra[AHEAD], rb[AHEAD];
  auto fetch = [&](int h0) {
#pragma unroll
    for (int t = 0; t < AHEAD; ++t) {
      const int h = h0 + t * step + h_lane;
      if (h < n_heads) ra[t].load(x + h * d + i0), rb[t].load(x + h * d + i1);
    }
  };
  fetch(h_warp);
  app_check_counts(p);

  const AppRow its = app_row(p, row, lane, live && turns, i0);
  if (!its.in) return;  // behind the last sequence: left as it was
  const bool ok = its.ok;
  const long long at = its.at;
  const float (&cs)[4] = its.cs, (&sn)[4] = its.sn;
  const float inv_d = 1.f / (float)d;
  // (the trip count is the warp's: its lanes shuffle together)
  for (int h0 = h_warp; h0 < n_heads; h0 += AHEAD * step) {
    float va[AHEAD][4], vb[AHEAD][4];
#pragma unroll
    for (int t = 0; t < AHEAD; ++t) ra[t].get(va[t]), rb[t].get(vb[t]);
    if (h0 + AHEAD * step < n_heads) fetch(h0 + AHEAD * step);
#pragma unroll
    for (int t = 0; t < AHEAD; ++t) {
      if (h0 + t * step >= n_heads) break;
      float(&a)[4] = va[t], (&b)[4] = vb[t];
      const int h = h0 + t * step + h_lane;
      const bool is_q = h < p.nq, is_k = !is_q && h < p.nq + p.kv.n_kv, is_v = !is_q && !is_k;
      const float* gain = is_q ? p.q_norm : is_k ? p.k_norm : nullptr;
      if (!live || h >= n_heads)
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = b[i] = 0.f;
      if (p.q_norm || p.k_norm) {
        float ss = app_squares(a[0], a[2], b[0], b[2]) + app_squares(a[1], a[3], b[1], b[3]);
#pragma unroll
        for (int o = LH / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
        if (gain) {
          const float r = rsqrtf(fmaf(ss, inv_d, p.eps));  // (2 ulp)
          const float4 g0 = *reinterpret_cast<const float4*>(gain + i0), g1 = *reinterpret_cast<const float4*>(gain + i1);
          a[0] *= r * g0.x, a[1] *= r * g0.y, a[2] *= r * g0.z, a[3] *= r * g0.w;
          b[0] *= r * g1.x, b[1] *= r * g1.y, b[2] *= r * g1.z, b[3] *= r * g1.w;
        }
      }
      if (turns && !is_v) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float u = a[i], w = b[i];
          a[i] = fmaf(w, -sn[i], __fmul_rn(u, cs[i])), b[i] = fmaf(u, sn[i], __fmul_rn(w, cs[i]));
        }
      }
      TO* dst = nullptr;
      if (is_q) dst = static_cast<TO*>(p.q) + (long long)row * p.q_ld + h * d;
      else if (ok) dst = static_cast<TO*>(is_k ? p.kv.k : p.kv.v) + at + (long long)(h - p.nq - (is_k ? 0 : p.kv.n_kv)) * p.kv.head_stride;
      if (dst && live && h < n_heads) {
        *reinterpret_cast<uint2*>(dst + i0) = make_uint2(pack2<TO>(a[0], a[1]), pack2<TO>(a[2], a[3]));
        *reinterpret_cast<uint2*>(dst + i1) = make_uint2(pack2<TO>(b[0], b[1]), pack2<TO>(b[2], b[3]));
      }
    }
  }
}

// Many rows: a warp per row, so that look-ups and sines are taken once for all heads.  Bound by the instructions per head as much as by the traffic (a loop
// over all heads alike issued 170 a turn and took 48 us for 9,200 rows of 48 heads), so queries, keys and values have a loop each: values move as they
// are, gains and addresses stay in registers, and the arithmetic is packed in pairs (in the order of the kernel above): 42 us, 4.6 TB/s, with norms or without - what is left is the
// way of a row, four dependent look-ups ahead of its first store, in less than three rows per warp place.  More warps with fewer loads in flight each: +5 to +15 %.
template <typename TI, typename TO, int LH>
__global__ void __launch_bounds__(APP_WARPS * 32) append_rows_kernel(const __grid_constant__ AppendParams p) {
  constexpr int HPW = 32 / LH, AHEAD = 4;
  typedef unsigned long long u64;
  const int lane = threadIdx.x & 31, row = blockIdx.x * APP_WARPS + (threadIdx.x >> 5);
  app_check_counts(p);
  if (row >= p.T) return;
  const int d = p.kv.d, c = lane & (LH - 1), h_lane = lane / LH;
  const bool live = c < d / 8, turns = 8 * c < p.rot;
  const int c0 = turns ? 4 * c : p.rot + 4 * (c - p.rot / 8), i0 = live ? c0 : 0, i1 = live ? i0 + (turns ? p.rot : d - p.rot) / 2 : 0;
  const TI* x = static_cast<const TI*>(p.qkv) + (long long)row * p.ld;
  AppRaw<TI> ra[AHEAD], rb[AHEAD];
  auto fetch = [&](const TI* from, int h0, int n) {
#pragma unroll
    for (int t = 0; t < AHEAD; ++t) {
      const int h = h0 + t * HPW + h_lane;
      if (h < n) ra[t].load(from + h * d + i0), rb[t].load(from + h * d + i1);
    }
  };
  fetch(x, 0, p.nq);
  const AppRow its = app_row(p, row, lane, live && turns, i0);
  if (!its.in) return;  // behind the last sequence: left as it was
  const u64 cs[2] = {two(its.cs[0], its.cs[1]), two(its.cs[2], its.cs[3])}, sn[2] = {two(its.sn[0], its.sn[1]), two(its.sn[2], its.sn[3])};
  const u64 ns[2] = {two(-its.sn[0], -its.sn[1]), two(-its.sn[2], -its.sn[3])};
  const float inv_d = 1.f / (float)d;

  // n heads from `from` (their first turns are on the way) to `to`, `stride` apart; then the first turns of the n_then heads at `then`
  auto heads = [&](auto kind, const TI* from, int n, TO* to, long long stride, bool stored, const float* gain, const TI* then, int n_then) {
    constexpr bool VALUES = decltype(kind)::value;
    u64 g[4] = {0, 0, 0, 0};
    if (!VALUES && gain) {
      const float4 g0 = *reinterpret_cast<const float4*>(gain + i0), g1 = *reinterpret_cast<const float4*>(gain + i1);
      g[0] = two(g0.x, g0.y), g[1] = two(g0.z, g0.w), g[2] = two(g1.x, g1.y), g[3] = two(g1.z, g1.w);
    }
#pragma unroll 1
    for (int h0 = 0; h0 < n; h0 += AHEAD * HPW) {
      AppRaw<TI> wa[AHEAD], wb[AHEAD];
#pragma unroll
      for (int t = 0; t < AHEAD; ++t) wa[t] = ra[t], wb[t] = rb[t];
      if (h0 + AHEAD * HPW < n) fetch(from, h0 + AHEAD * HPW, n);
      else fetch(then, 0, n_then);
#pragma unroll
      for (int t = 0; t < AHEAD; ++t) {
        if (h0 + t * HPW >= n) break;
        const int h = h0 + t * HPW + h_lane;
        const bool here = live && h < n;
        TO* dst = to + h * stride;
        if constexpr (VALUES && std::is_same<TI, TO>::value) {  // as they are
          if (here && stored) wa[t].store(dst + i0), wb[t].store(dst + i1);
          continue;
        } else {
          float f[8];
          wa[t].get(reinterpret_cast<float(&)[4]>(f[0])), wb[t].get(reinterpret_cast<float(&)[4]>(f[4]));
          u64 v[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = two(f[2 * i], f[2 * i + 1]);
          if (!VALUES) {
            if (gain) {
              u64 sq = mul2(v[0], v[0]);
#pragma unroll
              for (int i = 1; i < 4; ++i) sq = fma2(v[i], v[i], sq);
              float s0, s1;
              split(sq, s0, s1);
              float ss = here ? s0 + s1 : 0.f;
#pragma unroll
              for (int o = LH / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
              const float r = rsqrtf(fmaf(ss, inv_d, p.eps));  // (2 ulp)
              const u64 r2 = two(r, r);
#pragma unroll
              for (int i = 0; i < 4; ++i) v[i] = mul2(v[i], mul2(r2, g[i]));
            }
            if (turns) {
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                const u64 a = v[i], b = v[2 + i];
                v[i] = fma2(b, ns[i], mul2(a, cs[i])), v[2 + i] = fma2(a, sn[i], mul2(b, cs[i]));
              }
            }
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) split(v[i], f[2 * i], f[2 * i + 1]);
          if (here && stored) {
            *reinterpret_cast<uint2*>(dst + i0) = make_uint2(pack2<TO>(f[0], f[1]), pack2<TO>(f[2], f[3]));
            *reinterpret_cast<uint2*>(dst + i1) = make_uint2(pack2<TO>(f[4], f[5]), pack2<TO>(f[6], f[7]));
          }
        }
      }
    }
  };
  const TI *xk = x + (long long)p.nq * d, *xv = xk + (long long)p.kv.n_kv * d;
  if (p.nq == 0) fetch(xk, 0, p.kv.n_kv);
  heads(std::false_type(), x, p.nq, static_cast<TO*>(p.q) + (long long)row * p.q_ld, d, true, p.q_norm, xk, p.kv.n_kv);
  heads(std::false_type(), xk, p.kv.n_kv, static_cast<TO*>(p.kv.k) + its.at, p.kv.head_stride, its.ok, p.k_norm, xv, p.kv.n_kv);
  heads(std::true_type(), xv, p.kv.n_kv, static_cast<TO*>(p.kv.v) + its.at, p.kv.head_stride, its.ok, nullptr, xv, 0);
}

}  // namespace ls
