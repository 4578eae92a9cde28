// One token per row of logits by temperature, top-k, top-p and min-p from a given uniform number: w = exp((z - max) / T), ranked by logit (ties:
// lower index first); the token is the first, by index, at which the running sum of the kept weights exceeds u times their sum.
//
// Which side of a border a sum lies on decides the token, so no sum may depend on the order of its additions or lose what a 64-bit
// evaluation keeps: a weight is evaluated in fp64 (2^y by a table of 2^(j/64) and a polynomial of degree 4: 4e-14) and rounded ONCE to a multiple
// of 2^-S, S = 61 - ceil(log2 V) (44 at 128K tokens); from there on everything - sums over the vocabulary, p times a sum, u times a sum -
// is exact integer arithmetic.  Sums are the same in every order and for every number of CTAs.  A token below 2^-(S+1) of the best weighs nothing.
//
// A cluster of CTAs holds a row in shared memory: the logits are read from HBM once.
#pragma once
#include <cooperative_groups.h>

#include "op_common.cuh"

namespace ls {
namespace smp {
namespace cg = cooperative_groups;
typedef unsigned long long u64;

constexpr int THREADS = 512, WARPS = THREADS / 32;
constexpr int MAX_CS = 8;
constexpr int NV = 7;  // sums taken together

struct Params {
  const void* logits;
  long long ld;
  int rows, V, per;          // per: tokens of a CTA's slice (a multiple of 8)
  int shift;                 // S
  const float *u, *temperature, *top_p, *min_p;
  const int* top_k;
  int* token;
  float* prob;               // or null
};

// ordered like the value, -0 and 0 alike
__device__ __forceinline__ unsigned key_of(float z) {
  const unsigned b = __float_as_uint(z + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
// fp32 -> fp64 by its bits (conversions run at a quarter of the rate of fp64 sums); zero comes out as 2^-127, infinity as 2^128: both are
// what the sums here need
__device__ __forceinline__ double widen(float z) {
  const unsigned b = __float_as_uint(z);
  return __hiloint2double((int)((b & 0x80000000u) | (((b & 0x7fffffffu) >> 3) + (896u << 20))), (int)(b << 29));
}
// floor (or, with UP, ceiling) of x * m for a float x in [0, 1)
template <bool UP>
__device__ __forceinline__ u64 times(float x, u64 m) {
  const unsigned b = __float_as_uint(x);
  const int e = b >> 23;
  const u64 mant = e ? (b & 0x7fffffu) | 0x800000u : b & 0x7fffffu;
  const int s = e ? 150 - e : 149;  // x = mant * 2^-s
  const u64 hi = __umul64hi(mant, m), lo = mant * m;
  u64 r, rest;
  if (s >= 128) r = 0, rest = hi | lo;
  else if (s >= 64) r = s == 64 ? hi : hi >> (s - 64), rest = lo | (s == 64 ? 0 : hi << (128 - s));
  else r = (hi << (64 - s)) | (lo >> s), rest = lo << (64 - s);
  return r + (UP && rest != 0);
}

// the weight of a logit, scaled by 2^S
struct Weigher {
  const double* table;  // 2^(j / 64)
  double top, c;        // largest logit, log2(e) / T
  int shift;
  float none;           // logits up to this one weigh nothing: -inf, or all finite ones beside an infinity
  __device__ __forceinline__ double scaled(float z) const {
    const double y = (widen(z) - top) * c;
    if (!(z > none) || !(y > -(double)(shift + 2))) return 0.0;
    const double magic = 6755399441055744.0;  // 1.5 * 2^52: the sum's low word is 64 y to the nearest integer
    const double t = fma(y, 64.0, magic);
    const int k = __double2loint(t);
    const double f = fma(t - magic, -1.0 / 64, y) * 0.69314718055994530942;  // 2^y = 2^(k / 64) e^f, |f| <= ln 2 / 128
    const double q = fma(f, fma(f, fma(f, fma(f, 1.0 / 24, 1.0 / 6), 0.5), 1.0), 1.0);
    const double w = table[k & 63];
    return q * __hiloint2double(__double2hiint(w) + ((k >> 6) + shift) * (1 << 20), __double2loint(w));
  }
  __device__ __forceinline__ u64 rounded(double w) const { return (u64)__double_as_longlong(w + 4503599627370496.0) & 0xfffffffffffffull; }  // (below 2^52)
  __device__ __forceinline__ u64 operator()(float z) const { return rounded(scaled(z)); }
};

// Sums, minima and maxima over the cluster: warps, then the CTA's partials in every CTA's memory, two sets of slots in turn
struct Cluster {
  cg::cluster_group cl;
  int n, rank, phase;
  u64* sh;    // [WARPS][NV]
  u64* part;  // [2][MAX_CS][NV]

  template <int N, typename Op>
  __device__ __forceinline__ void fold(u64 (&v)[N], Op op) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) v[i] = op(v[i], __shfl_xor_sync(0xffffffffu, v[i], o));
    __syncthreads();
    if (lane == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) sh[warp * NV + i] = v[i];
    __syncthreads();
    if ((int)threadIdx.x < N) {
      u64 r = sh[threadIdx.x];
      for (int w = 1; w < WARPS; ++w) r = op(r, sh[w * NV + threadIdx.x]);
      for (int q = 0; q < n; ++q) *cl.map_shared_rank(part + (phase * MAX_CS + rank) * NV + threadIdx.x, q) = r;
    }
    cl.sync();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      u64 r = part[phase * MAX_CS * NV + i];
      for (int q = 1; q < n; ++q) r = op(r, part[(phase * MAX_CS + q) * NV + i]);
      v[i] = r;
    }
    phase ^= 1;
  }
  template <int N>
  __device__ __forceinline__ void sum(u64 (&v)[N]) {
    fold(v, [](u64 a, u64 b) { return a + b; });
  }
  __device__ __forceinline__ u64 sum(u64 x) {
    u64 v[1] = {x};
    sum(v);
    return v[0];
  }
  __device__ __forceinline__ u64 max(u64 x) {
    u64 v[1] = {x};
    fold(v, [](u64 a, u64 b) { return a > b ? a : b; });
    return v[0];
  }
  // What precedes this thread's x in the order (rank, thread), and the total
  __device__ __forceinline__ u64 scan(u64 x, u64& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    u64 inc = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const u64 t = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += t;
    }
    __syncthreads();
    if (lane == 31) sh[warp] = inc;
    __syncthreads();
    u64 before = inc - x, mine = 0;
    for (int w = 0; w < WARPS; ++w) {
      if (w < warp) before += sh[w];
      mine += sh[w];
    }
    if (threadIdx.x == 0)
      for (int q = 0; q < n; ++q) *cl.map_shared_rank(part + (phase * MAX_CS + rank) * NV, q) = mine;
    cl.sync();
    total = 0;
    for (int q = 0; q < n; ++q) {
      const u64 s = part[(phase * MAX_CS + q) * NV];
      if (q < rank) before += s;
      total += s;
    }
    phase ^= 1;
    return before;
  }
};

template <typename T>
__global__ void __launch_bounds__(THREADS) sample_kernel(const __grid_constant__ Params p) {
  extern __shared__ __align__(16) unsigned char smp_smem[];
  __shared__ double s_table[64];
  __shared__ u64 s_sh[WARPS * NV], s_part[2 * MAX_CS * NV];
  cg::cluster_group cl = cg::this_cluster();
  Cluster R{cl, (int)cl.num_blocks(), (int)cl.block_rank(), 0, s_sh, s_part};
  const int tid = threadIdx.x, row = blockIdx.x / R.n, V = p.V;
  const int v_lo = min(V, R.rank * p.per), n = min(V, v_lo + p.per) - v_lo;  // this CTA's tokens
  if (tid < 64) s_table[tid] = exp2((double)tid / 64);

  // ---- the slice, 16 bytes at a time but for its ends; an element that is no number counts as masked out ----
  const T* src = static_cast<const T*>(p.logits) + row * p.ld + v_lo;
  constexpr int VEC = 16 / sizeof(T);
  const int head = (int)((reinterpret_cast<uintptr_t>(src) & 15) / sizeof(T));  // elements from the 16-byte boundary before the slice
  T* z_sm = reinterpret_cast<T*>(smp_smem) + head;                              // z_sm[i]: token v_lo + i
  float top = -INFINITY;
  auto clean = [](float z) { return z == z ? z : -INFINITY; };
  {
    const int lead = min(n, head ? VEC - head : 0), n_vec = (n - lead) / VEC, tail = lead + n_vec * VEC;
    for (int i = tid; i < lead + n - tail; i += THREADS) {
      const int e = i < lead ? i : tail + i - lead;
      const float z = clean(to_f32<T>(src[e]));
      z_sm[e] = T(z), top = fmaxf(top, z);
    }
    const uint4* vs = reinterpret_cast<const uint4*>(src + lead);
    uint4* vd = reinterpret_cast<uint4*>(z_sm + lead);
#pragma unroll 4
    for (int i = tid; i < n_vec; i += THREADS) {
      uint4 w = __ldcs(vs + i);
      T* e = reinterpret_cast<T*>(&w);
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const float z = clean(to_f32<T>(e[j]));
        e[j] = T(z), top = fmaxf(top, z);
      }
      vd[i] = w;
    }
  }
  auto z_at = [&](int i) { return to_f32<T>(z_sm[i]); };
  const unsigned top_key = (unsigned)R.max(key_of(top));
  top = __uint_as_float(top_key & 0x80000000u ? top_key & 0x7fffffffu : ~top_key);
  const bool writer = R.rank == 0 && tid == 0;
  auto put = [&](int token, float prob) {
    p.token[row] = token;
    if (p.prob) p.prob[row] = prob;
  };
  if (top == -INFINITY) {  // nothing to choose from
    if (writer) put(-1, 0.f);
    return;
  }
  const float temp = p.temperature ? __ldg(p.temperature + row) : 1.f;
  if (!(temp > 0.f)) {  // greedy: the first of the largest
    u64 first = 0;
    for (int i = tid; i < n; i += THREADS)
      if (z_at(i) == top) {
        first = 0x7fffffffu - (unsigned)(v_lo + i);
        break;
      }
    first = R.max(first);
    if (writer) put((int)(0x7fffffffu - (unsigned)first), 1.f);
    return;
  }
  const Weigher weigh = {s_table, widen(top), 1.4426950408889634074 / (double)temp, p.shift, top == INFINITY ? 3.402823466e38f : -INFINITY};
  const int top_k = p.top_k ? __ldg(p.top_k + row) : 0;
  const float top_p = p.top_p ? __ldg(p.top_p + row) : 1.f, min_p = p.min_p ? __ldg(p.min_p + row) : 0.f;
  const double least = min_p > 0.f ? (double)fminf(min_p, 1.f) * (double)(1ull << p.shift) : 0.0;

  // ---- the cut: a token stays if its key is above `cut`, or equal to it and its index at most `last` ----
  unsigned cut = 0;
  int last = V - 1;
  auto kept = [&](unsigned k, int v) { return k > cut || (k == cut && v <= last); };
  const int seg = ((n + THREADS - 1) / THREADS) | 1, s_lo = min(n, tid * seg), s_hi = min(n, s_lo + seg);  // (odd: no bank twice)
  // index of the need-th token (from 1) of key c, by index
  auto nth_of_key = [&](unsigned c, u64 need) -> int {
    u64 mine = 0, total;
    for (int i = s_lo; i < s_hi; ++i) mine += key_of(z_at(i)) == c;
    u64 before = R.scan(mine, total);
    u64 at = 0;
    if (before < need && need <= before + mine)
      for (int i = s_lo; i < s_hi; ++i)
        if (key_of(z_at(i)) == c && ++before == need) at = v_lo + i;
    return (int)R.max(at);
  };
  // largest key c such that the sum of val(key, token) over the tokens of key >= c reaches `target` (three bits a pass)
  auto search = [&](auto val, u64 target) -> unsigned {
    unsigned c = 0;
    for (int shift = 30; shift >= 0; shift -= 3) {
      u64 s[NV];
#pragma unroll
      for (int k = 0; k < NV; ++k) s[k] = 0;
      for (int i = tid; i < n; i += THREADS) {
        const float z = z_at(i);
        const unsigned key = key_of(z);
        if (key < (c | (1u << shift))) continue;
        const u64 x = val(key, z, v_lo + i);
#pragma unroll
        for (int k = 0; k < NV; ++k) {
          const u64 cand = c + ((u64)(k + 1) << shift);  // (beyond 32 bits in the first pass: never reached)
          if (key >= cand) s[k] += x;
        }
      }
      R.sum(s);
      unsigned best = 0;
#pragma unroll
      for (int k = 0; k < NV; ++k)
        if (c + ((u64)(k + 1) << shift) <= 0xffffffffull && s[k] >= target) best = k + 1;
      c += best << shift;
    }
    return c;
  };
  if (top_k > 0 && top_k < V) {
    const unsigned c = search([](unsigned, float, int) -> u64 { return 1; }, top_k);
    u64 s[2] = {0, 0};
    for (int i = tid; i < n; i += THREADS) {
      const unsigned key = key_of(z_at(i));
      s[0] += key > c, s[1] += key == c;
    }
    R.sum(s);
    const u64 need = top_k - s[0];
    cut = c;
    if (need < s[1]) last = nth_of_key(c, need);
  }
  if (top_p > 0.f && top_p < 1.f) {
    auto mass = [&](unsigned key, float z, int v) -> u64 { return kept(key, v) ? weigh(z) : 0; };
    u64 all = 0;
    for (int i = tid; i < n; i += THREADS) all += mass(key_of(z_at(i)), z_at(i), v_lo + i);
    const u64 target = times<true>(top_p, R.sum(all));
    const unsigned c = search(mass, target);
    u64 s[3] = {0, 0, 0};  // mass above c, tokens of key c, their weight
    for (int i = tid; i < n; i += THREADS) {
      const float z = z_at(i);
      const unsigned key = key_of(z);
      if (key > c) s[0] += mass(key, z, v_lo + i);
      else if (key == c) s[1] += 1, s[2] += weigh(z);
    }
    R.sum(s);
    const u64 one = s[2] / s[1], need = (target - s[0] + one - 1) / one;
    if (c > cut) last = V - 1;
    if (need < s[1]) last = min(last, nth_of_key(c, need));  // (at the key where top-k cut, need stays within what it kept)
    cut = c;
  }

  // ---- the draw: every thread has a run of neighbouring tokens ----
  auto weight = [&](int i) -> double {
    const float z = z_at(i);
    if (!kept(key_of(z), v_lo + i)) return 0.0;
    const double w = weigh.scaled(z);
    return w >= least ? w : 0.0;
  };
  u64 mine = 0, total;
  for (int i = s_lo; i < s_hi; ++i) mine += weigh.rounded(weight(i));
  u64 before = R.scan(mine, total);
  const float u = __ldg(p.u + row);
  const u64 at = u > 0.f ? (u < 1.f ? times<false>(u, total) : total - 1) : 0;  // (total is 2^S at least: the largest logit stays)
  if (before <= at && at < before + mine)
    for (int i = s_lo; i < s_hi; ++i) {
      const double w = weight(i);
      before += weigh.rounded(w);
      if (before > at) {
        put(v_lo + i, (float)(w / (double)total));
        break;
      }
    }
}

}  // namespace smp
}  // namespace ls
