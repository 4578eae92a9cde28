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
constexpr int BINS = 2 * THREADS;  // of the distance from the best logit, as far down as a token weighs anything
constexpr int LIST = 2048;         // candidates that one CTA finishes alone

struct Params {
  const void* logits;
  long long ld;
  int rows, V, per;          // per: tokens of a CTA's slice (a multiple of 8)
  int shift;                 // S
  int hist_off;              // bytes from the slice to the histogram and the list behind it
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
  // What precedes this thread's x in this CTA, and its total
  __device__ __forceinline__ u64 block_scan(u64 x, u64& total) {
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
    u64 before = inc - x;
    total = 0;
    for (int w = 0; w < WARPS; ++w) {
      if (w < warp) before += sh[w];
      total += sh[w];
    }
    return before;
  }
  // a[0 .. n) ascending, n <= LIST (a has room for the next power of two)
  __device__ __forceinline__ void sort(u64* a, int n) {
    int size = 2;
    while (size < n) size *= 2;
    __syncthreads();
    for (int i = n + threadIdx.x; i < size; i += THREADS) a[i] = ~0ull;
    __syncthreads();
    for (int k = 2; k <= size; k *= 2)
      for (int j = k / 2; j > 0; j /= 2) {
        for (int i = threadIdx.x; i < size / 2; i += THREADS) {
          const int x = ((i & ~(j - 1)) << 1) | (i & (j - 1)), y = x | j;  // a pair that lies j apart
          const u64 p = a[x], q = a[y];
          if ((p > q) == ((x & k) == 0)) a[x] = q, a[y] = p;
        }
        __syncthreads();
      }
  }
  // What precedes this thread's x in the order (rank, thread), and the total
  __device__ __forceinline__ u64 scan(u64 x, u64& total) {
    u64 mine;
    u64 before = block_scan(x, mine);
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
  __shared__ u64 s_sh[WARPS * NV], s_part[2 * MAX_CS * NV], s_before[3];
  __shared__ int s_found[3];
  __shared__ unsigned s_count;
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
  const float u = __ldg(p.u + row);
  const bool by_k = top_k > 0 && top_k < V, by_p = top_p > 0.f && top_p < 1.f;
  if (by_k || by_p) {
    // Both cuts lie at a place in the ranking, and a histogram over the distance from the best logit says in which bin.  A bin's weights
    // lie between those of its ends, so it brackets the place of top-p, too.  Mostly few tokens rank that high: they are sent to one CTA,
    // which sorts them and does the rest alone.  Tokens too far down to weigh anything are in no bin: a cut among them cuts nothing.
    unsigned* hist = reinterpret_cast<unsigned*>(smp_smem + p.hist_off);
    u64* list = reinterpret_cast<u64*>(smp_smem + p.hist_off + BINS * 4);
    const float scale = (float)fmin(BINS / (double)(p.shift + 2) * weigh.c, 1e30);  // (rounded alike for all: the bins are as monotonous as the logits)
    const double step = weigh.c > 0.0 ? weigh.c / (double)scale : 0.0;             // log2 of the weights' ratio from one end of a bin to the other
    auto bin_of = [&](float z) -> int {  // BINS: none
      const float d = (z == top ? 0.f : top - z) * scale;
      return z > weigh.none && d < (float)BINS ? (int)d : BINS;
    };
    for (int i = tid; i < BINS; i += THREADS) hist[i] = 0;
    if (tid == 0) s_count = 0, s_found[0] = s_found[1] = s_found[2] = BINS;
    __syncthreads();
    u64 all = 0;
    for (int i = tid; i < n; i += THREADS) {
      const float z = z_at(i);
      const int b = bin_of(z);
      if (b < BINS) {
        atomicAdd(hist + b, 1u);
        if (!by_k) all += weigh(z);
      }
    }
    if (by_k) cl.sync();  // the histograms are complete
    else all = R.sum(all);
    // this thread's two bins in the whole cluster, and what lies above them
    u64 cnt[2] = {0, 0};
    for (int q = 0; q < R.n; ++q) {
      const uint2 c = *reinterpret_cast<const uint2*>(cl.map_shared_rank(hist + 2 * tid, q));
      cnt[0] += c.x, cnt[1] += c.y;
    }
    // the first bin at whose end the sum of w[] over the bins reaches target: s_found[slot], the sum before it: s_before[slot]
    auto crossing = [&](u64 w0, u64 w1, u64 target, int slot) {
      u64 total;
      const u64 before = R.block_scan(w0 + w1, total);
      if (before < target && target <= before + w0 + w1) {
        const int second = before + w0 < target;
        s_found[slot] = 2 * tid + second, s_before[slot] = before + (second ? w0 : 0);
      }
      __syncthreads();
    };
    int b_k = BINS;       // the bin where top-k cuts, and how many of it stay
    u64 of_b_k = 0;
    if (by_k) {
      crossing(cnt[0], cnt[1], top_k, 0);
      b_k = s_found[0];
      if (b_k < BINS) of_b_k = top_k - s_before[0];
    }
    auto count_to = [&](int b) -> u64 {  // tokens in the bins up to b
      u64 total;
      R.block_scan((2 * tid <= b ? cnt[0] : 0) + (2 * tid + 1 <= b ? cnt[1] : 0), total);
      return total;
    };
    // bins between which top-p cuts, given the mass it is to reach
    int b_lo = 0, b_hi = BINS - 1;
    auto bracket = [&](u64 target) {
      u64 up[2], down[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int b = 2 * tid + j;
        const u64 c = b < b_k ? cnt[j] : b == b_k ? of_b_k : 0;
        const double one = (double)(1ull << p.shift);
        up[j] = c * (u64)(exp2(-b * step * (1.0 - 1e-6)) * one * (1.0 + 1e-9) + 1.0);
        down[j] = c * (u64)(exp2(-(b + 1) * step * (1.0 + 1e-6)) * one * (1.0 - 1e-9));
      }
      crossing(up[0], up[1], target, 1);
      crossing(down[0], down[1], target, 2);
      b_lo = min(s_found[1], BINS - 1), b_hi = min(s_found[2], min(b_k, BINS - 1));
    };
    if (!by_k) bracket(times<true>(top_p, all));
    const int b_end = by_k ? min(b_k, BINS - 1) : b_hi;
    const u64 n_list = count_to(b_end);

    if (n_list <= LIST) {
      // ---- the candidates go to CTA 0 ----
      u64* far = cl.map_shared_rank(list, 0);
      unsigned* counter = cl.map_shared_rank(&s_count, 0);
      for (int i0 = 0; i0 < n; i0 += THREADS) {
        const int i = i0 + tid;
        const float z = i < n ? z_at(i) : -INFINITY;
        const bool in = i < n && bin_of(z) <= b_end;
        const unsigned who = __ballot_sync(0xffffffffu, in);
        if (who == 0) continue;
        unsigned at = 0;
        if ((tid & 31) == 0) at = atomicAdd(counter, (unsigned)__popc(who));
        at = __shfl_sync(0xffffffffu, at, 0) + __popc(who & ((1u << (tid & 31)) - 1));
        if (in) far[at] = (u64)~key_of(z) << 32 | (unsigned)(v_lo + i);
      }
      cl.sync();
      if (R.rank != 0) return;
      const int N = (int)n_list;
      R.sort(list, N);
      // rank j of the list: thread j / 4
      constexpr int PER = LIST / THREADS;
      auto z_of = [](unsigned key) { return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key); };
      u64 w[PER], sum = 0, total;
      double wd[PER];
      const int limit = by_k ? min(N, top_k) : N;
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        const int at = tid * PER + j;
        wd[j] = at < limit ? weigh.scaled(z_of(~(unsigned)(list[at] >> 32))) : 0.0;
        w[j] = weigh.rounded(wd[j]), sum += w[j];
      }
      u64 before = R.block_scan(sum, total);
      const u64 target = by_p ? (by_k ? times<true>(top_p, total) : times<true>(top_p, all)) : ~0ull;
      int stay = 0;  // of this thread's: those before the target is reached and not below min-p (a prefix of the ranking)
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        stay += tid * PER + j < limit && before < target && w[j] > 0 && wd[j] >= least;
        before += w[j];
      }
      u64 n_kept;
      R.block_scan(stay, n_kept);
      // the kept ones by index
      u64 mine[PER];
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        const u64 e = tid * PER + j < N ? list[tid * PER + j] : 0;
        mine[j] = e << 32 | e >> 32;
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < PER; ++j)
        if (tid * PER + j < (int)n_kept) list[tid * PER + j] = mine[j];
      __syncthreads();
      R.sort(list, (int)n_kept);
      sum = 0;
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        const int at = tid * PER + j;
        wd[j] = at < (int)n_kept ? weigh.scaled(z_of(~(unsigned)list[at])) : 0.0;
        w[j] = weigh.rounded(wd[j]), sum += w[j];
      }
      before = R.block_scan(sum, total);
      const u64 at = u > 0.f ? (u < 1.f ? times<false>(u, total) : total - 1) : 0;
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        if (before <= at && at < before + w[j]) put((int)(list[tid * PER + j] >> 32), (float)(wd[j] / (double)total));
        before += w[j];
      }
      return;
    }

    // ---- many tokens stay: the cuts are found by all CTAs together ----
    // this CTA's tokens of the bins b0 .. b1, listed where they fit (all CTAs decide alike)
    bool listed = false;
    unsigned n_mine = 0;
    auto gather = [&](int b0, int b1) {
      __syncthreads();
      if (tid == 0) s_count = 0;
      __syncthreads();
      for (int i = tid; i < n; i += THREADS) {
        const float z = z_at(i);
        const int b = bin_of(z);
        if (b < b0 || b > b1) continue;
        const unsigned at = atomicAdd(&s_count, 1u);
        if (at < LIST) list[at] = (u64)key_of(z) << 32 | (unsigned)(v_lo + i);
      }
      __syncthreads();
      n_mine = s_count;
      listed = R.max(n_mine) <= LIST;
    };
    auto each = [&](int b0, int b1, auto f) {  // f(key, logit, token) for this thread's tokens of the gathered bins
      if (listed) {
        for (unsigned i = tid; i < n_mine; i += THREADS) {
          const unsigned key = (unsigned)(list[i] >> 32);
          f(key, __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key), (int)(unsigned)list[i]);
        }
      } else {
        for (int i = tid; i < n; i += THREADS) {
          const float z = z_at(i);
          const int b = bin_of(z);
          if (b >= b0 && b <= b1) f(key_of(z), z, v_lo + i);
        }
      }
    };
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
    // largest key c such that the sum of val(key, logit, token) over the gathered tokens of key >= c reaches `target` (three bits a pass)
    auto search = [&](int b0, int b1, auto val, u64 target) -> unsigned {
      unsigned c = 0;
      for (int shift = 30; shift >= 0; shift -= 3) {
        u64 s[NV];
#pragma unroll
        for (int k = 0; k < NV; ++k) s[k] = 0;
        each(b0, b1, [&](unsigned key, float z, int v) {
          if (key < (c | (1u << shift))) return;
          const u64 x = val(key, z, v);
#pragma unroll
          for (int k = 0; k < NV; ++k) {
            const u64 cand = c + ((u64)(k + 1) << shift);  // (beyond 32 bits in the first pass: never reached)
            if (key >= cand) s[k] += x;
          }
        });
        R.sum(s);
        unsigned best = 0;
#pragma unroll
        for (int k = 0; k < NV; ++k)
          if (c + ((u64)(k + 1) << shift) <= 0xffffffffull && s[k] >= target) best = k + 1;
        c += best << shift;
      }
      return c;
    };
    if (b_k < BINS) {
      gather(b_k, b_k);
      const unsigned c = search(b_k, b_k, [](unsigned, float, int) -> u64 { return 1; }, of_b_k);
      u64 s[2] = {0, 0};
      each(b_k, b_k, [&](unsigned key, float, int) { s[0] += key > c, s[1] += key == c; });
      R.sum(s);
      const u64 need = of_b_k - s[0];
      cut = c;
      if (need < s[1]) last = nth_of_key(c, need);
    }
    if (by_p) {
      auto mass = [&](unsigned key, float z, int v) -> u64 { return kept(key, v) ? weigh(z) : 0; };
      if (by_k) {
        all = 0;
        for (int i = tid; i < n; i += THREADS) all += mass(key_of(z_at(i)), z_at(i), v_lo + i);
        all = R.sum(all);
        bracket(times<true>(top_p, all));
      }
      u64 above = 0;
      for (int i = tid; i < n; i += THREADS) {
        const float z = z_at(i);
        if (bin_of(z) < b_lo) above += weigh(z);
      }
      const u64 target = times<true>(top_p, all) - R.sum(above);
      gather(b_lo, b_hi);
      const unsigned c = search(b_lo, b_hi, mass, target);
      u64 s[3] = {0, 0, 0};  // mass above c, tokens of key c, their weight
      each(b_lo, b_hi, [&](unsigned key, float z, int v) {
        if (key > c) s[0] += mass(key, z, v);
        else if (key == c) s[1] += 1, s[2] += weigh(z);
      });
      R.sum(s);
      const u64 one = s[2] / s[1], need = (target - s[0] + one - 1) / one;
      if (c > cut) last = V - 1;
      if (need < s[1]) last = min(last, nth_of_key(c, need));  // (at the key where top-k cut, need stays within what it kept)
      cut = c;
    }
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
