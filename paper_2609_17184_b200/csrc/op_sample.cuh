// One token per row of logits by temperature, top-k, top-p and min-p from a given uniform number: w = exp((z - max) / T), ranked by logit (ties:
// lower index first); the token is the first, by index, at which the running sum of the kept weights exceeds u times their sum.
//
// Which side of a border a sum lies on decides the token, so no sum may depend on the order of its additions: a weight is evaluated in fp64 (2^y by a table of 2^(j/256) and a polynomial of degree 3: 1.4e-13) and rounded ONCE to a multiple
// of 2^-S, S = 61 - ceil(log2 V) (44 at 128K tokens, 48 at most); from there on everything - sums over the vocabulary, p times a sum, u times a sum -
// is exact integer arithmetic.  Sums are the same in every order and for every number of CTAs.  A token below 2^-(S+1) of the best weighs nothing, and a sum is off by
// at most V 2^-(S+1) of the best (2^-26 for the largest vocabulary, 2^-36 for 8192 tokens): a uniform number in fp32 is one of 2^-24 apart at 1.
//
// A cluster of CTAs holds a row in shared memory, so the logits are read from HBM once; what bounds a call is then the chain of passes over
// a CTA's slice and of hand-overs in the cluster (some 1000 cycles each):
//   1  load, largest logit                                                     all rows
//   2  tokens that a small k may keep, by the threads' own maxima              rows with a top-k of few
//   3  histogram over the distance from the best: tokens and places in a bin   other rows with top-k or top-p
//   4  exact mass, tokens of the bins where top-p may cut                      rows with top-p
//   5  exact mass of what stays, by index                                      all rows of many kept tokens
// 256 rows of 50,001 16-bit logits with k = 50 take 28 us (41 by way of the histogram), 64 rows of 128,256 with settings of their own 70 us, one row of
// 49,152 with top-p 22 us, 8 rows without filters 8 us.  Measured and left out: 1024 threads a CTA (+5 to +100 %), logits left in the L2 instead of shared
// memory (+10 to +20 % a pass), sorting up to 512 candidates instead of comparing up to 256 with each other (+30 %).
#pragma once
#include <cooperative_groups.h>

#include "op_common.cuh"

namespace ls {
namespace smp {
namespace cg = cooperative_groups;
typedef unsigned long long u64;

constexpr int THREADS = 512, WARPS = THREADS / 32;
constexpr int MAX_CS = 8;
constexpr int NV = 7;              // sums taken together
constexpr int BINS = 2 * THREADS;  // of the distance from the best logit, as far down as a token weighs anything
constexpr int LIST = 2048;         // tokens one CTA can be sent, an equal part of them by each CTA
constexpr int SOLO = 256;          // candidates with which one CTA finishes a row alone
static_assert(2 * SOLO == THREADS, "the list's companion holds a pair for each of them, or a sum for each thread");
constexpr int QUICK = 192;         // top-k times CTAs of a row up to which that is tried without a histogram (some half as many tokens more are sent)
constexpr int LINE = 160;          // tokens a warp has room for: 31 that wait and four a lane
static_assert(WARPS * LINE * 4 <= (LIST + 2 * SOLO) * 8, "in the list's place");
constexpr int MAX_VOCAB_BITS = 18;

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
__device__ __forceinline__ float logit_of(unsigned key) { return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key); }
// a token's place in the ranking, ascending
__device__ __forceinline__ u64 place_of(float z, int v) { return (u64)~key_of(z) << MAX_VOCAB_BITS | (unsigned)v; }
__device__ __forceinline__ float logit_at(u64 place) { return logit_of(~(unsigned)(place >> MAX_VOCAB_BITS)); }
__device__ __forceinline__ int token_at(u64 place) { return (int)((unsigned)place & ((1u << MAX_VOCAB_BITS) - 1)); }
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
  const double* table;  // 2^(j / 256)
  double top, c;        // largest logit, 256 log2(e) / T
  int shift;
  float none;           // logits up to this one weigh nothing: -inf, or all finite ones beside an infinity
  unsigned far;         // high word of -256 (S + 2): what lies further down is taken to lie there (and weighs nothing)
  // No branch, so that the chains of neighbouring tokens overlap (one alone takes some 250 cycles).
  __device__ __forceinline__ double scaled(float z) const {
    double y = (widen(z) - top) * c;
    // (y <= 0: a larger high word is further down; the low word does not matter there)
    y = __hiloint2double((int)min(z > none ? (unsigned)__double2hiint(y) : 0xffffffffu, far), __double2loint(y));
    return power(y);
  }
  // 2^(S + y / 256) for a y from 0 down to -256 (S + 2)
  __device__ __forceinline__ double power(double y) const {
    const double magic = 6755399441055744.0;  // 1.5 * 2^52: the sum's low word is y to the nearest integer
    const double t = y + magic;
    const int k = __double2loint(t);
    const double f = y - (t - magic);  // 2^(y / 256) = 2^(k / 256) 2^(f / 256), |f| <= 1 / 2
    constexpr double a = 0.69314718055994530942 / 256;
    const double q = fma(f, fma(f, fma(f, a * a * a / 6, a * a / 2), a), 1.0);
    const double w = table[k & 255];
    return q * __hiloint2double(__double2hiint(w) + ((k >> 8) + shift) * (1 << 20), __double2loint(w));
  }
  __device__ __forceinline__ static u64 rounded(double w) { return (u64)__double_as_longlong(w + 4503599627370496.0) & 0xfffffffffffffull; }  // (below 2^52)
  __device__ __forceinline__ u64 operator()(float z) const { return rounded(scaled(z)); }
};

// Sums and maxima over a CTA or the cluster: warps, then the CTA's partials in every CTA's memory, two sets of slots in turn
struct Cluster {
  cg::cluster_group cl;
  int n, rank, phase;
  u64* sh;    // [WARPS][NV]
  u64* part;  // [2][MAX_CS][NV]

  template <int N, typename Op>
  __device__ __forceinline__ void fold_block(u64 (&v)[N], Op op) {  // v valid in thread i < N as v[0], for value i
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
  }
  template <int N, typename Op>
  __device__ __forceinline__ void fold(u64 (&v)[N], Op op) {
    fold_block(v, op);
    if ((int)threadIdx.x < N * n) {  // one thread per value and CTA that is told
      const int i = threadIdx.x % N, q = threadIdx.x / N;
      u64 r = sh[i];
      for (int w = 1; w < WARPS; ++w) r = op(r, sh[w * NV + i]);
      *cl.map_shared_rank(part + (phase * MAX_CS + rank) * NV + i, q) = r;
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
  __device__ __forceinline__ u64 max(u64 x) {
    u64 v[1] = {x};
    fold(v, [](u64 a, u64 b) { return a > b ? a : b; });
    return v[0];
  }
  template <int N>
  __device__ __forceinline__ void sum_block(u64 (&v)[N]) {
    fold_block(v, [](u64 a, u64 b) { return a + b; });
#pragma unroll
    for (int i = 0; i < N; ++i) {
      u64 r = 0;
      for (int w = 0; w < WARPS; ++w) r += sh[w * NV + i];
      v[i] = r;
    }
  }
  // What precedes this thread's x in this CTA, and its total; and the same of a second value
  __device__ __forceinline__ u64 scan_block(u64 x, u64& total, u64 x2, u64& before2, u64& total2) const {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    u64 inc = x, inc2 = x2;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const u64 t = __shfl_up_sync(0xffffffffu, inc, o), t2 = __shfl_up_sync(0xffffffffu, inc2, o);
      if (lane >= o) inc += t, inc2 += t2;
    }
    __syncthreads();
    if (lane == 31) sh[warp] = inc, sh[WARPS + warp] = inc2;
    __syncthreads();
    u64 before = inc - x;
    before2 = inc2 - x2, total = total2 = 0;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
      const u64 s = sh[w], s2 = sh[WARPS + w];
      if (w < warp) before += s, before2 += s2;
      total += s, total2 += s2;
    }
    return before;
  }
  __device__ __forceinline__ u64 scan_block(u64 x, u64& total) const {
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
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
      const u64 s = sh[w];
      if (w < warp) before += s;
      total += s;
    }
    return before;
  }
  // a[0 .. n) ascending (a has room for the next power of two)
  __device__ __noinline__ void sort(u64* a, int n) const {
    int size = 2;
    while (size < n) size *= 2;
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
    u64 before = scan_block(x, mine);
    if ((int)threadIdx.x < n) *cl.map_shared_rank(part + (phase * MAX_CS + rank) * NV, threadIdx.x) = mine;
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

// four neighbouring logits of a slice
template <typename T>
__device__ __forceinline__ float4 quad_of(const T* z_sm, int i) {
  if constexpr (sizeof(T) == 4) {
    return reinterpret_cast<const float4*>(z_sm)[i];
  } else {
    const uint2 w = reinterpret_cast<const uint2*>(z_sm)[i];
    const T* e = reinterpret_cast<const T*>(&w);
    return make_float4(to_f32<T>(e[0]), to_f32<T>(e[1]), to_f32<T>(e[2]), to_f32<T>(e[3]));
  }
}
// One logit's weight where few are taken.  (Out of line: a row runs this code once, and what is not in the instruction cache costs its way from the
// L2 - inlined throughout, the kernel was 390 KB.)
__device__ __noinline__ double weigh_one(const Weigher& g, float z) { return g.scaled(z); }

template <typename T>
__global__ void __launch_bounds__(THREADS, 2) sample_kernel(const __grid_constant__ Params p) {
  extern __shared__ __align__(16) unsigned char smp_smem[];
  __shared__ double s_table[256];
  __shared__ u64 s_sh[WARPS * NV], s_part[2 * MAX_CS * NV], s_before[3], s_upto, s_cut;
  __shared__ int s_found[3];
  __shared__ unsigned s_mine[3], s_sent[3][MAX_CS];  // tokens this CTA has sent, and what every CTA has, each time
  cg::cluster_group cl = cg::this_cluster();
  Cluster R{cl, (int)cl.num_blocks(), (int)cl.block_rank(), 0, s_sh, s_part};
  const int tid = threadIdx.x, row = blockIdx.x / R.n, V = p.V;
  const int v_lo = min(V, R.rank * p.per), n = min(V, v_lo + p.per) - v_lo;  // this CTA's tokens
  const float temp = p.temperature ? __ldg(p.temperature + row) : 1.f, u = __ldg(p.u + row);
  const float top_p = p.top_p ? __ldg(p.top_p + row) : 1.f, min_p = p.min_p ? __ldg(p.min_p + row) : 0.f;
  const int top_k = p.top_k ? __ldg(p.top_k + row) : 0;
  // Another CTA's shared memory is there only once that CTA has started: each says so here, and the slice's load covers the wait for the others
  if (R.n > 1) asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");

  // ---- the slice as it lies in memory, 16 bytes at a time; what of the first and the last 16 is not the slice's counts as masked out.  (A logit that is
  // no number is treated so wherever it is compared.) ----
  constexpr int VEC = 16 / sizeof(T);
  const T* src = static_cast<const T*>(p.logits) + row * p.ld + v_lo;
  const int head = (int)((reinterpret_cast<uintptr_t>(src) & 15) / sizeof(T));  // elements from the 16-byte boundary before the slice
  const int n_piece = (head + n + VEC - 1) / VEC, whole = (head + n) / VEC, n_quad = n_piece * (VEC / 4), v_first = v_lo - head;
  T* z_sm = reinterpret_cast<T*>(smp_smem);  // element e: token v_first + e
  float top = -INFINITY;
  {
    const uint4* vs = reinterpret_cast<const uint4*>(src - head);
#pragma unroll 4
    for (int i = tid + (head != 0); i < whole; i += THREADS) {
      const uint4 w = __ldcs(vs + i);
      reinterpret_cast<uint4*>(z_sm)[i] = w;
      const T* e = reinterpret_cast<const T*>(&w);
#pragma unroll
      for (int j = 0; j < VEC; ++j) top = fmaxf(top, to_f32<T>(e[j]));  // (of a number and none: the number)
    }
    const int e = tid < VEC ? tid : whole * VEC + tid - VEC;  // the first piece's and the last one's elements
    if (tid < VEC ? head != 0 || whole == 0 : tid < 2 * VEC && whole < n_piece && (whole > 0 || head == 0)) {
      const T z = e >= head && e < head + n ? src[e - head] : T(-INFINITY);
      z_sm[e] = z, top = fmaxf(top, to_f32<T>(z));
    }
  }
  if (tid < 256) s_table[tid] = exp2((double)tid / 256);
  const float own_top = top;
  if (R.n > 1) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");  // (before the first word that goes to another CTA)
  const unsigned top_key = (unsigned)R.max(key_of(top));
  top = logit_of(top_key);
  auto put = [&](int token, float prob) {
    p.token[row] = token;
    if (p.prob) p.prob[row] = prob;
  };
  const bool writer = R.rank == 0 && tid == 0;
  if (top == -INFINITY) {  // nothing to choose from
    if (writer) put(-1, 0.f);
    return;
  }
  if (!(temp > 0.f)) {  // greedy: the first of the largest
    unsigned first = 0;
#pragma unroll 1
    for (int i = tid; i < n_quad; i += THREADS) {
      const float4 q = quad_of(z_sm, i);
      const int j = q.x == top ? 0 : q.y == top ? 1 : q.z == top ? 2 : q.w == top ? 3 : 4;
      if (j < 4) first = max(first, 0x7fffffffu - (unsigned)(v_first + i * 4 + j));
    }
    first = (unsigned)R.max(first);
    if (writer) put((int)(0x7fffffffu - first), 1.f);
    return;
  }
  const double log2_t = 1.4426950408889634074 / (double)temp;
  const Weigher weigh = {s_table, widen(top), 256.0 * log2_t, p.shift, top == INFINITY ? 3.402823466e38f : -INFINITY,
                         (unsigned)__double2hiint(-256.0 * (p.shift + 2))};
  const double one = (double)(1ull << p.shift), least = min_p > 0.f ? (double)fminf(min_p, 1.f) * one : 0.0;
  const bool by_k = top_k > 0 && top_k < V, by_p = top_p > 0.f && top_p < 1.f;

  // ---- the cut: tokens of places up to this one stay ----
  u64 cut = ~0ull;
  if (by_k || by_p) {
    // A histogram over the distance from the best logit says in which bin a cut lies.  Beside its tokens a bin counts how far down in it they
    // lie, in 1 / 1024 of its width: by the chord and the tangent of 2^-x that brackets its mass to some 2^-10 of the width's 3 %, so the place
    // of top-p comes out to within a bin or two.  Tokens too far down to weigh anything are in no bin: a cut among them cuts nothing.
    unsigned* hist = reinterpret_cast<unsigned*>(smp_smem + p.hist_off);  // [BINS]: tokens, then [BINS]: how far down
    u64* list = reinterpret_cast<u64*>(hist + 2 * BINS);
    u64* weights = list + LIST;
    const float scale = (float)fmin(BINS / (double)(p.shift + 2) * log2_t, 1e30);  // (rounded alike for all: the bins are as monotonous as the logits)
    const double step = log2_t > 0.0 ? log2_t / (double)scale : 0.0;               // log2 of the weights' ratio from one end of a bin to the other
    auto depth_of = [&](float z) -> float {  // BINS or more: in no bin
      const float d = (z == top ? 0.f : top - z) * scale;
      return z > weigh.none ? d : (float)BINS;
    };
    if (tid == 0) s_cut = ~0ull, s_mine[0] = s_mine[1] = s_mine[2] = 0, s_found[0] = s_found[1] = s_found[2] = BINS;
    // the first bin at whose end the sum of w over the bins reaches target: s_found[slot]; the sum before it: s_before[slot]
    auto crossing = [&](u64 before, u64 w0, u64 w1, u64 target, int slot) {
      if (before < target && target <= before + w0 + w1) {
        const int second = before + w0 < target;
        s_found[slot] = 2 * tid + second, s_before[slot] = before + (second ? w0 : 0);
      }
    };
    const unsigned room = LIST / R.n;
    bool solo = false;
    u64 all = 0;  // the mass top-p is a part of
    u64 cnt[2] = {0, 0}, low[2] = {0, 0}, n_before = 0, n_all;  // this thread's two bins in the whole cluster, and tokens of the bins above them
    int b_k = BINS;                                             // the bin where top-k cuts, and how many of it stay
    u64 of_b_k = 0;
    // First top-k (or, where few tokens are candidates at all, whatever cuts there are), then top-p.  Before that, for a small k: at least k tokens reach
    // the k-th largest of the threads' own maxima, and mostly not many more; if they are as few as that, no histogram of all tokens is needed.
#pragma unroll 1
    for (int step_ = by_k && top_k * R.n <= QUICK ? -1 : 0; step_ < 2; ++step_) {
      int b_lo = 0, b_hi = BINS - 1;
      if (step_ <= 0) {
        for (int i = tid; i < BINS / 2; i += THREADS) reinterpret_cast<uint4*>(hist)[i] = make_uint4(0, 0, 0, 0);
        __syncthreads();
        if (step_ < 0) {
          const float d = depth_of(own_top);
          if (d < (float)BINS) atomicAdd(hist + (int)d, 1u);
          __syncthreads();
          const uint2 c = *reinterpret_cast<const uint2*>(hist + 2 * tid);
          crossing(R.scan_block(c.x + c.y, n_all), c.x, c.y, top_k, 0);
          __syncthreads();
          b_hi = min(s_found[0], BINS - 1);
          solo = true;
        } else {
          solo = false;
#pragma unroll 2
          for (int i = tid; i < n_quad; i += THREADS) {
            const float4 q = quad_of(z_sm, i);
            const float z[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float d = depth_of(z[j]);
              if (d < (float)BINS) {
                const int b = (int)d;
                atomicAdd(hist + b, 1u);
                if (by_p) atomicAdd(hist + BINS + b, (unsigned)((d - (float)b) * 1024.f));
              }
            }
          }
          cl.sync();
#pragma unroll 8
          for (int q = 0; q < R.n; ++q) {
            const unsigned* h = cl.map_shared_rank(hist, q) + 2 * tid;
            const uint2 c = *reinterpret_cast<const uint2*>(h), l = *reinterpret_cast<const uint2*>(h + BINS);
            cnt[0] += c.x, cnt[1] += c.y, low[0] += l.x, low[1] += l.y;
          }
          n_before = R.scan_block(cnt[0] + cnt[1], n_all);
          if (by_k) {
            if (tid == 0) s_found[0] = BINS;
            __syncthreads();
            crossing(n_before, cnt[0], cnt[1], top_k, 0);
            __syncthreads();
            b_k = s_found[0];
            if (b_k < BINS) of_b_k = top_k - s_before[0];
          }
        }
      }
      if (by_p && step_ >= 0 && by_k == (step_ == 1)) {
        // Bins between which top-p cuts.  Weights of a bin of c tokens and summed depths D (in bins; c / 1024 may be missing): with r = 2^-step, at
        // depth x of it r^x <= 1 - x (1 - r) (chord) and r^x >= 1 + x ln r (tangent), times the weight at the bin's upper end.
        u64 up[2], down[2];
        const double limit = -256.0 * (p.shift + 2), r = weigh.power(fmax(-256.0 * step, limit)) / one;
#pragma unroll 1
        for (int j = 0; j < 2; ++j) {
          const int b = 2 * tid + j;
          const bool part = b == b_k;  // of the bin where top-k cut only of_b_k tokens are left, whichever
          const double c = b < b_k ? (double)(j ? cnt[1] : cnt[0]) : part ? (double)of_b_k : 0.0, deep = (double)(j ? low[1] : low[0]) / 1024;
          const double at = weigh.power(fmax(-256.0 * step * b, limit));
          const double d0 = part ? 0.0 : deep, d1 = part ? c : fmin(c, deep + c / 1024);
          const u64 hi = (u64)(at * (c - d0 * (1.0 - r)) * (1.0 + 1e-5) + c);
          u64 lo = (u64)(at * fmax(c + d1 * -0.69314718055994530942 * step, c * r) * (1.0 - 1e-5));  // (1e-5: the roundings of a depth)
          lo = lo > (u64)c ? lo - (u64)c : 0;                                                        // (weights are rounded)
          if (j) up[1] = hi, down[1] = lo;
          else up[0] = hi, down[0] = lo;
        }
        u64 up_all, down_all, down_before;
        const u64 up_before = R.scan_block(up[0] + up[1], up_all, down[0] + down[1], down_before, down_all);
        crossing(up_before, up[0], up[1], times<true>(top_p, down_all), 1);      // the mass may be this small: it is reached here at the earliest
        crossing(down_before, down[0], down[1], times<true>(top_p, up_all), 2);  // ... or this large
        __syncthreads();
        b_lo = min(s_found[1], BINS - 1), b_hi = min(s_found[2], min(b_k, BINS - 1));
      }
      if (step_ < 0) {
      } else if (step_ == 0) {
        const int b_end = by_k ? min(b_k, BINS - 1) : b_hi;
        if (2 * tid == (b_end & ~1)) s_upto = n_before + cnt[0] + (b_end & 1 ? cnt[1] : 0);
        __syncthreads();
        solo = s_upto <= SOLO;
        if (solo) b_lo = 0, b_hi = b_end;
        else if (b_k < BINS) b_lo = b_hi = b_k;
        else if (!by_p || by_k) continue;  // (no cut, or top-p's is to come)
      } else if (!by_p || !by_k) {
        break;  // (found in the first turn)
      }
      const bool k_cut = by_k && step_ <= 0, mass = by_p && !k_cut;
      // ---- this CTA's tokens of the bins b_lo .. b_hi go, in no order, to its part of CTA 0's list, and their number to all; with `mass`, also: the exact weight
      // of what is kept so far, and the part of it in the bins before b_lo ----
      u64 sums[2] = {0, 0};
      {
        u64* to = cl.map_shared_rank(list, 0) + R.rank * room;
        const float f0 = (float)b_lo, f1 = (float)(b_hi + 1);  // (b_hi < BINS)
#pragma unroll 2
        for (int i = tid; i < n_quad; i += THREADS) {
          const float4 q = quad_of(z_sm, i);
          const float z[4] = {q.x, q.y, q.z, q.w};
          if (mass) {
            u64 w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = weigh(z[j]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              if (cut != ~0ull && place_of(z[j], v_first + i * 4 + j) > cut) w[j] = 0;
              sums[0] += w[j], sums[1] += depth_of(z[j]) < f0 ? w[j] : 0;
            }
          }
          if (!(depth_of(fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3]))) < f1)) continue;  // (the nearest of the four)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float d = depth_of(z[j]);
            if (d >= f0 && d < f1) {
              const unsigned at = atomicAdd(s_mine + step_ + 1, 1u);
              if (at < room) to[at] = place_of(z[j], v_first + i * 4 + j);
            }
          }
        }
        __syncthreads();
        if (tid < R.n) *cl.map_shared_rank(&s_sent[step_ + 1][R.rank], tid) = s_mine[step_ + 1];
      }
      R.sum(sums);  // (and what was sent has arrived)
      if (mass) all = sums[0];
      unsigned most = 0, of_all = 0;
      for (int q = 0; q < R.n; ++q) most = max(most, s_sent[step_ + 1][q]), of_all += s_sent[step_ + 1][q];
      if (step_ < 0 && (most > room || of_all > SOLO)) continue;
      const u64 target = k_cut ? of_b_k : times<true>(top_p, all) - sums[1];
      if (most <= room) {
        if (R.rank == 0) {
          // ---- CTA 0 closes the gaps in its list ----
          int N = 0;
          {
            u64 e[LIST / THREADS];
            int at[LIST / THREADS];
#pragma unroll
            for (int j = 0; j < LIST / THREADS; ++j) {
              const int i = tid + j * THREADS, q = i / (int)room, k = i - q * (int)room;
              e[j] = list[i], at[j] = -1;
              if (q < R.n && k < (int)s_sent[step_ + 1][q]) {
                at[j] = k;
                for (int x = 0; x < q; ++x) at[j] += s_sent[step_ + 1][x];
              }
            }
            for (int q = 0; q < R.n; ++q) N += s_sent[step_ + 1][q];
            __syncthreads();
#pragma unroll
            for (int j = 0; j < LIST / THREADS; ++j)
              if (at[j] >= 0) list[at[j]] = e[j];
            __syncthreads();
          }
          auto tell = [&](u64 c) {
            for (int q = 0; q < R.n; ++q) *cl.map_shared_rank(&s_cut, q) = c;
          };
          auto worth = [&](u64 place) -> u64 {  // in the sum that is to reach the target
            return k_cut ? 1 : place <= cut ? Weigher::rounded(weigh_one(weigh, logit_at(place))) : 0;
          };
          u64 goal = target;
          if (N > SOLO) {
            // the bins are cut finer, a thread each, and only the part where the target is reached stays in the list
            u64* fine = weights;  // [THREADS]
            fine[tid] = 0;
            if (tid == 0) s_mine[0] = 0;
            __syncthreads();
            const float f0 = (float)b_lo, per = THREADS / (float)(b_hi + 1 - b_lo);
            auto part_of = [&](u64 place) -> int { return min((int)((depth_of(logit_at(place)) - f0) * per), THREADS - 1); };
            u64 e[LIST / THREADS];
#pragma unroll 1
            for (int i = tid; i < N; i += THREADS) {
              const u64 place = list[i];
              atomicAdd(fine + part_of(place), worth(place));
            }
            __syncthreads();
            u64 total;
            const u64 mine = fine[tid], before = R.scan_block(mine, total);
            if (before < goal && goal <= before + mine) s_found[0] = tid, s_before[0] = before;
            __syncthreads();
            const int where = s_found[0];
            goal -= s_before[0];
#pragma unroll
            for (int j = 0; j < LIST / THREADS; ++j) e[j] = tid + j * THREADS < N ? list[tid + j * THREADS] : ~0ull;
            __syncthreads();
#pragma unroll
            for (int j = 0; j < LIST / THREADS; ++j)
              if (e[j] != ~0ull && part_of(e[j]) == where) list[atomicAdd(s_mine, 1u)] = e[j];
            __syncthreads();
            N = (int)s_mine[0];
          }
          if (N <= SOLO) {
            // Few tokens: a group of threads for each, which goes over all others.  First what precedes it in the ranking: how many, and their weight
            ulonglong2* pairs = reinterpret_cast<ulonglong2*>(weights);  // [SOLO]: place, weight
            int lanes = 32;
            while (lanes * N > THREADS) lanes >>= 1;
            const int at_ = tid / lanes, part = tid & (lanes - 1);
            const bool have = at_ < N, first = have && part == 0;
            const u64 place = have ? list[at_] : ~0ull;
            double wd = 0.0;
            u64 w = 0;
            if (have) {
              if (solo) wd = weigh_one(weigh, logit_at(place)), w = Weigher::rounded(wd);
              else w = worth(place);
            }
            if (first) pairs[at_] = make_ulonglong2(place, w);
            __syncthreads();
            u64 before = 0;
            int rank = 0;
#pragma unroll 4
            for (int i = part; i < N; i += lanes) {
              const ulonglong2 x = pairs[i];
              if (x.x < place) before += x.y, ++rank;
            }
            for (int o = lanes >> 1; o > 0; o >>= 1) before += __shfl_xor_sync(0xffffffffu, before, o), rank += __shfl_xor_sync(0xffffffffu, rank, o);
            if (!solo) {
              if (first && before < goal && goal <= before + w) tell(place);
            } else {
              const bool in_k = have && (!by_k || rank < top_k);
              u64 s[1] = {first && in_k ? w : 0};
              if (by_k && by_p) R.sum_block(s);
              const u64 reach = by_p ? times<true>(top_p, by_k ? s[0] : all) : ~0ull;
              const bool stays = in_k && before < reach && wd >= least;
              __syncthreads();
              if (first && !stays) pairs[at_].y = 0;
              s[0] = first && stays ? w : 0;
              R.sum_block(s);
              const u64 total = s[0], at = u > 0.f ? (u < 1.f ? times<false>(u, total) : total - 1) : 0;
              // ... and now, of those that stay, what precedes it by index
              const unsigned token = (unsigned)token_at(place);
              before = 0;
#pragma unroll 4
              for (int i = part; i < N; i += lanes) {
                const ulonglong2 x = pairs[i];
                if ((unsigned)token_at(x.x) < token) before += x.y;
              }
              for (int o = lanes >> 1; o > 0; o >>= 1) before += __shfl_xor_sync(0xffffffffu, before, o);
              if (first && stays && before <= at && at < before + w) put((int)token, (float)(wd / (double)total));
              return;
            }
          } else {
            R.sort(list, N);
            constexpr int PER = LIST / THREADS;
            u64 w[PER], sum = 0, total;
#pragma unroll
            for (int j = 0; j < PER; ++j) w[j] = tid * PER + j < N ? worth(list[tid * PER + j]) : 0, sum += w[j];
            u64 before = R.scan_block(sum, total);
#pragma unroll
            for (int j = 0; j < PER; ++j) {
              if (before < goal && goal <= before + w[j]) tell(list[tid * PER + j]);
              before += w[j];
            }
          }
        }
        if (solo) return;
        cl.sync();
        cut = min(cut, s_cut);
      } else {
        // ---- more than fit (many equal logits): the smallest place c such that the sum over the places up to c reaches target, three bits of it a pass of all CTAs ----
        u64 c = 0, base = 0;
#pragma unroll 1
        for (int shift = 48; shift >= 0; shift -= 3) {
          u64 s[NV];
#pragma unroll
          for (int k = 0; k < NV; ++k) s[k] = 0;
#pragma unroll 1
          for (int e = tid; e < n_quad * 4; e += THREADS) {
            const float z = to_f32<T>(z_sm[e]), d = depth_of(z);
            const u64 place = place_of(z, v_first + e);
            if (!(d >= (float)b_lo && d < (float)(b_hi + 1)) || place >> (shift + 3) != c >> (shift + 3)) continue;
            const u64 x = k_cut ? 1 : place <= cut ? Weigher::rounded(weigh_one(weigh, z)) : 0;
            const int digit = (int)(place >> shift) & 7;
#pragma unroll
            for (int k = 0; k < NV; ++k) s[k] += digit <= k ? x : 0;
          }
          R.sum(s);
          int digit = NV;
          u64 skipped = 0;
#pragma unroll
          for (int k = NV - 1; k >= 0; --k)
            if (base + s[k] >= target) digit = k;
#pragma unroll
          for (int k = 0; k < NV; ++k)
            if (k + 1 == digit) skipped = s[k];
          base += skipped, c |= (u64)digit << shift;
        }
        cut = min(cut, c);
      }
    }
  }

  // ---- the draw: every warp has a run of neighbouring quads, its lanes take them in turn ----
  const int lane = tid & 31, warp = tid >> 5, run = ((n_quad + THREADS - 1) / THREADS) * 32, r_lo = min(n_quad, warp * run), r_hi = min(n_quad, r_lo + run);
  u64 mine = 0, total;
  if (cut == ~0ull && least == 0.0) {
#pragma unroll 2
    for (int i = r_lo + lane; i < r_hi; i += 32) {
      const float4 q = quad_of(z_sm, i);
      mine += (weigh(q.x) + weigh(q.y)) + (weigh(q.z) + weigh(q.w));
    }
  } else {
    // Mostly few stay: those that rank ahead of the cut and are not far below what min-p asks for are put in a row, and weighed 32 at a time
    const float low = least > 0.0 && top < INFINITY ? top + temp * (1.001f * __logf(fminf(min_p, 1.f)) - 1e-5f) - 1e-6f * fabsf(top) : -INFINITY;
    const unsigned key_lo = max(~(unsigned)(cut >> MAX_VOCAB_BITS), low > -INFINITY ? key_of(low) : 0u);  // (of no cut: 0)
    // (in the list's place: the histogram ahead of it may still be read by the cluster's other CTAs, where no cut was looked for in the list)
    unsigned* line = reinterpret_cast<unsigned*>(smp_smem + p.hist_off + BINS * 8) + warp * LINE;
    int in_line = 0;
    auto worth = [&](unsigned e) -> u64 {
      const double w = weigh_one(weigh, to_f32<T>(z_sm[e]));
      return w >= least ? Weigher::rounded(w) : 0;
    };
#pragma unroll 1
    for (int i0 = r_lo; i0 < r_hi; i0 += 32) {
      const int i = i0 + lane;
      const float4 q = quad_of(z_sm, min(i, r_hi - 1));
      const float z[4] = {q.x, q.y, q.z, q.w};
      unsigned stays[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) stays[j] = __ballot_sync(0xffffffffu, i < r_hi && key_of(z[j]) >= key_lo && place_of(z[j], v_first + i * 4 + j) <= cut);
      if ((stays[0] | stays[1] | stays[2] | stays[3]) == 0) continue;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (stays[j] >> lane & 1) line[in_line + __popc(stays[j] & ((1u << lane) - 1))] = i * 4 + j;
        in_line += __popc(stays[j]);
      }
      __syncwarp();
#pragma unroll 1
      for (; in_line >= 32; in_line -= 32) mine += worth(line[in_line - 32 + lane]);
      __syncwarp();
    }
    if (lane < in_line) mine += worth(line[lane]);
  }
  u64 before = R.scan(mine, total);
  const u64 at = u > 0.f ? (u < 1.f ? times<false>(u, total) : total - 1) : 0;  // (total is 2^S at least: the largest logit stays)
  // ... is in one warp's run, which all of its CTA go over again
  if (tid == 0) s_found[0] = -1;
  const u64 end = __shfl_sync(0xffffffffu, before + mine, 31);
  __syncthreads();
  if (lane == 0 && before <= at && at < end) s_found[0] = warp, s_before[0] = before;
  __syncthreads();
  if (s_found[0] < 0) return;
  const int per = (run + THREADS - 1) / THREADS, f_lo = s_found[0] * run, f_hi = min(n_quad, f_lo + run);
  const int e_lo = min(f_hi, f_lo + tid * per) * 4, e_hi = min(f_hi, f_lo + (tid + 1) * per) * 4;
  mine = 0;
#pragma unroll 1
  for (int i = e_lo / 4; i < e_hi / 4; ++i) {
    const float4 q = quad_of(z_sm, i);
    const float z[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const double w = weigh.scaled(z[j]);
      mine += w >= least && place_of(z[j], v_first + i * 4 + j) <= cut ? Weigher::rounded(w) : 0;
    }
  }
  u64 sum;
  before = s_before[0];
  before += R.scan_block(mine, sum);
  if (before <= at && at < before + mine) {
#pragma unroll 1
    for (int e = e_lo; e < e_hi; ++e) {
      const float z = to_f32<T>(z_sm[e]);
      const double w = weigh_one(weigh, z);
      if (w < least || place_of(z, v_first + e) > cut) continue;
      before += Weigher::rounded(w);
      if (before > at) {
        put(v_first + e, (float)(w / (double)total));
        break;
      }
    }
  }
}

}  // namespace smp
}  // namespace ls
