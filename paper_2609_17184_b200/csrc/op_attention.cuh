// Attention of a batch whose sequences share a prefix, over a paged cache: o = softmax(scale q [Kp; Ks]^T) [Vp; Vs] with one Kp, Vp for all
// sequences and a Ks, Vs of each sequence's own.  A softmax over a union of keys is the merge of the softmaxes over its parts (running
// maximum, sum and weighted values), so the two parts are separate problems:
//
//   prefix_rows_kernel     problems of few rows against many keys: a sequence's own keys (its new rows x the query heads of a kv head), and
//                          the prefix where the whole batch has few rows.  Bound by the stream of keys and values.
//   prefix_tc_kernel       the prefix against the rows of a larger batch, on tcgen05 (op_prefix_tc.cuh).
//   prefix_merge_kernel    folds a row's parts in a fixed order, writes it and its log-sum-exp.
//
// Scores are bf16 / fp16 products summed in fp32; maximum, sum and weighted values are fp32.  The softmax weights are rounded to the cache's
// type for the second contraction (at most 1): an error of half a step of the output's own type per weight, averaged over the keys.
#pragma once
#include "op_common.cuh"

namespace ls {

constexpr int PXR_WARPS = 4;   // warps of a CTA, each with a ring and problems of its own
constexpr int PXR_STAGES = 3;  // tiles in flight per warp: 8 warps x 3 x 8 KB per SM cover the latency of HBM several times
constexpr int PXR_KEYS = 16;   // keys of a tile
constexpr int PXR_MAX_SEQS = 2048;

struct PrefixParams {
  const void* q;
  long long q_ld;
  PagedKv kv;
  const int* prefix_pages;
  int prefix_len;
  int prefix_rows;         // 1: the prefix is problem 0 of prefix_rows_kernel
  const int* page_table;
  long long table_ld;
  int table_w;
  const int *lens, *cu_rows;
  int B, T, nq, G;
  float scale_log2;        // scale * log2(e)
  int max_tiles;           // row tiles (of 16 rows) a kv head can have
  int n_warps;             // warps the units are dealt to
  int* plan;               // [2 NP + 2]: units before problem i, row tiles before it (the last entries: their totals)
  float *item_o, *item_ml; // partials of the tiles whose first key is in the segment: [kv head][row tile][16][D], ..[2]
  float *warp_o, *warp_ml; // partials of the segments that begin inside a tile's keys: [warp][16][D], ..[2]
  int tc_tiles, tc_splits; // prefix_tc_kernel: tiles of 128 rows, parts of the prefix (0: it does not run)
  float *tc_o, *tc_ml;     // its partials: [kv head][row tile][part][128][D], ..[2]
  void* out;
  long long out_ld;
  float* lse;              // [T][nq] or null
  int* flag;
};

// a problem: rows row0 .. row0 + n - 1 of the batch against len keys; a row that lies j-th sees the first len - (n - 1 - j) of them (all of them
// in the prefix)
struct PxProblem {
  int row0, n, len;
  bool prefix;
};
__device__ __forceinline__ PxProblem px_problem(const PrefixParams& p, int i) {
  PxProblem r;
  r.prefix = p.prefix_rows && i == 0;
  if (r.prefix) {
    r.row0 = 0, r.n = p.T, r.len = p.prefix_len;
    return r;
  }
  const int b = i - p.prefix_rows;
  const int r0 = __ldg(p.cu_rows + b), r1 = __ldg(p.cu_rows + b + 1);
  const long long cap = (long long)p.table_w << p.kv.page_shift;
  const int len = __ldg(p.lens + b);
  r.row0 = r0, r.n = (r0 < 0 || r1 < r0 || r1 > p.T) ? 0 : r1 - r0;
  r.len = len < 0 ? 0 : (int)min((long long)len, cap);
  return r;
}
// row counts or a length that are not what they should be
__device__ __forceinline__ bool px_bad(const PrefixParams& p, int i, const PxProblem& r) {
  if (r.prefix) return false;
  const int b = i - p.prefix_rows;
  return r.len != __ldg(p.lens + b) || r.n != __ldg(p.cu_rows + b + 1) - __ldg(p.cu_rows + b);
}

__device__ __forceinline__ int px_block_scan(int v, int* s_w) {  // inclusive, 128 threads
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += u;
  }
  __syncthreads();
  if (lane == 31) s_w[warp] = v;
  __syncthreads();
  for (int w = 0; w < warp; ++w) v += s_w[w];
  return v;
}

template <typename T>
__device__ __forceinline__ void px_mma(float (&c)[4], const unsigned (&a)[4], unsigned b0, unsigned b1) {
  if constexpr (sizeof(T) == 2 && std::is_same<T, __half>::value)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void px_ldsm4(unsigned (&r)[4], unsigned addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void px_ldsm4t(unsigned (&r)[4], unsigned addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ float px_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));  // (2 ulp: far below the rounding of a weight)
  return y;
}
__device__ __forceinline__ void px_cp16(unsigned dst, const void* src, bool valid) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(valid ? 16 : 0) : "memory");
}

// warps that U units are dealt to: none goes empty (the slot of a warp without units would be read, but never written)
__device__ __forceinline__ int px_warps(const PrefixParams& p, long long U) { return (int)min((long long)p.n_warps, U); }
// unit -> warp, when U units are dealt to W warps in equal contiguous shares (warp w has [w U / W, (w + 1) U / W))
__device__ __forceinline__ int px_warp_of(long long u, long long U, int W) { return (int)(((u + 1) * W - 1) / U); }

constexpr int px_rows_smem(int D, int np) { return PXR_WARPS * PXR_STAGES * 2 * PXR_KEYS * D * 2 + (2 * np + 2) * 4; }

// The work of all problems is one line of units, a unit being 16 keys for 16 rows of a problem and kv head, ordered [kv head][problem][row
// tile][keys], and every warp takes an equal share of it: lengths may be as ragged as they like.  A warp's ring of tiles runs on across
// its segments; a segment leaves one partial (weighted values, maximum, sum) of up to 16 rows.  Rows are the 16-row operand of mma.sync: with
// one to four live rows most of it is idle, but at 32 MMAs per 8 KB of keys and values the tensor pipe is busy a fifth of the time the
// stream takes.
template <typename T, int D>
__global__ void __launch_bounds__(PXR_WARPS * 32, 2) prefix_rows_kernel(const __grid_constant__ PrefixParams p) {
  constexpr int ROW = D * 2, CH = D / 8, TILE = PXR_KEYS * ROW, KS = D / 16, NT = D / 8, KPI = 32 / CH;
  extern __shared__ __align__(128) unsigned char px_smem[];
  __shared__ int s_w[PXR_WARPS];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  const int NP = p.B + p.prefix_rows;
  int* s_unit = reinterpret_cast<int*>(px_smem + PXR_WARPS * PXR_STAGES * 2 * TILE);  // [NP + 1]
  int* s_item = s_unit + NP + 1;                                                       // [NP + 1]
  pdl_launch_dependents();

  // ---- the line of units: every CTA adds it up for itself ----
  int base_i = 0, base_u = 0;
  for (int i0 = 0; i0 < NP; i0 += PXR_WARPS * 32) {
    const int i = i0 + tid;
    PxProblem r = {0, 0, 0, false};
    bool bad = false;
    if (i < NP) r = px_problem(p, i), bad = px_bad(p, i, r);
    const int rt = r.len > 0 ? (r.n * p.G + 15) / 16 : 0;
    const int e_i = base_i + px_block_scan(rt, s_w);
    const bool fits = e_i <= p.max_tiles;  // (always, unless the row counts overlap)
    const int units = fits ? rt * ((r.len + PXR_KEYS - 1) / PXR_KEYS) : 0;
    const int e_u = base_u + px_block_scan(units, s_w);
    if (i < NP) s_item[i] = e_i - rt, s_unit[i] = e_u - units;
    if ((bad || !fits) && p.flag && blockIdx.x == 0) atomicOr(p.flag, OP_BAD_ROWS);
    __syncthreads();
    if (tid == PXR_WARPS * 32 - 1) s_w[0] = e_i, s_w[1] = e_u;
    __syncthreads();
    base_i = s_w[0], base_u = s_w[1];
    __syncthreads();
  }
  if (tid == 0) s_unit[NP] = base_u, s_item[NP] = base_i;
  __syncthreads();
  if (blockIdx.x == 0)
    for (int i = tid; i < 2 * NP + 2; i += PXR_WARPS * 32) p.plan[i] = s_unit[i];
  const int Us = base_u;
  const long long U = (long long)Us * p.kv.n_kv;
  const int w = blockIdx.x * PXR_WARPS + warp;
  const int W = px_warps(p, U);
  // (every thread waits before it ends: this kernel may run beside prefix_tc_kernel, and the merge waits for this one only)
  if (w >= W) {
    pdl_wait();
    return;
  }
  const long long u_lo = w * U / W, u_hi = (w + 1) * U / W;

  // a place on the line
  struct Cursor {
    int h, i, rt, k;       // kv head, problem, row tile, tile of keys
    int n_rt, n_k;
    PxProblem r;
  };
  auto enter = [&](Cursor& c) {
    c.r = px_problem(p, c.i);
    c.n_rt = (c.r.n * p.G + 15) / 16, c.n_k = (c.r.len + PXR_KEYS - 1) / PXR_KEYS;
  };
  auto advance = [&](Cursor& c) {
    if (++c.k < c.n_k) return;
    c.k = 0;
    if (++c.rt < c.n_rt) return;
    c.rt = 0;
    do {
      if (++c.i == NP) c.i = 0, ++c.h;
    } while (s_unit[c.i] == s_unit[c.i + 1]);
    enter(c);
  };
  Cursor cc;
  {
    const int r = (int)(u_lo % Us);
    cc.h = (int)(u_lo / Us);
    int lo = 0, hi = NP - 1;  // the last problem that begins at or before r (one of no units is never the last: the next begins there too)
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (s_unit[mid] <= r) lo = mid;
      else hi = mid - 1;
    }
    cc.i = lo;
    enter(cc);
    const int at = r - s_unit[lo];
    cc.rt = at / cc.n_k, cc.k = at - cc.rt * cc.n_k;
  }
  Cursor ci = cc;  // where the requests are

  const unsigned ring = (unsigned)__cvta_generic_to_shared(px_smem) + warp * PXR_STAGES * 2 * TILE;
  // the page of lane's key (lanes 0 .. 15) of the tile at ci: looked up a tile ahead of its use
  int page = -1;
  bool page_ok = false;
  auto look_up = [&]() {
    const int pos = ci.k * PXR_KEYS + (lane & 15);
    page_ok = pos < ci.r.len;
    if (page_ok) {
      const int pg = pos >> p.kv.page_shift;
      page = __ldg(ci.r.prefix ? p.prefix_pages + pg : p.page_table + (ci.i - p.prefix_rows) * p.table_ld + pg);
    }
  };
  auto request = [&](int stage) {
    const int pos = ci.k * PXR_KEYS + (lane & 15);
    bool ok = page_ok;
    if (ok && (page < 0 || page >= p.kv.n_pages)) {
      ok = false;
      if (p.flag) atomicOr(p.flag, OP_BAD_PAGE);
    }
    const long long off = ok ? page * p.kv.page_stride + (pos & ((1 << p.kv.page_shift) - 1)) * p.kv.slot_stride + ci.h * p.kv.head_stride : 0;
    const unsigned dst = ring + stage * 2 * TILE;
#pragma unroll
    for (int j = 0; j < PXR_KEYS / KPI; ++j) {
      const int key = lane / CH + j * KPI, ch = lane & (CH - 1);
      const long long o = __shfl_sync(0xffffffffu, off, key);
      const bool v = __shfl_sync(0xffffffffu, (int)ok, key) != 0;
      const unsigned at = dst + key * ROW + ((ch ^ (key & 7)) << 4);
      px_cp16(at, static_cast<const T*>(p.kv.k) + o + (v ? ch * 8 : 0), v);
      px_cp16(at + TILE, static_cast<const T*>(p.kv.v) + o + (v ? ch * 8 : 0), v);
    }
  };
  long long u_req = u_lo;
  look_up();
  auto feed = [&](int stage) {
    if (u_req < u_hi) {
      request(stage);
      if (++u_req < u_hi) {
        advance(ci);
        look_up();
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int s = 0; s < PXR_STAGES - 1; ++s) feed(s);

  int stage = 0;
  for (long long u = u_lo; u < u_hi;) {
    // ---- a segment: the tiles of keys that this warp has of one row tile ----
    const int first_k = cc.k, seg = (int)min((long long)(cc.n_k - cc.k), u_hi - u), R = cc.r.n * p.G, r0 = cc.rt * 16;
    unsigned qf[KS][4];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int r = r0 + g + 8 * half, j = r / p.G;
      const T* src = static_cast<const T*>(p.q) + (long long)(cc.r.row0 + j) * p.q_ld + (cc.h * p.G + (r - j * p.G)) * D + 2 * t;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        qf[ks][half] = r < R ? *reinterpret_cast<const unsigned*>(src + 16 * ks) : 0u;
        qf[ks][2 + half] = r < R ? *reinterpret_cast<const unsigned*>(src + 16 * ks + 8) : 0u;
      }
    }
    // keys that rows g and g + 8 see; the fewest any live row of the tile sees
    int sees[2];
#pragma unroll
    for (int half = 0; half < 2; ++half) sees[half] = cc.r.prefix ? cc.r.len : cc.r.len - (cc.r.n - 1 - min((r0 + g + 8 * half) / p.G, cc.r.n - 1));
    const int sees_all = cc.r.prefix ? cc.r.len : cc.r.len - (cc.r.n - 1 - r0 / p.G);
    float o[NT][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[n][i] = 0.f;

    for (int it = 0; it < seg; ++it) {
      asm volatile("cp.async.wait_group %0;" ::"n"(PXR_STAGES - 2) : "memory");
      __syncwarp();
      feed(stage == 0 ? PXR_STAGES - 1 : stage - 1);  // (the stage that the last tile has left)
      const unsigned sk = ring + stage * 2 * TILE, sv = sk + TILE;
      const int k0 = (first_k + it) * PXR_KEYS;
      float s[2][4];
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[j][i] = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const int key = (lane >> 4) * 8 + (lane & 7), ch = 2 * ks + ((lane >> 3) & 1);
        unsigned b[4];
        px_ldsm4(b, sk + key * ROW + ((ch ^ (key & 7)) << 4));
        px_mma<T>(s[0], qf[ks], b[0], b[1]);
        px_mma<T>(s[1], qf[ks], b[2], b[3]);
      }
      // ---- running softmax; this lane: rows g (elements 0, 1) and g + 8 (2, 3), keys 8 j + 2 t, + 1 ----
      float alpha[2];
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        float mx = -INFINITY;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float& x = s[j][2 * half + e];
            x = k0 + 8 * j + 2 * t + e < sees[half] ? x * p.scale_log2 : -INFINITY;
            mx = fmaxf(mx, x);
          }
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
        mx = fmaxf(mx, m[half]);
        const float ref = mx == -INFINITY ? 0.f : mx;  // (a row that has seen no key, or whose scores are all -inf)
        alpha[half] = px_exp2(m[half] - ref);
        m[half] = mx;
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float& x = s[j][2 * half + e];
            x = px_exp2(x - ref);
            sum += x;
          }
        l[half] = fmaf(l[half], alpha[half], sum);  // (this lane's keys; summed over the lanes when the segment is done)
      }
      if (__any_sync(0xffffffffu, alpha[0] != 1.f || alpha[1] != 1.f)) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[n][i] *= alpha[i >> 1];
      }
      const unsigned pf[4] = {pack2<T>(s[0][0], s[0][1]), pack2<T>(s[0][2], s[0][3]), pack2<T>(s[1][0], s[1][1]), pack2<T>(s[1][2], s[1][3])};
      // Keys that some rows of the tile see and others do not: an infinity or NaN among their values must not reach the latter as 0 * inf.
      // Where there is one, those keys are added row by row and their values zeroed ahead of the contraction.
      if (k0 + PXR_KEYS > sees_all && sees_all < cc.r.len) {
        const int ka = max(sees_all - k0, 0), kb = min(PXR_KEYS, cc.r.len - k0);
        T* vp = reinterpret_cast<T*>(px_smem + (sv - (unsigned)__cvta_generic_to_shared(px_smem)));
        bool odd = false;
        for (int e = lane; e < (kb - ka) * D; e += 32) {
          const float x = to_f32<T>(vp[ka * D + e]);
          odd |= !(fabsf(x) <= 3.4e38f);
        }
        if (__any_sync(0xffffffffu, odd)) {
          for (int key = ka; key < kb; ++key) {
            const int j = key >> 3, from = (lane & ~3) | ((key & 7) >> 1);
            float w[2];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              const unsigned pr = __shfl_sync(0xffffffffu, j ? pf[2 + half] : pf[half], from);
              const T* two = reinterpret_cast<const T*>(&pr);
              w[half] = to_f32<T>(two[key & 1]);
            }
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const float x = to_f32<T>(vp[key * D + ((n ^ (key & 7)) << 3) + 2 * t + (i & 1)]);
                if (k0 + key < sees[i >> 1]) o[n][i] = fmaf(w[i >> 1], x, o[n][i]);
              }
          }
          __syncwarp();
          for (int e = lane; e < (kb - ka) * D; e += 32) vp[ka * D + e] = T(0.f);
          __syncwarp();
        }
      }
#pragma unroll
      for (int n2 = 0; n2 < NT / 2; ++n2) {
        const int key = ((lane >> 3) & 1) * 8 + (lane & 7), ch = 2 * n2 + (lane >> 4);
        unsigned b[4];
        px_ldsm4t(b, sv + key * ROW + ((ch ^ (key & 7)) << 4));
        px_mma<T>(o[2 * n2], pf, b[0], b[1]);
        px_mma<T>(o[2 * n2 + 1], pf, b[2], b[3]);
      }
      __syncwarp();  // the tile may be overwritten
      if (++stage == PXR_STAGES) stage = 0;
    }

    // ---- the segment is done ----
    const bool whole = first_k == 0;
    const long long slot = whole ? (long long)cc.h * p.max_tiles + s_item[cc.i] + cc.rt : w;
    float* po = (whole ? p.item_o : p.warp_o) + slot * 16 * D;
    float* pm = (whole ? p.item_ml : p.warp_ml) + slot * 32;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      l[half] += __shfl_xor_sync(0xffffffffu, l[half], 1);
      l[half] += __shfl_xor_sync(0xffffffffu, l[half], 2);
      if (r0 + g + 8 * half >= R) continue;
#pragma unroll
      for (int n = 0; n < NT; ++n) __stcg(reinterpret_cast<float2*>(po + (g + 8 * half) * D + 8 * n + 2 * t), make_float2(o[n][2 * half], o[n][2 * half + 1]));
      if (t == 0) __stcg(reinterpret_cast<float2*>(pm + (g + 8 * half) * 2), make_float2(m[half], l[half]));
    }
    u += seg;
    if (u < u_hi) {
      cc.k += seg - 1;
      advance(cc);
    }
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");  // (only empty groups are left)
  pdl_wait();
}

// One warp per (row, query head): the parts of the prefix and of the sequence's own keys in a fixed order.
template <typename T, int D>
__global__ void __launch_bounds__(128) prefix_merge_kernel(const __grid_constant__ PrefixParams p) {
  constexpr int V = D / 32;  // elements per lane
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, h = blockIdx.x, b = blockIdx.y, NP = p.B + p.prefix_rows;
  const int i_own = b + p.prefix_rows;
  const PxProblem own = px_problem(p, i_own);
  pdl_wait();
  const int Us = __ldcg(p.plan + NP);
  const long long U = (long long)Us * p.kv.n_kv;
  const int W = px_warps(p, U);
  struct Part {          // the segments of a row tile: one in the tile's own slot, the others in the slots of the warps that follow
    long long item;
    int w0, n;
  };
  auto part_of = [&](int i, int len, int rt) {
    Part q = {0, 0, 0};
    const int u0 = __ldcg(p.plan + i), u1 = __ldcg(p.plan + i + 1);
    if (u1 <= u0) return q;
    const int n_k = (len + PXR_KEYS - 1) / PXR_KEYS;
    const long long a = (long long)h * Us + u0 + (long long)rt * n_k;
    q.item = (long long)h * p.max_tiles + __ldcg(p.plan + NP + 1 + i) + rt;
    q.w0 = px_warp_of(a, U, W), q.n = 1 + px_warp_of(a + n_k - 1, U, W) - q.w0;
    return q;
  };
  const int R = own.n * p.G;
  for (int r = warp + blockIdx.z * 4; r < R; r += 4 * gridDim.z) {
    const int j = r / p.G, row = own.row0 + j, head = h * p.G + (r - j * p.G);
    float m = -INFINITY, l = 0.f, acc[V];
#pragma unroll
    for (int e = 0; e < V; ++e) acc[e] = 0.f;
    // parts of a problem: count of them, and where part x has its row of weighted values and its (maximum, sum)
    auto fold = [&](int count, auto o_at, auto ml_at) {
      for (int x0 = 0; x0 < count; x0 += 32) {
        const int cnt = min(32, count - x0);
        float2 ml = make_float2(-INFINITY, 0.f);
        if (lane < cnt) ml = __ldcg(reinterpret_cast<const float2*>(ml_at(x0 + lane)));
        const float mx = fmaxf(m, warp_max(ml.x)), ref = mx == -INFINITY ? 0.f : mx;
        const float wt = px_exp2(ml.x - ref), keep = px_exp2(m - ref);
        m = mx;
        l = l * keep + warp_sum(ml.y * wt);
#pragma unroll
        for (int e = 0; e < V; ++e) acc[e] *= keep;
#pragma unroll 4
        for (int y = 0; y < cnt; ++y) {
          const float f = __shfl_sync(0xffffffffu, wt, y);
          const float* src = o_at(x0 + y) + lane * V;
          float v[V];
          if constexpr (V == 4) {
            const float4 z = __ldcg(reinterpret_cast<const float4*>(src));
            v[0] = z.x, v[1] = z.y, v[2] = z.z, v[3] = z.w;
          } else {
            const float2 z = __ldcg(reinterpret_cast<const float2*>(src));
            v[0] = z.x, v[1] = z.y;
          }
#pragma unroll
          for (int e = 0; e < V; ++e) acc[e] = fmaf(f, v[e], acc[e]);
        }
      }
    };
    const int pr = row * p.G + (r - j * p.G);  // the row's number in the prefix problem
    if (p.tc_splits) {
      const long long slot = (long long)(h * p.tc_tiles + (pr >> 7)) * p.tc_splits * 128 + (pr & 127);
      fold(p.tc_splits, [&](int x) { return p.tc_o + (slot + x * 128) * D; }, [&](int x) { return p.tc_ml + (slot + x * 128) * 2; });
    }
    for (int which = p.prefix_rows ? 0 : 1; which < 2; ++which) {
      const int rr = which ? r : pr;
      const Part q = part_of(which ? i_own : 0, which ? own.len : p.prefix_len, rr >> 4);
      fold(q.n, [&](int x) { return (x == 0 ? p.item_o + q.item * 16 * D : p.warp_o + (long long)(q.w0 + x) * 16 * D) + (rr & 15) * D; },
           [&](int x) { return (x == 0 ? p.item_ml + q.item * 32 : p.warp_ml + (long long)(q.w0 + x) * 32) + (rr & 15) * 2; });
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;  // a row that sees no key: zeros
    T* dst = static_cast<T*>(p.out) + (long long)row * p.out_ld + head * D + lane * V;
#pragma unroll
    for (int e = 0; e < V; e += 2) *reinterpret_cast<unsigned*>(dst + e) = pack2<T>(acc[e] * inv, acc[e + 1] * inv);
    if (p.lse && lane == 0) p.lse[(long long)row * p.nq + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
  }
}

}  // namespace ls
