// Attention of a batch whose sequences share a prefix, over a paged cache: o = softmax(scale q [Kp; Ks]^T) [Vp; Vs] with one Kp, Vp for all
// sequences and a Ks, Vs of each sequence's own.  A softmax over a union of keys is the merge of the softmaxes over its parts (running
// maximum, sum and weighted values), so the call is a set of problems - the prefix against the rows of the whole batch, every sequence's own keys
// against its rows - that leave partials, and two kernels:
//
//   prefix_kernel        one CTA per SM, in one of two roles:
//     tiles              (op_prefix_tiles.cuh) the prefix of a larger batch on tcgen05, bound by the tensor core and the exponentials
//     rows               problems of few rows against many keys, bound by the stream of keys and values
//   prefix_merge_kernel  folds a row's partials in a fixed order, writes it and its log-sum-exp
//
// The two kinds of work want different parts of the machine, so they run side by side: every CTA adds up from the lengths what there is of either
// and takes the role that makes both end together.  (One after the other, 256 sequences of 16 heads behind 16384 positions took 122 us
// where the stream alone takes 57 and the prefix alone 62; side by side they take 102.)
//
// Scores are bf16 / fp16 products summed in fp32; maximum, sum and weighted values are fp32.  The softmax weights are rounded to the cache's
// type for the second contraction: an error of half a step of the output's own type per weight, averaged over the keys (large batches in
// bf16: 0.0023 from 64 bits where weights in 32 bits leave 0.0017, the rounding of the output; fp16 0.00026 and 0.00021).
#pragma once
#include <cuda.h>

#include "op_common.cuh"
#include "tc.cuh"

namespace ls {

constexpr int PX_THREADS = 384;      // tiles: 4 + 4 softmax warps, two producers, two MMA issuers; rows: the first eight
constexpr int PX_SMS = 148;
constexpr int PX_MAX_SEQS = 2048;
constexpr int PXR_WARPS = 8;         // warps of a CTA in the rows' role, each with a ring and problems of its own
constexpr int PXR_KEYS = 16;         // keys of a tile
constexpr int PXT_ROWS = 128, PXT_KEYS = 128;
constexpr int PXT_K_STAGES = 3, PXT_V_STAGES = 2;  // tiles of keys and of values in flight
constexpr float PX_SLACK = 8.f;  // (log2) how far a row's maximum may run ahead of its reference
constexpr long long PX_WAIT_CYCLES = 400000000LL;  // ~0.2 s: a wait that runs this long gives up: its rows become NaN, and it leaves its flag

template <int D>
struct PxCfg {
  static constexpr int TILE = PXR_KEYS * D * 2;            // rows: keys or values of a tile
  static constexpr int STAGES = D == 128 ? 3 : 6;          // ... tiles in flight per warp: 192 KB per SM cover the latency of HBM several times
  static constexpr int TC_TILE = PXT_KEYS * D * 2;
  static constexpr int ROWS_BYTES = PXR_WARPS * STAGES * 2 * TILE, TILES_BYTES = (1 + PXT_K_STAGES + PXT_V_STAGES) * TC_TILE;
  static constexpr int MAIN = 1024 + (ROWS_BYTES > TILES_BYTES ? ROWS_BYTES : TILES_BYTES);
  static constexpr int smem(int np) { return MAIN + (np + 1) * 4; }
};

struct PrefixParams {
  const void* q;
  long long q_ld;
  PagedKv kv;
  const int* prefix_pages;
  int prefix_len;
  int prefix_rows;         // 1: the prefix is problem 0 of the rows' role
  int tc_tiles;            // tiles of 128 rows of the batch and a kv head (0: nothing for the tiles' role)
  const int* page_table;
  long long table_ld;
  int table_w;
  const int *lens, *cu_rows;
  int B, T, nq, G;
  float scale_log2;        // scale * log2(e)
  int max_tiles;           // row tiles (of 16 rows) a kv head can have
  // partials of the rows' role: of the segments that begin with a problem's first key [kv head][row tile][16][D], ..[2], and of the others [warp][16][D], ..[2]
  float *item_o, *item_ml, *warp_o, *warp_ml;
  // ... of the tiles' role: [kv head][row tile][128][D], ..[2]; [worker][row tile][128][D], ..[2]
  float *tc_item_o, *tc_item_ml, *tc_work_o, *tc_work_ml;
  int* state;              // 1: the row counts are not what they should be, and nothing of the rows' is done
  int2 *item_seg, *tc_seg; // for every row tile (of either role): the worker of its first segment and how many workers, one after the other, have segments of it
  void* out;
  long long out_ld;
  float* lse;              // [T][nq] or null
  int* flag;
  long long wait_cycles;   // how long a wait may take (PX_WAIT_CYCLES)
  int stop_tile;           // test hook: no CTA requests its tiles of keys and values from this one on (INT_MAX: all are), so that the waits for them run out
};

// a problem: rows row0 .. row0 + n - 1 of the batch against len keys; a row that lies j-th sees the first len - (n - 1 - j) of them (all of them
// in the prefix)
struct PxProblem {
  int row0, n, len;
  bool prefix, bad_rows, bad_len;  // row counts that do not ascend in [0, T]; a length beyond the table (cut to it)
};
__device__ __forceinline__ PxProblem px_problem(const PrefixParams& p, int i) {
  PxProblem r;
  r.prefix = p.prefix_rows && i == 0, r.bad_rows = r.bad_len = false;
  if (r.prefix) {
    r.row0 = 0, r.n = p.T, r.len = p.prefix_len;
    return r;
  }
  const int b = i - p.prefix_rows;
  const int r0 = __ldg(p.cu_rows + b), r1 = __ldg(p.cu_rows + b + 1), len = __ldg(p.lens + b);
  const long long cap = (long long)p.table_w << p.kv.page_shift;
  const bool rows = r0 >= 0 && r1 >= r0 && r1 <= p.T;
  r.row0 = r0, r.n = rows ? r1 - r0 : 0;
  r.len = len < 0 ? 0 : (int)min((long long)len, cap);
  r.bad_rows = !rows, r.bad_len = r.len != len;
  return r;
}

// The first of a problem's row tiles: a rule of its own rows, so that nothing has to be added up to find a partial.  (Tiles of 16 rows per sequence are at
// most its rows / 16 + 1, so that those of two sequences do not meet.)
__device__ __forceinline__ int px_first_tile(const PrefixParams& p, int i, const PxProblem& r) {
  return r.prefix ? 0 : (p.prefix_rows ? (p.T * p.G + 15) / 16 : 0) + r.row0 * p.G / 16 + i - p.prefix_rows;
}

// What precedes x in this CTA plus x, and the total (all threads of the CTA)
__device__ __forceinline__ int px_block_scan(int x, int* s_w, int& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 31) s_w[warp] = x;
  __syncthreads();
  total = 0;
  int add = 0;
  for (int w = 0; w < PX_THREADS / 32; ++w) {
    if (w == warp) add = total;
    total += s_w[w];
  }
  return x + add;
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

__device__ __forceinline__ void px_tma_4d(unsigned dst, const CUtensorMap* map, unsigned bar, int x, int y, int z, int w) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(dst),
               "l"(reinterpret_cast<unsigned long long>(map)), "r"(bar), "r"(x), "r"(y), "r"(z), "r"(w)
               : "memory");
}
// Bounded wait: false when it gave up.  `failed` says so to the whole CTA (before whatever this warp hands on next), whose later waits give up at once.
// Most find their phase complete: they read neither that nor the clock.
__device__ __forceinline__ bool px_wait(const PrefixParams& p, unsigned long long* bar, unsigned parity, int& failed) {
  unsigned done;
  asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
               : "=r"(done)
               : "r"(tc_smem_u32(bar)), "r"(parity)
               : "memory");
  if (!done && !tc_mbar_wait(tc_smem_u32(bar), parity, *const_cast<volatile int*>(&failed) ? 2000LL : p.wait_cycles)) {
    *const_cast<volatile int*>(&failed) = 1;
    __threadfence_block();
    return false;
  }
  return true;
}
// Work is dealt as a line of U units, of which worker w of W has [w U / W, (w + 1) U / W); no worker goes empty (the slot of one without units would be
// read, but never written), so there are at most as many as units.
__device__ __forceinline__ int px_workers(int W, long long U) { return (int)min((long long)W, U); }
__device__ __forceinline__ int px_worker_of(long long u, long long U, int W) { return (int)(((u + 1) * W - 1) / U); }

// Which CTAs take which role: the first `tiles` the tiles', the others the rows'.
struct PxRoles {
  int workers, tiles;  // a worker: one CTA per row tile, side by side, so that their keys and values come from HBM once
};
// All threads of the CTA; every CTA comes to the same answer.  In ns: a tile of 128 x 128 takes 1200 (head size 64: 900), a segment 5000 more (queries,
// first keys, last weights, partial), an SM streams some 50 bytes a ns.  Of all numbers of workers that leave the rows a CTA, the one with which the later of
// the two roles ends first, a thread for each; as many as a multiple of the heads, or a part of them, have no segment cut at the end of one.
template <int D>
__device__ __forceinline__ PxRoles px_roles(const PrefixParams& p, long long row_units, unsigned long long* s_w) {
  PxRoles r = {0, 0};
  if (p.tc_tiles == 0) return r;
  const int all = (p.prefix_len + PXT_KEYS - 1) / PXT_KEYS, most = PX_SMS - (row_units > 0), w = threadIdx.x + 1, lane = threadIdx.x & 31;
  const long long U = (long long)p.kv.n_kv * all;
  const int n_w = (int)min((long long)max(1, most / p.tc_tiles), U);
  // (one worker of more row tiles than CTAs: even rounds of them)
  auto tiles_of = [&](int w, int& rounds) {
    rounds = (p.tc_tiles * w + most - 1) / most;
    return (p.tc_tiles * w + rounds - 1) / rounds;
  };
  int rounds;
  unsigned long long best = ~0ull;
  if (w <= n_w) {
    const float rows = (float)row_units * (PXR_KEYS * D * 4) / 50.f, n = (float)((U + w - 1) / w);
    const float cuts = w % p.kv.n_kv == 0 ? 1.f : p.kv.n_kv % w == 0 ? (float)(p.kv.n_kv / w) : floorf(n / all) + 2.f;
    const int x = tiles_of(w, rounds);
    const float t = fmaxf((n * (D == 128 ? 1200.f : 900.f) + cuts * 5000.f) * rounds, row_units > 0 ? rows / (PX_SMS - x) + 4000.f : 0.f);
    best = (unsigned long long)__float_as_uint(t) << 32 | (unsigned)w;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) best = min(best, __shfl_xor_sync(0xffffffffu, best, o));
  __syncthreads();
  if (lane == 0) s_w[threadIdx.x >> 5] = best;
  __syncthreads();
  for (int i = 0; i < PX_THREADS / 32; ++i) best = min(best, s_w[i]);
  r.workers = (int)(unsigned)best, r.tiles = tiles_of(r.workers, rounds);
  return r;
}

// The work of all problems is one line of units, a unit being 16 keys for 16 rows of a problem and kv head, ordered [kv head][problem][row
// tile][keys], and every warp takes an equal share of it: lengths may be as ragged as they like.  A warp's ring of tiles runs on across
// its segments; a segment leaves one partial (weighted values, maximum, sum) of up to 16 rows.  Rows are the 16-row operand of mma.sync: with
// one to four live rows most of it is idle, but at 32 MMAs per 8 KB of keys and values the tensor pipe is busy a fifth of the time the
// stream takes.
//
// Tiles come by cp.async, whatever the pages (boxes of 16 keys x 64 elements by TMA, for pages of 8 and more: 46 against 42 us for 270 MB).  As in the tiles'
// role a row's reference moves only when a tile's maximum runs more than 2^8 ahead of it, so that a tile mostly needs neither a maximum over its lanes
// nor a rescaled accumulator.
template <typename T, int D>
__device__ __forceinline__ void px_rows_role(const PrefixParams& p, unsigned char* raw, const int* s_unit, int Us, int cta, int n_cta) {
  constexpr int TILE = PxCfg<D>::TILE, STAGES = PxCfg<D>::STAGES, KS = D / 16, NT = D / 8, NH = D / 64, PIECE = PXR_KEYS * 128;
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), g = lane >> 2, t = lane & 3;
  const int NP = p.B + p.prefix_rows;
  const long long U = (long long)Us * p.kv.n_kv;
  const int W = px_workers(n_cta * PXR_WARPS, U), w = cta + warp * n_cta;  // (neighbouring shares on different SMs)
  if (warp >= PXR_WARPS || w >= W) return;
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

  const unsigned base = (tc_smem_u32(raw) + 1023u) & ~1023u, ring = base + warp * STAGES * 2 * TILE;
  unsigned char* ring_ptr = raw + (ring - tc_smem_u32(raw));
  // the page of lane's key (lanes 0 .. 15, and again 16 .. 31) of the tile at ci: looked up a tile ahead of its use
  int page = -1;
  bool mine = false;
  auto look_up = [&]() {
    const int pos = ci.k * PXR_KEYS + (lane & 15);
    mine = pos < ci.r.len;
    if (mine) {
      const int pg = pos >> p.kv.page_shift;
      page = __ldg(ci.r.prefix ? p.prefix_pages + pg : p.page_table + (ci.i - p.prefix_rows) * p.table_ld + pg);
    }
  };
  auto request = [&](int stage) {
    const int pos = ci.k * PXR_KEYS + (lane & 15);
    bool there = mine;
    if (there && (page < 0 || page >= p.kv.n_pages)) {
      there = false;
      if (p.flag) atomicOr(p.flag, OP_BAD_PAGE);
    }
    const unsigned dst = ring + stage * 2 * TILE;
    const long long off = there ? page * p.kv.page_stride + (pos & ((1 << p.kv.page_shift) - 1)) * p.kv.slot_stride + ci.h * p.kv.head_stride : 0;
#pragma unroll
    for (int j = 0; j < PXR_KEYS * NH / 4; ++j) {  // 32 lanes: 128 bytes of four keys
      const int key = (lane >> 3) + 4 * (j / NH), piece = j % NH, ch = lane & 7;
      const long long o = __shfl_sync(0xffffffffu, off, key);
      const bool v = __shfl_sync(0xffffffffu, (int)there, key) != 0;
      const unsigned at = dst + piece * PIECE + key * 128 + ((ch ^ (key & 7)) << 4);
      px_cp16(at, static_cast<const T*>(p.kv.k) + o + (v ? piece * 64 + ch * 8 : 0), v);  // (zeros behind the last key)
      px_cp16(at + TILE, static_cast<const T*>(p.kv.v) + o + (v ? piece * 64 + ch * 8 : 0), v);
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
  for (int s = 0; s < STAGES - 1; ++s) feed(s);

  // this lane's part of the fragments' addresses: keys (row operand by pairs of 8), values (transposed)
  const int k_key = (lane >> 4) * 8 + (lane & 7), v_key = ((lane >> 3) & 1) * 8 + (lane & 7);
  unsigned k_at[4], v_at[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) k_at[i] = k_key * 128 + (((2 * i + ((lane >> 3) & 1)) ^ (k_key & 7)) << 4), v_at[i] = v_key * 128 + (((2 * i + (lane >> 4)) ^ (v_key & 7)) << 4);
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
    float o[NT][4], ref[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[n][i] = 0.f;

    for (int it = 0; it < seg; ++it) {
      const int k0 = (first_k + it) * PXR_KEYS;
      asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 2) : "memory");
      __syncwarp();
      feed(stage == 0 ? STAGES - 1 : stage - 1);  // (the stage that the last tile has left)
      const unsigned sk = ring + stage * 2 * TILE, sv = sk + TILE;
      unsigned char* v_ptr = ring_ptr + stage * 2 * TILE + TILE;
      float s[2][2][4];  // of 8 keys each; even and odd steps of 16 dims in chains of their own
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[j][x][i] = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        unsigned b[4];
        px_ldsm4(b, sk + (ks >> 2) * PIECE + k_at[ks & 3]);
        px_mma<T>(s[0][ks & 1], qf[ks], b[0], b[1]);
        px_mma<T>(s[1][ks & 1], qf[ks], b[2], b[3]);
      }
      // ---- running softmax; this lane: rows g (elements 0, 1) and g + 8 (2, 3), keys 8 j + 2 t, + 1 ----
      float mx[2];
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[j][0][i] = (s[j][0][i] + s[j][1][i]) * p.scale_log2;
      if (k0 + PXR_KEYS > sees_all) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (k0 + 8 * j + 2 * t + (i & 1) >= sees[i >> 1]) s[j][0][i] = -INFINITY;
      }
#pragma unroll
      for (int half = 0; half < 2; ++half) mx[half] = fmaxf(fmaxf(s[0][0][2 * half], s[0][0][2 * half + 1]), fmaxf(s[1][0][2 * half], s[1][0][2 * half + 1]));
      if (__any_sync(0xffffffffu, mx[0] > ref[0] + PX_SLACK || mx[1] > ref[1] + PX_SLACK)) {
        float f[2];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          mx[half] = fmaxf(mx[half], __shfl_xor_sync(0xffffffffu, mx[half], 1));
          mx[half] = fmaxf(mx[half], __shfl_xor_sync(0xffffffffu, mx[half], 2));
          const float to = fmaxf(mx[half], ref[half]);
          f[half] = to == ref[half] ? 1.f : px_exp2(ref[half] - to);
          ref[half] = to, l[half] *= f[half];
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[n][i] *= f[i >> 1];
      }
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const float sub = ref[half] == -INFINITY ? 0.f : ref[half];  // (a row that has seen no key, or whose scores are all -inf)
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float& x = s[j][0][2 * half + e];
            x = px_exp2(x - sub);
            sum += x;
          }
        l[half] += sum;  // (this lane's keys; summed over the lanes when the segment is done)
      }
      const unsigned pf[4] = {pack2<T>(s[0][0][0], s[0][0][1]), pack2<T>(s[0][0][2], s[0][0][3]), pack2<T>(s[1][0][0], s[1][0][1]), pack2<T>(s[1][0][2], s[1][0][3])};
      // Keys that some rows of the tile see and others do not: an infinity or NaN among their values must not reach the latter as 0 * inf.
      // Where there is one, those keys are added row by row and their values zeroed ahead of the contraction.
      if (k0 + PXR_KEYS > sees_all && sees_all < cc.r.len) {
        const int ka = max(sees_all - k0, 0), kb = min(PXR_KEYS, cc.r.len - k0);
        auto value = [&](int key, int c) -> T& { return *reinterpret_cast<T*>(v_ptr + (c >> 6) * PIECE + key * 128 + ((((c >> 3) & 7) ^ (key & 7)) << 4) + (c & 7) * 2); };
        bool odd = false;
        for (int e = lane; e < (kb - ka) * D; e += 32) odd |= !(fabsf(to_f32<T>(value(ka + e / D, e % D))) <= 3.4e38f);
        if (__any_sync(0xffffffffu, odd)) {
          for (int key = ka; key < kb; ++key) {
            const int j = key >> 3, from = (lane & ~3) | ((key & 7) >> 1);
            float wt[2];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              const unsigned pr = __shfl_sync(0xffffffffu, j ? pf[2 + half] : pf[half], from);
              const T* two = reinterpret_cast<const T*>(&pr);
              wt[half] = to_f32<T>(two[key & 1]);
            }
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const float x = to_f32<T>(value(key, 8 * n + 2 * t + (i & 1)));
                if (k0 + key < sees[i >> 1]) o[n][i] = fmaf(wt[i >> 1], x, o[n][i]);
              }
          }
          __syncwarp();
          for (int e = lane; e < (kb - ka) * D; e += 32) value(ka + e / D, e % D) = T(0.f);
          __syncwarp();
        }
      }
#pragma unroll
      for (int n2 = 0; n2 < NT / 2; ++n2) {
        unsigned b[4];
        px_ldsm4t(b, sv + (n2 >> 2) * PIECE + v_at[n2 & 3]);
        px_mma<T>(o[2 * n2], pf, b[0], b[1]);
        px_mma<T>(o[2 * n2 + 1], pf, b[2], b[3]);
      }
      __syncwarp();  // the tile may be overwritten
      if (++stage == STAGES) stage = 0;
    }

    // ---- the segment is done ----
    const bool whole = first_k == 0;
    const long long slot = whole ? (long long)cc.h * p.max_tiles + px_first_tile(p, cc.i, cc.r) + cc.rt : w;
    if (whole && lane == 0) p.item_seg[slot] = make_int2(w, seg == cc.n_k ? 1 : 1 + px_worker_of(u + cc.n_k - 1, U, W) - w);
    float* po = (whole ? p.item_o : p.warp_o) + slot * 16 * D;
    float* pm = (whole ? p.item_ml : p.warp_ml) + slot * 32;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      l[half] += __shfl_xor_sync(0xffffffffu, l[half], 1);
      l[half] += __shfl_xor_sync(0xffffffffu, l[half], 2);
      if (r0 + g + 8 * half >= R) continue;
#pragma unroll
      for (int n = 0; n < NT; ++n) __stcg(reinterpret_cast<float2*>(po + (g + 8 * half) * D + 8 * n + 2 * t), make_float2(o[n][2 * half], o[n][2 * half + 1]));
      if (t == 0) __stcg(reinterpret_cast<float2*>(pm + (g + 8 * half) * 2), make_float2(ref[half], l[half]));
    }
    u += seg;
    if (u < u_hi) {
      cc.k += seg - 1;
      advance(cc);
    }
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");  // (only empty groups are left)
}

}  // namespace ls
