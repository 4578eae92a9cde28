// The tiles' role of prefix_kernel: many rows against the shared prefix on the fifth-generation tensor cores.
//
// A worker's CTA takes 128 rows - token rows x the query heads of a kv head - and a range of 128-key tiles of the line [kv head][keys].  Scores
// Q K^T land in tensor memory, a thread per row reads its 128 of them and puts the weights there as the 16-bit A operand of P V.  The tiles go to two
// streams in turn, each with scores, weights and four softmax warps of its own, so that the tensor core multiplies while either takes
// exponentials; as scores and weights do not share their place, a stream's next scores are multiplied as soon as its last ones have been read.
//
// Both streams add to ONE accumulator in tensor memory (two would take the room of the weights), so a row has one reference that its weights are
// relative to, handed from tile to tile: it moves, and the accumulator is rescaled, only when a tile's maximum exceeds it by more than 2^8 (weights up
// to 256 keep their relative precision), in the order of the tiles.  The CTA leaves one partial per row and kv head.
//
// A tile's keys and values arrive by TMA, one box per page and 64 elements of a head (the page table is read by the producer's lanes, so a tile
// of small pages is 32 requests of a warp at once), 128-byte swizzle: K as a K-major operand, V - rows of keys - as an MN-major one.
//
// What bounds it: at head size 128 the two products of a tile take 1024 cycles at best (both operands of the first come from shared memory, which
// 128 x 128 tiles saturate) and its 16,384 exponentials, at 16 a cycle, as many.  It takes 1570: a stream's tile is a chain of about 3100 (scores
// 100, their read 250, maximum 500, reference 500, weights 1400, hand-over), and there are two streams.  384 rows of 16 heads against 16,384 keys
// take 63 us, 0.8 PFLOP/s.  Measured and left out: a quarter of the exponentials by a polynomial on the FMA pipe (no change; half: 5 %
// slower), two threads per row (no change).  Not measured: an accumulator per stream (weights in the place of their scores, two accumulators: 512 columns as well),
// which would take the hand-over of the reference out of the chain.  The 168 registers of the launch are not enough for it all: 68 bytes a thread are spilled at
// head size 128, 100 at 64, all in this role's softmax.
#pragma once
#include "op_attention.cuh"

namespace ls {

__device__ __forceinline__ void pxt_ld32(unsigned (&v)[32], unsigned taddr) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
               : "r"(taddr)
               : "memory");
}
__device__ __forceinline__ void pxt_st16(unsigned taddr, const unsigned (&v)[16]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};" ::"r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(taddr)
               : "memory");
}
__device__ __forceinline__ void pxt_ld16(unsigned (&v)[16], unsigned taddr) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
               : "r"(taddr)
               : "memory");
}
__device__ __forceinline__ float pxt_max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ void pxt_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void pxt_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// One arrival for a warp, its lanes' accesses before it (an mbarrier takes arrivals one by one: 32 of them cost as many turns)
__device__ __forceinline__ void pxt_arrive(unsigned bar, int lane) {
  __syncwarp();
  if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
// A in tensor memory (two 16-bit values a column), B in shared memory
__device__ __forceinline__ void pxt_mma_ts(unsigned d, unsigned a, unsigned long long b, unsigned idesc, unsigned accumulate) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b),
               "r"(idesc), "r"(accumulate)
               : "memory");
}

constexpr unsigned PXT_P = 256, PXT_O = 384;  // tensor memory: scores of either stream, 64 columns of weights of either, the accumulator

struct PxtShared {
  unsigned long long kfull[PXT_K_STAGES], kempty[PXT_K_STAGES], vfull[PXT_V_STAGES], vempty[PXT_V_STAGES];  // rings of keys and of values
  unsigned long long sc[2], sr[2];     // a stream's scores: multiplied, read
  unsigned long long rf[2][4];         // ... references of its tile known, to a warp's rows
  unsigned long long pw[2][2], pv[2];  // ... weights there (of either half of the keys), multiplied
  unsigned tmem;
  int failed;  // a wait has run out
  float m[2][PXT_ROWS], l[2][PXT_ROWS];
};

// What the warps of a CTA in the tiles' role have in common: CTA `cta` has row tile cta % tc_tiles of worker cta / tc_tiles or, where the row tiles are
// more than the CTAs, row tiles cta, cta + n_cta, .. of the one worker.
struct PxtWork {
  long long u_lo, u_hi;
  int worker, workers, rt0, rt_step, all, last_keys, R;
  unsigned base, k_ring, v_ring;  // shared addresses: queries, rings
  unsigned char* base_ptr;
  template <int D>
  __device__ __forceinline__ static PxtWork of(const PrefixParams& p, const PxRoles& roles, unsigned char* raw, int cta) {
    PxtWork w;
    const bool one = p.tc_tiles > roles.tiles;
    w.all = (p.prefix_len + PXT_KEYS - 1) / PXT_KEYS, w.last_keys = p.prefix_len - (w.all - 1) * PXT_KEYS, w.R = p.T * p.G;
    w.workers = roles.workers, w.worker = one ? 0 : cta / p.tc_tiles, w.rt0 = one ? cta : cta % p.tc_tiles, w.rt_step = one ? roles.tiles : p.tc_tiles;
    const long long U = (long long)p.kv.n_kv * w.all;
    w.u_lo = w.worker * U / roles.workers, w.u_hi = (w.worker + 1) * U / roles.workers;
    w.base = (tc_smem_u32(raw) + 1023u) & ~1023u, w.k_ring = w.base + PxCfg<D>::TC_TILE, w.v_ring = w.k_ring + PXT_K_STAGES * PxCfg<D>::TC_TILE;
    w.base_ptr = raw + (w.base - tc_smem_u32(raw));
    return w;
  }
  // f(row tile, kv head, first tile, tiles) for every segment
  template <typename F>
  __device__ __forceinline__ void each(const PrefixParams& p, F f) const {
    for (int rt = rt0; rt < p.tc_tiles; rt += rt_step)
      for (long long u = u_lo; u < u_hi;) {
        const int h = (int)(u / all), k_lo = (int)(u - (long long)h * all), n = (int)min((long long)(all - k_lo), u_hi - u);
        u += n;
        f(rt, h, k_lo, n);
      }
  }
  __device__ __forceinline__ int keys(int tile) const { return tile == all - 1 ? last_keys : PXT_KEYS; }
};
// the softmax warps and the MMA issuers: the segment's queries are there, the last one's accumulators have been read
__device__ __forceinline__ void pxt_segment_sync() {
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  asm volatile("bar.sync 2, 320;" ::: "memory");
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
}

// Producer of the keys or of the values: a lane per box (a tile is D / 64 pieces of [128 keys][64 elements])
template <int D, int STAGES>
__device__ __forceinline__ void pxt_produce(const CUtensorMap& map, const PrefixParams& p, unsigned long long* full, unsigned long long* empty, unsigned ring, const PxtWork& w,
                                            int lane, int& failed) {
  constexpr int TILE = PxCfg<D>::TC_TILE, HALF = PXT_KEYS * 128, NH = D / 64;
  const int slots = min(PXT_KEYS, 1 << p.kv.page_shift), boxes = PXT_KEYS / slots;
  const int box = lane % boxes, half = lane / boxes;
  int s = 0, units = 0;
  unsigned par = 1;
  bool ok = true;
  w.each(p, [&](int, int h, int k_lo, int n) {
    // (after a wait that gave up nothing more is requested: a stage may still be read, or be on its way.  Who waits for it gives up, too)
    for (int i = 0; i < n && ok && units < p.stop_tile; ++i) {
      const int live = (w.keys(k_lo + i) + slots - 1) / slots;  // boxes with keys in them
      const int pos = (k_lo + i) * PXT_KEYS + box * slots;
      const bool mine = half < NH && box < live;
      int page = p.kv.n_pages;
      if (mine) {
        page = __ldg(p.prefix_pages + (pos >> p.kv.page_shift));
        if (page < 0 || page >= p.kv.n_pages) {  // (out of the map's bounds: zeros arrive)
          page = p.kv.n_pages;
          if (p.flag) atomicOr(p.flag, OP_BAD_PAGE);
        }
      }
      if (units >= STAGES) {
        ok = __all_sync(0xffffffffu, px_wait(p, empty + s, par, failed));
        if (!ok) break;
      }
      const unsigned bar = tc_smem_u32(full + s);
      if (lane == 0) tc_mbar_expect_tx(bar, (unsigned)(live * NH * slots * 128));
      __syncwarp();
      if (mine) px_tma_4d(ring + s * TILE + half * HALF + box * slots * 128, &map, bar, half * 64, pos & ((1 << p.kv.page_shift) - 1), h, page);
      ++units;
      if (++s == STAGES) s = 0, par ^= 1u;
    }
  });
}

template <typename T>
__host__ __device__ constexpr unsigned pxt_idesc(int n, bool b_mn_major) {
  return (1u << 4) | (std::is_same<T, __half>::value ? 0u : (1u << 7) | (1u << 10)) | (b_mn_major ? 1u << 16 : 0u) | ((unsigned)(n >> 3) << 17) | ((unsigned)(PXT_ROWS >> 4) << 24);
}

// Issuers of the two products, a warp each (one for both, with five waits a tile, took 2500 cycles of it): a warp walks the tiles together, one elected
// lane issues.  S = Q K^T of a tile into its stream's scores, as soon as the last ones there have been read:
template <typename T, int D>
__device__ __forceinline__ void pxt_scores(const PrefixParams& p, PxtShared& sh, const PxtWork& w, unsigned tmem) {
  constexpr int TILE = PxCfg<D>::TC_TILE, HALF = PXT_KEYS * 128;
  bool ok = true;
  const unsigned long long desc = tc_smem_desc(0), q = desc | ((w.base >> 4) & 0x3FFF);  // 8-row groups 1024 bytes apart
  int s = 0, read[2] = {0, 0};  // ring stage; scores of a stream that have been waited for
  unsigned par = 0;
  w.each(p, [&](int, int, int, int n) {
    pxt_segment_sync();
    for (int i = 0; i < n; ++i) {
      if (i >= 2) ok &= px_wait(p, &sh.sr[i & 1], read[i & 1]++ & 1, sh.failed);
      ok &= px_wait(p, &sh.kfull[s], par, sh.failed);
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      if (tc_elect_one()) {
        const unsigned long long k = desc | (((w.k_ring + s * TILE) >> 4) & 0x3FFF);
        const unsigned d = tmem + (i & 1) * 128;
        if (ok)
#pragma unroll
          for (int ks = 0; ks < D / 16; ++ks) tc_mma(d, q + ((ks >> 2) * HALF + (ks & 3) * 32) / 16, k + ((ks >> 2) * HALF + (ks & 3) * 32) / 16, pxt_idesc<T>(PXT_KEYS, false), ks != 0);
        tc_commit(tc_smem_u32(&sh.kempty[s]));
        tc_commit(tc_smem_u32(&sh.sc[i & 1]));
      }
      __syncwarp();
      if (++s == PXT_K_STAGES) s = 0, par ^= 1u;
    }
    for (int i = max(0, n - 2); i < n; ++i) ok &= px_wait(p, &sh.sr[i & 1], read[i & 1]++ & 1, sh.failed);  // (no phase is missed)
  });
}
// O += P V of a tile as its weights come, the first half of its keys while the second half's exponentials are taken:
template <typename T, int D>
__device__ __forceinline__ void pxt_values(const PrefixParams& p, PxtShared& sh, const PxtWork& w, unsigned tmem, int lane) {
  constexpr int TILE = PxCfg<D>::TC_TILE, HALF = PXT_KEYS * 128, NH = D / 64;
  bool ok = true;
  const unsigned long long desc = tc_smem_desc(0) | (unsigned long long)(HALF >> 4) << 16;  // 8-key groups 1024 bytes apart, the pieces of 64 elements HALF
  int s = 0, done[2] = {0, 0};  // ring stage, tiles of a stream
  unsigned par = 0;
  w.each(p, [&](int, int, int k_lo, int n) {
    pxt_segment_sync();
    for (int i = 0; i < n; ++i) {
      const int keys = w.keys(k_lo + i), steps = (keys + 15) / 16, st = i & 1;
      const unsigned v = w.v_ring + s * TILE;
      ok &= px_wait(p, &sh.vfull[s], par, sh.failed);
      if (keys & 15) {  // values behind the last key, up to a whole step: whatever they are, 0 times them must be 0
        for (int e = lane; e < (steps * 16 - keys) * NH * 8; e += 32) {
          const int c = e & 7, x = (e >> 3) % NH, r = keys + (e >> 3) / NH;
          *reinterpret_cast<uint4*>(w.base_ptr + (v - w.base) + x * HALF + r * 128 + c * 16) = make_uint4(0, 0, 0, 0);
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
      }
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        ok &= px_wait(p, &sh.pw[st][half], done[st] & 1, sh.failed);
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        if (tc_elect_one()) {
          const unsigned long long b = desc | ((v >> 4) & 0x3FFF);
          const unsigned a = tmem + PXT_P + st * 64;
          if (ok)
#pragma unroll
            for (int ks = 4 * half; ks < 4 * half + 4; ++ks)
              if (ks < steps) pxt_mma_ts(tmem + PXT_O, a + ks * 8, b + ks * 128, pxt_idesc<T>(D, true), (i | ks) != 0);
          if (half == 1) {
            tc_commit(tc_smem_u32(&sh.vempty[s]));
            tc_commit(tc_smem_u32(&sh.pv[st]));
          }
        }
        __syncwarp();
      }
      ++done[st];
      if (++s == PXT_V_STAGES) s = 0, par ^= 1u;
    }
  });
}

template <typename T, int D>
__device__ __forceinline__ void pxt_softmax(const PrefixParams& p, PxtShared& sh, const PxtWork& w, unsigned tmem, int tid, int warp, int lane) {
  constexpr int HALF = PXT_KEYS * 128;
  int done = 0, done_other = 0;  // tiles this warp's stream has had, and the other
  w.each(p, [&](int rt, int h, int k_lo, int n) {
    const int r0 = rt * PXT_ROWS;
    // the queries, K-major with the same swizzle; rows beyond the batch are zeros
    for (int i = tid; i < PXT_ROWS * (D / 8); i += 256) {
      const int r = i / (D / 8), c = i % (D / 8), row = r0 + r;
      uint4 v = make_uint4(0, 0, 0, 0);
      if (row < w.R) {
        const int t = row / p.G;
        v = *reinterpret_cast<const uint4*>(static_cast<const T*>(p.q) + (long long)t * p.q_ld + (h * p.G + row - t * p.G) * D + c * 8);
      }
      *reinterpret_cast<uint4*>(w.base_ptr + (c >> 3) * HALF + r * 128 + (((c & 7) ^ (r & 7)) << 4)) = v;
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    pxt_segment_sync();
    // ---- softmax: stream st, a thread per row ----
    const int st = warp >> 2, row = (warp & 3) * 32 + lane;
    const unsigned lanes = (unsigned)((warp & 3) * 32) << 16, t_s = tmem + lanes + st * 128, t_p = tmem + lanes + PXT_P + st * 64, t_o = tmem + lanes + PXT_O;
    const int mine = (n - st + 1) / 2;  // tiles of this stream
    float ref = -INFINITY, l = 0.f;
    for (int j = 0; j < mine; ++j) {
      const int i = 2 * j + st;
      px_wait(p, &sh.sc[st], (done + j) & 1, sh.failed);
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      unsigned v[4][32];
#pragma unroll
      for (int c = 0; c < 4; ++c) pxt_ld32(v[c], t_s + 32 * c);
      pxt_wait_ld();
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      pxt_arrive(tc_smem_u32(&sh.sr[st]), lane);
      const int keys = w.keys(k_lo + i);
      if (keys < PXT_KEYS) {
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int e = 0; e < 32; ++e)
            if (32 * c + e >= keys) v[c][e] = 0xff800000u;
      }
      float mx[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        mx[c] = fmaxf(__uint_as_float(v[c][0]), __uint_as_float(v[c][1]));
#pragma unroll
        for (int e = 2; e < 32; e += 2) mx[c] = pxt_max3(mx[c], __uint_as_float(v[c][e]), __uint_as_float(v[c][e + 1]));
      }
      const float m = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * p.scale_log2;
      // the reference: that of the tile before, unless this one's maximum runs too far ahead of it
      float to = m;
      bool moves = false;
      if (i > 0) {
        px_wait(p, &sh.rf[st ^ 1][warp & 3], (done_other + (st ? j : j - 1)) & 1, sh.failed);
        const float prev = sh.m[st ^ 1][row];
        moves = m > prev + PX_SLACK;
        to = moves ? m : prev;
        if (__any_sync(0xffffffffu, moves)) {  // the accumulator is at rest when the tile before is multiplied: this one's weights are not there yet
          if (j > 0) px_wait(p, &sh.pv[st], (done + j - 1) & 1, sh.failed);  // (tiles are multiplied in order: then the other stream's last phase but one is over)
          px_wait(p, &sh.pv[st ^ 1], (done_other + (st ? j : j - 1)) & 1, sh.failed);
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const float f = to == -INFINITY ? 1.f : px_exp2(prev - to);
#pragma unroll
          for (int c = 0; c < D / 16; ++c) {
            unsigned o[16];
            pxt_ld16(o, t_o + 16 * c);
            pxt_wait_ld();
#pragma unroll
            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
            pxt_st16(t_o + 16 * c, o);
          }
          pxt_wait_st();
        }
      }
      sh.m[st][row] = to;
      pxt_arrive(tc_smem_u32(&sh.rf[st][warp & 3]), lane);
      if (__any_sync(0xffffffffu, to != ref)) l *= to == ref || j == 0 ? 1.f : px_exp2(ref - to);
      ref = to;
      const float sub = ref == -INFINITY ? 0.f : ref;
      const unsigned long long sc2 = two(p.scale_log2, p.scale_log2), sub2 = two(-sub, -sub);
      if (j > 0) px_wait(p, &sh.pv[st], (done + j - 1) & 1, sh.failed);  // this stream's last weights are used up
      unsigned long long sum[2] = {0, 0};
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        unsigned wt[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          float a, b;
          split(fma2(two(__uint_as_float(v[c][2 * e]), __uint_as_float(v[c][2 * e + 1])), sc2, sub2), a, b);
          a = px_exp2(a), b = px_exp2(b);
          sum[e & 1] = add2(sum[e & 1], two(a, b));
          wt[e] = pack2<T>(a, b);
        }
        pxt_st16(t_p + 16 * c, wt);
        if (c & 1) {
          pxt_wait_st();
          asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
          pxt_arrive(tc_smem_u32(&sh.pw[st][c >> 1]), lane);
        }
      }
      float a, b;
      split(add2(sum[0], sum[1]), a, b);
      l += a + b;
    }
    // ---- the row's partial: warps 0 .. 3 the first half of its elements, 4 .. 7 the second ----
    sh.l[st][row] = l;
    if (mine > 0) px_wait(p, &sh.pv[st], (done + mine - 1) & 1, sh.failed);
    done += mine, done_other += n - mine;
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    asm volatile("bar.sync 1, 256;" ::: "memory");
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    // the accumulator is relative to the last tile's reference, a stream's sum to that of its own last tile
    const int end = (n - 1) & 1;
    const float top = sh.m[end][row];
    float mass = sh.l[end][row];
    if (n > 1) {
      const float other = sh.m[end ^ 1][row];
      mass += sh.l[end ^ 1][row] * (other == top ? 1.f : px_exp2(other - (top == -INFINITY ? 0.f : top)));
    }
    const long long tile = k_lo == 0 ? (long long)h * p.tc_tiles + rt : (long long)w.worker * p.tc_tiles + rt;
    float* po = (k_lo == 0 ? p.tc_item_o : p.tc_work_o) + (tile * PXT_ROWS + row) * D;
    float* pm = (k_lo == 0 ? p.tc_item_ml : p.tc_work_ml) + (tile * PXT_ROWS + row) * 2;
    const bool live = r0 + row < w.R;
    if (*const_cast<volatile int*>(&sh.failed)) mass = CUDART_NAN_F;  // whatever was multiplied: no number for a caller without a flag
    if (live && st == 0) __stcg(reinterpret_cast<float2*>(pm), make_float2(top, mass));
    if (k_lo == 0 && tid == 0) p.tc_seg[tile] = make_int2(w.worker, n == w.all ? 1 : 1 + px_worker_of((long long)(h + 1) * w.all - 1, (long long)p.kv.n_kv * w.all, w.workers) - w.worker);
#pragma unroll
    for (int c = 0; c < D / 64; ++c) {
      unsigned o[32];
      pxt_ld32(o, t_o + st * (D / 2) + 32 * c);
      pxt_wait_ld();
      float* dst = po + st * (D / 2) + 32 * c;
      if (live)
#pragma unroll
        for (int e = 0; e < 32; e += 4)
          __stcg(reinterpret_cast<float4*>(dst + e), make_float4(__uint_as_float(o[e]), __uint_as_float(o[e + 1]), __uint_as_float(o[e + 2]), __uint_as_float(o[e + 3])));
    }
  });
}

// Before the warps part: barriers, tensor memory
__device__ __forceinline__ void pxt_begin(PxtShared& sh, int tid, int warp) {
  if (tid == 0) {
    sh.failed = 0;
    for (int s = 0; s < PXT_K_STAGES; ++s) tc_mbar_init(tc_smem_u32(&sh.kfull[s]), 1), tc_mbar_init(tc_smem_u32(&sh.kempty[s]), 1);
    for (int s = 0; s < PXT_V_STAGES; ++s) tc_mbar_init(tc_smem_u32(&sh.vfull[s]), 1), tc_mbar_init(tc_smem_u32(&sh.vempty[s]), 1);
    for (int s = 0; s < 2; ++s) {
      tc_mbar_init(tc_smem_u32(&sh.sc[s]), 1), tc_mbar_init(tc_smem_u32(&sh.pv[s]), 1);
      tc_mbar_init(tc_smem_u32(&sh.sr[s]), 4);
      for (int w = 0; w < 4; ++w) tc_mbar_init(tc_smem_u32(&sh.rf[s][w]), 1);
      tc_mbar_init(tc_smem_u32(&sh.pw[s][0]), 4), tc_mbar_init(tc_smem_u32(&sh.pw[s][1]), 4);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 9) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tc_smem_u32(&sh.tmem)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
}
// ... and after they have met again
__device__ __forceinline__ void pxt_end(const PrefixParams& p, PxtShared& sh, unsigned tmem, int tid, int warp) {
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  const bool failed = *const_cast<volatile int*>(&sh.failed) != 0;
  if (failed && p.flag && tid == 0) atomicOr(p.flag, OP_TIMEOUT);
  if (warp == 9) {
    // a wait that gave up may have left copies in flight: give them a bounded time to land before the memory is freed
    if (failed) {
      const long long t0 = clock64();
      while (clock64() - t0 < 2000000LL) {
      }
    }
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
  }
}

}  // namespace ls
