// Attention of many rows to the shared prefix on the fifth-generation tensor cores (see op_attention.cuh for the problem it solves).
//
// A CTA takes 128 rows - token rows x the query heads of a kv head - and a range of 128-key tiles.  Scores Q K^T land in tensor memory, a thread
// per row reads its 128 of them, and the weights go back over them as the 16-bit A operand of P V, whose accumulator stays in tensor
// memory.  The tiles go to two streams in turn, each with scores, weights, accumulator and four softmax warps of its own: while one stream's
// warps take their exponentials the tensor core multiplies for the other.  A row's accumulator is rescaled only when its maximum has
// grown by more than 2^8 (weights up to 256 keep their relative precision); the streams are merged at the end, and a CTA leaves one partial
// per row.
//
// A tile's keys and values arrive by TMA, one box per page and 64 elements of a head (the page table is read by the producer's lanes, so a tile
// of small pages is 32 requests of a warp at once), 128-byte swizzle: K as a K-major operand, V - rows of keys - as an MN-major one.
//
// What bounds it: 16,384 exponentials per tile at 16 a cycle and SM and, at head size 128, the two products take 1024 cycles of a tile each.
#pragma once
#include <cuda.h>

#include "op_attention.cuh"
#include "tc.cuh"

namespace ls {

constexpr int PXT_THREADS = 320;  // 4 + 4 softmax warps, producer, MMA issuer
constexpr int PXT_ROWS = 128, PXT_KEYS = 128;
constexpr int PXT_STAGES = 5;     // keys or values of a tile each
constexpr float PXT_SLACK = 8.f;  // (log2) how far a row's maximum may run ahead of its reference
constexpr long long PXT_WAIT_CYCLES = 400000000LL;  // ~0.2 s: a wait that runs this long gives up and leaves its flag

__host__ __device__ constexpr int pxt_tile_bytes(int D) { return PXT_KEYS * D * 2; }
__host__ __device__ constexpr int pxt_smem(int D) { return 1024 + (1 + PXT_STAGES) * pxt_tile_bytes(D); }

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
__device__ __forceinline__ void pxt_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void pxt_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void pxt_arrive(unsigned bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void pxt_tma_4d(unsigned dst, const CUtensorMap* map, unsigned bar, int x, int y, int z, int w) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(dst),
               "l"(reinterpret_cast<unsigned long long>(map)), "r"(bar), "r"(x), "r"(y), "r"(z), "r"(w)
               : "memory");
}
// A in tensor memory (two 16-bit values a column), B in shared memory
__device__ __forceinline__ void pxt_mma_ts(unsigned d, unsigned a, unsigned long long b, unsigned idesc, unsigned accumulate) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b),
               "r"(idesc), "r"(accumulate)
               : "memory");
}

template <typename T, int D>
__global__ void __launch_bounds__(PXT_THREADS, 1)
    prefix_tc_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const __grid_constant__ PrefixParams p) {
  constexpr int TILE = pxt_tile_bytes(D), HALF = PXT_KEYS * 128, NH = D / 64;  // a tile is NH pieces of [128 keys][64 elements]
  extern __shared__ unsigned char pxt_raw[];
  __shared__ __align__(8) unsigned long long s_full[PXT_STAGES], s_empty[PXT_STAGES], s_sc[2], s_pw[2], s_ov[2];
  __shared__ unsigned s_tmem;
  __shared__ float s_m[2][PXT_ROWS], s_l[2][PXT_ROWS];
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const unsigned base = (tc_smem_u32(pxt_raw) + 1023u) & ~1023u, ring = base + TILE;
  unsigned char* base_ptr = pxt_raw + (base - tc_smem_u32(pxt_raw));

  // (row tiles fastest: those that read the same keys run next to each other)
  const int rt = blockIdx.x % p.tc_tiles, rest = blockIdx.x / p.tc_tiles, sp = rest % p.tc_splits, h = rest / p.tc_splits;
  const int R = p.T * p.G, r0 = rt * PXT_ROWS;
  const int all = (p.prefix_len + PXT_KEYS - 1) / PXT_KEYS, k_lo = (int)((long long)all * sp / p.tc_splits);
  const int n = (int)((long long)all * (sp + 1) / p.tc_splits) - k_lo;  // tiles of this CTA (at least one)
  const int last_keys = p.prefix_len - (all - 1) * PXT_KEYS;            // keys of the last tile of all
  auto keys_of = [&](int i) { return k_lo + i == all - 1 ? last_keys : PXT_KEYS; };

  pdl_launch_dependents();
  if (tid == 0) {
    for (int s = 0; s < PXT_STAGES; ++s) tc_mbar_init(tc_smem_u32(&s_full[s]), 1), tc_mbar_init(tc_smem_u32(&s_empty[s]), 1);
    for (int s = 0; s < 2; ++s) tc_mbar_init(tc_smem_u32(&s_sc[s]), 1), tc_mbar_init(tc_smem_u32(&s_pw[s]), 128), tc_mbar_init(tc_smem_u32(&s_ov[s]), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 9) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tc_smem_u32(&s_tmem)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  } else if (warp < 8) {  // the queries, K-major with the same swizzle; rows beyond the batch are zeros
    for (int i = tid; i < PXT_ROWS * (D / 8); i += 256) {
      const int r = i / (D / 8), c = i % (D / 8), row = r0 + r;
      uint4 v = make_uint4(0, 0, 0, 0);
      if (row < R) {
        const int t = row / p.G;
        v = *reinterpret_cast<const uint4*>(static_cast<const T*>(p.q) + (long long)t * p.q_ld + (h * p.G + row - t * p.G) * D + c * 8);
      }
      *reinterpret_cast<uint4*>(base_ptr + (c >> 3) * HALF + r * 128 + (((c & 7) ^ (r & 7)) << 4)) = v;
    }
  }
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const unsigned tmem = s_tmem;
  bool ok = true;
  auto wait = [&](unsigned long long* bar, unsigned parity) {  // bounded; after the first failure every later wait gives up at once
    if (!tc_mbar_wait(tc_smem_u32(bar), parity, ok ? PXT_WAIT_CYCLES : 2000LL)) ok = false;
  };

  if (warp == 8) {
    // ---- producer: keys 0, keys 1, values 0, keys 2, values 1, ... a lane per box ----
    const int slots = min(PXT_KEYS, 1 << p.kv.page_shift), boxes = PXT_KEYS / slots;
    const int box = lane % boxes, half = lane / boxes;
    int s = 0, u = 0;
    unsigned par = 1;
    auto load = [&](int i, const CUtensorMap* map) {
      if (u >= PXT_STAGES) wait(&s_empty[s], par);
      const int live = (keys_of(i) + slots - 1) / slots;  // boxes with keys in them
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
      const unsigned bar = tc_smem_u32(&s_full[s]);
      if (lane == 0) tc_mbar_expect_tx(bar, (unsigned)(live * NH * slots * 128));
      __syncwarp();
      if (mine) pxt_tma_4d(ring + s * TILE + half * HALF + box * slots * 128, map, bar, half * 64, pos & ((1 << p.kv.page_shift) - 1), h, page);
      ++u;
      if (++s == PXT_STAGES) s = 0, par ^= 1u;
    };
    load(0, &map_k);
    if (n > 1) load(1, &map_k);
    for (int i = 0; i < n; ++i) {
      load(i, &map_v);
      if (i + 2 < n) load(i + 2, &map_k);
    }
  } else if (warp == 9) {
    // ---- MMA issuer: the warp walks the tiles together, one elected lane issues ----
    constexpr unsigned fmt = std::is_same<T, __half>::value ? 0u : 1u;
    constexpr unsigned idesc_qk = (1u << 4) | (fmt << 7) | (fmt << 10) | ((unsigned)(PXT_KEYS >> 3) << 17) | ((unsigned)(PXT_ROWS >> 4) << 24);
    constexpr unsigned idesc_pv = (1u << 4) | (fmt << 7) | (fmt << 10) | (1u << 16) | ((unsigned)(D >> 3) << 17) | ((unsigned)(PXT_ROWS >> 4) << 24);
    const unsigned long long desc = tc_smem_desc(0);  // 8-row groups 1024 bytes apart; for the values also: their two halves HALF bytes apart
    const unsigned long long desc_v = desc | (unsigned long long)(HALF >> 4) << 16;
    int s = 0;
    unsigned par = 0;
    auto next = [&]() {
      if (++s == PXT_STAGES) s = 0, par ^= 1u;
    };
    auto scores = [&](int i) {  // S = Q K^T of tile i into its stream's scores
      wait(&s_full[s], par);
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      if (tc_elect_one()) {
        const unsigned k = ring + s * TILE;
        if (ok)
#pragma unroll
          for (int ks = 0; ks < D / 16; ++ks) {
            const unsigned off = (ks >> 2) * HALF + (ks & 3) * 32;
            tc_mma(tmem + (i & 1) * 128, desc | ((base + off) >> 4 & 0x3FFF), desc | ((k + off) >> 4 & 0x3FFF), idesc_qk, ks != 0);
          }
        tc_commit(tc_smem_u32(&s_empty[s]));
        tc_commit(tc_smem_u32(&s_sc[i & 1]));
      }
      __syncwarp();
      next();
    };
    scores(0);
    if (n > 1) scores(1);
    for (int i = 0; i < n; ++i) {
      wait(&s_full[s], par);
      const int keys = keys_of(i), steps = (keys + 15) / 16;
      const unsigned v = ring + s * TILE;
      if (keys & 15) {  // values behind the last key, up to a whole step: whatever they are, 0 times them must be 0
        for (int e = lane; e < (steps * 16 - keys) * NH * 8; e += 32) {
          const int c = e & 7, x = (e >> 3) % NH, r = keys + (e >> 3) / NH;
          *reinterpret_cast<uint4*>(base_ptr + (v - base) + x * HALF + r * 128 + c * 16) = make_uint4(0, 0, 0, 0);
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
      }
      wait(&s_pw[i & 1], (i >> 1) & 1);
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      if (tc_elect_one()) {
        if (ok)
#pragma unroll
          for (int ks = 0; ks < PXT_KEYS / 16; ++ks)
            if (ks < steps) pxt_mma_ts(tmem + 256 + (i & 1) * 128, tmem + (i & 1) * 128 + ks * 8, desc_v | ((v + ks * 2048) >> 4 & 0x3FFF), idesc_pv, (i >= 2) | (ks != 0));
        tc_commit(tc_smem_u32(&s_empty[s]));
        tc_commit(tc_smem_u32(&s_ov[i & 1]));
      }
      __syncwarp();
      next();
      if (i + 2 < n) scores(i + 2);
    }
  } else {
    // ---- softmax: stream st, a thread per row ----
    const int st = warp >> 2, row = (warp & 3) * 32 + lane;
    const unsigned lanes = (unsigned)((warp & 3) * 32) << 16, t_s = tmem + lanes + st * 128, t_o = tmem + lanes + 256;
    const int mine = (n - st + 1) / 2;  // tiles of this stream
    float ref = -INFINITY, l = 0.f;
    for (int j = 0; j < mine; ++j) {
      wait(&s_sc[st], j & 1);
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      unsigned v[4][32];
#pragma unroll
      for (int c = 0; c < 4; ++c) pxt_ld32(v[c], t_s + 32 * c);
      pxt_wait_ld();
      const int keys = keys_of(2 * j + st);
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
        mx[c] = __uint_as_float(v[c][0]);
#pragma unroll
        for (int e = 1; e < 32; ++e) mx[c] = fmaxf(mx[c], __uint_as_float(v[c][e]));
      }
      const float m = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * p.scale_log2;
      if (j > 0) wait(&s_ov[st], (j - 1) & 1);  // (done by now: the scores were multiplied after it) the accumulator is at rest until these weights are handed over
      if (j == 0) ref = m;
      else if (__any_sync(0xffffffffu, m > ref + PXT_SLACK)) {
        const float to = fmaxf(m, ref), f = to == -INFINITY ? 1.f : px_exp2(ref - to);
        ref = to, l *= f;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {
          unsigned o[16];
          pxt_ld16(o, t_o + st * 128 + 16 * c);
          pxt_wait_ld();
#pragma unroll
          for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
          pxt_st16(t_o + st * 128 + 16 * c, o);
        }
      }
      const float sub = ref == -INFINITY ? 0.f : ref;
      float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        unsigned w[16];
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
          const float a = px_exp2(fmaf(__uint_as_float(v[c][e]), p.scale_log2, -sub)), b = px_exp2(fmaf(__uint_as_float(v[c][e + 1]), p.scale_log2, -sub));
          sum[(e >> 1) & 3] += a + b;
          w[e >> 1] = pack2<T>(a, b);
        }
        pxt_st16(t_s + 16 * c, w);
      }
      l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
      pxt_wait_st();
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      pxt_arrive(tc_smem_u32(&s_pw[st]));
    }
    // ---- the streams' parts of a row are merged: warps 0 .. 3 the first half of its elements, 4 .. 7 the second ----
    s_m[st][row] = ref, s_l[st][row] = l;
    if (mine > 0) wait(&s_ov[st], (mine - 1) & 1);
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    asm volatile("bar.sync 1, 256;" ::: "memory");
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const float m0 = s_m[0][row], m1 = s_m[1][row], top = fmaxf(m0, m1), sub = top == -INFINITY ? 0.f : top;
    const float f0 = px_exp2(m0 - sub), f1 = n > 1 ? px_exp2(m1 - sub) : 0.f;
    const long long slot = ((long long)(h * p.tc_tiles + rt) * p.tc_splits + sp) * PXT_ROWS + row;
    const bool live = r0 + row < R;
    if (live && st == 0) __stcg(reinterpret_cast<float2*>(p.tc_ml + slot * 2), make_float2(top, s_l[0][row] * f0 + (n > 1 ? s_l[1][row] * f1 : 0.f)));
#pragma unroll
    for (int c = 0; c < D / 64; ++c) {
      unsigned a[32], b[32];
      const unsigned at = t_o + st * (D / 2) + 32 * c;
      pxt_ld32(a, at);
      if (n > 1) pxt_ld32(b, at + 128);  // (uniform; without a second tile the second accumulator holds nothing)
      pxt_wait_ld();
      float* dst = p.tc_o + slot * D + st * (D / 2) + 32 * c;
      if (live) {
#pragma unroll
        for (int e = 0; e < 32; e += 4) {
          float x[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            x[i] = __uint_as_float(a[e + i]) * f0;
            if (n > 1) x[i] = fmaf(__uint_as_float(b[e + i]), f1, x[i]);
          }
          __stcg(reinterpret_cast<float4*>(dst + e), make_float4(x[0], x[1], x[2], x[3]));
        }
      }
    }
  }
  if (!ok && p.flag) atomicOr(p.flag, OP_TIMEOUT);
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  const int failed = __syncthreads_or(!ok);
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
