// The kernels of prefix_attention: roles, and the fold of their partials (see op_attention.cuh).
#pragma once
#include "op_prefix_tiles.cuh"

namespace ls {

template <typename T, int D>
__global__ void __launch_bounds__(PX_THREADS, 1)
    prefix_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const __grid_constant__ PrefixParams p) {
  extern __shared__ __align__(128) unsigned char px_smem[];
  __shared__ __align__(8) PxtShared s_tiles;
  __shared__ int s_w[PX_THREADS / 32];
  __shared__ unsigned long long s_best[PX_THREADS / 32];
  const int tid = threadIdx.x, NP = p.B + p.prefix_rows;
  int* s_unit = reinterpret_cast<int*>(px_smem + PxCfg<D>::MAIN);  // [NP + 1]
  pdl_launch_dependents();

  // ---- the line of the rows' units: every CTA adds it up for itself ----
  int base_u = 0, bad_rows = 0;
  for (int i0 = 0; i0 < NP; i0 += PX_THREADS) {
    const int i = i0 + tid;
    PxProblem r = {0, 0, 0, false, false, false};
    if (i < NP) r = px_problem(p, i);
    bad_rows |= r.bad_rows;
    if ((r.bad_rows || r.bad_len) && p.flag && blockIdx.x == 0) atomicOr(p.flag, OP_BAD_ROWS);
    const int units = (r.n * p.G + 15) / 16 * ((r.len + PXR_KEYS - 1) / PXR_KEYS);
    int total;
    const int before = base_u + px_block_scan(units, s_w, total) - units;
    base_u += total;
    if (i < NP) s_unit[i] = before;
  }
  if (tid == 0) s_unit[NP] = base_u;
  bad_rows = __syncthreads_or(bad_rows);
  if (bad_rows) base_u = 0;  // (rows could belong to several sequences: their units would not be what the host has made room for)
  if (blockIdx.x == 0 && tid == 0) *p.state = bad_rows;
  PxRoles roles = px_roles<D>(p, (long long)base_u * p.kv.n_kv, s_best);
  // (uniform to the compiler, and with them all that the loops below run over: the MMAs' operands have to sit in uniform registers)
  base_u = __shfl_sync(0xffffffffu, base_u, 0), roles.workers = __shfl_sync(0xffffffffu, roles.workers, 0), roles.tiles = __shfl_sync(0xffffffffu, roles.tiles, 0);
  // Registers go where the work is: 168 a thread at launch (12 warps), from here on 216 for the first eight warps and 72 for the others
  // (2 x 216 + 72 = 3 x 168: px_launch makes sure of the 168).
  const int lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  const bool tiles = (int)blockIdx.x < roles.tiles;
  PxtWork w;
  unsigned tmem = 0;
  if (tiles) {
    w = PxtWork::of<D>(p, roles, px_smem, blockIdx.x);
    pxt_begin(s_tiles, tid, warp);
    tmem = s_tiles.tmem;
  }
  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    if (tiles && warp == 8) pxt_produce<D, PXT_K_STAGES>(map_k, p, s_tiles.kfull, s_tiles.kempty, w.k_ring, w, lane, s_tiles.failed);
    if (tiles && warp == 9) pxt_scores<T, D>(p, s_tiles, w, tmem);
    if (tiles && warp == 10) pxt_values<T, D>(p, s_tiles, w, tmem, lane);
    if (tiles && warp == 11) pxt_produce<D, PXT_V_STAGES>(map_v, p, s_tiles.vfull, s_tiles.vempty, w.v_ring, w, lane, s_tiles.failed);
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
    if (tiles) pxt_softmax<T, D>(p, s_tiles, w, tmem, tid, warp, lane);
    else if (base_u > 0) px_rows_role<T, D>(p, px_smem, s_unit, base_u, blockIdx.x - roles.tiles, PX_SMS - roles.tiles);
  }
  if (tiles) pxt_end(p, s_tiles, tmem, tid, warp);
}

// WPR warps per sequence and query head: a row's partials - of the prefix and of the sequence's own keys - in a fixed order, a lane looking one up each.  A
// chain of a few dependent reads that a warp runs once or twice: what counts is that it is short, in code most of all, which is not in the
// instruction cache (16 KB of it took 10 us where there were 35 partials to fold).
template <typename T, int D, int WPR>
__global__ void __launch_bounds__(128) prefix_merge_kernel(const __grid_constant__ PrefixParams p) {
  constexpr int V = D / 32, AHEAD = WPR > 1 ? 12 : 4;  // elements per lane, partials in flight
  __shared__ float s_o[WPR > 1 ? 4 : 1][D], s_ml[4][2];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, at = WPR > 1 ? blockIdx.x : blockIdx.x * 4 + warp;
  const int b = at / p.nq, head = at - b * p.nq, h = head / p.G;
  if (b >= p.B) return;
  const PxProblem own = px_problem(p, b + p.prefix_rows);
  const int own_tile = h * p.max_tiles + px_first_tile(p, b + p.prefix_rows, own);
  pdl_wait();
  const bool there = __ldcg(p.state) == 0;
#pragma unroll 1
  for (int j = blockIdx.y; j < own.n; j += gridDim.y) {
    const int row = own.row0 + j, r = j * p.G + head - h * p.G, pr = row * p.G + head - h * p.G;  // the row's numbers in its own problem and in the prefix'
    // its tiles' slots, and the segments there are: first worker, number
    const int tc_tile = h * p.tc_tiles + (pr >> 7), pre_tile = h * p.max_tiles + (pr >> 4), mine = own_tile + (r >> 4);
    int2 st = make_int2(0, 0), sp = st, so = st;
    if (p.tc_tiles) st = __ldcg(p.tc_seg + tc_tile);
    if (p.prefix_rows) sp = __ldcg(p.item_seg + pre_tile);
    if (own.len > 0) so = __ldcg(p.item_seg + mine);
    const int count = there ? st.y + sp.y + so.y : 0;
    float m = -INFINITY, l = 0.f, acc[V];
#pragma unroll
    for (int e = 0; e < V; ++e) acc[e] = 0.f;
#pragma unroll 1
    for (int x0 = WPR > 1 ? warp : 0; x0 < count; x0 += 32 * WPR) {  // (the warps take them in turn)
      // this lane's partial: the first of a tile is in the tile's own slot, the others in those of the workers that follow
      int x = x0 + lane * WPR;
      const int cnt = min(32, (count - x0 + WPR - 1) / WPR);
      const float *po = p.item_o, *pm = p.item_ml;
      long long slot = 0;
      if (x < st.y) {
        slot = (long long)(x == 0 ? tc_tile : (st.x + x) * p.tc_tiles + (pr >> 7)) * 128 + (pr & 127);
        po = x == 0 ? p.tc_item_o : p.tc_work_o, pm = x == 0 ? p.tc_item_ml : p.tc_work_ml;
      } else if (x < count) {
        x -= st.y;
        const bool pre = x < sp.y;
        x -= pre ? 0 : sp.y;
        slot = (long long)(x == 0 ? (pre ? pre_tile : mine) : (pre ? sp.x : so.x) + x) * 16 + ((pre ? pr : r) & 15);
        if (x) po = p.warp_o, pm = p.warp_ml;
      }
      float2 ml = make_float2(-INFINITY, 0.f);
      if (lane < cnt) ml = __ldcg(reinterpret_cast<const float2*>(pm) + slot);
      unsigned long long src = reinterpret_cast<unsigned long long>(po + slot * D);
      const float mx = fmaxf(m, warp_max(ml.x)), ref = mx == -INFINITY ? 0.f : mx;
      const float wt = px_exp2(ml.x - ref), keep = px_exp2(m - ref);
      m = mx;
      l = l * keep + warp_sum(ml.y * wt);
#pragma unroll
      for (int e = 0; e < V; ++e) acc[e] *= keep;
#pragma unroll 1
      for (int y0 = 0; y0 < cnt; y0 += AHEAD) {
        float v[AHEAD][V], f[AHEAD];
#pragma unroll
        for (int y = 0; y < AHEAD; ++y) {  // (behind the last: the last again, with a weight of 0)
          const float* s = reinterpret_cast<const float*>(__shfl_sync(0xffffffffu, src, min(y0 + y, cnt - 1))) + lane * V;
          f[y] = __shfl_sync(0xffffffffu, wt, y0 + y < cnt ? y0 + y : 31);
          if (y0 + y >= cnt) f[y] = 0.f;
          if constexpr (V == 4) *reinterpret_cast<float4*>(v[y]) = __ldcg(reinterpret_cast<const float4*>(s));
          else *reinterpret_cast<float2*>(v[y]) = __ldcg(reinterpret_cast<const float2*>(s));
        }
#pragma unroll
        for (int y = 0; y < AHEAD; ++y)
#pragma unroll
          for (int e = 0; e < V; ++e)
            if (y0 + y < cnt) acc[e] = fmaf(f[y], v[y][e], acc[e]);
      }
    }
    if constexpr (WPR > 1) {  // the warps' sums, in order
      __syncthreads();
#pragma unroll
      for (int e = 0; e < V; ++e) s_o[warp][lane * V + e] = acc[e];
      if (lane == 0) s_ml[warp][0] = m, s_ml[warp][1] = l;
      __syncthreads();
      if (warp) continue;
      const float top = fmaxf(fmaxf(s_ml[0][0], s_ml[1][0]), fmaxf(s_ml[2][0], s_ml[3][0])), ref = top == -INFINITY ? 0.f : top;
      m = top, l = 0.f;
#pragma unroll
      for (int e = 0; e < V; ++e) acc[e] = 0.f;
#pragma unroll 1
      for (int w = 0; w < 4; ++w) {
        const float f = px_exp2(s_ml[w][0] - ref);
        l = fmaf(s_ml[w][1], f, l);
#pragma unroll
        for (int e = 0; e < V; ++e) acc[e] = fmaf(s_o[w][lane * V + e], f, acc[e]);
      }
    }
    const float inv = l == 0.f ? 0.f : __fdividef(1.f, l);  // a row that sees no key: zeros
    T* dst = static_cast<T*>(p.out) + (long long)row * p.out_ld + head * D + lane * V;
#pragma unroll
    for (int e = 0; e < V; e += 2) *reinterpret_cast<unsigned*>(dst + e) = pack2<T>(acc[e] * inv, acc[e + 1] * inv);
    if (p.lse && lane == 0) p.lse[(long long)row * p.nq + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
  }
}

}  // namespace ls
