// The kernels of prefix_attention: roles, and the fold of their partials (see op_attention.cuh).
#pragma once
#include "op_prefix_tiles.cuh"

namespace ls {

template <typename T, int D>
__global__ void __launch_bounds__(PX_THREADS, 1)
    prefix_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const __grid_constant__ PrefixParams p) {
  extern __shared__ __align__(128) unsigned char px_smem[];
  __shared__ __align__(8) PxtShared s_tiles;
  __shared__ long long s_w[PX_THREADS / 32];
  const int tid = threadIdx.x, NP = p.B + p.prefix_rows;
  int* s_unit = reinterpret_cast<int*>(px_smem + PxCfg<D>::MAIN);  // [NP + 1]
  int* s_item = s_unit + NP + 1;                                    // [NP + 1]
  pdl_launch_dependents();

  // ---- the line of the rows' units: every CTA adds it up for itself ----
  long long before = 0;  // row tiles (upper word) and units of the problems so far
  for (int i0 = 0; i0 < NP; i0 += PX_THREADS) {
    const int i = i0 + tid;
    PxProblem r = {0, 0, 0, false, false};
    if (i < NP) r = px_problem(p, i);
    if (r.bad && p.flag && blockIdx.x == 0) atomicOr(p.flag, OP_BAD_ROWS);
    const int rt = r.len > 0 ? (r.n * p.G + 15) / 16 : 0;
    const long long x = (long long)rt << 32 | (unsigned)(rt * ((r.len + PXR_KEYS - 1) / PXR_KEYS));
    long long total;
    const long long mine = before + px_block_scan(x, s_w, total) - x;
    before += total;
    if (i < NP) s_item[i] = (int)(mine >> 32), s_unit[i] = (int)(unsigned)mine;
  }
  if (tid == 0) s_item[NP] = (int)(before >> 32), s_unit[NP] = (int)(unsigned)before;
  __syncthreads();
  int base_u = (int)(unsigned)before;
  if ((before >> 32) > p.max_tiles) {  // row counts that overlap: no room for their partials, so nothing of the rows' is done
    if (p.flag && tid == 0 && blockIdx.x == 0) atomicOr(p.flag, OP_BAD_ROWS);
    for (int i = tid; i <= NP; i += PX_THREADS) s_item[i] = s_unit[i] = 0;
    base_u = 0;
    __syncthreads();
  }
  PxRoles roles = px_roles<D>(p, (long long)base_u * p.kv.n_kv, s_w);
  // (uniform to the compiler, and with them all that the loops below run over: the MMAs' operands have to sit in uniform registers)
  base_u = __shfl_sync(0xffffffffu, base_u, 0), roles.workers = __shfl_sync(0xffffffffu, roles.workers, 0), roles.tiles = __shfl_sync(0xffffffffu, roles.tiles, 0);
  if (blockIdx.x == 0) {
    for (int i = tid; i < 2 * NP + 2; i += PX_THREADS) p.plan[i] = s_unit[i];
    if (tid == 0) p.plan[2 * NP + 2] = roles.workers, p.plan[2 * NP + 3] = PX_SMS - roles.tiles;
  }
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
  bool ok = true;
  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    if (tiles && warp == 8) pxt_produce<D, PXT_K_STAGES>(map_k, p, s_tiles.kfull, s_tiles.kempty, w.k_ring, w, lane, ok);
    if (tiles && warp == 9) pxt_scores<T, D>(p, s_tiles, w, tmem, ok);
    if (tiles && warp == 10) pxt_values<T, D>(p, s_tiles, w, tmem, lane, ok);
    if (tiles && warp == 11) pxt_produce<D, PXT_V_STAGES>(map_v, p, s_tiles.vfull, s_tiles.vempty, w.v_ring, w, lane, ok);
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
    if (tiles) pxt_softmax<T, D>(p, s_tiles, w, tmem, tid, warp, lane, ok);
    else if (base_u > 0) px_rows_role<T, D>(p, px_smem, s_unit, s_item, base_u, blockIdx.x - roles.tiles, PX_SMS - roles.tiles);
  }
  if (tiles) pxt_end(p, tmem, warp, ok);
}

// WPR warps per (row, query head): its partials - of the prefix and of the sequence's own keys - in a fixed order, a lane looking one up each.
template <typename T, int D, int WPR>
__global__ void __launch_bounds__(128) prefix_merge_kernel(const __grid_constant__ PrefixParams p) {
  constexpr int V = D / 32;  // elements per lane
  __shared__ float s_o[WPR > 1 ? 4 : 1][D], s_ml[4][2];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, h = blockIdx.x, b = blockIdx.y, NP = p.B + p.prefix_rows, i_own = b + p.prefix_rows;
  const PxProblem own = px_problem(p, i_own);
  const int R = own.n * p.G, all = (p.prefix_len + PXT_KEYS - 1) / PXT_KEYS;
  pdl_wait();
  // the lines the work was dealt on
  const int Us = __ldcg(p.plan + NP), o0 = __ldcg(p.plan + i_own), o1 = __ldcg(p.plan + i_own + 1), o_item = __ldcg(p.plan + NP + 1 + i_own);
  const int p1 = p.prefix_rows ? __ldcg(p.plan + 1) : 0, workers = __ldcg(p.plan + 2 * NP + 2), n_cta = __ldcg(p.plan + 2 * NP + 3);
  const long long U = (long long)Us * p.kv.n_kv, Ut = (long long)p.kv.n_kv * all;
  const int W = px_workers(n_cta * PXR_WARPS, U);
  // a problem's segments are in its row tile's own slot, then in those of the workers that follow
  struct Line {
    int w0, n;
  };
  auto line_of = [&](long long first, int count, long long units, int w) -> Line {
    const int w0 = px_worker_of(first, units, w);
    return {w0, 1 + px_worker_of(first + count - 1, units, w) - w0};
  };
  Line lt = {0, 0};
  if (workers) lt = line_of((long long)h * all, all, Ut, workers);
  for (int r = WPR > 1 ? blockIdx.z : blockIdx.z * 4 + warp; r < R; r += WPR > 1 ? gridDim.z : 4 * gridDim.z) {
    const int j = r / p.G, row = own.row0 + j, head = h * p.G + (r - j * p.G), pr = row * p.G + (r - j * p.G);  // pr: the row's number in the prefix problem
    Line lp = {0, 0}, lo = {0, 0};
    const int kp = (p.prefix_len + PXR_KEYS - 1) / PXR_KEYS, ko = (own.len + PXR_KEYS - 1) / PXR_KEYS;
    if (p1 > 0) lp = line_of((long long)h * Us + (long long)(pr >> 4) * kp, kp, U, W);
    if (o1 > o0) lo = line_of((long long)h * Us + o0 + (long long)(r >> 4) * ko, ko, U, W);
    const int count = lt.n + lp.n + lo.n;
    float m = -INFINITY, l = 0.f, acc[V];
#pragma unroll
    for (int e = 0; e < V; ++e) acc[e] = 0.f;
    for (int x0 = WPR > 1 ? warp * 32 : 0; x0 < count; x0 += 32 * WPR) {
      // this lane's partial
      int x = x0 + lane;
      const float *po = p.item_o, *pm = nullptr;
      if (x < count) {
        if (x < lt.n) {
          const long long at = ((x == 0 ? (long long)h : (long long)(lt.w0 + x)) * p.tc_tiles + (pr >> 7)) * 128 + (pr & 127);
          po = (x == 0 ? p.tc_item_o : p.tc_work_o) + at * D, pm = (x == 0 ? p.tc_item_ml : p.tc_work_ml) + at * 2;
        } else {
          x -= lt.n;
          const bool pre = x < lp.n;
          if (!pre) x -= lp.n;
          const int rr = pre ? pr : r;
          const long long at = (x == 0 ? (long long)h * p.max_tiles + (pre ? 0 : o_item) + (rr >> 4) : (long long)((pre ? lp.w0 : lo.w0) + x)) * 16 + (rr & 15);
          po = (x == 0 ? p.item_o : p.warp_o) + at * D, pm = (x == 0 ? p.item_ml : p.warp_ml) + at * 2;
        }
      }
      const float2 ml = pm ? __ldcg(reinterpret_cast<const float2*>(pm)) : make_float2(-INFINITY, 0.f);
      const float mx = fmaxf(m, warp_max(ml.x)), ref = mx == -INFINITY ? 0.f : mx;
      const float wt = px_exp2(ml.x - ref), keep = px_exp2(m - ref);
      m = mx;
      l = l * keep + warp_sum(ml.y * wt);
#pragma unroll
      for (int e = 0; e < V; ++e) acc[e] *= keep;
      const int cnt = min(32, count - x0);
      for (int y0 = 0; y0 < cnt; y0 += 8) {
        float v[8][V];
#pragma unroll
        for (int y = 0; y < 8; ++y) {
          const float* src = reinterpret_cast<const float*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(po), y0 + y)) + lane * V;
#pragma unroll
          for (int e = 0; e < V; ++e) v[y][e] = 0.f;
          if (y0 + y < cnt) {
            if constexpr (V == 4) {
              const float4 z = __ldcg(reinterpret_cast<const float4*>(src));
              v[y][0] = z.x, v[y][1] = z.y, v[y][2] = z.z, v[y][3] = z.w;
            } else {
              const float2 z = __ldcg(reinterpret_cast<const float2*>(src));
              v[y][0] = z.x, v[y][1] = z.y;
            }
          }
        }
#pragma unroll
        for (int y = 0; y < 8; ++y) {
          const float f = __shfl_sync(0xffffffffu, wt, y0 + y);
#pragma unroll
          for (int e = 0; e < V; ++e) acc[e] = y0 + y < cnt ? fmaf(f, v[y][e], acc[e]) : acc[e];
        }
      }
    }
    if constexpr (WPR > 1) {  // the warps' sums, in order
      __syncthreads();
#pragma unroll
      for (int e = 0; e < V; ++e) s_o[warp][lane * V + e] = acc[e];
      if (lane == 0) s_ml[warp][0] = m, s_ml[warp][1] = l;
      __syncthreads();
      if (warp) continue;
      float top = m;
      for (int w = 1; w < 4; ++w) top = fmaxf(top, s_ml[w][0]);
      const float ref = top == -INFINITY ? 0.f : top;
      l = 0.f;
#pragma unroll
      for (int e = 0; e < V; ++e) acc[e] = 0.f;
      for (int w = 0; w < 4; ++w) {
        const float f = px_exp2(s_ml[w][0] - ref);
        l = fmaf(s_ml[w][1], f, l);
#pragma unroll
        for (int e = 0; e < V; ++e) acc[e] = fmaf(s_o[w][lane * V + e], f, acc[e]);
      }
      m = top;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;  // a row that sees no key: zeros
    T* dst = static_cast<T*>(p.out) + (long long)row * p.out_ld + head * D + lane * V;
#pragma unroll
    for (int e = 0; e < V; e += 2) *reinterpret_cast<unsigned*>(dst + e) = pack2<T>(acc[e] * inv, acc[e + 1] * inv);
    if (p.lse && lane == 0) p.lse[(long long)row * p.nq + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
  }
}

}  // namespace ls
