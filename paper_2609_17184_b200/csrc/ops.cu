// C ABI of the operators between the linear maps (see include/loopspec.h): checks of the arguments, rules that choose a kernel's
// variant, launches.  No call synchronises, allocates or keeps anything (but which kernels may use how much shared memory, and the driver's
// function that encodes tensor maps).
#include "../../include/loopspec.h"

#include <algorithm>
#include <atomic>
#include <climits>
#include <cmath>
#include <cstring>

#include "op_append.cuh"
#include "op_prefix.cuh"
#include "op_sample.cuh"

using namespace ls;

namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
bool pow2(int x) { return x > 0 && (x & (x - 1)) == 0; }
int log2_of(int x) {
  int s = 0;
  while ((1 << s) < x) ++s;
  return s;
}

// pdl: the kernel may start while its predecessor still runs and orders itself with griddepcontrol.wait
template <typename P>
int launch(void (*fn)(const P), dim3 grid, int block, size_t smem, void* stream, const P& params, bool pdl = false, int cluster = 0) {
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof cfg);
  cfg.gridDim = grid, cfg.blockDim = dim3(block), cfg.dynamicSmemBytes = smem, cfg.stream = static_cast<cudaStream_t>(stream);
  cudaLaunchAttribute at[2];
  int n = 0;
  if (pdl) at[n].id = cudaLaunchAttributeProgrammaticStreamSerialization, at[n++].val.programmaticStreamSerializationAllowed = 1;
  if (cluster > 0) {
    at[n].id = cudaLaunchAttributeClusterDimension;
    at[n].val.clusterDim.x = cluster, at[n].val.clusterDim.y = 1, at[n].val.clusterDim.z = 1;
    ++n;
  }
  cfg.attrs = at, cfg.numAttrs = n;
  if (cudaLaunchKernelEx(&cfg, fn, params) == cudaSuccess) return LOOPSPEC_OK;
  (void)cudaGetLastError();
  return LOOPSPEC_ECUDA;
}

// the cache as the kernels see it; false: not a cache they take
bool paged_kv(const loopspec_paged_kv* c, PagedKv* o) {
  if (!c || !c->k || !c->v || !aligned16(c->k) || !aligned16(c->v) || (c->dtype != 1 && c->dtype != 2)) return false;
  if (c->page_stride % 8 || c->head_stride % 8 || c->slot_stride % 8 || c->page_stride < 0 || c->head_stride < 0 || c->slot_stride < 0) return false;
  if (!pow2(c->page_size) || c->page_size > 65536 || c->n_pages < 0 || c->n_kv_heads < 1 || c->head_dim < 8 || c->head_dim > 256 || c->head_dim % 8) return false;
  o->k = c->k, o->v = c->v, o->page_stride = c->page_stride, o->head_stride = c->head_stride, o->slot_stride = c->slot_stride;
  o->n_pages = c->n_pages, o->page_shift = log2_of(c->page_size), o->n_kv = c->n_kv_heads, o->d = c->head_dim;
  return true;
}

using AppendFn = void (*)(const AppendParams);
template <typename TI, typename TO>
AppendFn append_fn(int lh, bool rows) {
  switch (lh) {
    case 1: return rows ? append_rows_kernel<TI, TO, 1> : append_kernel<TI, TO, 1>;
    case 2: return rows ? append_rows_kernel<TI, TO, 2> : append_kernel<TI, TO, 2>;
    case 4: return rows ? append_rows_kernel<TI, TO, 4> : append_kernel<TI, TO, 4>;
    case 8: return rows ? append_rows_kernel<TI, TO, 8> : append_kernel<TI, TO, 8>;
    case 16: return rows ? append_rows_kernel<TI, TO, 16> : append_kernel<TI, TO, 16>;
    default: return rows ? append_rows_kernel<TI, TO, 32> : append_kernel<TI, TO, 32>;
  }
}
template <typename TO>
AppendFn append_fn(int dtype, int lh, bool rows) {
  return dtype == 0 ? append_fn<float, TO>(lh, rows) : dtype == 1 ? append_fn<__nv_bfloat16, TO>(lh, rows) : append_fn<__half, TO>(lh, rows);
}

constexpr int kSms = 148;
// Token rows from which append_kv gives each a warp of its own; below, a row's heads are spread over warps [us spread / a warp each, 16 bits: 48 heads of 128 with
// norms 100 rows 3.8 / 7.7, 300 5.6 / 7.7, 600 6.6 / 8.6, 1000 9.7 / 8.8, 1990 14.8 / 11.5, 8000 50 / 36; 48 heads of 64 with norms 300 5.1 / 5.5, 600 5.0 / 6.1, 1000
// 6.7 / 6.0; without 300 4.8 / 4.5, 600 4.4 / 4.9, 1000 5.9 / 5.0; 6 heads of 64 100 3.0 / 3.5, 600 3.8 / 3.9, 1000 5.0 / 3.8, 8000 20 / 10: the crossing lies
// between 600 and 1000 rows throughout, but for 300 rows of heads of 64 without norms, which the rule costs 0.3 us]
constexpr int APP_ROWS = 1000;

// Lets a kernel ask for `bytes` of dynamic shared memory; `done` remembers, a bit per device, that it may.  regs: registers a thread that it must have
// been compiled to (0: any)
bool allow_smem(const void* fn, int bytes, std::atomic<unsigned long long>& done, int regs = 0) {
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0) return false;
  const unsigned long long bit = 1ull << (dev & 63);
  if (dev < 64 && (done.load(std::memory_order_relaxed) & bit)) return true;
  cudaFuncAttributes a;
  if (regs && (cudaFuncGetAttributes(&a, fn) != cudaSuccess || a.numRegs != regs)) {
    (void)cudaGetLastError();
    return false;
  }
  if (cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) {
    (void)cudaGetLastError();
    return false;
  }
  if (dev < 64) done.fetch_or(bit, std::memory_order_relaxed);
  return true;
}

// ---- attention behind a shared prefix ----
struct PxPlan {
  int max_tiles, tc_tiles;
  size_t state, item_seg, tc_seg, item_ml, item_o, warp_ml, warp_o, tc_item_ml, tc_item_o, tc_work_ml, tc_work_o, total;
};
constexpr int PX_MAX_LEN = INT32_MAX - 128;  // positions: a tile's last still has a number
constexpr int PXT_MIN_ROWS = 33;  // rows of the batch and a kv head from which on the prefix goes to the tensor cores' tiles
bool px_plan(int T, int B, int nq, int nkv, int d, int P, PxPlan* o) {
  if (T < 0 || B < 0 || B > PX_MAX_SEQS || nq < 1 || nkv < 1 || nq % nkv || (d != 64 && d != 128) || P < 0) return false;
  if ((int64_t)T * nq > (1 << 27) || nkv > 65535 || (int64_t)B * nq > (1 << 30) || P > PX_MAX_LEN) return false;
  const int rows = T * (nq / nkv);
  o->max_tiles = rows / 16 + B + 1 + (P > 0 ? rows / 16 + 1 : 0);
  o->tc_tiles = rows >= PXT_MIN_ROWS && P > 0 ? (rows + PXT_ROWS - 1) / PXT_ROWS : 0;
  size_t at = 0;
  auto take = [&](size_t n) {
    const size_t r = at;
    at += (n + 255) / 256 * 256;
    return r;
  };
  o->state = take(4), o->item_seg = take((size_t)nkv * o->max_tiles * 8), o->tc_seg = take((size_t)nkv * o->tc_tiles * 8);
  o->item_ml = take((size_t)nkv * o->max_tiles * 128);
  o->item_o = take((size_t)nkv * o->max_tiles * 16 * d * 4);
  o->warp_ml = take((size_t)PX_SMS * PXR_WARPS * 128);
  o->warp_o = take((size_t)PX_SMS * PXR_WARPS * 16 * d * 4);
  const size_t items = (size_t)nkv * o->tc_tiles * PXT_ROWS, work = o->tc_tiles ? (size_t)PX_SMS * PXT_ROWS : 0;
  o->tc_item_ml = take(items * 8), o->tc_item_o = take(items * d * 4);
  o->tc_work_ml = take(work * 8), o->tc_work_o = take(work * d * 4);
  o->total = at;
  return true;
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                                  CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn encode_tiled_fn() {
  static std::atomic<EncodeTiledFn> fn;
  EncodeTiledFn f = fn.load(std::memory_order_acquire);
  if (!f) {
    void* ptr = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &ptr, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) {
      (void)cudaGetLastError();
      return nullptr;
    }
    f = reinterpret_cast<EncodeTiledFn>(ptr);
    fn.store(f, std::memory_order_release);
  }
  return f;
}
// keys or values as (element, slot, head, page); boxes of 64 elements of `box` slots
bool cache_map(CUtensorMap* map, const PagedKv& kv, const void* ptr, int dtype, int box) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (!fn) return false;
  cuuint64_t dims[4] = {(cuuint64_t)kv.d, (cuuint64_t)1 << kv.page_shift, (cuuint64_t)kv.n_kv, (cuuint64_t)kv.n_pages};
  cuuint64_t strides[3] = {(cuuint64_t)kv.slot_stride * 2, (cuuint64_t)kv.head_stride * 2, (cuuint64_t)kv.page_stride * 2};
  cuuint32_t boxes[4] = {64, (cuuint32_t)box, 1, 1}, estr[4] = {1, 1, 1, 1};
  return fn(map, dtype == 1 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, const_cast<void*>(ptr), dims, strides, boxes, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int D>
int px_launch(PrefixParams& p, const PxPlan& t, int dtype, void* stream) {
  static std::atomic<unsigned long long> allowed;
  if (!allow_smem((const void*)prefix_kernel<T, D>, PxCfg<D>::smem(PX_MAX_SEQS + 1), allowed, 168)) return LOOPSPEC_ECUDA;
  // The prefix on tcgen05: pages of at least 8 slots (a swizzled group of rows) and strides that a tensor map takes; else it is one more problem of few rows.
  CUtensorMap mk, mv;
  memset(&mk, 0, sizeof mk), memset(&mv, 0, sizeof mv);
  const int page = 1 << p.kv.page_shift, box = std::min(page, PXT_KEYS);
  const bool tc = t.tc_tiles && page >= 8 && cache_map(&mk, p.kv, p.kv.k, dtype, box) && cache_map(&mv, p.kv, p.kv.v, dtype, box);
  p.tc_tiles = tc ? t.tc_tiles : 0, p.prefix_rows = p.prefix_len > 0 && !tc;
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof cfg);
  cfg.gridDim = dim3(PX_SMS), cfg.blockDim = dim3(PX_THREADS), cfg.dynamicSmemBytes = PxCfg<D>::smem(p.B + p.prefix_rows), cfg.stream = static_cast<cudaStream_t>(stream);
  if (cudaLaunchKernelEx(&cfg, prefix_kernel<T, D>, mk, mv, static_cast<const PrefixParams&>(p)) != cudaSuccess) {
    (void)cudaGetLastError();
    return LOOPSPEC_ECUDA;
  }
  // the fold: a CTA per sequence and query head while there are few rows, else a warp (16 rows x heads 9.0 / 10.6 us, 640 15.7 / 18.5, 2048 45.9 / 37.4);
  // long runs of rows over several
  const int64_t heads = (int64_t)p.B * p.nq;
  const unsigned y = (unsigned)std::min<int64_t>(64, std::max<int64_t>(1, ((int64_t)p.T * 2 + p.B - 1) / p.B));
  if ((int64_t)p.T * p.nq <= 8 * kSms) return launch(prefix_merge_kernel<T, D, 4>, dim3((unsigned)heads, y), 128, 0, stream, p, true);
  return launch(prefix_merge_kernel<T, D, 1>, dim3((unsigned)((heads + 3) / 4), y), 128, 0, stream, p, true);
}

// stop_tile, wait_us: see loopspec_debug_prefix_attention
int prefix_attention(const void* q, int64_t q_ld, int32_t T, int32_t n_q_heads, const loopspec_paged_kv* kv, const int32_t* prefix_pages, int32_t prefix_len,
                     const int32_t* page_table, int64_t table_ld, int32_t table_width, const int32_t* lens, const int32_t* cu_rows, int32_t n_seqs, float scale,
                     void* out, int64_t out_ld, float* lse, int32_t* flag, void* scratch, size_t scratch_bytes, void* cuda_stream, int32_t stop_tile,
                     int32_t wait_us) {
  PrefixParams p;
  memset(&p, 0, sizeof p);
  PxPlan t;
  if (!paged_kv(kv, &p.kv) || !px_plan(T, n_seqs, n_q_heads, p.kv.n_kv, p.kv.d, prefix_len, &t) || !(scale >= 0.f) || std::isinf(scale)) return LOOPSPEC_EINVAL;
  if (table_width < 0 || table_ld < table_width || (int64_t)table_width * kv->page_size > PX_MAX_LEN) return LOOPSPEC_EINVAL;
  if (T == 0 || n_seqs == 0) return LOOPSPEC_OK;  // (every row is padding)
  const int64_t width = (int64_t)n_q_heads * p.kv.d;
  if (!q || !aligned16(q) || q_ld % 8 || (T > 1 && q_ld < width) || !out || !aligned16(out) || out_ld % 8 || (T > 1 && out_ld < width)) return LOOPSPEC_EINVAL;
  if (!lens || !cu_rows || (table_width && !page_table) || (prefix_len && !prefix_pages)) return LOOPSPEC_EINVAL;
  p.G = n_q_heads / p.kv.n_kv;
  // units of 16 keys x 16 rows of a kv head, counted in 32 bits
  const double units = ((double)T * p.G / 16 + n_seqs) * ((double)table_width * kv->page_size / 16 + 1) + ((double)T * p.G / 16 + 1) * ((double)prefix_len / 16 + 1);
  if (units >= 2147483648.0) return LOOPSPEC_EINVAL;
  if (!scratch || scratch_bytes < t.total || (reinterpret_cast<uintptr_t>(scratch) & 255)) return LOOPSPEC_ECAPACITY;
  p.q = q, p.q_ld = q_ld, p.prefix_pages = prefix_pages, p.prefix_len = prefix_len;
  p.page_table = page_table, p.table_ld = table_ld, p.table_w = table_width, p.lens = lens, p.cu_rows = cu_rows;
  p.B = n_seqs, p.T = T, p.nq = n_q_heads;
  p.scale_log2 = (scale == 0.f ? 1.f / std::sqrt((float)p.kv.d) : scale) * 1.4426950408889634f;
  p.max_tiles = t.max_tiles;
  unsigned char* sc = static_cast<unsigned char*>(scratch);
  p.state = reinterpret_cast<int*>(sc + t.state), p.item_seg = reinterpret_cast<int2*>(sc + t.item_seg), p.tc_seg = reinterpret_cast<int2*>(sc + t.tc_seg);
  p.item_ml = reinterpret_cast<float*>(sc + t.item_ml), p.item_o = reinterpret_cast<float*>(sc + t.item_o);
  p.warp_ml = reinterpret_cast<float*>(sc + t.warp_ml), p.warp_o = reinterpret_cast<float*>(sc + t.warp_o);
  p.tc_item_ml = reinterpret_cast<float*>(sc + t.tc_item_ml), p.tc_item_o = reinterpret_cast<float*>(sc + t.tc_item_o);
  p.tc_work_ml = reinterpret_cast<float*>(sc + t.tc_work_ml), p.tc_work_o = reinterpret_cast<float*>(sc + t.tc_work_o);
  p.out = out, p.out_ld = out_ld, p.lse = lse, p.flag = flag;
  p.stop_tile = stop_tile >= 0 ? stop_tile : INT_MAX, p.wait_cycles = stop_tile >= 0 && wait_us > 0 ? (long long)wait_us * 2000 : PX_WAIT_CYCLES;
  if (p.kv.d == 128) return kv->dtype == 1 ? px_launch<__nv_bfloat16, 128>(p, t, 1, cuda_stream) : px_launch<__half, 128>(p, t, 2, cuda_stream);
  return kv->dtype == 1 ? px_launch<__nv_bfloat16, 64>(p, t, 1, cuda_stream) : px_launch<__half, 64>(p, t, 2, cuda_stream);
}

// ---- sampling ----
constexpr int SMP_MAX_VOCAB = 1 << 18, SMP_SMEM = 200 * 1024;
template <typename T>
int smp_launch(smp::Params& p, void* stream) {
  static std::atomic<unsigned long long> allowed;
  constexpr int extra = 32 + smp::BINS * 8 + (smp::LIST + 2 * smp::SOLO) * 8;
  // CTAs per row: up to three for every two SMs (two share one; a cluster's hand-overs cost more than a wider one gains: 64 rows of 32,000 take 10.2 us
  // with two each, 11.4 with four; with top-p 0.9 32 and 38, with k = 50 13.6 and 17.4), none with less than 2048 tokens; more where a slice would not fit
  int cs = 1;
  while (cs < smp::MAX_CS && ((p.V > 2048 * cs && p.rows * cs * 2 <= kSms * 3 / 2) || (p.V / cs + 8) * (int)sizeof(T) + extra > SMP_SMEM)) cs *= 2;
  p.per = ((p.V + cs - 1) / cs + 7) / 8 * 8;
  p.hist_off = p.per * (int)sizeof(T) + 32;  // (a piece more than the slice: it need not begin on a boundary)
  const int bytes = p.hist_off - 32 + extra;
  if (!allow_smem((const void*)smp::sample_kernel<T>, SMP_SMEM, allowed)) return LOOPSPEC_ECUDA;
  return launch(smp::sample_kernel<T>, dim3(p.rows * cs), smp::THREADS, bytes, stream, p, false, cs);
}

}  // namespace

extern "C" {

int loopspec_op_append_kv(const void* qkv, int32_t qkv_dtype, int64_t qkv_ld, int32_t T, int32_t n_q_heads, const loopspec_paged_kv* kv,
                          const int32_t* page_table, int64_t table_ld, int32_t table_width, const int32_t* cached, const int32_t* cu_rows, int32_t n_seqs,
                          const int32_t* pos_offset, const double* inv_freq, int32_t rot_dim, const float* q_norm, const float* k_norm, float eps,
                          void* q_out, int64_t q_ld, int32_t* flag, void* cuda_stream) {
  AppendParams p;
  memset(&p, 0, sizeof p);
  if (!paged_kv(kv, &p.kv) || qkv_dtype < 0 || qkv_dtype > 2 || T < 0 || T > INT32_MAX - APP_WARPS || n_seqs < 0 || n_q_heads < 0 || n_q_heads > 65536 || p.kv.n_kv > 65536) return LOOPSPEC_EINVAL;
  if ((q_norm && !aligned16(q_norm)) || (k_norm && !aligned16(k_norm))) return LOOPSPEC_EINVAL;
  if (rot_dim < 0 || rot_dim > p.kv.d || rot_dim % 8 || (rot_dim && !inv_freq)) return LOOPSPEC_EINVAL;
  if (table_width < 0 || table_ld < table_width) return LOOPSPEC_EINVAL;
  if (T == 0 || n_seqs == 0) return LOOPSPEC_OK;  // (every row is padding)
  const int64_t width = ((int64_t)n_q_heads + 2 * (int64_t)p.kv.n_kv) * p.kv.d;
  if (!qkv || !aligned16(qkv) || qkv_ld % 8 || (T > 1 && qkv_ld < width) || !cached || !cu_rows || (table_width && !page_table)) return LOOPSPEC_EINVAL;
  if (n_q_heads && (!q_out || !aligned16(q_out) || q_ld % 8 || (T > 1 && q_ld < (int64_t)n_q_heads * p.kv.d))) return LOOPSPEC_EINVAL;
  p.qkv = qkv, p.ld = qkv_ld, p.q = q_out, p.q_ld = q_ld;
  p.page_table = page_table, p.table_ld = table_ld, p.table_w = table_width;
  p.cached = cached, p.cu_rows = cu_rows, p.pos_offset = pos_offset, p.inv_freq = inv_freq, p.q_norm = q_norm, p.k_norm = k_norm, p.eps = eps;
  p.T = T, p.B = n_seqs, p.nq = n_q_heads, p.rot = rot_dim, p.err = flag;
  int lh = 1;
  while (lh < p.kv.d / 8) lh *= 2;
  const bool rows = T >= APP_ROWS;
  const AppendFn fn = kv->dtype == 1 ? append_fn<__nv_bfloat16>(qkv_dtype, lh, rows) : append_fn<__half>(qkv_dtype, lh, rows);
  if (rows) return launch(fn, dim3((T + APP_WARPS - 1) / APP_WARPS, 1), APP_WARPS * 32, 0, cuda_stream, p);
  const int per_turn = APP_WARPS * (32 / lh), turns = (int)((n_q_heads + 2 * (int64_t)p.kv.n_kv + per_turn - 1) / per_turn);
  return launch(fn, dim3(T, std::max(1, std::min(turns, 1184 / T))), APP_WARPS * 32, 0, cuda_stream, p);
}

size_t loopspec_prefix_attention_scratch_bytes(int32_t T, int32_t n_seqs, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t prefix_len) {
  PxPlan t;
  return px_plan(T, n_seqs, n_q_heads, n_kv_heads, head_dim, prefix_len, &t) ? t.total : 0;
}

int loopspec_op_prefix_attention(const void* q, int64_t q_ld, int32_t T, int32_t n_q_heads, const loopspec_paged_kv* kv, const int32_t* prefix_pages,
                                 int32_t prefix_len, const int32_t* page_table, int64_t table_ld, int32_t table_width, const int32_t* lens,
                                 const int32_t* cu_rows, int32_t n_seqs, float scale, void* out, int64_t out_ld, float* lse, int32_t* flag, void* scratch,
                                 size_t scratch_bytes, void* cuda_stream) {
  return prefix_attention(q, q_ld, T, n_q_heads, kv, prefix_pages, prefix_len, page_table, table_ld, table_width, lens, cu_rows, n_seqs, scale, out, out_ld, lse, flag,
                          scratch, scratch_bytes, cuda_stream, -1, 0);
}

int loopspec_debug_prefix_attention(const void* q, int64_t q_ld, int32_t T, int32_t n_q_heads, const loopspec_paged_kv* kv, const int32_t* prefix_pages,
                                    int32_t prefix_len, const int32_t* page_table, int64_t table_ld, int32_t table_width, const int32_t* lens,
                                    const int32_t* cu_rows, int32_t n_seqs, float scale, void* out, int64_t out_ld, float* lse, int32_t* flag, void* scratch,
                                    size_t scratch_bytes, void* cuda_stream, int32_t stop_tile, int32_t wait_us) {
  return prefix_attention(q, q_ld, T, n_q_heads, kv, prefix_pages, prefix_len, page_table, table_ld, table_width, lens, cu_rows, n_seqs, scale, out, out_ld, lse, flag,
                          scratch, scratch_bytes, cuda_stream, stop_tile, wait_us);
}

int loopspec_op_sample(const void* logits, int32_t dtype, int64_t ld, int32_t rows, int32_t vocab, const float* uniforms, const float* temperature,
                       const int32_t* top_k, const float* top_p, const float* min_p, int32_t* tokens, float* probs, void* cuda_stream) {
  if (dtype < 0 || dtype > 2 || rows < 0 || rows > (1 << 24) || vocab < 1 || vocab > SMP_MAX_VOCAB || (rows > 1 && ld < vocab)) return LOOPSPEC_EINVAL;
  if (rows == 0) return LOOPSPEC_OK;
  if (!logits || !uniforms || !tokens || (reinterpret_cast<uintptr_t>(logits) & (dtype ? 1 : 3))) return LOOPSPEC_EINVAL;
  smp::Params p;
  memset(&p, 0, sizeof p);
  p.logits = logits, p.ld = ld, p.rows = rows, p.V = vocab, p.shift = std::min(48, 61 - log2_of(vocab));
  p.u = uniforms, p.temperature = temperature, p.top_k = top_k, p.top_p = top_p, p.min_p = min_p, p.token = tokens, p.prob = probs;
  return dtype == 0 ? smp_launch<float>(p, cuda_stream) : dtype == 1 ? smp_launch<__nv_bfloat16>(p, cuda_stream) : smp_launch<__half>(p, cuda_stream);
}

}  // extern "C"
