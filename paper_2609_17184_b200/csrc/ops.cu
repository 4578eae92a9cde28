// C ABI of the operators between the linear maps (see include/loopspec.h): checks of the arguments, rules that choose a kernel's
// variant, launches.  No call synchronises, allocates or keeps anything.
#include "../../include/loopspec.h"

#include <algorithm>
#include <cstring>

#include "op_append.cuh"

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
int launch(void (*fn)(const P), dim3 grid, int block, size_t smem, void* stream, const P& params, bool pdl = false, int cluster = 1) {
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof cfg);
  cfg.gridDim = grid, cfg.blockDim = dim3(block), cfg.dynamicSmemBytes = smem, cfg.stream = static_cast<cudaStream_t>(stream);
  cudaLaunchAttribute at[2];
  int n = 0;
  if (pdl) at[n].id = cudaLaunchAttributeProgrammaticStreamSerialization, at[n++].val.programmaticStreamSerializationAllowed = 1;
  if (cluster > 1) {
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
AppendFn append_fn(int lh) {
  switch (lh) {
    case 1: return append_kernel<TI, TO, 1>;
    case 2: return append_kernel<TI, TO, 2>;
    case 4: return append_kernel<TI, TO, 4>;
    case 8: return append_kernel<TI, TO, 8>;
    case 16: return append_kernel<TI, TO, 16>;
    default: return append_kernel<TI, TO, 32>;
  }
}
template <typename TO>
AppendFn append_fn(int dtype, int lh) {
  return dtype == 0 ? append_fn<float, TO>(lh) : dtype == 1 ? append_fn<__nv_bfloat16, TO>(lh) : append_fn<__half, TO>(lh);
}

}  // namespace

extern "C" {

int loopspec_op_append_kv(const void* qkv, int32_t qkv_dtype, int64_t qkv_ld, int32_t T, int32_t n_q_heads, const loopspec_paged_kv* kv,
                          const int32_t* page_table, int64_t table_ld, int32_t table_width, const int32_t* cached, const int32_t* cu_rows, int32_t n_seqs,
                          const int32_t* pos_offset, const double* inv_freq, int32_t rot_dim, const float* q_norm, const float* k_norm, float eps,
                          void* q_out, int64_t q_ld, int32_t* flag, void* cuda_stream) {
  AppendParams p;
  memset(&p, 0, sizeof p);
  if (!paged_kv(kv, &p.kv) || qkv_dtype < 0 || qkv_dtype > 2 || T < 0 || n_seqs < 0 || n_q_heads < 0 || n_q_heads > 65536 || p.kv.n_kv > 65536) return LOOPSPEC_EINVAL;
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
  const AppendFn fn = kv->dtype == 1 ? append_fn<__nv_bfloat16>(qkv_dtype, lh) : append_fn<__half>(qkv_dtype, lh);
  // few rows: a row's heads over several CTAs
  const int per_cta = APP_WARPS * (32 / lh), iters = (int)((n_q_heads + 2 * (int64_t)p.kv.n_kv + per_cta - 1) / per_cta);
  const int split = std::max(1, std::min(iters, 1184 / T));
  return launch(fn, dim3(T, split), APP_WARPS * 32, 0, cuda_stream, p);
}

}  // extern "C"
