// Embedding lookup and its gradient.
//   x[t] = s E[ids[t]];   G[v] (=|+=) s sum_{t: ids[t] = v} dx[t]
// Bound by memory.  Ids outside [0, V) name no row.
#include <type_traits>

#include "dev_common.h"
#include "taw_internal.h"

namespace taw {

// the id of token t, or -1 where it names no row
template <typename TI>
__device__ __forceinline__ int row_id(const TI* __restrict__ ids, int64_t t, int V) {
  const TI v = ids[t];
  return v >= 0 && v < (TI)V ? (int)v : -1;
}

// =============================================================================== forward
// one workgroup per token
template <typename T, typename TI>
__global__ void __launch_bounds__(256) embed_fwd_kernel(const TI* __restrict__ ids, const T* __restrict__ table, T* __restrict__ x, int H, int V, int64_t ld_table,
                                                        int64_t ld_x, float scale) {
  const int64_t t = blockIdx.x;
  const int v = row_id(ids, t, V);
  const T* src = table + (int64_t)(v < 0 ? 0 : v) * ld_table;
  T* dst = x + t * ld_x;
  for (int i = threadIdx.x; i < H; i += 256) dst[i] = v < 0 ? (T)0.f : (T)((float)src[i] * scale);
}

// =============================================================================== backward
// one workgroup per row of the table and 256 columns; it looks through all the ids, in order
template <typename T, typename TI>
__global__ void __launch_bounds__(256) embed_bwd_kernel(const TI* __restrict__ ids, const T* __restrict__ dx, float* __restrict__ G, int T_, int H, int V, int64_t ld_table,
                                                        int64_t ld_x, float scale, int accumulate) {
  const int v = blockIdx.x, col = blockIdx.y * 256 + threadIdx.x, lane = threadIdx.x & 63;
  float s = 0.f;
  bool any = false;
  for (int t0 = 0; t0 < T_; t0 += 64) {
    const bool mine = t0 + lane < T_ && row_id(ids, t0 + lane, V) == v;
    unsigned long long who = __ballot(mine);
    while (who) {
      const int t = t0 + __builtin_ctzll(who);
      who &= who - 1;
      any = true;
      if (col < H) s += (float)dx[(int64_t)t * ld_x + col];
    }
  }
  if (col >= H) return;
  float* g = G + (int64_t)v * ld_table + col;
  if (!accumulate) *g = scale * s;
  else if (any) *g += scale * s;
}

// =============================================================================== launchers
static inline int last_err() { return (int)hipGetLastError(); }

template <typename F>
static int by_types(int dtype, int id_type, F f) {
  if (dtype == DT_BF16) return id_type == IDX_I64 ? f((bf16_t*)nullptr, (int64_t*)nullptr) : f((bf16_t*)nullptr, (int32_t*)nullptr);
  return id_type == IDX_I64 ? f((float*)nullptr, (int64_t*)nullptr) : f((float*)nullptr, (int32_t*)nullptr);
}

int launch_embed_fwd(const EmbedArgs& a, const void* ids, const void* table, void* x, hipStream_t st) {
  return by_types(a.dtype, a.id_type, [&](auto* t, auto* i) {
    using T = std::remove_pointer_t<decltype(t)>;
    using TI = std::remove_pointer_t<decltype(i)>;
    hipLaunchKernelGGL((embed_fwd_kernel<T, TI>), dim3((unsigned)a.T), dim3(256), 0, st, (const TI*)ids, (const T*)table, (T*)x, a.H, a.V, a.ld_table, a.ld_x, a.scale);
    return last_err();
  });
}

size_t embed_bwd_workspace_bytes(int, int, int) { return 0; }

int launch_embed_bwd(const EmbedArgs& a, const void* ids, const void* dx, float* G, void*, hipStream_t st) {
  return by_types(a.dtype, a.id_type, [&](auto* t, auto* i) {
    using T = std::remove_pointer_t<decltype(t)>;
    using TI = std::remove_pointer_t<decltype(i)>;
    hipLaunchKernelGGL((embed_bwd_kernel<T, TI>), dim3((unsigned)a.V, (unsigned)((a.H + 255) / 256)), dim3(256), 0, st, (const TI*)ids, (const T*)dx, G, a.T, a.H, a.V,
                       a.ld_table, a.ld_x, a.scale, a.accumulate);
    return last_err();
  });
}

}  // namespace taw
