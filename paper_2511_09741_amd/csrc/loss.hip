// Cross entropy over the vocabulary, with label smoothing and z-loss, and its gradient.
//   lse = log sum_v exp l_v;  row = lse - (1 - eps) l_y - eps/V sum_v l_v + z lse^2
//   dl_v = up ((1 + 2 z lse) exp(l_v - lse) - (1 - eps) [v = y] - eps/V)
// Bound by memory: the logits are read once and the gradient is written once.
#include <type_traits>

#include "dev_common.h"
#include "taw_internal.h"

namespace taw {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kInf = __builtin_huge_valf();

// the label of row t, or -1 where the row is not counted
template <typename TI>
__device__ __forceinline__ int label_of(const TI* __restrict__ labels, int64_t t, int V) {
  const TI y = labels[t];
  return y >= 0 && y < (TI)V ? (int)y : -1;
}

// sum and maximum over a workgroup of NW wavefronts, for every thread, in wavefront order
template <int NW>
__device__ __forceinline__ float block_sum(float x, float* red) {
  x = wave_sum(x);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
  __syncthreads();
  float s = 0.f;
#pragma unroll
  for (int w = 0; w < NW; ++w) s += red[w];
  return s;
}
template <int NW>
__device__ __forceinline__ float block_max(float x, float* red) {
  x = wave_max(x);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
  __syncthreads();
  float s = -kInf;
#pragma unroll
  for (int w = 0; w < NW; ++w) s = fmaxf(s, red[w]);
  return s;
}

struct RowTerms {                 // of the loss
  float eps, z, grad_scale;
  int mean;
};

// =============================================================================== counted rows
template <typename TI>
__global__ void __launch_bounds__(1024) loss_count_kernel(const TI* __restrict__ labels, int T_, int V, int* __restrict__ count) {
  __shared__ int red[16];
  int n = 0;
  for (int t = threadIdx.x; t < T_; t += 1024) n += label_of(labels, t, V) >= 0;
  for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = n;
  __syncthreads();
  if (threadIdx.x == 0) {
    n = 0;
    for (int w = 0; w < 16; ++w) n += red[w];
    *count = n;
  }
}

// =============================================================================== rows
// A workgroup per row: maximum, sum of exponentials, gradient.
template <typename TL, typename TG, typename TI, bool GRAD>
__global__ void __launch_bounds__(256) loss_row_kernel(const TL* logits, const TI* __restrict__ labels, int V, int V_pad, int64_t ld, int64_t ld_grad, RowTerms c,
                                                       const int* __restrict__ count, float* __restrict__ rows, float* __restrict__ lse_out, TG* dlogits) {
  __shared__ float red[4];
  const int64_t t = blockIdx.x;
  const int y = label_of(labels, t, V);
  const TL* l = logits + t * ld;
  TG* d = dlogits + t * ld_grad;
  if (y < 0) {
    if (threadIdx.x == 0) {
      rows[t] = 0.f;
      if (lse_out) lse_out[t] = 0.f;
    }
    if (GRAD)
      for (int v = threadIdx.x; v < V_pad; v += 256) d[v] = (TG)0.f;
    return;
  }
  float top = -kInf, total = 0.f;
  for (int v = threadIdx.x; v < V; v += 256) {
    const float x = (float)l[v];
    top = fmaxf(top, x);
    total += x;
  }
  top = block_max<4>(top, red);
  const float m = top == -kInf ? 0.f : top;
  float sum = 0.f;
  for (int v = threadIdx.x; v < V; v += 256) sum += exp2f(((float)l[v] - m) * kLog2e);
  sum = block_sum<4>(sum, red);
  total = c.eps != 0.f ? block_sum<4>(total, red) : 0.f;
  const float lse = m + logf(sum);              // -inf where nothing but -inf is there
  const float ly = (float)l[y];
  __syncthreads();                              // dlogits may be the logits
  if (threadIdx.x == 0) {
    float r = sum == 0.f ? kInf : lse - (1.f - c.eps) * ly;
    if (c.eps != 0.f) r -= c.eps / (float)V * total;
    if (c.z != 0.f) r += c.z * lse * lse;
    rows[t] = r;
    if (lse_out) lse_out[t] = lse;
  }
  if (!GRAD) return;
  const float up = sum == 0.f ? 0.f : c.mean ? c.grad_scale / (float)*count : c.grad_scale;
  const float p1 = c.z != 0.f && sum != 0.f ? 1.f + 2.f * c.z * lse : 1.f, share = c.eps / (float)V;
  for (int v = threadIdx.x; v < V_pad; v += 256) {
    float g = 0.f;
    if (v < V && sum != 0.f) {
      g = exp2f(((float)l[v] - lse) * kLog2e) * p1 - share - (v == y ? 1.f - c.eps : 0.f);
      g *= up;
    }
    d[v] = (TG)g;
  }
}

// the gradient from a saved lse
template <typename TL, typename TG, typename TI>
__global__ void __launch_bounds__(256) loss_bwd_kernel(const TL* logits, const TI* __restrict__ labels, int V, int V_pad, int64_t ld, int64_t ld_grad, RowTerms c,
                                                       const float* __restrict__ lse_in, const float* __restrict__ dloss, TG* dlogits) {
  const int64_t t = blockIdx.x;
  const int y = label_of(labels, t, V);
  const TL* l = logits + t * ld;
  TG* d = dlogits + t * ld_grad;
  const float lse = lse_in[t], up = dloss[t], share = c.eps / (float)V;
  const float p1 = c.z != 0.f ? 1.f + 2.f * c.z * lse : 1.f;
  const bool none = y < 0 || lse == -kInf;
  for (int v = threadIdx.x; v < V_pad; v += 256) {
    float g = 0.f;
    if (v < V && !none) g = up * (exp2f(((float)l[v] - lse) * kLog2e) * p1 - share - (v == y ? 1.f - c.eps : 0.f));
    d[v] = (TG)g;
  }
}

// =============================================================================== sum of the rows' losses
template <typename TI>
__global__ void __launch_bounds__(1024) loss_sum_kernel(const float* __restrict__ rows, const TI* __restrict__ labels, int T_, int V, int mean, float* __restrict__ loss) {
  __shared__ double red[16];
  __shared__ int redn[16];
  double s = 0.0;
  int n = 0;
  for (int t = threadIdx.x; t < T_; t += 1024) {
    s += (double)rows[t];
    n += label_of(labels, t, V) >= 0;
  }
  for (int o = 32; o > 0; o >>= 1) {
    s += __shfl_xor(s, o, 64);
    n += __shfl_xor(n, o, 64);
  }
  if ((threadIdx.x & 63) == 0) {
    red[threadIdx.x >> 6] = s;
    redn[threadIdx.x >> 6] = n;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    s = 0.0;
    n = 0;
    for (int w = 0; w < 16; ++w) {
      s += red[w];
      n += redn[w];
    }
    loss[0] = n == 0 ? 0.f : (float)(mean ? s / (double)n : s);
    loss[1] = (float)n;
  }
}

// =============================================================================== launchers
static inline int last_err() { return (int)hipGetLastError(); }

size_t loss_workspace_bytes(int T_) { return 256 + ((size_t)T_ * 4 + 255) / 256 * 256; }      // the count; the rows' losses where the caller has no use for them

template <typename F>
static int by_types(const LossArgs& a, F f) {
  const auto with_labels = [&](auto* l, auto* g) { return a.label_type == IDX_I64 ? f(l, g, (int64_t*)nullptr) : f(l, g, (int32_t*)nullptr); };
  if (a.dtype == DT_BF16) return with_labels((bf16_t*)nullptr, (bf16_t*)nullptr);
  if (a.grad_dtype == DT_BF16) return with_labels((float*)nullptr, (bf16_t*)nullptr);
  return with_labels((float*)nullptr, (float*)nullptr);
}

int launch_loss(const LossArgs& a, const void* logits, const void* labels, float* loss, float* rows, float* lse, void* dlogits, void* ws, hipStream_t st) {
  int* count = (int*)ws;
  if (!rows) rows = (float*)((char*)ws + 256);
  const RowTerms c{a.eps, a.z, a.grad_scale, a.mean};
  return by_types(a, [&](auto* pl, auto* pg, auto* pi) {
    using TL = std::remove_pointer_t<decltype(pl)>;
    using TG = std::remove_pointer_t<decltype(pg)>;
    using TI = std::remove_pointer_t<decltype(pi)>;
    if (a.T) {
      if (dlogits && a.mean) hipLaunchKernelGGL((loss_count_kernel<TI>), dim3(1), dim3(1024), 0, st, (const TI*)labels, a.T, a.V, count);
      if (dlogits)
        hipLaunchKernelGGL((loss_row_kernel<TL, TG, TI, true>), dim3((unsigned)a.T), dim3(256), 0, st, (const TL*)logits, (const TI*)labels, a.V, a.V_pad, a.ld, a.ld_grad, c,
                           count, rows, lse, (TG*)dlogits);
      else
        hipLaunchKernelGGL((loss_row_kernel<TL, TG, TI, false>), dim3((unsigned)a.T), dim3(256), 0, st, (const TL*)logits, (const TI*)labels, a.V, a.V_pad, a.ld, a.ld_grad, c,
                           count, rows, lse, (TG*)nullptr);
      const int e = last_err();
      if (e) return e;
    }
    hipLaunchKernelGGL((loss_sum_kernel<TI>), dim3(1), dim3(1024), 0, st, rows, (const TI*)labels, a.T, a.V, a.mean, loss);
    return last_err();
  });
}

int launch_loss_bwd(const LossArgs& a, const void* logits, const void* labels, const float* lse, const float* dloss, void* dlogits, hipStream_t st) {
  const RowTerms c{a.eps, a.z, 0.f, 0};
  return by_types(a, [&](auto* pl, auto* pg, auto* pi) {
    using TL = std::remove_pointer_t<decltype(pl)>;
    using TG = std::remove_pointer_t<decltype(pg)>;
    using TI = std::remove_pointer_t<decltype(pi)>;
    hipLaunchKernelGGL((loss_bwd_kernel<TL, TG, TI>), dim3((unsigned)a.T), dim3(256), 0, st, (const TL*)logits, (const TI*)labels, a.V, a.V_pad, a.ld, a.ld_grad, c, lse, dloss,
                       (TG*)dlogits);
    return last_err();
  });
}

}  // namespace taw
