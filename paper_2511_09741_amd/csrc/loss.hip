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

// =============================================================================== a row as vectors
// A row is taken as 16-byte vectors aligned in memory, whatever its first element is aligned to: the first vector starts `lead` elements before the
// row, and what of the first and the last one lies outside the row is neither read nor written.
template <typename TL, typename TG>
struct RowVecs {
  static constexpr int VW = 16 / sizeof(TL);
  const TL* in;               // the first vector
  TG* out;                    // the gradient at the same place
  int lead, end, count;       // elements [lead, end) of the vectors are the row
  bool wide;                  // the gradient's vectors are aligned too
  typedef Vec<TL, VW> vec_t;

  __device__ __forceinline__ RowVecs(const TL* logits, TG* dlogits, int64_t t, int V, int64_t ld, int64_t ld_grad) {
    const int64_t at = t * ld;
    lead = (int)(at & (VW - 1));
    end = lead + V;
    count = (end + VW - 1) / VW;
    in = logits + (at - lead);
    const int64_t to = t * ld_grad - lead;
    out = dlogits + to;
    wide = (to & (VW - 1)) == 0;
  }
  __device__ __forceinline__ bool inside(int c) const { return c * VW >= lead && (c + 1) * VW <= end; }
  // outside the row: -inf, a class of probability 0
  __device__ __forceinline__ void load(int c, vec_t& x) const {
    if (inside(c)) {
      x.load_nt(in + (int64_t)c * VW);
    } else {
#pragma unroll
      for (int j = 0; j < VW; ++j) {
        const int e = c * VW + j;
        x.set(j, -kInf);
        if (e >= lead && e < end) x.raw[j] = in[e];
      }
    }
  }
  __device__ __forceinline__ void store(int c, const float* g) const {
    if (wide && inside(c)) {
      typedef TG out_t __attribute__((ext_vector_type(VW)));
      out_t o;
#pragma unroll
      for (int j = 0; j < VW; ++j) o[j] = (TG)g[j];
      __builtin_nontemporal_store(o, reinterpret_cast<out_t*>(out + (int64_t)c * VW));
    } else {
#pragma unroll
      for (int j = 0; j < VW; ++j) {
        const int e = c * VW + j;
        if (e >= lead && e < end) out[e] = (TG)g[j];
      }
    }
  }
};

// exp(l - m) = exp2(l s - m s) with s = log2 e, one fused multiply-add and one exponential.  m s is exact as far as the sum of exponentials and its
// logarithm go, since both are taken from the rounded m s.  Beyond 1e30 the values of a row are equal or further apart than any exponential reaches:
// s = 1 does for them, and m s does not overflow.
struct Shift {
  float s, ms;
  bool huge;
  __device__ __forceinline__ explicit Shift(float m) : s(fabsf(m) > 1e30f ? 1.f : kLog2e), ms(m * s), huge(fabsf(m) > 1e30f) {}
  __device__ __forceinline__ float exp(float l) const { return __builtin_amdgcn_exp2f(__builtin_fmaf(l, s, -ms)); }
  __device__ __forceinline__ float lse(float m, float sum) const { return huge ? m + logf(sum) : (ms + log2f(sum)) * kLn2; }
};

// the gradient of VW logits: scale * exp(l) - share, and less by `own` at the label
template <typename R>
__device__ __forceinline__ void gradient(const R& row, int c, const typename R::vec_t& x, const Shift& sh, float scale, float share, float own, int y) {
  float g[R::VW];
#pragma unroll
  for (int j = 0; j < R::VW; ++j) g[j] = __builtin_fmaf(scale, sh.exp(x.get(j)), -share);
  const int at = y + row.lead - c * R::VW;
  if (at >= 0 && at < R::VW) {
#pragma unroll
    for (int j = 0; j < R::VW; ++j)
      if (j == at) g[j] -= own;
  }
  row.store(c, g);
}

// =============================================================================== rows
// A workgroup of NT threads per row, which stays packed in registers (MAXC vectors a thread) between its maximum, its sum of exponentials and its
// gradient: the logits are read once.  What does not fit (MORE) is summed on the way with a running maximum, and read a second time for the gradient.
template <typename TL, typename TG, typename TI, int NT, int MAXC, bool MORE, bool GRAD>
__global__ void __launch_bounds__(NT) loss_row_kernel(const TL* logits, const TI* __restrict__ labels, int T_, int V, int V_pad, int64_t ld, int64_t ld_grad, RowTerms c,
                                                      const int* __restrict__ count, float* __restrict__ rows, float* __restrict__ lse_out, TG* dlogits) {
  typedef RowVecs<TL, TG> R;
  constexpr int NW = NT / 64;
  __shared__ float red[NW];
  const int64_t t = blockIdx.x;
  const int y = label_of(labels, t, V), tid = threadIdx.x;
  if (y < 0) {
    if (tid == 0) {
      rows[t] = 0.f;
      if (lse_out) lse_out[t] = 0.f;
    }
    if (GRAD) {
      const R row(logits, dlogits, t, V, ld, ld_grad);
      const float zero[R::VW] = {};
      for (int i = tid; i < row.count; i += NT) row.store(i, zero);
      for (int v = V + tid; v < V_pad; v += NT) dlogits[t * ld_grad + v] = (TG)0.f;
    }
    return;
  }
  const R row(logits, dlogits, t, V, ld, ld_grad);
  const float ly = (float)logits[t * ld + y];      // before anything is written: dlogits may be the logits
  float counted = 1.f;
  if (GRAD && c.mean) {
    if (count) {
      counted = (float)*count;
    } else {
      int n = 0;
      for (int i = tid; i < T_; i += NT) n += label_of(labels, i, V) >= 0;
      counted = block_sum<NW>((float)n, red);      // exact: T is small here
    }
  }
  float top = -kInf, total = 0.f, sum = 0.f;
  if (MORE) {
    constexpr int U = 4;
    for (int i = tid + MAXC * NT; i < row.count; i += U * NT) {
      typename R::vec_t x[U];
#pragma unroll
      for (int k = 0; k < U; ++k)
        if (i + k * NT < row.count) row.load(i + k * NT, x[k]);
      float m = top;
#pragma unroll
      for (int k = 0; k < U; ++k)
        if (i + k * NT < row.count)
#pragma unroll
          for (int j = 0; j < R::VW; ++j) m = fmaxf(m, x[k].get(j));
      const float ref = m == -kInf ? 0.f : m;
      sum *= __builtin_amdgcn_exp2f((top - ref) * kLog2e);
#pragma unroll
      for (int k = 0; k < U; ++k)
        if (i + k * NT < row.count)
#pragma unroll
          for (int j = 0; j < R::VW; ++j) {
            const float l = x[k].get(j);
            sum += __builtin_amdgcn_exp2f((l - ref) * kLog2e);
            const int e = (i + k * NT) * R::VW + j;
            if (c.eps != 0.f && e >= row.lead && e < row.end) total += l;
          }
      top = m;
    }
  }
  typename R::vec_t x[MAXC];
#pragma unroll
  for (int k = 0; k < MAXC; ++k)
    if (tid + k * NT < row.count) row.load(tid + k * NT, x[k]);
  const float mine = top;
#pragma unroll
  for (int k = 0; k < MAXC; ++k)
    if (tid + k * NT < row.count) {
#pragma unroll
      for (int j = 0; j < R::VW; ++j) top = fmaxf(top, x[k].get(j));
      if (c.eps != 0.f)
#pragma unroll
        for (int j = 0; j < R::VW; ++j) {
          const int e = (tid + k * NT) * R::VW + j;
          if (e >= row.lead && e < row.end) total += x[k].get(j);
        }
    }
  top = block_max<NW>(top, red);
  const float m = top == -kInf ? 0.f : top;
  const Shift sh(m);
  if (MORE) sum *= sh.exp(mine);
#pragma unroll
  for (int k = 0; k < MAXC; ++k) {
    x[k].pin();
    if (tid + k * NT < row.count)
#pragma unroll
      for (int j = 0; j < R::VW; ++j) sum += sh.exp(x[k].get(j));
  }
  sum = block_sum<NW>(sum, red);
  if (c.eps != 0.f) total = block_sum<NW>(total, red);
  const float lse = sum == 0.f ? -kInf : sh.lse(m, sum);
  if (tid == 0) {
    float r = sum == 0.f ? kInf : lse - (1.f - c.eps) * ly;
    if (c.eps != 0.f) r -= c.eps / (float)V * total;
    if (c.z != 0.f) r += c.z * lse * lse;
    rows[t] = r;
    if (lse_out) lse_out[t] = lse;
  }
  if (!GRAD) return;
  const bool none = sum == 0.f;                    // nothing but -inf
  const float up = none ? 0.f : c.mean ? c.grad_scale / counted : c.grad_scale;
  const float scale = none ? 0.f : up * (c.z != 0.f ? 1.f + 2.f * c.z * lse : 1.f) / sum, share = up * c.eps / (float)V, own = up * (1.f - c.eps);
#pragma unroll
  for (int k = 0; k < MAXC; ++k) {
    x[k].pin();
    if (tid + k * NT < row.count) gradient(row, tid + k * NT, x[k], sh, scale, share, own, y);
  }
  if (MORE) {
    constexpr int U = 4;                           // backwards: what was read last is the likeliest to be in a cache
    const int n = (row.count - tid + NT - 1) / NT;
    for (int k0 = n - 1; k0 >= MAXC; k0 -= U) {
      typename R::vec_t z[U];
#pragma unroll
      for (int k = 0; k < U; ++k)
        if (k0 - k >= MAXC) row.load(tid + (k0 - k) * NT, z[k]);
#pragma unroll
      for (int k = 0; k < U; ++k)
        if (k0 - k >= MAXC) gradient(row, tid + (k0 - k) * NT, z[k], sh, scale, share, own, y);
    }
  }
  for (int v = V + tid; v < V_pad; v += NT) dlogits[t * ld_grad + v] = (TG)0.f;
}

// The gradient from a saved lse: nothing is summed, so a row is cut into parts of kPart vectors.
constexpr int kPart = 1024;
template <typename TL, typename TG, typename TI>
__global__ void __launch_bounds__(256) loss_bwd_kernel(const TL* logits, const TI* __restrict__ labels, int V, int V_pad, int64_t ld, int64_t ld_grad, RowTerms c,
                                                       const float* __restrict__ lse_in, const float* __restrict__ dloss, TG* dlogits, unsigned parts) {
  typedef RowVecs<TL, TG> R;
  constexpr int U = kPart / 256;
  const int64_t t = blockIdx.x / parts;
  const unsigned part = blockIdx.x - (unsigned)t * parts;
  const int y = label_of(labels, t, V);
  const R row(logits, dlogits, t, V, ld, ld_grad);
  const float lse = lse_in[t];
  const bool none = y < 0 || lse == -kInf;
  const int first = part * kPart + threadIdx.x;
  typename R::vec_t x[U];
  if (!none) {
#pragma unroll
    for (int k = 0; k < U; ++k)
      if (first + k * 256 < row.count) row.load(first + k * 256, x[k]);
  }
  const Shift sh(lse);
  const float up = none ? 0.f : dloss[t];
  // what the rounding of lse s leaves out
  const float rest = sh.huge ? 1.f : __builtin_amdgcn_exp2f(-__builtin_fmaf(lse, sh.s, -sh.ms));
  const float scale = up * (c.z != 0.f ? 1.f + 2.f * c.z * lse : 1.f) * rest, share = up * c.eps / (float)V, own = up * (1.f - c.eps);
#pragma unroll
  for (int k = 0; k < U; ++k) {
    const int i = first + k * 256;
    if (i >= row.count) break;
    if (none) {
      const float zero[R::VW] = {};
      row.store(i, zero);
    } else {
      gradient(row, i, x[k], sh, scale, share, own, y);
    }
  }
  if (part == parts - 1)
    for (int v = V + threadIdx.x; v < V_pad; v += 256) dlogits[t * ld_grad + v] = (TG)0.f;
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

// rows up to which a workgroup counts the labels itself: a launch costs more than reading this many
constexpr int kCountedInline = 2048;

int launch_loss(const LossArgs& a, const void* logits, const void* labels, float* loss, float* rows, float* lse, void* dlogits, void* ws, hipStream_t st) {
  int* count = dlogits && a.mean && a.T > kCountedInline ? (int*)ws : nullptr;
  if (!rows) rows = (float*)((char*)ws + 256);
  const RowTerms c{a.eps, a.z, a.grad_scale, a.mean};
  return by_types(a, [&](auto* pl, auto* pg, auto* pi) {
    using TL = std::remove_pointer_t<decltype(pl)>;
    using TG = std::remove_pointer_t<decltype(pg)>;
    using TI = std::remove_pointer_t<decltype(pi)>;
    if (a.T) {
      if (count) hipLaunchKernelGGL((loss_count_kernel<TI>), dim3(1), dim3(1024), 0, st, (const TI*)labels, a.T, a.V, count);
      constexpr int VW = 16 / sizeof(TL);
      const int vecs = (a.V + 2 * (VW - 1)) / VW;      // at most, wherever a row starts
#define TAW_LOSS(NT, MAXC, MORE)                                                                                                                                    \
  do {                                                                                                                                                              \
    if (dlogits)                                                                                                                                                    \
      hipLaunchKernelGGL((loss_row_kernel<TL, TG, TI, NT, MAXC, MORE, true>), dim3((unsigned)a.T), dim3(NT), 0, st, (const TL*)logits, (const TI*)labels, a.T, a.V,  \
                         a.V_pad, a.ld, a.ld_grad, c, count, rows, lse, (TG*)dlogits);                                                                              \
    else                                                                                                                                                            \
      hipLaunchKernelGGL((loss_row_kernel<TL, TG, TI, NT, MAXC, MORE, false>), dim3((unsigned)a.T), dim3(NT), 0, st, (const TL*)logits, (const TI*)labels, a.T, a.V, \
                         a.V_pad, a.ld, a.ld_grad, c, count, rows, lse, (TG*)nullptr);                                                                              \
  } while (0)
      if (vecs <= 64 * 8) TAW_LOSS(64, 8, false);
      else if (vecs <= 256 * 8) TAW_LOSS(256, 8, false);
      else if (vecs <= 512 * 8) TAW_LOSS(512, 8, false);
      else if (vecs <= 1024 * 8) TAW_LOSS(1024, 8, false);
      else if (vecs <= 1024 * 16) TAW_LOSS(1024, 16, false);
      else TAW_LOSS(1024, 16, true);
#undef TAW_LOSS
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
    constexpr int VW = 16 / sizeof(TL);
    const uint64_t parts = ((a.V + 2 * (VW - 1)) / VW + kPart - 1) / kPart, blocks = parts * a.T;
    if (blocks > 0x7fffffffu) return (int)hipErrorInvalidValue;
    hipLaunchKernelGGL((loss_bwd_kernel<TL, TG, TI>), dim3((unsigned)blocks), dim3(256), 0, st, (const TL*)logits, (const TI*)labels, a.V, a.V_pad, a.ld, a.ld_grad, c, lse, dloss,
                       (TG*)dlogits, (unsigned)parts);
    return last_err();
  });
}

}  // namespace taw
