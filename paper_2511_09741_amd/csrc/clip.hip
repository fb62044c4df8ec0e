// Global gradient norm over a list of tensors, and clipping by it.
//   sumsq = sum g^2 (fp64);  norm = |s| sqrt(sumsq);  coef = min(1, max_norm / norm)
// Bound by memory: the norm reads every gradient once, the scaling in place reads and writes it once more.
#include <cmath>
#include <type_traits>

#include "dev_common.h"
#include "taw_internal.h"

namespace taw {

// Tensors travel as kernel arguments, so a call copies nothing to the device and can be captured; a longer list takes several launches.  A short one
// is a smaller argument (of 2.5 KB they made a launch from the host 1 us longer).
template <int N>
struct TensorList {
  static constexpr int kMax = N;
  void* data[N];
  unsigned long long n[N];
  unsigned first[N + 1];                      // piece number of the tensor's first piece
  unsigned char bf16[N];
  int count;
  int piece;                                  // elements of a tensor that a workgroup takes at a time
};

template <typename L>
__device__ __forceinline__ int tensor_of(const L& l, unsigned piece) {
  int lo = 0, hi = l.count - 1;               // the last tensor that starts at or before the piece
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (l.first[mid] <= piece) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ double wave_sum_f64(double x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
  return x;
}

// sum over a workgroup of NW wavefronts, in wavefront order; thread 0 has it
template <int NW>
__device__ __forceinline__ double block_sum_f64(double x) {
  __shared__ double red[NW];
  x = wave_sum_f64(x);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
  __syncthreads();
  double s = 0.0;
  if (threadIdx.x == 0)
    for (int w = 0; w < NW; ++w) s += red[w];
  return s;
}

// =============================================================================== sum of squares
// Squares and sums in fp64: an fp32 square overflows from 1.8e19 on, and the fp64 units keep up with memory.
// A piece that is whole is read with 8 vectors in flight a thread.
template <typename T>
__device__ __forceinline__ double piece_sumsq(const T* __restrict__ p, int m) {
  constexpr int VW = VecWidth<T>::value, U = 8;
  double s[4] = {0.0, 0.0, 0.0, 0.0};
  const auto add = [&](const Vec<T, VW>& x) {
#pragma unroll
    for (int j = 0; j < VW; ++j) {
      const double v = (double)x.get(j);
      s[j & 3] = fma(v, v, s[j & 3]);
    }
  };
  const int nv = m / VW;
  int i = threadIdx.x;
  for (; i + (U - 1) * 256 < nv; i += U * 256) {
    Vec<T, VW> x[U];
#pragma unroll
    for (int k = 0; k < U; ++k) x[k].load_nt(p + (size_t)(i + k * 256) * VW);
#pragma unroll
    for (int k = 0; k < U; ++k) add(x[k]);
  }
#pragma unroll 2
  for (; i < nv; i += 256) {
    Vec<T, VW> x;
    x.load_nt(p + (size_t)i * VW);
    add(x);
  }
  const int e = nv * VW + threadIdx.x;
  if (e < m) {
    const double v = (double)(float)p[e];
    s[0] = fma(v, v, s[0]);
  }
  return (s[0] + s[1]) + (s[2] + s[3]);
}

// f(data, elements) for the pieces of this workgroup; data points to float or bf16
template <typename L, typename F>
__device__ __forceinline__ void over_pieces(const L& l, F f) {
  const unsigned pieces = l.first[l.count];
  for (unsigned piece = blockIdx.x; piece < pieces; piece += gridDim.x) {
    const int t = tensor_of(l, piece);
    const unsigned long long at = (unsigned long long)(piece - l.first[t]) * l.piece;
    const int m = (int)(l.n[t] - at < l.piece ? l.n[t] - at : l.piece);
    if (l.bf16[t]) f((bf16_t*)l.data[t] + at, m);
    else f((float*)l.data[t] + at, m);
  }
}

template <typename L>
__global__ void __launch_bounds__(256) sumsq_kernel(const L l, double* __restrict__ partials) {
  double s = 0.0;
  over_pieces(l, [&](const auto* p, int m) { s += piece_sumsq(p, m); });
  s = block_sum_f64<4>(s);
  if (threadIdx.x == 0) partials[blockIdx.x] = s;
}

__device__ __forceinline__ void finish_clip(double sumsq, float max_norm, float grad_scale, taw_clip_state* state) {
  const float norm = (float)(fabs((double)grad_scale) * sqrt(sumsq));
  const bool fine = norm <= 3.402823466e38f;  // false for NaN too
  state->norm = norm;
  state->coef = !fine ? 0.f : norm > max_norm ? max_norm / norm : 1.f;
  state->nonfinite = fine ? 0 : 1;
  for (int i = 0; i < 3; ++i) state->reserved[i] = 0;
}

__global__ void __launch_bounds__(256) sumsq_finish_kernel(const double* __restrict__ partials, int np, int set, int finish, float max_norm, float grad_scale,
                                                           taw_clip_state* __restrict__ state) {
  double s = 0.0;
  for (int i = threadIdx.x; i < np; i += 256) s += partials[i];
  s = block_sum_f64<4>(s);
  if (threadIdx.x == 0) {
    if (!set) s += state->sumsq;
    state->sumsq = s;
    if (finish) finish_clip(s, max_norm, grad_scale, state);
  }
}

__global__ void __launch_bounds__(64) clip_coef_kernel(float max_norm, float grad_scale, taw_clip_state* __restrict__ state) {
  if (threadIdx.x == 0) finish_clip(state->sumsq, max_norm, grad_scale, state);
}

// =============================================================================== scaling in place
// A workgroup to a piece, and pieces that are one batch of loads and then one of stores.  364 M fp32 in 26 tensors, us where they are scaled and where
// there is nothing to do (the launch of wavefronts that end at once): pieces of 4096 476 and 20, 8192 495 and 11, 16384 547 and 6, 2048 workgroups
// that go from piece to piece 590 and 4.5.  8192: most steps of a training run clip nothing.
constexpr int kScalePiece = 8192;
template <typename T>
__device__ __forceinline__ void piece_scale(T* __restrict__ p, int m, float c) {
  constexpr int VW = VecWidth<T>::value, U = kScalePiece / (256 * VW);
  const auto scaled = [&](const Vec<T, VW>& x) {
    Vec<T, VW> o;
#pragma unroll
    for (int j = 0; j < VW; ++j) o.set(j, x.get(j) * c);
    return o;
  };
  const int nv = m / VW;
  int i = threadIdx.x;
  for (; i + (U - 1) * 256 < nv; i += U * 256) {
    Vec<T, VW> x[U];
#pragma unroll
    for (int k = 0; k < U; ++k) x[k].load_nt(p + (size_t)(i + k * 256) * VW);
#pragma unroll
    for (int k = 0; k < U; ++k) scaled(x[k]).store_nt(p + (size_t)(i + k * 256) * VW);
  }
#pragma unroll 2
  for (; i < nv; i += 256) {
    Vec<T, VW> x;
    x.load_nt(p + (size_t)i * VW);
    scaled(x).store_nt(p + (size_t)i * VW);
  }
  const int e = nv * VW + threadIdx.x;
  if (e < m) p[e] = (T)((float)p[e] * c);
}

template <typename L>
__global__ void __launch_bounds__(256) clip_kernel(const L l, const taw_clip_state* __restrict__ state) {
  const float c = state->coef;
  if (c == 1.f || state->nonfinite) return;
  over_pieces(l, [&](auto* p, int m) { piece_scale(p, m, c); });
}

// =============================================================================== launchers
static inline int last_err() { return (int)hipGetLastError(); }

// Where a list is too short for the chip its pieces are of 2048 elements; the norm's otherwise of 16384, 8 vectors in flight a thread.
static int piece_of(const taw_tensor* t, int count, int most) {
  size_t n = 0;
  for (int i = 0; i < count; ++i) n += t[i].n;
  return n < ((size_t)1 << 22) ? 2048 : most;
}
constexpr int kSumPiece = 16384;
constexpr unsigned kSumGrid = 2048, kScaleGrid = 1 << 23;

// cuts the list into launches; f(list, grid) returns a status
template <typename L, typename F>
static int over_list_as(const taw_tensor* t, int count, int piece, unsigned grid, F f) {
  L l;
  l.piece = piece_of(t, count, piece);
  int i = 0;
  while (i < count) {
    l.count = 0;
    unsigned pieces = 0;
    for (; i < count && l.count < L::kMax; ++i) {
      if (!t[i].n) continue;
      const unsigned long long np = (t[i].n + l.piece - 1) / l.piece;
      if (np > 0x7fffffffull) return (int)hipErrorInvalidValue;
      if (pieces + np > 0x7fffffffull) break;
      l.data[l.count] = t[i].data;
      l.n[l.count] = t[i].n;
      l.bf16[l.count] = t[i].dtype == DT_BF16;
      l.first[l.count++] = pieces;
      pieces += (unsigned)np;
    }
    if (!pieces) continue;
    l.first[l.count] = pieces;
    const int e = f(l, pieces < grid ? pieces : grid);
    if (e) return e;
  }
  return 0;
}

template <typename F>
static int over_list(const taw_tensor* t, int count, int piece, unsigned grid, F f) {
  return count <= 16 ? over_list_as<TensorList<16>>(t, count, piece, grid, f) : over_list_as<TensorList<120>>(t, count, piece, grid, f);
}

size_t grad_norm_workspace_bytes(const taw_tensor* t, int count) {
  size_t blocks = 0;
  over_list(t, count, kSumPiece, kSumGrid, [&](const auto&, unsigned grid) { blocks += grid; return 0; });
  return blocks * sizeof(double) + 16;
}

int launch_grad_sumsq(const taw_tensor* t, int count, int set, int finish, float max_norm, float grad_scale, taw_clip_state* state, void* ws, hipStream_t st) {
  double* partials = (double*)ws;
  int np = 0;
  const int e = over_list(t, count, kSumPiece, kSumGrid, [&](const auto& l, unsigned grid) {
    hipLaunchKernelGGL((sumsq_kernel<std::decay_t<decltype(l)>>), dim3(grid), dim3(256), 0, st, l, partials + np);
    np += (int)grid;
    return last_err();
  });
  if (e) return e;
  hipLaunchKernelGGL(sumsq_finish_kernel, dim3(1), dim3(256), 0, st, partials, np, set, finish, max_norm, grad_scale, state);
  return last_err();
}

int launch_clip_coef(float max_norm, float grad_scale, taw_clip_state* state, hipStream_t st) {
  hipLaunchKernelGGL(clip_coef_kernel, dim3(1), dim3(64), 0, st, max_norm, grad_scale, state);
  return last_err();
}

int launch_grad_clip(const taw_tensor* t, int count, const taw_clip_state* state, hipStream_t st) {
  return over_list(t, count, kScalePiece, kScaleGrid, [&](const auto& l, unsigned grid) {
    hipLaunchKernelGGL((clip_kernel<std::decay_t<decltype(l)>>), dim3(grid), dim3(256), 0, st, l, state);
    return last_err();
  });
}

}  // namespace taw
