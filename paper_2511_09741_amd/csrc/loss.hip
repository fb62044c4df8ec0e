// Cross entropy over the vocabulary, with label smoothing and z-loss, and its gradient.
//   lse = log sum_v exp l_v;  row = lse - (1 - eps) l_y - eps/V sum_v l_v + z lse^2
//   dl_v = up ((1 + 2 z lse) exp(l_v - lse) - (1 - eps) [v = y] - eps/V)
// Bound by memory: the logits are read once (rows of more than 8192 vectors of 16 bytes twice) and the gradient is written once.
#include <type_traits>

#include "dev_common.h"
#include "taw_internal.h"

namespace taw {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kInf = __builtin_huge_valf();

// the label of a row, or -1 where the row is not counted
struct Labels {
  const void* p;
  int wide, V;                // int64
  Labels from(int64_t t) const { return Labels{static_cast<const char*>(p) + t * (wide ? 8 : 4), wide, V}; }
  __device__ __forceinline__ int operator[](int64_t t) const {
    const int64_t y = wide ? static_cast<const int64_t*>(p)[t] : static_cast<const int32_t*>(p)[t];
    return y >= 0 && y < V ? (int)y : -1;
  }
};

// sum and maximum over a workgroup of NW wavefronts, for every thread, in wavefront order
template <int NW>
__device__ __forceinline__ float block_sum(float x, float* red) {
  x = wave_sum(x);
  if (NW == 1) return x;
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
  if (NW == 1) return x;
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
  float each;                     // eps / V: the logits are weighted with it before they are summed, or classes masked by the type's lowest value overflow the sum
  int mean;
};

// =============================================================================== counted rows
__device__ __forceinline__ int wave_count(int n) {
  for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o, 64);
  return n;
}

// of each workgroup
__global__ void __launch_bounds__(1024) loss_count_kernel(const Labels labels, int T_, int* __restrict__ count) {
  __shared__ int red[16];
  int n = 0;
  for (int t = blockIdx.x * 1024 + threadIdx.x; t < T_; t += gridDim.x * 1024) n += labels[t] >= 0;
  n = wave_count(n);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = n;
  __syncthreads();
  if (threadIdx.x == 0) {
    n = 0;
    for (int w = 0; w < 16; ++w) n += red[w];
    count[blockIdx.x] = n;
  }
}

// of 64 workgroups
__global__ void __launch_bounds__(64) loss_count_join_kernel(int* count) {
  const int n = wave_count(count[threadIdx.x]);
  if (threadIdx.x == 0) *count = n;
}

// by one thread
__device__ __forceinline__ void store_loss(double s, int64_t n, int mean, float* __restrict__ loss) {
  loss[0] = n == 0 ? 0.f : (float)(mean ? s / (double)n : s);
  loss[1] = (float)n;
}

// =============================================================================== a row as vectors
// A row is taken as `count` vectors of 16 bytes that are aligned in memory, whatever its first element is aligned to, and the up to VW - 1 elements
// before and behind them, its edge, of which each of the first threads has one.  SAME: the gradient's rows start as far from a vector as the logits',
// so that its vectors are aligned too; without it they are stored element by element, which costs (rows of 32003 logits, us with the gradient's stride
// 32064 and the logits' 32003 / 32064): gradient from a saved lse, 2048 rows of bf16 63 / 43; with the loss, 8192 rows of bf16 218 / 187, fp32 to bf16
// 286 / 250, fp32 397 / 354.
template <typename TL, typename TG, bool SAME>
struct RowVecs {
  static constexpr int VW = 16 / sizeof(TL);
  typedef Vec<TL, VW> vec_t;
  static constexpr bool kHoldsExp = sizeof(TL) == 4;
  const TL* in;               // the first vector
  TG* out;                    // the gradient at the same place
  int head, count, tail;      // elements before the vectors, vectors, elements behind them

  __device__ __forceinline__ RowVecs(const TL* logits, TG* dlogits, int64_t t, int V, int64_t ld, int64_t ld_grad) {
    const int64_t at = t * ld, to = t * ld_grad;
    head = (int)(-at & (VW - 1));
    head = head < V ? head : V;
    count = (V - head) / VW;
    tail = V - head - count * VW;
    in = logits + (at + head);
    out = dlogits + (to + head);
  }
  // KEEP: leave it in the caches, it will be read again
  template <bool KEEP = false>
  __device__ __forceinline__ void load(unsigned c, vec_t& x) const {
    if (KEEP) x.load(in + (size_t)c * VW);
    else x.load_nt(in + (size_t)c * VW);
  }
  __device__ __forceinline__ void store(unsigned c, const float* g) const {
    if (SAME) {
      typedef TG out_t __attribute__((ext_vector_type(VW)));
      out_t o;
#pragma unroll
      for (int j = 0; j < VW; ++j) o[j] = (TG)g[j];
      __builtin_nontemporal_store(o, reinterpret_cast<out_t*>(out + (size_t)c * VW));
    } else {
#pragma unroll
      for (int j = 0; j < VW; ++j) out[(size_t)c * VW + j] = (TG)g[j];
    }
  }
  // the element of the edge that is thread i's, relative to the first vector; there is none where edge() is false
  __device__ __forceinline__ bool edge(int i, int* e) const {
    *e = i < head ? i - head : i - head + count * VW;
    return i < head + tail;
  }
};

// exp(l - m) = exp2(l s - m s) with s = log2 e, one fused multiply-add and one exponential.  What the rounding of m s leaves out is a factor of all the
// exponentials of a row, which its sum has too.  Up to |m| = 2^30 that factor lies within 2^-64 .. 2^64 (half a step of a product below 2^31), and with
// it the sum of 2^24 classes; beyond it would leave fp32's range.  There s = 1 does: m s is exact, and a logit that is not m is at least 128 away from
// it, further than any exponential reaches.
struct Shift {
  float s, ms;
  bool far;
  __device__ __forceinline__ explicit Shift(float m) {
#pragma clang fp contract(off)        // everything rests on the rounded product: it is not to be fused with what it is added to
    far = fabsf(m) > 0x1p30f;
    s = far ? 1.f : kLog2e;
    ms = m * s;
  }
  __device__ __forceinline__ float exp(float l) const { return __builtin_amdgcn_exp2f(__builtin_fmaf(l, s, -ms)); }
  // log sum exp(l - m), of the sum of exp()
  __device__ __forceinline__ float log_sum(float m, float sum) const { return (log2f(sum) - __builtin_fmaf(m, s, -ms)) * kLn2; }
};

// A vector that a row's workgroup holds.  fp32: the exponentials take the place of the logits, and are not formed a second time for the gradient (which
// took a third of the kernel's instructions).  bf16: they would take twice the registers, so the logits stay.
template <typename R>
__device__ __forceinline__ void sum_exp(typename R::vec_t& x, const Shift& sh, float& sum) {
#pragma unroll
  for (int j = 0; j < R::VW; ++j) {
    const float e = sh.exp(x.get(j));
    sum += e;
    if (R::kHoldsExp) x.set(j, e);
  }
}

// the gradient of VW logits: scale * exp(l) - share, and less by `own` at the label.  HELD: sum_exp() has seen the vector
template <bool HELD, typename R>
__device__ __forceinline__ void gradient(const R& row, unsigned c, const typename R::vec_t& x, const Shift& sh, float scale, float share, float own, int y) {
  float g[R::VW];
#pragma unroll
  for (int j = 0; j < R::VW; ++j) g[j] = __builtin_fmaf(scale, HELD && R::kHoldsExp ? x.get(j) : sh.exp(x.get(j)), -share);
  const unsigned at = (unsigned)(y - row.head) - c * R::VW;
  if (at < (unsigned)R::VW) {
#pragma unroll
    for (int j = 0; j < R::VW; ++j)
      if (j == (int)at) g[j] -= own;
  }
  row.store(c, g);
}

// what a row comes to, from its maximum m, its sum of exponentials and (label smoothing) its weighted sum of logits; the thread that is told to stores it.
// The loss is the maximum less the label's logit, which is exact where they are close, and log sum exp(l - m), not lse less the logit: that would have the
// roundings of lse, which are of the logits' size (5e-4 at 1e4).  lse is rounded once from both: far from zero it does not fall below the maximum.
struct RowResult {
  float scale, share, own;                         // gradient: scale * exp(l) - share, - own at the label
  float loss = 0.f;                                // for the thread that stores it
  __device__ __forceinline__ RowResult(const Shift& sh, float m, float sum, float total, float ly, const RowTerms& c, float counted, int64_t t, bool store,
                                       float* __restrict__ rows, float* __restrict__ lse_out) {
    const bool none = sum == 0.f;                  // nothing but -inf
    const float log_sum = sh.log_sum(m, sum), lse = none ? -kInf : m + log_sum;
    if (store) {
      float r = none ? kInf : __builtin_fmaf(2.f * (1.f - c.eps), 0.5f * m - 0.5f * ly, log_sum);      // halves: the whole may be more than fp32 holds
      if (c.each != 0.f) r += __builtin_fmaf(c.eps, m, -total);
      if (c.z != 0.f) r += c.z * lse * lse;
      rows[t] = loss = r;
      if (lse_out) lse_out[t] = lse;
    }
    const float up = none ? 0.f : c.mean ? c.grad_scale / counted : c.grad_scale;
    scale = none ? 0.f : up * (c.z != 0.f ? 1.f + 2.f * c.z * lse : 1.f) / sum;
    share = up * c.each;
    own = up * (1.f - c.eps);
  }
};

// The maximum of a held row of bf16, two values an instruction: as signed integers the bits of floats that are not negative are in the floats' order,
// and above those of the negative ones.  Where the row's maximum is negative (none() after the workgroup's maximum) it is formed in floats after all.
typedef short s16x2_t __attribute__((ext_vector_type(2)));
template <typename R>
struct PairMax {
  s16x2_t m = {-32768, -32768};
  __device__ __forceinline__ void add(const typename R::vec_t& x) {
    const u32x4_t w = __builtin_bit_cast(u32x4_t, x.raw);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const unsigned two = w[j];
      m = __builtin_elementwise_max(m, __builtin_bit_cast(s16x2_t, two));
    }
  }
  __device__ __forceinline__ float top() const {
    const int i = m[0] > m[1] ? m[0] : m[1];
    return i >= 0 ? __uint_as_float((unsigned)i << 16) : -kInf;
  }
  static __device__ __forceinline__ bool none(float top) { return !(top >= 0.f); }
};

// the edge of a row: a logit a thread, -inf (a class of probability 0) where it has none
template <typename R>
struct Edge {
  int e;
  bool have;
  float l;
  __device__ __forceinline__ Edge(const R& row, int tid, float each, float& top, float& total) {
    have = row.edge(tid, &e);
    l = have ? (float)row.in[e] : -kInf;
    top = fmaxf(top, l);
    if (have && each != 0.f) total = __builtin_fmaf(each, l, total);
  }
  template <typename G>
  __device__ __forceinline__ void store(const R& row, const Shift& sh, const G& g, int y) const {
    if (have) row.out[e] = __builtin_fmaf(g.scale, sh.exp(l), -g.share) - (e + row.head == y ? g.own : 0.f);
  }
};

// a row that is not counted
template <int NT, bool GRAD, bool SAME, typename TL, typename TG>
__device__ __forceinline__ void empty_row(const TL* logits, TG* dlogits, int64_t t, int tid, int V, int V_pad, int64_t ld, int64_t ld_grad, float* __restrict__ rows,
                                          float* __restrict__ lse_out) {
  typedef RowVecs<TL, TG, SAME> R;
  if (tid == 0) {
    rows[t] = 0.f;
    if (lse_out) lse_out[t] = 0.f;
  }
  if (!GRAD) return;
  const R row(logits, dlogits, t, V, ld, ld_grad);
  const float zero[R::VW] = {};
  for (int i = tid; i < row.count; i += NT) row.store(i, zero);
  int e;
  if (row.edge(tid, &e)) row.out[e] = (TG)0.f;
  for (int v = V + tid; v < V_pad; v += NT) dlogits[t * ld_grad + v] = (TG)0.f;
}

// =============================================================================== rows
// A workgroup of NT threads per row, which stays packed in registers (MAXC vectors a thread) between its maximum, its sum of exponentials and its
// gradient: the logits are read once.  MORE: of a row that is longer, the rest is summed on the way with a running maximum, and read a second time for the
// gradient, backwards (what was read last is the likeliest to be in a cache).
// Row t by the threads tid = 0 .. NT - 1; counted: the rows that are, for the mean's gradient.  Returns the row's loss (tid 0).
template <int NT, int MAXC, bool MORE, bool GRAD, bool SAME, typename TL, typename TG, typename C>
__device__ __forceinline__ float loss_row(const TL* logits, const Labels& labels, int64_t t, int tid, int V, int V_pad, int64_t ld, int64_t ld_grad,
                                          const RowTerms& c, C rows_counted, float* __restrict__ rows, float* __restrict__ lse_out, TG* dlogits, float* red) {
  typedef RowVecs<TL, TG, SAME> R;
  constexpr int NW = NT / 64;
  const int y = labels[t];
  const R row(logits, dlogits, t, V, ld, ld_grad);
  // The logits wait for the label.  Asked for before it is there, they come no sooner (40 to 1536 rows of 1000 to 32000 bf16: within 2%), and those of rows
  // that are not counted are read for nothing: 1024 rows of 32000, a third of them such, 12.9 us waiting, 14.7 asked for at once.
  if (y < 0) {
    empty_row<NT, GRAD, SAME>(logits, dlogits, t, tid, V, V_pad, ld, ld_grad, rows, lse_out);
    return 0.f;
  }
  typename R::vec_t x[MAXC];
  if (row.count)
#pragma unroll
    for (int k = 0; k < MAXC; ++k) row.load(tid + k * NT < row.count ? tid + k * NT : row.count - 1, x[k]);      // always a load: none waits for a branch
  const float ly = (float)logits[t * ld + y];      // before anything is written: dlogits may be the logits
  const float counted = GRAD && c.mean ? rows_counted() : 1.f;
  float top = -kInf, total = 0.f, sum = 0.f;
  const int n = row.count > tid ? (row.count - tid + NT - 1) / NT : 0;                 // vectors of this thread
  if (MORE) {
    constexpr int U = 4;
    for (int k0 = MAXC; k0 < n; k0 += U) {
      typename R::vec_t z[U];
#pragma unroll
      for (int k = 0; k < U; ++k) row.template load<true>(tid + (k0 + k < n ? k0 + k : k0) * NT, z[k]);
      const float was = top;
#pragma unroll
      for (int k = 0; k < U; ++k)
        if (k0 + k < n)
#pragma unroll
          for (int j = 0; j < R::VW; ++j) top = fmaxf(top, z[k].get(j));
      const float ref = top == -kInf ? 0.f : top;
      sum *= __builtin_amdgcn_exp2f((was - ref) * kLog2e);
#pragma unroll
      for (int k = 0; k < U; ++k)
        if (k0 + k < n)
#pragma unroll
          for (int j = 0; j < R::VW; ++j) {
            const float l = z[k].get(j);
            sum += __builtin_amdgcn_exp2f((l - ref) * kLog2e);
            if (c.each != 0.f) total = __builtin_fmaf(c.each, l, total);
          }
    }
  }
  const float before = top;                        // what sum is relative to
  const Edge<R> edge(row, tid, c.each, top, total);
  const auto exact_top = [&]() {
#pragma unroll
    for (int k = 0; k < MAXC; ++k)
      if (k < n)
#pragma unroll
        for (int j = 0; j < R::VW; ++j) top = fmaxf(top, x[k].get(j));
    return block_max<NW>(top, red);
  };
  if constexpr (sizeof(TL) == 2) {
    PairMax<R> pairs;
#pragma unroll
    for (int k = 0; k < MAXC; ++k)
      if (k < n) pairs.add(x[k]);
    const float all = block_max<NW>(fmaxf(top, pairs.top()), red);
    top = pairs.none(all) ? exact_top() : all;
  } else {
    top = exact_top();
  }
  if (c.each != 0.f) {
#pragma unroll
    for (int k = 0; k < MAXC; ++k)
      if (k < n)
#pragma unroll
        for (int j = 0; j < R::VW; ++j) total = __builtin_fmaf(c.each, x[k].get(j), total);
    total = block_sum<NW>(total, red);
  }
  const float m = top == -kInf ? 0.f : top;
  const Shift sh(m);
  if (MORE && n > MAXC) sum *= sh.exp(before);
  sum += sh.exp(edge.l);
#pragma unroll
  for (int k = 0; k < MAXC; ++k) {
    x[k].pin();
    if (k < n) sum_exp<R>(x[k], sh, sum);
  }
  sum = block_sum<NW>(sum, red);
  const RowResult g(sh, m, sum, total, ly, c, counted, t, tid == 0, rows, lse_out);
  if (!GRAD) return g.loss;
#pragma unroll
  for (int k = 0; k < MAXC; ++k) {
    x[k].pin();
    if (k < n) gradient<true>(row, tid + k * NT, x[k], sh, g.scale, g.share, g.own, y);
  }
  if (MORE) {
    constexpr int U = 4;
    for (int k0 = n - 1; k0 >= MAXC; k0 -= U) {
      typename R::vec_t z[U];
#pragma unroll
      for (int k = 0; k < U; ++k) row.load(tid + (k0 - k >= MAXC ? k0 - k : k0) * NT, z[k]);
#pragma unroll
      for (int k = 0; k < U; ++k)
        if (k0 - k >= MAXC) gradient<false>(row, tid + (k0 - k) * NT, z[k], sh, g.scale, g.share, g.own, y);
    }
  }
  edge.store(row, sh, g, y);
  for (int v = V + tid; v < V_pad; v += NT) dlogits[t * ld_grad + v] = (TG)0.f;
  return g.loss;
}

// ROWS: of a workgroup, more than one where a wavefront takes a row (NT = 64)
template <typename TL, typename TG, int ROWS, int NT, int MAXC, bool MORE, bool GRAD, bool SAME>
__global__ void __launch_bounds__(NT* ROWS) loss_row_kernel(const TL* logits, const Labels labels, int T_, int V, int V_pad, int64_t ld, int64_t ld_grad, RowTerms c,
                                                            const int* __restrict__ count, float* __restrict__ rows, float* __restrict__ lse_out, TG* dlogits, int n_rows) {
  static_assert(ROWS == 1 || NT == 64, "");
  __shared__ float red[NT / 64];
  const int tid = ROWS == 1 ? threadIdx.x : threadIdx.x & 63, t = ROWS == 1 ? blockIdx.x : blockIdx.x * ROWS + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (ROWS > 1 && t >= n_rows) return;
  const auto counted = [&]() {
    if (count) return (float)*count;
    int n = 0;
    for (int i = tid; i < T_; i += NT) n += labels[i] >= 0;
    return block_sum<NT / 64>((float)n, red);      // exact: T is small here
  };
  loss_row<NT, MAXC, MORE, GRAD, SAME>(logits, labels, t, tid, V, V_pad, ld, ld_grad, c, counted, rows, lse_out, dlogits, red);
}

// Up to 16 short rows (kFewVecs vectors together): one workgroup for all of them and their sum, a wavefront on each, and so one launch.  8 rows of 1024 bf16:
// 3.4 us, with gradient 4.1 (rows and sum in a launch each: 5.2, 6.3); 16 rows of 2048: 4.6, 6.5 (5.2, 6.4).  A second row a wavefront loses: 32 of 1024 take 6.1, 8.5 (5.1, 6.1).
constexpr int kFewRows = 16, kFewVecs = 4096;
template <typename TL, typename TG, bool GRAD, bool SAME>
__global__ void __launch_bounds__(64 * kFewRows) loss_few_kernel(const TL* logits, const Labels labels, int T_, int V, int V_pad, int64_t ld, int64_t ld_grad, RowTerms c,
                                                        float* __restrict__ loss, float* __restrict__ rows, float* __restrict__ lse_out, TG* dlogits) {
  __shared__ double red[kFewRows];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int n = __popcll(__ballot(lane < T_ && labels[lane < T_ ? lane : 0] >= 0));
  double s = 0.0;
  if (wave < T_)
    s = (double)loss_row<64, 8, false, GRAD, SAME>(logits, labels, wave, lane, V, V_pad, ld, ld_grad, c, [&]() { return (float)n; }, rows, lse_out, dlogits, nullptr);
  if (lane == 0) red[wave] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    s = 0.0;
    for (int w = 0; w < kFewRows; ++w) s += red[w];
    store_loss(s, n, c.mean, loss);
  }
}

// The gradient from a saved lse: nothing is summed, so a row is cut into parts of kPart vectors, and ROWS short ones share a workgroup (65536 rows of 256 bf16
// 12 us, 44 with a workgroup each).
constexpr int kPart = 1024;
template <typename TL, typename TG, bool SAME, int ROWS>
__global__ void __launch_bounds__(256) loss_bwd_kernel(const TL* logits, const Labels labels, int V, int V_pad, int64_t ld, int64_t ld_grad, RowTerms c,
                                                       const float* __restrict__ lse_in, const float* __restrict__ dloss, TG* dlogits, unsigned parts, unsigned n_rows) {
  typedef RowVecs<TL, TG, SAME> R;
  constexpr int U = kPart / 256, NT = 256 / ROWS;
  const int tid = threadIdx.x % NT;
  const int64_t t = ROWS == 1 ? blockIdx.x / parts : blockIdx.x * ROWS + threadIdx.x / NT;
  if (ROWS > 1 && t >= n_rows) return;
  const unsigned part = ROWS == 1 ? blockIdx.x - (unsigned)t * parts : 0;
  const int y = labels[t];
  const R row(logits, dlogits, t, V, ld, ld_grad);
  const float lse = lse_in[t];
  const bool none = y < 0 || lse == -kInf;
  const int first = part * kPart + tid;
  typename R::vec_t x[U];
  if (!none) {
#pragma unroll
    for (int k = 0; k < U; ++k)
      if (first + k * NT < row.count) row.load(first + k * NT, x[k]);
  }
  const Shift sh(lse);
  const float up = none ? 0.f : dloss[t];
  const float rest = sh.far ? 1.f : __builtin_amdgcn_exp2f(-__builtin_fmaf(lse, sh.s, -sh.ms));     // what the rounding of lse s leaves out
  struct {
    float scale, share, own;
  } const g{up * (c.z != 0.f ? 1.f + 2.f * c.z * lse : 1.f) * rest, up * c.each, up * (1.f - c.eps)};
#pragma unroll
  for (int k = 0; k < U; ++k) {
    const int i = first + k * NT;
    if (i >= row.count) break;
    if (none) {
      const float zero[R::VW] = {};
      row.store(i, zero);
    } else {
      gradient<false>(row, i, x[k], sh, g.scale, g.share, g.own, y);
    }
  }
  if (part) return;
  int e;
  if (row.edge(tid, &e)) row.out[e] = none ? 0.f : __builtin_fmaf(g.scale, sh.exp((float)row.in[e]), -g.share) - (e + row.head == y ? g.own : 0.f);
  for (int v = V + tid; v < V_pad; v += NT) dlogits[t * ld_grad + v] = (TG)0.f;
}

// =============================================================================== few rows
// A few rows that are more than a workgroup holds: each is cut into `parts` runs of at most kSplitVecs vectors, a workgroup on each, which leaves the run's
// maximum, sum of exponentials and sum of logits; whoever needs the row's joins those of its parts, in order.  With a gradient the logits are read
// twice, the second time from the memory-side cache.  131072 classes, us without and with the cut: gradient from bf16, 1 row 20 and 10, 128 rows 25 and 20,
// 333 rows 48 and 43, 512 rows 59 and 64; from fp32, 1 row 23 and 10, 128 rows 32 and 28, 200 rows 39 and 42; the loss alone of fp32, 1 row 14 and 7, 32 rows
// 18 and 11, 128 rows 19 and 25 (one workgroup joins them all).  A row that a workgroup does hold gains nothing (50001 classes of bf16, 1 row 11.1 and
// 11.2, 333 rows 21 and 23).
constexpr int kSplitVecs = 2048, kSplitMax = 64, kSplitRows = 128, kSplitRowsAlone = 64;
struct PartSum {
  float m, sum, total, ly;                         // ly: the logit at the label, in part 0 (dlogits may take the logits' place before a row is joined)
};

template <typename TL>
__global__ void __launch_bounds__(256) loss_part_kernel(const TL* __restrict__ logits, const Labels labels, int V, int64_t ld, float each, int len, unsigned parts,
                                                        PartSum* __restrict__ out) {
  typedef RowVecs<TL, TL, true> R;
  constexpr int NT = 256, U = kSplitVecs / NT, NW = NT / 64;
  __shared__ float red[NW];
  const int64_t t = blockIdx.x / parts;
  const int part = (int)(blockIdx.x - (unsigned)t * parts), y = labels[t], tid = threadIdx.x;
  if (y < 0) return;
  const R row(logits, nullptr, t, V, ld, ld);
  const int from = part * len, left = row.count - from, m_ = left < len ? left : len, n = m_ > tid ? (m_ - tid + NT - 1) / NT : 0;
  typename R::vec_t x[U];
  if (m_ > 0)
#pragma unroll
    for (int k = 0; k < U; ++k) row.template load<true>(from + (k < n ? tid + k * NT : m_ - 1), x[k]);
  float top = -kInf, total = 0.f, sum = 0.f, edge = -kInf;
  int e;
  if (part == 0 && row.edge(tid, &e)) {
    top = edge = (float)row.in[e];
    if (each != 0.f) total = each * edge;
  }
#pragma unroll
  for (int k = 0; k < U; ++k)
    if (k < n)
#pragma unroll
      for (int j = 0; j < R::VW; ++j) top = fmaxf(top, x[k].get(j));
  top = block_max<NW>(top, red);
  const Shift sh(top == -kInf ? 0.f : top);
  sum = sh.exp(edge);
#pragma unroll
  for (int k = 0; k < U; ++k) {
    x[k].pin();
    if (k < n)
#pragma unroll
      for (int j = 0; j < R::VW; ++j) {
        sum += sh.exp(x[k].get(j));
        if (each != 0.f) total = __builtin_fmaf(each, x[k].get(j), total);
      }
  }
  sum = block_sum<NW>(sum, red);
  if (each != 0.f) total = block_sum<NW>(total, red);
  if (tid == 0) out[blockIdx.x] = PartSum{top, sum, total, part == 0 ? (float)logits[t * ld + y] : 0.f};
}

// what a part's sum counts for beside the row's maximum m
__device__ __forceinline__ float part_weight(const PartSum& p, float m) {
#pragma clang fp contract(off)        // of the rounded products, as in the sums: with either unrounded, logits around 1e4 are off by up to 3e-4
  if (p.m == -kInf) return 0.f;
  const Shift a(p.m), b(m);
  return p.m == m ? 1.f : a.far != b.far ? 0.f : __builtin_amdgcn_exp2f(a.ms - b.ms);      // p.m <= m: one that is far and one that is not are 128 apart
}

// joined by a wavefront, a part a lane: every lane has the result
__device__ __forceinline__ PartSum join_parts(const PartSum* __restrict__ p, int parts) {
  const int lane = threadIdx.x & 63;
  PartSum mine = lane < parts ? p[lane] : PartSum{-kInf, 0.f, 0.f, 0.f}, all;
  all.m = wave_max(mine.m);
  all.sum = wave_sum(mine.sum * part_weight(mine, all.m));
  all.total = wave_sum(mine.total);
  all.ly = __shfl(mine.ly, 0, 64);
  return all;
}

// the gradient of a part, from the sums of all of its row's
template <typename TL, typename TG, bool SAME>
__global__ void __launch_bounds__(256) loss_part_grad_kernel(const TL* logits, const Labels labels, int T_, int V, int V_pad, int64_t ld, int64_t ld_grad, RowTerms c, int len,
                                                             unsigned parts, const PartSum* __restrict__ sums, float* __restrict__ rows, float* __restrict__ lse_out,
                                                             TG* dlogits) {
  typedef RowVecs<TL, TG, SAME> R;
  constexpr int NT = 256, U = kSplitVecs / NT, NW = NT / 64;
  __shared__ float red[NW];
  const int64_t t = blockIdx.x / parts;
  const int part = (int)(blockIdx.x - (unsigned)t * parts), y = labels[t], tid = threadIdx.x;
  const R row(logits, dlogits, t, V, ld, ld_grad);
  const int from = part * len, left = row.count - from, m_ = left < len ? left : len, n = m_ > tid ? (m_ - tid + NT - 1) / NT : 0;
  int e;
  const bool edge = part == 0 && row.edge(tid, &e);
  if (y < 0) {
    const float zero[R::VW] = {};
    for (int k = 0; k < n; ++k) row.store(from + tid + k * NT, zero);
    if (edge) row.out[e] = (TG)0.f;
    if (part == 0 && tid == 0) {
      rows[t] = 0.f;
      if (lse_out) lse_out[t] = 0.f;
    }
  } else {
    typename R::vec_t x[U];
    if (m_ > 0)
#pragma unroll
      for (int k = 0; k < U; ++k) row.load(from + (k < n ? tid + k * NT : m_ - 1), x[k]);
    const float le = edge ? (float)row.in[e] : 0.f;
    const PartSum all = join_parts(sums + t * parts, (int)parts);
    float counted = 1.f;
    if (c.mean) {
      int k = 0;
      for (int i = tid; i < T_; i += NT) k += labels[i] >= 0;
      counted = block_sum<NW>((float)k, red);
    }
    const float m = all.m == -kInf ? 0.f : all.m;
    const Shift sh(m);
    const RowResult g(sh, m, all.sum, all.total, all.ly, c, counted, t, part == 0 && tid == 0, rows, lse_out);
#pragma unroll
    for (int k = 0; k < U; ++k)
      if (k < n) gradient<false>(row, from + tid + k * NT, x[k], sh, g.scale, g.share, g.own, y);
    if (edge) row.out[e] = __builtin_fmaf(g.scale, sh.exp(le), -g.share) - (e + row.head == y ? g.own : 0.f);
  }
  if (part == 0)
    for (int v = V + tid; v < V_pad; v += NT) dlogits[t * ld_grad + v] = (TG)0.f;
}

// =============================================================================== sum of the rows' losses
struct LossSum {
  double s;
  int64_t n;
};

// parts != 0: the rows' losses are formed here, from the sums of their parts, a wavefront on each.  out: one workgroup of several, which leaves its sum
__global__ void __launch_bounds__(1024) loss_sum_kernel(float* rows, const Labels labels, int T_, int mean, float* __restrict__ loss, int parts, const PartSum* __restrict__ sums,
                                                        RowTerms c, float* __restrict__ lse_out, LossSum* __restrict__ out) {
  __shared__ double red[16];
  __shared__ int redn[16];
  if (parts) {
    const bool first = (threadIdx.x & 63) == 0;
    for (int t = threadIdx.x >> 6; t < T_; t += 16) {
      if (labels[t] < 0) {
        if (first) {
          rows[t] = 0.f;
          if (lse_out) lse_out[t] = 0.f;
        }
        continue;
      }
      const PartSum all = join_parts(sums + (size_t)t * parts, parts);
      const float m = all.m == -kInf ? 0.f : all.m;
      const RowResult g(Shift(m), m, all.sum, all.total, all.ly, c, 1.f, t, first, rows, lse_out);
    }
    __syncthreads();
  }
  double s = 0.0;
  int n = 0;
  for (int t = blockIdx.x * 1024 + threadIdx.x; t < T_; t += gridDim.x * 1024) {
    s += (double)rows[t];
    n += labels[t] >= 0;
  }
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  n = wave_count(n);
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
    if (out) out[blockIdx.x] = LossSum{s, n};
    else store_loss(s, n, mean, loss);
  }
}

__global__ void __launch_bounds__(64) loss_sum_join_kernel(const LossSum* __restrict__ sums, int mean, float* __restrict__ loss) {
  double s = sums[threadIdx.x].s;
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  const int n = wave_count((int)sums[threadIdx.x].n);
  if (threadIdx.x == 0) store_loss(s, n, mean, loss);
}

// =============================================================================== launchers
static inline int last_err() { return (int)hipGetLastError(); }

constexpr int kHeldVecs = 512 * 16;      // of a row, at most, by a workgroup

// parts that a row is cut into, 0: not cut
static int parts_of(const LossArgs& a, bool grad) {
  const int64_t vecs = a.V / (a.dtype == DT_BF16 ? 8 : 4);
  if (!a.T || a.T > (grad ? kSplitRows : kSplitRowsAlone) || vecs <= kHeldVecs) return 0;
  const int64_t least = (vecs + kSplitVecs - 1) / kSplitVecs, want = 1024 / a.T, most = vecs / 512;
  const int64_t parts = want < least ? least : want < most ? want : most;
  return least > kSplitMax ? 0 : parts < kSplitMax ? (int)parts : kSplitMax;
}

// 64 counts; 64 sums; the rows' losses where the caller has no use for them; the sums of parts
constexpr size_t kHeadBytes = 64 * sizeof(int) + 64 * sizeof(LossSum);
static size_t rows_bytes(int T_) { return ((size_t)T_ * 4 + 255) / 256 * 256; }
size_t loss_workspace_bytes(const LossArgs& a) {
  return kHeadBytes + rows_bytes(a.T) + (size_t)a.T * parts_of(a, true) * sizeof(PartSum);
}

template <typename F>
static int by_types(const LossArgs& a, F f) {
  const auto with = [&](auto* l, auto* g) {
    constexpr int64_t VW = 16 / sizeof(*l);
    return (a.ld - a.ld_grad) % VW == 0 ? f(l, g, std::true_type{}) : f(l, g, std::false_type{});
  };
  if (a.dtype == DT_BF16) return with((bf16_t*)nullptr, (bf16_t*)nullptr);
  if (a.grad_dtype == DT_BF16) return with((float*)nullptr, (bf16_t*)nullptr);
  return with((float*)nullptr, (float*)nullptr);
}

// Rows up to which a workgroup counts the labels itself.  us so and with a launch for the count: 256 rows of 1000 7.8 and 10.3, 1024 rows of 1000 10.2 and
// 10.4, of 32000 26.9 and 29.6; 2048 rows of 1000 13.6 and 10.3, 3000 rows of 32000 81 and 76.
constexpr int kCountedInline = 1024;
// More rows than this that a wavefront holds lie four to a workgroup: with gradient, 65536 rows of 4000 bf16 187 us (201 with a workgroup to a row), 16384 57 and 60,
// 4096 the same.  Those of at most a vector a lane always do, with registers for no more: 2^20 rows of 256 453 us (516 with room for eight), 333 of 30 the same.
constexpr int kWaveRows = 2047;
// Rows up to which one workgroup counts the labels, and one adds up the losses, not 64 and another launch.  us with one and with 64, rows of 64 bf16, loss
// alone / with gradient: 4096 rows 7.6 and 9.8 / 10.9 and 14.8, 8192 10.0 and 9.8 / 14.5 and 16.4, 16384 15.1 and 10.8 / 22.0 and 17.1, 65536 53 and 23 /
// 74 and 36, 2^20 902 and 288.
constexpr int kOneGroup = 16384;

int launch_loss(const LossArgs& a, const void* logits, const void* labels, float* loss, float* rows, float* lse, void* dlogits, void* ws, hipStream_t st) {
  int* count = (int*)ws;
  if (!rows) rows = (float*)((char*)ws + kHeadBytes);
  const RowTerms c{a.eps, a.z, a.grad_scale, a.eps / (float)a.V, a.mean};
  const Labels y{labels, a.label_type == IDX_I64, a.V};
  return by_types(a, [&](auto* pl, auto* pg, auto same) {
    using TL = std::remove_pointer_t<decltype(pl)>;
    using TG = std::remove_pointer_t<decltype(pg)>;
    constexpr bool SAME = decltype(same)::value;
    const TL* l = (const TL*)logits;
    TG* d = (TG*)dlogits;
    constexpr int VW = 16 / sizeof(TL);
    const bool many = a.T > kOneGroup;
    const int vecs = a.V / VW, parts = parts_of(a, d != nullptr);
    PartSum* sums = (PartSum*)((char*)ws + kHeadBytes + rows_bytes(a.T));
    if (a.T && a.T <= kFewRows && vecs <= 64 * 8 && a.T * vecs <= kFewVecs) {
      const auto kernel = d ? loss_few_kernel<TL, TG, true, SAME> : loss_few_kernel<TL, TG, false, true>;
      hipLaunchKernelGGL(kernel, dim3(1), dim3(64 * kFewRows), 0, st, l, y, a.T, a.V, a.V_pad, a.ld, a.ld_grad, c, loss, rows, lse, d);
      return last_err();
    }
    if (parts) {
      const int len = (vecs + parts - 1) / parts;
      hipLaunchKernelGGL((loss_part_kernel<TL>), dim3((unsigned)(a.T * parts)), dim3(256), 0, st, l, y, a.V, a.ld, c.each, len, (unsigned)parts, sums);
      int e = last_err();
      if (e) return e;
      if (d) {
        hipLaunchKernelGGL((loss_part_grad_kernel<TL, TG, SAME>), dim3((unsigned)(a.T * parts)), dim3(256), 0, st, l, y, a.T, a.V, a.V_pad, a.ld, a.ld_grad, c, len, (unsigned)parts,
                           sums, rows, lse, d);
        e = last_err();
        if (e) return e;
      }
    } else if (a.T) {
      if (d && a.mean && a.T > kCountedInline) {
        hipLaunchKernelGGL(loss_count_kernel, dim3(many ? 64 : 1), dim3(1024), 0, st, y, a.T, count);
        if (many) hipLaunchKernelGGL(loss_count_join_kernel, dim3(1), dim3(64), 0, st, count);
      } else {
        count = nullptr;
      }
#define TAW_LOSS(ROWS, NT, MAXC, MORE)                                                                                                                         \
  do {                                                                                                                                                         \
    const auto kernel = d ? loss_row_kernel<TL, TG, ROWS, NT, MAXC, MORE, true, SAME> : loss_row_kernel<TL, TG, ROWS, NT, MAXC, MORE, false, true>;            \
    over_blocks(a.T, kMostBlocks, [&](int64_t t, unsigned n) {                                                                                                 \
      hipLaunchKernelGGL(kernel, dim3((n + ROWS - 1) / ROWS), dim3(NT * ROWS), 0, st, l + t * a.ld, y.from(t), a.T, a.V, a.V_pad, a.ld, a.ld_grad, c, count,   \
                         rows + t, lse ? lse + t : lse, d ? d + t * a.ld_grad : d, (int)n);                                                                    \
    });                                                                                                                                                        \
  } while (0)
      if (vecs <= 64) TAW_LOSS(4, 64, 1, false);
      else if (vecs <= 64 * 8 && a.T > kWaveRows) TAW_LOSS(4, 64, 8, false);
      else if (vecs <= 64 * 8) TAW_LOSS(1, 64, 8, false);
      else if (vecs <= 256 * 8) TAW_LOSS(1, 256, 8, false);
      else if (vecs <= 512 * 8) TAW_LOSS(1, 512, 8, false);
      else if (vecs <= kHeldVecs) TAW_LOSS(1, 512, 16, false);
      else TAW_LOSS(1, 512, 16, true);
#undef TAW_LOSS
      const int e = last_err();
      if (e) return e;
    }
    LossSum* part = (LossSum*)((char*)ws + 64 * sizeof(int));
    hipLaunchKernelGGL(loss_sum_kernel, dim3(many ? 64 : 1), dim3(1024), 0, st, rows, y, a.T, a.mean, loss, d ? 0 : parts, sums, c, lse, many ? part : nullptr);
    if (many) hipLaunchKernelGGL(loss_sum_join_kernel, dim3(1), dim3(64), 0, st, part, a.mean, loss);
    return last_err();
  });
}

int launch_loss_bwd(const LossArgs& a, const void* logits, const void* labels, const float* lse, const float* dloss, void* dlogits, hipStream_t st) {
  const RowTerms c{a.eps, a.z, 0.f, a.eps / (float)a.V, 0};
  const Labels y{labels, a.label_type == IDX_I64, a.V};
  return by_types(a, [&](auto* pl, auto* pg, auto same) {
    using TL = std::remove_pointer_t<decltype(pl)>;
    using TG = std::remove_pointer_t<decltype(pg)>;
    constexpr int VW = 16 / sizeof(TL);
    const unsigned vecs = a.V / VW, parts = vecs ? (vecs + kPart - 1) / kPart : 1;
#define TAW_LOSS_BWD(ROWS)                                                                                                                                             \
  over_blocks(a.T, kMostBlocks / parts & ~7ull, [&](int64_t t, unsigned n) { /* multiples of 8 rows: as aligned as the first */                                        \
    hipLaunchKernelGGL((loss_bwd_kernel<TL, TG, decltype(same)::value, ROWS>), dim3((n + ROWS - 1) / ROWS * parts), dim3(256), 0, st, (const TL*)logits + t * a.ld,    \
                       y.from(t), a.V, a.V_pad, a.ld, a.ld_grad, c, lse + t, dloss + t, (TG*)dlogits + t * a.ld_grad, parts, n);                                       \
  })
    if (vecs <= kPart / 16) TAW_LOSS_BWD(16);
    else if (vecs <= kPart / 4) TAW_LOSS_BWD(4);
    else TAW_LOSS_BWD(1);
#undef TAW_LOSS_BWD
    return last_err();
  });
}

}  // namespace taw
