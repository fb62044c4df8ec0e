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
// A thread moves one vector of each of U consecutive tokens' rows, and stores it past L2 (the batch is larger than that, and leaves it to the table's
// frequent rows).  65536 tokens of 2048, 32000 rows: U = 1 94 us, 2 57 us, 4 58 us, 8 59 us; U = 4 with ordinary stores 80 us.
template <typename T, int VW, int U, typename TI>
__global__ void __launch_bounds__(256) embed_fwd_kernel(const TI* __restrict__ ids, const T* __restrict__ table, T* __restrict__ x, int T_, int H, int V, int64_t ld_table,
                                                        int64_t ld_x, float scale) {
  const unsigned cpr = (unsigned)(H / VW);
  const uint64_t idx = (uint64_t)blockIdx.x * 256 + threadIdx.x;
  const uint64_t group = idx / cpr;
  const int64_t t0 = (int64_t)group * U;
  if (t0 >= T_) return;
  const int col = (int)(idx - group * cpr) * VW;
  int v[U];
#pragma unroll
  for (int k = 0; k < U; ++k) v[k] = t0 + k < T_ ? row_id(ids, t0 + k, V) : -1;
  Vec<T, VW> r[U];
#pragma unroll
  for (int k = 0; k < U; ++k)
    if (v[k] >= 0) r[k].load(table + (int64_t)v[k] * ld_table + col);
#pragma unroll
  for (int k = 0; k < U; ++k) {
    if (t0 + k >= T_) break;
    Vec<T, VW> o;
#pragma unroll
    for (int j = 0; j < VW; ++j) o.set(j, v[k] >= 0 ? r[k].get(j) * scale : 0.f);
    o.store_nt(x + (t0 + k) * ld_x + col);
  }
}

// =============================================================================== backward
// The tokens are sorted by id (stable: tokens of one id keep their order), then the sorted sequence is cut into pieces of K tokens, and the rows of
// dx of a piece are summed id by id.  An id with at most K tokens is summed whole, by the piece it starts in (which so reads up to K - 1 tokens
// beyond its end); one with more leaves a partial sum in every piece it has a part in, and a last kernel adds those up in order.  So no thread reads
// more than 2 K rows whatever the ids are, every row of dx is read once, and the result does not depend on scheduling.

constexpr int kSortWaves = 16;
constexpr int kSortMaxOwn = 1024;              // ids that a workgroup of the sort owns at most

// The order of the sorted ids is by place_of(v), any order being as good as another: workgroup w of the sort owns the nb-th part of the ids whose low
// bits come to w, so that the frequent ids of a vocabulary, which lie together, are spread over all of them.
struct SortShape {
  int lb, own;                                 // nb = 1 << lb workgroups, each with `own` ids: id r of workgroup w is (r << lb) | ((w - r) & (nb - 1))
  __host__ __device__ int group_of(int v) const { return (v + (v >> lb)) & ((1 << lb) - 1); }
  __host__ __device__ int place_of(int v) const { return group_of(v) * own + (v >> lb); }
  __host__ __device__ int64_t places() const { return ((int64_t)own << lb) + 1; }
};
static SortShape sort_shape(int V) {
  SortShape s{0, 0};
  while (s.lb < 8 && (1 << s.lb) < V) ++s.lb;
  while (((V - 1) >> s.lb) >= kSortMaxOwn) ++s.lb;
  s.own = ((V - 1) >> s.lb) + 1;
  return s;
}

// A workgroup goes through all the tokens twice: to count its own ids by wavefront (each has a contiguous run of tokens) and the tokens of the
// workgroups before it, which is where its part of the sorted sequence starts; and to place its own.  No workgroup waits for another, nothing is
// cleared beforehand.  The ids are read from L2 (256 times 128 KiB at 32768 tokens).
// perm: token at a sorted place; sid: its id; start[place_of(v)], start[own nb]: where the tokens of v start, and the number of tokens that name a row.
template <typename TI>
__global__ void __launch_bounds__(1024) embed_sort_kernel(const TI* __restrict__ ids, int T_, int V, SortShape sh, int* __restrict__ perm, int* __restrict__ sid,
                                                          int* __restrict__ start) {
  extern __shared__ int cnt[];                 // [kSortWaves][own]
  __shared__ int wsum[kSortWaves], lsum[kSortWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, R = sh.own, w0 = blockIdx.x;
  for (int i = threadIdx.x; i < kSortWaves * R; i += 1024) cnt[i] = 0;
  __syncthreads();
  const int run = ((T_ + kSortWaves - 1) / kSortWaves + 63) / 64 * 64;
  const int t0 = wave * run, t1 = t0 + run < T_ ? t0 + run : T_;
  int* mycnt = cnt + wave * R;
  int less = 0;
  constexpr int U = 16;
  for (int t = t0; t < t1; t += 64 * U) {
    int v[U];
#pragma unroll
    for (int k = 0; k < U; ++k) {                // all the loads first, whatever lies behind the run
      const int at = t + 64 * k + lane;
      v[k] = row_id(ids, at < t1 ? at : t1 - 1, V);
      if (at >= t1) v[k] = -1;
    }
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int g = v[k] < 0 ? 0x7fffffff : sh.group_of(v[k]);
      less += g < w0;
      if (g == w0) atomicAdd(&mycnt[v[k] >> sh.lb], 1);
    }
  }
  for (int o = 32; o > 0; o >>= 1) less += __shfl_xor(less, o, 64);
  if (lane == 0) lsum[wave] = less;
  __syncthreads();
  // where each id's tokens start, and within them each wavefront's
  int total = 0;
  const int r = threadIdx.x;                   // R <= 1024
  if (r < R)
    for (int w = 0; w < kSortWaves; ++w) total += cnt[w * R + r];
  int incl = total;
  for (int o = 1; o < 64; o <<= 1) {
    const int up = __shfl_up(incl, o, 64);
    if (lane >= o) incl += up;
  }
  if (lane == 63) wsum[wave] = incl;
  __syncthreads();
  int at = incl - total;
  for (int w = 0; w < kSortWaves; ++w) {
    at += lsum[w];
    if (w < wave) at += wsum[w];
  }
  if (r < R) {
    start[w0 * R + r] = at;
    int off = at;
    for (int w = 0; w < kSortWaves; ++w) {
      const int c = cnt[w * R + r];
      cnt[w * R + r] = off;
      off += c;
    }
    if (r == R - 1 && w0 == (int)gridDim.x - 1) start[w0 * R + R] = off;
  }
  __syncthreads();
  for (int t = t0; t < t1; t += 64 * U) {
    int v[U];
#pragma unroll
    for (int k = 0; k < U; ++k) {                // all the loads first, whatever lies behind the run
      const int at = t + 64 * k + lane;
      v[k] = row_id(ids, at < t1 ? at : t1 - 1, V);
      if (at >= t1) v[k] = -1;
    }
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const bool mine = v[k] >= 0 && sh.group_of(v[k]) == w0;
      unsigned long long left = __ballot(mine);
      while (left) {                           // one turn for each different id of the 64: mostly none or one
        const int f = __builtin_ctzll(left);
        const int id = __builtin_amdgcn_readlane(v[k], f);
        const unsigned long long same = __ballot(mine && v[k] == id);
        const int base = mycnt[id >> sh.lb];
        if (mine && v[k] == id) {
          const int pos = base + __popcll(same & ((1ull << lane) - 1));
          perm[pos] = t + 64 * k + lane;
          sid[pos] = id;
        }
        if (lane == f) mycnt[id >> sh.lb] = base + __popcll(same);
        left &= ~same;
      }
    }
  }
}

// Sums of pieces: a thread has one vector of columns of a piece.  part: [pieces][2][H]: the sum of the long id that a piece starts within (0), and of
// the one that starts in it and goes on behind it (1).  The threads behind those of the pieces zero the rows that no token names.
constexpr int kZeroRows = 4;
template <typename T, int VW>
__global__ void __launch_bounds__(256) embed_rows_kernel(const int* __restrict__ perm, const int* __restrict__ sid, const int* __restrict__ start, const T* __restrict__ dx,
                                                         float* __restrict__ G, float* __restrict__ part, int H, int V, SortShape sh, int64_t ld_table, int64_t ld_x,
                                                         float scale, int accumulate, int K, unsigned piece_blocks) {
  constexpr int U = 8;
  const unsigned cpr = (unsigned)(H / VW);
  typedef float fv_t __attribute__((ext_vector_type(VW), aligned(VW * 4 < 16 ? VW * 4 : 16)));
  if (blockIdx.x >= piece_blocks) {
    constexpr int ZW = VW < 4 ? VW : 4;        // 16 bytes a store
    typedef float zv_t __attribute__((ext_vector_type(ZW)));
    const unsigned zpr = (unsigned)(H / ZW);
    const uint64_t idx = (uint64_t)(blockIdx.x - piece_blocks) * 256 + threadIdx.x;
    const uint64_t q = idx / zpr;
    const int col = (int)(idx - q * zpr) * ZW;
#pragma unroll
    for (int k = 0; k < kZeroRows; ++k) {
      const int64_t v = (int64_t)q * kZeroRows + k;
      if (v >= V) break;
      const int at = sh.place_of((int)v);
      if (start[at] == start[at + 1]) __builtin_nontemporal_store(zv_t(0.f), reinterpret_cast<zv_t*>(G + v * ld_table + col));
    }
    return;
  }
  const uint64_t idx = (uint64_t)blockIdx.x * 256 + threadIdx.x;
  const uint64_t p = idx / cpr;
  const int col = (int)(idx - p * cpr) * VW;
  const int n = start[sh.places() - 1];
  if (p * K >= (uint64_t)n) return;
  const int p0 = (int)p * K, p1 = p0 + K < n ? p0 + K : n;
  int from = p0, to = p1;
  bool head = false, tail = false;
  {
    const int v = sh.place_of(sid[p0]), s = start[v], e = start[v + 1];
    if (s < p0) {
      head = e - s > K;
      if (!head) from = e;                     // its start's piece has it whole
    }
  }
  {
    const int v = sh.place_of(sid[p1 - 1]), s = start[v], e = start[v + 1];
    if (e > p1) {
      tail = e - s > K;
      if (!tail) to = e;
    }
  }
  if (from >= to) return;
  fv_t acc = fv_t(0.f);
  int cur = sid[from];
  auto flush = [&](bool last) {
    if (head || (last && tail)) {
      *reinterpret_cast<fv_t*>(part + ((int64_t)p * 2 + (head ? 0 : 1)) * H + col) = acc;
    } else {
      float* g = G + (int64_t)cur * ld_table + col;
      fv_t o = acc * scale;
      if (accumulate) o += *reinterpret_cast<const fv_t*>(g);
      *reinterpret_cast<fv_t*>(g) = o;
    }
    head = false;
  };
  for (int q = from; q < to; q += U) {
    int who[U], id[U];
    Vec<T, VW> r[U];
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int at = q + k < to ? q + k : to - 1;
      who[k] = perm[at];
      id[k] = sid[at];
    }
#pragma unroll
    for (int k = 0; k < U; ++k) r[k].load(dx + (int64_t)who[k] * ld_x + col);
#pragma unroll
    for (int k = 0; k < U; ++k) {
      if (q + k >= to) break;
      if (id[k] != cur) {
        flush(false);
        cur = id[k];
        acc = fv_t(0.f);
      }
#pragma unroll
      for (int j = 0; j < VW; ++j) acc[j] += r[k].get(j);
    }
  }
  flush(true);
}

// The ids with more than K tokens: the workgroup of the kJoinPieces pieces that such an id starts in adds up its partial sums, wavefront w those of the
// pieces w, w + kJoinWaves, ... counted from there, then the wavefronts in order.
constexpr int kJoinWaves = 8, kJoinPieces = 16;
template <int VW>
__global__ void __launch_bounds__(64 * kJoinWaves) embed_join_kernel(const int* __restrict__ sid, const int* __restrict__ start, const float* __restrict__ part,
                                                                     float* __restrict__ G, int H, SortShape sh, int64_t ld_table, float scale, int accumulate, int K) {
  typedef float fv_t __attribute__((ext_vector_type(VW)));
  __shared__ fv_t red[kJoinWaves][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = start[sh.places() - 1];
  // lane i looks at piece i: the id at its end, if that starts in it, goes on behind it and is long
  const int64_t end = ((int64_t)blockIdx.x * kJoinPieces + lane + 1) * K;
  int v = 0, np = 0;
  if (lane < kJoinPieces && end < n) {
    v = sid[end - 1];
    const int at = sh.place_of(v), s = start[at], e = start[at + 1];
    if (s >= end - K && e > end && e - s > K) np = (int)((e - 1) / K - (end / K - 1)) + 1;
  }
  for (unsigned long long left = __ballot(np > 0); left; left &= left - 1) {
    const int f = __builtin_ctzll(left);
    const int id = __builtin_amdgcn_readlane(v, f), count = __builtin_amdgcn_readlane(np, f);
    const int64_t p = (int64_t)blockIdx.x * kJoinPieces + f;
    for (int c0 = blockIdx.y * 64 * VW; c0 < H; c0 += gridDim.y * 64 * VW) {
      const int col = c0 + lane * VW;
      fv_t t = fv_t(0.f);
      if (col < H) {
#pragma unroll 8
        for (int k = wave; k < count; k += kJoinWaves) t += *reinterpret_cast<const fv_t*>(part + ((p + k) * 2 + (k ? 0 : 1)) * H + col);
      }
      red[wave][lane] = t;
      __syncthreads();
      if (wave == 0 && col < H) {
#pragma unroll
        for (int w = 1; w < kJoinWaves; ++w) t += red[w][lane];
        t *= scale;
        fv_t* g = reinterpret_cast<fv_t*>(G + (int64_t)id * ld_table + col);
        *g = accumulate ? *g + t : t;
      }
      __syncthreads();
    }
  }
}

// =============================================================================== launchers
static inline int last_err() { return (int)hipGetLastError(); }

// the widest vector of 1, 2, 4 (8 for bf16) elements that the row length and the strides are multiples of
static int width_of(int dtype, int64_t a, int64_t b, int64_t c) {
  const int64_t m = a | b | c;
  return m % 8 == 0 && dtype == DT_BF16 ? 8 : m % 4 == 0 ? 4 : m % 2 == 0 ? 2 : 1;
}

template <int VW> using width_t = std::integral_constant<int, VW>;
template <typename F>
static int by_types(const EmbedArgs& a, F f) {
  const int w = width_of(a.dtype, a.H, a.ld_table, a.ld_x);
  const auto sized = [&](auto* t, auto* i) {
    using T = std::remove_pointer_t<decltype(t)>;
    if constexpr (sizeof(T) == 2)
      if (w == 8) return f(t, i, width_t<8>{});
    return w == 4 ? f(t, i, width_t<4>{}) : w == 2 ? f(t, i, width_t<2>{}) : f(t, i, width_t<1>{});
  };
  if (a.dtype == DT_BF16) return a.id_type == IDX_I64 ? sized((bf16_t*)nullptr, (int64_t*)nullptr) : sized((bf16_t*)nullptr, (int32_t*)nullptr);
  return a.id_type == IDX_I64 ? sized((float*)nullptr, (int64_t*)nullptr) : sized((float*)nullptr, (int32_t*)nullptr);
}

static bool grid_of(uint64_t threads, uint64_t* blocks) {
  *blocks = (threads + 255) / 256;
  return *blocks <= 0x7fffffffu;
}

int launch_embed_fwd(const EmbedArgs& a, const void* ids, const void* table, void* x, hipStream_t st) {
  return by_types(a, [&](auto* t, auto* i, auto w) {
    using T = std::remove_pointer_t<decltype(t)>;
    using TI = std::remove_pointer_t<decltype(i)>;
    constexpr int VW = decltype(w)::value, U = 2;
    uint64_t blocks;
    if (!grid_of((uint64_t)((a.T + U - 1) / U) * (a.H / VW), &blocks)) return (int)hipErrorInvalidValue;
    hipLaunchKernelGGL((embed_fwd_kernel<T, VW, U, TI>), dim3((unsigned)blocks), dim3(256), 0, st, (const TI*)ids, (const T*)table, (T*)x, a.T, a.H, a.V, a.ld_table, a.ld_x,
                       a.scale);
    return last_err();
  });
}

// tokens of a piece: 32, or fewer where that leaves the chip fewer than 8 wavefronts a compute unit
static int piece_of(int64_t T_, int64_t cpr) {
  int K = 32;
  while (K > 8 && T_ * cpr < (int64_t)K * 131072) K /= 2;
  return K;
}

struct EmbedWork {
  int *perm, *sid, *start;
  float* part;
  size_t bytes;
};
static EmbedWork embed_work(const EmbedArgs& a, int K, void* base) {
  size_t off = 0;
  const auto take = [&](size_t bytes) {
    char* p = (char*)base + off;
    off += (bytes + 255) / 256 * 256;
    return (void*)p;
  };
  EmbedWork w;
  w.perm = (int*)take((size_t)a.T * 4);
  w.sid = (int*)take((size_t)a.T * 4);
  w.start = (int*)take((size_t)sort_shape(a.V).places() * 4);
  const size_t pieces = ((size_t)a.T + K - 1) / K;
  w.part = (float*)take(pieces > 1 ? pieces * 2 * a.H * 4 : 0);
  w.bytes = off;
  return w;
}

size_t embed_bwd_workspace_bytes(const EmbedArgs& a) { return embed_work(a, piece_of(a.T, a.H / width_of(a.dtype, a.H, a.ld_table, a.ld_x)), nullptr).bytes; }

int launch_embed_bwd(const EmbedArgs& a, const void* ids, const void* dx, float* G, void* ws, hipStream_t st) {
  return by_types(a, [&](auto* t, auto* i, auto w) {
    using T = std::remove_pointer_t<decltype(t)>;
    using TI = std::remove_pointer_t<decltype(i)>;
    constexpr int VW = decltype(w)::value;
    const uint64_t cpr = a.H / VW;
    const int K = piece_of(a.T, (int64_t)cpr);
    const EmbedWork k = embed_work(a, K, ws);
    const SortShape sh = sort_shape(a.V);
    TAW_SET_LDS_LIMIT_ONCE((embed_sort_kernel<TI>), kSortWaves * kSortMaxOwn * sizeof(int));
    hipLaunchKernelGGL((embed_sort_kernel<TI>), dim3(1u << sh.lb), dim3(1024), kSortWaves * sh.own * sizeof(int), st, (const TI*)ids, a.T, a.V, sh, k.perm, k.sid, k.start);
    int e = last_err();
    if (e) return e;
    const uint64_t pieces = (a.T + K - 1) / K;
    uint64_t pb, zb;
    if (!grid_of(pieces * cpr, &pb) || !grid_of(a.accumulate ? 0 : (uint64_t)((a.V + kZeroRows - 1) / kZeroRows) * (a.H / (VW < 4 ? VW : 4)), &zb) || pb + zb > 0x7fffffffu) return (int)hipErrorInvalidValue;
    if (pb + zb) {
      hipLaunchKernelGGL((embed_rows_kernel<T, VW>), dim3((unsigned)(pb + zb)), dim3(256), 0, st, k.perm, k.sid, k.start, (const T*)dx, G, k.part, a.H, a.V, sh, a.ld_table, a.ld_x,
                         a.scale, a.accumulate, K, (unsigned)pb);
      e = last_err();
      if (e) return e;
    }
    if (pieces > 1) {
      constexpr int JW = VW < 4 ? VW : 4;
      const unsigned cols = (unsigned)((a.H + 64 * JW - 1) / (64 * JW));
      hipLaunchKernelGGL((embed_join_kernel<JW>), dim3((unsigned)((pieces + kJoinPieces - 1) / kJoinPieces), cols < 64 ? cols : 64), dim3(64 * kJoinWaves), 0, st, k.sid, k.start, k.part, G, a.H, sh, a.ld_table,
                         a.scale, a.accumulate, K);
      e = last_err();
    }
    return e;
  });
}

}  // namespace taw
