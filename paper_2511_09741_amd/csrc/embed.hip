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
                                                        int64_t ld_x, float scale, uint64_t block0) {
  const unsigned cpr = (unsigned)(H / VW);
  const uint64_t idx = (block0 + blockIdx.x) * 256 + threadIdx.x;
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
// more than 2 K rows whatever the ids are, and the result does not depend on scheduling.  Every row of dx is added once, but the rows at a piece's start
// that the piece before has summed are loaded again and passed over: counted, 5% more loads at 32768 tokens of 4096 and at 65536 of 2048 with ids as text
// has them, 2% at 4503 of 1024 with padding; 23 to 39% where every id has 30 to 50 tokens and a piece 64.

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

// A workgroup goes through all the tokens to count its own ids by wavefront (each has a contiguous run of tokens) and the tokens of the workgroups
// before it, which is where its part of the sorted sequence starts; then it places its own, which the wavefronts have listed in LDS (one that found
// more than kSortList goes through its run again).  No workgroup waits for another, nothing is cleared beforehand.  The ids are read from L2 (256 times
// 128 KiB at 32768 tokens).  So the work is tokens times workgroups, which beyond 2^18 ids become more than 256.  Rows of 8 added to a shard, whole calls, us,
// ids evenly spread: 32000 ids, 16384 tokens 19, 65536 30, 262144 91, 10^6 267 (as text has them 642: the workgroup of the most frequent id); 65536
// tokens, 2^18 ids 31, 2^20 67, 2^22 207, 2^24 760.
// perm: token at a sorted place; sid: its id (0 and -1 behind the tokens that name a row); start[place_of(v)], start[own nb]: where the tokens of v start,
// and how many name a row.
constexpr int kSortList = 1024;               // 16384 tokens of 2048, half of them one id: the sort takes 15 us, 18 with 512, where a run goes through its ids twice
constexpr int kRunBits = 20;                   // T <= 2^24: a run has at most 2^20 tokens, and an id is one of 2^10 of its workgroup
template <typename TI>
__global__ void __launch_bounds__(1024) embed_sort_kernel(const TI* __restrict__ ids, int T_, int V, SortShape sh, int* __restrict__ perm, int* __restrict__ sid,
                                                          int* __restrict__ start) {
  extern __shared__ int cnt[];                 // [kSortWaves][own]
  __shared__ int list[kSortWaves][kSortList], wsum[kSortWaves], lsum[kSortWaves], placed;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, R = sh.own, w0 = blockIdx.x;
  for (int i = threadIdx.x; i < kSortWaves * R; i += 1024) cnt[i] = 0;
  __syncthreads();
  const int run = ((T_ + kSortWaves - 1) / kSortWaves + 63) / 64 * 64;
  const int t0 = wave * run, t1 = t0 + run < T_ ? t0 + run : T_;
  int* mycnt = cnt + wave * R;
  int less = 0, found = 0;
  constexpr int U = 16;
  const auto load_ids = [&](int t, int* v) {     // all the loads first, whatever lies behind the run
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int at = t + 64 * k + lane;
      v[k] = row_id(ids, at < t1 ? at : t1 - 1, V);
      if (at >= t1) v[k] = -1;
    }
  };
  for (int t = t0; t < t1; t += 64 * U) {
    int v[U];
    load_ids(t, v);
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int g = v[k] < 0 ? 0x7fffffff : sh.group_of(v[k]);
      less += g < w0;
      const unsigned long long mine = __ballot(g == w0);
      if (!mine) continue;
      if (g == w0) {
        const int r = v[k] >> sh.lb, at = found + __popcll(mine & ((1ull << lane) - 1));
        atomicAdd(&mycnt[r], 1);
        if (at < kSortList) list[wave][at] = (r << kRunBits) | (t - t0 + 64 * k + lane);
      }
      found += __popcll(mine);
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
    if (r == R - 1) placed = off;
  }
  __syncthreads();
  if (w0 == (int)gridDim.x - 1) {              // behind the last of all
    if (threadIdx.x == 0) start[w0 * R + R] = placed;
    for (int i = placed + threadIdx.x; i < T_; i += 1024) {
      perm[i] = 0;
      sid[i] = -1;
    }
  }
  // places 64 tokens of the run, in order: one turn for each different id among them
  auto place = [&](bool mine, int own, int token) {
    unsigned long long left = __ballot(mine);
    while (left) {
      const int f = __builtin_ctzll(left);
      const int id = __builtin_amdgcn_readlane(own, f);
      const unsigned long long same = __ballot(mine && own == id);
      const int base = mycnt[id];
      if (mine && own == id) {
        const int pos = base + __popcll(same & ((1ull << lane) - 1));
        perm[pos] = token;
        sid[pos] = (id << sh.lb) | ((w0 - id) & ((1 << sh.lb) - 1));
      }
      if (lane == f) mycnt[id] = base + __popcll(same);
      left &= ~same;
    }
  };
  if (found <= kSortList) {
    for (int i = 0; i < found; i += 64) {
      const int e = i + lane < found ? list[wave][i + lane] : 0;
      place(i + lane < found, e >> kRunBits, t0 + (e & ((1 << kRunBits) - 1)));
    }
  } else {
    for (int t = t0; t < t1; t += 64 * U) {
      int v[U];
      load_ids(t, v);
#pragma unroll
      for (int k = 0; k < U; ++k) place(v[k] >= 0 && sh.group_of(v[k]) == w0, v[k] >> sh.lb, t + 64 * k + lane);
    }
  }
}

// Sums of pieces: a thread has one vector of columns of a piece.  part: [pieces][2][H]: the sum of the long id that a piece starts within (0), and of
// the one that starts in it and goes on behind it (1).  The workgroups behind those of the pieces zero the rows that no token names, a vector a
// thread (163 us for 32768 tokens of 4096; four rows a thread 173; zeroed by the sort's workgroups instead, beside its latency, 182).
// Four columns a thread, also of bf16: the sums are stored 16 bytes a lane side by side (32768 tokens of 4096 into 32000 rows: 185 us with four, 192 with
// eight).  STREAM: dx and G go past L2 (180 us; 4503 tokens of 1024, which L2 has room for: 24.8 against 23.3).
template <typename T, int VW, bool STREAM>
__global__ void __launch_bounds__(256) embed_rows_kernel(const int* __restrict__ perm, const int* __restrict__ sid, const int* __restrict__ start, const T* __restrict__ dx,
                                                         float* __restrict__ G, float* __restrict__ part, int H, SortShape sh, int64_t ld_table, int64_t ld_x,
                                                         float scale, int accumulate, int K, uint64_t piece_blocks, int V, int T_, uint64_t block0) {
  constexpr int U = 8;
  const unsigned cpr = (unsigned)(H / VW);
  typedef float fv_t __attribute__((ext_vector_type(VW), aligned(VW * 4 < 16 ? VW * 4 : 16)));
  const uint64_t block = block0 + blockIdx.x;
  if (block >= piece_blocks) {
    const uint64_t idx = (block - piece_blocks) * 256 + threadIdx.x;
    const int64_t v = (int64_t)(idx / cpr);
    if (v >= V) return;
    const int col = (int)(idx - v * cpr) * VW, at = sh.place_of((int)v);
    if (start[at] == start[at + 1]) __builtin_nontemporal_store(fv_t(0.f), reinterpret_cast<fv_t*>(G + v * ld_table + col));
    return;
  }
  const uint64_t idx = block * 256 + threadIdx.x;
  const uint64_t p = idx / cpr;
  const int col = (int)(idx - p * cpr) * VW;
  const int p0 = (int)p * K;
  if (p * K >= (uint64_t)T_) return;
  int p1 = p0 + K < T_ ? p0 + K : T_;
  int who[U], id[U];
  Vec<T, VW> r[U];
  // the first tokens are asked for before it is known which of them are this piece's, and so are their rows
  const auto tokens = [&](int q, int to) {
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int at = q + k < to ? q + k : to - 1;
      who[k] = perm[at];
      id[k] = sid[at];
    }
  };
  const auto load_rows = [&]() {
#pragma unroll
    for (int k = 0; k < U; ++k) {
      if (STREAM) r[k].load_nt(dx + (int64_t)who[k] * ld_x + col);
      else r[k].load(dx + (int64_t)who[k] * ld_x + col);
    }
  };
  tokens(p0, p1);
  int last_id = sid[p1 - 1];
  if (id[0] < 0) return;
  if (last_id < 0) {                             // behind the last of all
    p1 = start[sh.places() - 1];
    last_id = sid[p1 - 1];
  }
  load_rows();
  int from = p0, to = p1;
  bool head = false, tail = false;
  {
    const int v = sh.place_of(id[0]), w = sh.place_of(last_id), s = start[v], e = start[v + 1], s1 = start[w], e1 = start[w + 1];
    if (s < p0) {
      head = e - s > K;
      if (!head) from = e;                       // its start's piece has it whole
    }
    if (e1 > p1) {
      tail = e1 - s1 > K;
      if (!tail) to = e1;
    }
  }
  if (from >= to) return;
  fv_t acc = fv_t(0.f);
  int cur = -1;
  auto flush = [&](bool last) {
    if (head || (last && tail)) {
      *reinterpret_cast<fv_t*>(part + ((int64_t)p * 2 + (head ? 0 : 1)) * H + col) = acc;
    } else {
      float* g = G + (int64_t)cur * ld_table + col;
      fv_t o = acc * scale;
      if (accumulate) o += *reinterpret_cast<const fv_t*>(g);
      if (STREAM) __builtin_nontemporal_store(o, reinterpret_cast<fv_t*>(g));
      else *reinterpret_cast<fv_t*>(g) = o;
    }
    head = false;
  };
  for (int q = p0; q < to; q += U) {
    if (q != p0) {                               // U <= K: the first ones are there
      tokens(q, to);
      load_rows();
    }
#pragma unroll
    for (int k = 0; k < U; ++k) r[k].pin();       // all are under way before the first is used
#pragma unroll
    for (int k = 0; k < U; ++k) {
      if (q + k >= to) break;
      if (q + k < from) continue;
      if (id[k] != cur) {
        if (cur >= 0) flush(false);
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
                                                                     float* __restrict__ G, int H, SortShape sh, int64_t ld_table, float scale, int accumulate, int K, int T_) {
  typedef float fv_t __attribute__((ext_vector_type(VW)));
  __shared__ fv_t red[kJoinWaves][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  // lane i looks at piece i: the id at its end, if that starts in it, goes on behind it and is long
  const int64_t end = ((int64_t)blockIdx.x * kJoinPieces + lane + 1) * K;
  int v = 0, np = 0;
  if (lane < kJoinPieces && end < T_ && (v = sid[end - 1]) >= 0) {
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

// A few tokens: one launch, no sort.  A workgroup per token and 64 VW columns marks the tokens with the same id; if its own is the first of them it sums
// their rows: of rows with fewer than 64 vectors a wavefront takes several at a time, in `groups` of lanes, and wavefront w the places w, w + 4, ... of
// its groups in the list; then groups and wavefronts are added in order.  The first zero_blocks workgroups zero the rows that no token names.  Looking
// through the ids costs T * T / 64 loads for each column block, sorting them two launches more (few_tokens() has the line).
constexpr int kFewTokens = 2048, kZeroBlocks = 2048;
template <typename T, int VW, typename TI>
__global__ void __launch_bounds__(256) embed_few_kernel(const TI* __restrict__ ids, const T* __restrict__ dx, float* __restrict__ G, int T_, int H, int V, int64_t ld_table,
                                                        int64_t ld_x, float scale, int accumulate, int zero_blocks) {
  typedef float fv_t __attribute__((ext_vector_type(VW)));
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if ((int)blockIdx.x < zero_blocks) {
    __shared__ unsigned named[(1 << 24) / kZeroBlocks / 32 + 1];
    const int per = (V + zero_blocks - 1) / zero_blocks, v0 = blockIdx.x * per, n = V - v0 < per ? V - v0 : per;
    for (int i = threadIdx.x; i <= per / 32; i += 256) named[i] = 0;
    __syncthreads();
    for (int t = threadIdx.x; t < T_; t += 256) {
      const int r = row_id(ids, t, V) - v0;
      if (r >= 0 && r < n) atomicOr(&named[r >> 5], 1u << (r & 31));
    }
    __syncthreads();
    for (int r = wave; r < n; r += 4) {
      if ((named[r >> 5] >> (r & 31)) & 1) continue;
      float* g = G + (int64_t)(v0 + r) * ld_table;
      for (int c = lane * VW; c < H; c += 64 * VW) __builtin_nontemporal_store(fv_t(0.f), reinterpret_cast<fv_t*>(g + c));
    }
    return;
  }
  __shared__ unsigned long long mask[kFewTokens / 64];
  __shared__ int list[kFewTokens];
  __shared__ fv_t red[4][64];
  const unsigned b = blockIdx.x - zero_blocks, ncb = (unsigned)((H + 64 * VW - 1) / (64 * VW));
  const int t = (int)(b / ncb), v = row_id(ids, t, V), nb = (T_ + 63) / 64;
  if (v < 0) return;
  int id[kFewTokens / 256];                     // all are under way before the first is looked at
#pragma unroll
  for (int k = 0; k < kFewTokens / 256; ++k) {
    const int at = (k * 4 + wave) * 64 + lane;
    id[k] = row_id(ids, at < T_ ? at : 0, V);
  }
#pragma unroll
  for (int k = 0; k < kFewTokens / 256; ++k) {
    const unsigned long long same = __ballot((k * 4 + wave) * 64 + lane < T_ && id[k] == v);
    if (lane == 0) mask[k * 4 + wave] = same;
  }
  __syncthreads();
  // lane i looks at the 64 tokens i
  const unsigned long long mine = lane < nb ? mask[lane] : 0;
  const unsigned long long before = lane < (t >> 6) ? mine : lane == (t >> 6) ? mine & ((1ull << (t & 63)) - 1) : 0;
  if (__ballot(before != 0)) return;            // not the first
  int upto = __popcll(mine);
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int up = __shfl_up(upto, o, 64);
    if (lane >= o) upto += up;
  }
  const int n = __shfl(upto, 63, 64);
  if ((lane & 3) == wave) {
    int at = upto - __popcll(mine);
    for (unsigned long long left = mine; left; left &= left - 1) list[at++] = lane * 64 + __builtin_ctzll(left);
  }
  __syncthreads();
  int width = 64;                               // lanes of a group
  while (width > 1 && (width / 2) * VW >= H) width /= 2;
  const int groups = 64 / width, col = (int)(b % ncb) * 64 * VW + (lane & (width - 1)) * VW;
  fv_t acc = fv_t(0.f);
  if (col < H) {
    const int step = 4 * groups;
    int q = wave * groups + lane / width;
    const auto rows = [&](auto u) {
      constexpr int U = decltype(u)::value;
      Vec<T, VW> r[U];
#pragma unroll
      for (int k = 0; k < U; ++k) r[k].load(dx + (int64_t)list[q + k * step < n ? q + k * step : q] * ld_x + col);
#pragma unroll
      for (int k = 0; k < U; ++k) r[k].pin();     // all are under way before the first is used
#pragma unroll
      for (int k = 0; k < U; ++k)
        if (q + k * step < n)
#pragma unroll
          for (int j = 0; j < VW; ++j) acc[j] += r[k].get(j);
      q += U * step;
    };
    while (q + 8 * step < n) rows(std::integral_constant<int, 16>{});
    while (q < n) rows(std::integral_constant<int, 4>{});      // most ids have one token or two
  }
  for (int o = width; o < 64; o <<= 1)
#pragma unroll
    for (int j = 0; j < VW; ++j) acc[j] += __shfl_xor(acc[j], o, 64);
  red[wave][lane] = acc;
  __syncthreads();
  if (wave || lane >= width || col >= H) return;
  acc = scale * (((acc + red[1][lane]) + red[2][lane]) + red[3][lane]);
  fv_t* g = reinterpret_cast<fv_t*>(G + (int64_t)v * ld_table + col);
  *g = accumulate ? *g + acc : acc;
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

static uint64_t blocks_of(uint64_t threads) { return (threads + 255) / 256; }

int launch_embed_fwd(const EmbedArgs& a, const void* ids, const void* table, void* x, hipStream_t st) {
  return by_types(a, [&](auto* t, auto* i, auto w) {
    using T = std::remove_pointer_t<decltype(t)>;
    using TI = std::remove_pointer_t<decltype(i)>;
    constexpr int VW = decltype(w)::value, U = 2;
    over_blocks(blocks_of((uint64_t)((a.T + U - 1) / U) * (a.H / VW)), kMostBlocks, [&](uint64_t block0, unsigned blocks) {
      hipLaunchKernelGGL((embed_fwd_kernel<T, VW, U, TI>), dim3(blocks), dim3(256), 0, st, (const TI*)ids, (const T*)table, (T*)x, a.T, a.H, a.V, a.ld_table, a.ld_x, a.scale,
                         block0);
    });
    return last_err();
  });
}

// Tokens of a piece: 64, or fewer where that leaves the chip fewer than 32 wavefronts a compute unit (8192 tokens of 4096 added to a shard: 75 us with 64,
// 61 with 32, 58 with 16; 4503 of 1024: 24 us with 8, 27 with 16, 33 with 32; 32768 of 4096 the same with all).
static int piece_of(int64_t T_, int64_t cpr) {
  int K = 64;
  while (K > 8 && T_ * cpr < (int64_t)K * 524288) K /= 2;
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
  w.part = (float*)take(pieces * 2 * a.H * 4);
  w.bytes = off;
  return w;
}

constexpr uint64_t kStreamBytes = (uint64_t)64 << 20;       // dx: more than the L2 caches hold

// columns of a thread of the backward
static int bwd_width_of(const EmbedArgs& a) {
  const int w = width_of(a.dtype, a.H, a.ld_table, a.ld_x);
  return w < 4 ? w : 4;
}

// Rows added to a shard of 32000, us without and with the sort, ids as text has them / a third of them one row: 512 tokens of 4096 12 / 17 and 20 / 17,
// 1024 27 / 33 and 23 / 23; 1024 of 1024 8 / 16 and 19 / 19, 2048 17 / 29 and 22 / 21; 2048 of 256 9 / 18 and 19 / 19.
static bool few_tokens(const EmbedArgs& a) { return a.T <= kFewTokens && (int64_t)a.T * a.T * ((a.H + 255) / 256) <= 1 << 22; }

size_t embed_bwd_workspace_bytes(const EmbedArgs& a) { return few_tokens(a) ? 0 : embed_work(a, piece_of(a.T, a.H / bwd_width_of(a)), nullptr).bytes; }

int launch_embed_bwd(const EmbedArgs& a, const void* ids, const void* dx, float* G, void* ws, hipStream_t st) {
  return by_types(a, [&](auto* t, auto* i, auto w) {
    using T = std::remove_pointer_t<decltype(t)>;
    using TI = std::remove_pointer_t<decltype(i)>;
    constexpr int VW = decltype(w)::value < 4 ? decltype(w)::value : 4;
    if (few_tokens(a)) {
      const int zero = a.accumulate ? 0 : a.V < kZeroBlocks ? a.V : kZeroBlocks;
      const uint64_t blocks = zero + (uint64_t)a.T * ((a.H + 64 * VW - 1) / (64 * VW));
      if (blocks > 1 << 23) return (int)hipErrorInvalidValue;      // there are fewer: few_tokens()
      hipLaunchKernelGGL((embed_few_kernel<T, VW, TI>), dim3((unsigned)blocks), dim3(256), 0, st, (const TI*)ids, (const T*)dx, G, a.T, a.H, a.V, a.ld_table, a.ld_x, a.scale,
                         a.accumulate, zero);
      return last_err();
    }
    const uint64_t cpr = a.H / VW;
    const int K = piece_of(a.T, (int64_t)cpr);
    const EmbedWork k = embed_work(a, K, ws);
    const SortShape sh = sort_shape(a.V);
    const uint64_t pieces = (a.T + K - 1) / K, blocks = blocks_of(pieces * cpr);
    const uint64_t zero = blocks_of(a.accumulate ? 0 : (uint64_t)a.V * cpr);
    TAW_SET_LDS_LIMIT_ONCE((embed_sort_kernel<TI>), kSortWaves * kSortMaxOwn * sizeof(int));
    hipLaunchKernelGGL((embed_sort_kernel<TI>), dim3(1u << sh.lb), dim3(1024), kSortWaves * sh.own * sizeof(int), st, (const TI*)ids, a.T, a.V, sh, k.perm, k.sid, k.start);
    int e = last_err();
    if (e) return e;
    const auto rows = (uint64_t)a.T * a.H * sizeof(T) > kStreamBytes ? embed_rows_kernel<T, VW, true> : embed_rows_kernel<T, VW, false>;
    over_blocks(blocks + zero, kMostBlocks, [&](uint64_t block0, unsigned n) {
      hipLaunchKernelGGL(rows, dim3(n), dim3(256), 0, st, k.perm, k.sid, k.start, (const T*)dx, G, k.part, a.H, sh, a.ld_table, a.ld_x, a.scale, a.accumulate, K, blocks, a.V, a.T,
                         block0);
    });
    e = last_err();
    if (e) return e;
    const unsigned cols = (unsigned)((a.H + 64 * VW - 1) / (64 * VW));
    hipLaunchKernelGGL((embed_join_kernel<VW>), dim3((unsigned)((pieces + kJoinPieces - 1) / kJoinPieces), cols < 64 ? cols : 64), dim3(64 * kJoinWaves), 0, st, k.sid, k.start,
                       k.part, G, a.H, sh, a.ld_table, a.scale, a.accumulate, K, a.T);
    return last_err();
  });
}

}  // namespace taw
