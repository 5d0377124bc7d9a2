// Lookup of tokens in a table, times a scale, and the table's gradient.
//
//   forward    y_i = scale W[token_i]
//   backward   dW_v = scale * sum over i with token_i = v of dy_i
//
// Both are bound by memory.  The gradient needs the rows of dy by token, and in an order that does not depend on timing.  Up to 256 rows one launch
// finds and adds them, more take three:
//   1. sort   A workgroup owns the tokens with one remainder modulo the number of workgroups, reads all tokens, counts its own and those
//             before them, and lists its own rows by token, in their order (integers, read from the caches: no word from another
//             workgroup is needed).
//   2. sum    The list is cut into pieces of equal length; a piece adds rows in registers and writes the sums of the tokens that begin in it, to
//             their ends.  Tokens with more rows than a piece leave a partial sum in each.  Other workgroups write the zeros of tokens that
//             do not occur.
//   3. join   Adds the partial sums of each long token, in order.
//
// Measured (bf16): 32768 tokens of 65536 by 2048 lookup 41 us (4.3 TB/s), sort 14, sum 82 (4.9 TB/s), join 7; 65536 of 131072 by 4096, added to the
// table's other gradient, 145, 20, 193, 17; 64 tokens by 2048 2.4 us, which is a launch's own length.
#include "label_sums.h"
#include "seq_common.h"

namespace pbkd {
namespace {

constexpr int kMaxRows = 1 << 23, kMaxVocab = 1 << 22, kMaxD = 65536;
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kMostBins = 512;       // tokens a workgroup of the sort owns: their counts for each wave fill 32 KB of LDS

struct FwdArgs {
  const void *tokens, *w;
  void *y;
  long long rows, ws, ys;
  int v, d;
  float scale;
};

// A group of TPR threads takes ROWS rows, eight elements a thread at a time: their tokens, then their reads, are on their way together.
template <typename T, typename IT, int TPR, int ROWS, bool FAR>
__global__ __launch_bounds__(256) void embed_fwd_kernel(FwdArgs A) {
  const long long row = ((long long)blockIdx.x * (256 / TPR) + threadIdx.x / TPR) * ROWS;
  if (row >= A.rows) return;
  bool live[ROWS], in[ROWS];
  const T *w[ROWS];
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    in[r] = row + r < A.rows;
    const IT v = in[r] ? static_cast<const IT *>(A.tokens)[row + r] : IT(-1);
    live[r] = v >= 0 && v < A.v;
    w[r] = static_cast<const T *>(A.w) + (live[r] ? (long long)v : 0) * A.ws;
  }
  T *y = static_cast<T *>(A.y) + row * A.ys;
  for (int c = threadIdx.x % TPR * 8; c < A.d; c += TPR * 8) {
    float x[ROWS][8];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) load_n<T, 8>(w[r] + c, live[r] ? A.d - c : 0, x[r]);
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
#pragma unroll
      for (int k = 0; k < 8; ++k) x[r][k] = live[r] ? x[r][k] * A.scale : 0.f;
      store_n<T, 8, FAR>(y + r * A.ys + c, in[r] ? A.d - c : 0, x[r]);
    }
  }
}

// The sorted list's layout in the workspace.  Token v belongs to workgroup v % groups, where it has bin v / groups.
struct Plan {
  int groups, bins;          // of the sort
  int piece;                 // rows a piece of the list has
  long long pieces;
  size_t order, keys, ranges, live, partial, bytes;   // offsets
};

inline Plan make_plan(long long rows, int vocab, int d) {
  Plan p;
  p.groups = 1;
  while (p.groups < 256 && p.groups * 16 < vocab) p.groups *= 2;
  while ((long long)p.groups * kMostBins < vocab) p.groups *= 2;
  p.bins = (vocab + p.groups - 1) / p.groups;
  p.piece = rows <= 16384 ? 8 : 32;      // few rows: more pieces fill the chip; many: fewer partial sums
  p.pieces = cdiv64(rows, p.piece);
  auto up = [](size_t n) { return (n + 255) / 256 * 256; };
  p.order = 0;
  p.keys = p.order + up(rows * 4);
  p.ranges = p.keys + up(rows * 4);
  p.live = p.ranges + up((size_t)p.groups * p.bins * 8);
  p.partial = p.live + 256;
  p.bytes = p.partial + up((size_t)p.pieces * 2 * d * 4) + 256;
  return p;
}

struct Range {
  int start, count;          // of a token in the list
};

struct SortArgs {
  const void *tokens;
  int *order, *keys, *live;
  Range *ranges;
  int rows, v, groups, bins;
  int *slot;                 // null, or [v]: where a token's rows begin in the list, -1 for none
};

// The lists of 16 waves, each of which reads a sixteenth of the tokens, follow each other within a token: rows stay in order.
// A wave keeps its rows in LDS as it counts them; one that finds more than kQueue reads the tokens again.
constexpr int kQueue = 1024;        // 65536 tokens of which one makes 9 %: 61 us with 256

template <typename IT>
__global__ __launch_bounds__(kSortThreads) void embed_sort_kernel(SortArgs A) {
  __shared__ int at[kSortWaves][kMostBins];   // first counts, then where the wave's next row of this token goes
  __shared__ int rows[kSortWaves][kQueue];
  __shared__ unsigned short bins[kSortWaves][kQueue];
  __shared__ int wave_sum[kSortWaves], before_sum[kSortWaves];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, mine = blockIdx.x, mask = A.groups - 1;
  const int shift = 31 - __builtin_clz(A.groups);
  const unsigned long long below = (1ull << lane) - 1;
  const IT *tokens = static_cast<const IT *>(A.tokens);
  const int per = (A.rows + kSortThreads - 1) / kSortThreads * 64;
  const long long lo = (long long)wave * per;
  const int n = lo < A.rows ? (A.rows - lo < per ? (int)(A.rows - lo) : per) : 0;
  constexpr int U = 16;
  auto read = [&](int i, IT (&w)[U]) {
#pragma unroll
    for (int k = 0; k < U; ++k) w[k] = i + k * 64 + lane < n ? tokens[lo + i + k * 64 + lane] : IT(-1);
  };
  IT w[U], ahead[U];
  read(0, ahead);
  for (int i = lane; i < kMostBins; i += 64) at[wave][i] = 0;
  int before = 0, found = 0;
  for (int i = 0; i < n; i += 64 * U) {
#pragma unroll
    for (int k = 0; k < U; ++k) w[k] = ahead[k];
    if (i + 64 * U < n) read(i + 64 * U, ahead);
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const bool live = w[k] >= 0 && w[k] < A.v;
      const int t = live ? (int)w[k] : 0, g = t & mask;
      const bool own = live && g == mine;
      before += live && g < mine;
      const unsigned long long all = __ballot(own);
      if (!all) continue;
      if (own) {
        atomicAdd(&at[wave][t >> shift], 1);
        const int to = found + __popcll(all & below);
        if (to < kQueue) rows[wave][to] = (int)(lo + i + k * 64 + lane), bins[wave][to] = (unsigned short)(t >> shift);
      }
      found += __popcll(all);
    }
  }
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) before += __shfl_xor(before, k, 64);
  if (lane == 0) before_sum[wave] = before;
  __syncthreads();
  // a thread's bin: rows in all waves, and where they start
  int total = 0;
  if (tid < A.bins)
    for (int k = 0; k < kSortWaves; ++k) total += at[k][tid];
  int scan = total;
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) {
    const int x = __shfl_up(scan, k, 64);
    if (lane >= k) scan += x;
  }
  if (lane == 63) wave_sum[wave] = scan;
  __syncthreads();
  int first = scan - total;
  for (int k = 0; k < kSortWaves; ++k) first += before_sum[k] + (k < wave ? wave_sum[k] : 0);
  if (tid < A.bins) {
    A.ranges[mine * A.bins + tid] = Range{first, total};
    if (A.slot && (tid << shift | mine) < A.v) A.slot[tid << shift | mine] = total ? first : -1;
    for (int k = 0; k < kSortWaves; ++k) {
      const int x = at[k][tid];
      at[k][tid] = first;
      first += x;
    }
  }
  if (mine == A.groups - 1 && tid == kSortThreads - 1) *A.live = first;   // bins behind the last are empty: the end of all
  __syncthreads();
  // Lanes with the same bin find each other and take their places in the order of the lanes: bin by bin where there are few, which is
  // how frequent tokens come, otherwise bit by bit.
  const int bits = A.bins > 1 ? 32 - __builtin_clz(A.bins - 1) : 0;
  auto place = [&](bool own, int bin, int row) {
    const unsigned long long all = __ballot(own);
    unsigned long long todo = all, same = 0;
#pragma unroll 1
    for (int k = 0; k < 4 && todo; ++k) {
      const int b = __builtin_amdgcn_readlane(bin, __builtin_ctzll(todo));
      const unsigned long long these = __ballot(own && bin == b);
      if (bin == b) same = these;
      todo &= ~these;
    }
    if (todo) {
      same = all;
#pragma unroll 1
      for (int b = 0; b < bits; ++b) {
        const unsigned long long ones = __ballot(bin >> b & 1);
        same &= bin >> b & 1 ? ones : ~ones;
      }
    }
    int to = 0;
    if (own) to = at[wave][bin] + __popcll(same & below);
    __builtin_amdgcn_wave_barrier();             // all lanes have read their place
    if (own) {
      if (!(same & below)) at[wave][bin] += __popcll(same);
      A.order[to] = row;
      A.keys[to] = bin << shift | mine;
    }
    __builtin_amdgcn_wave_barrier();
  };
  if (found <= kQueue) {
    for (int i = 0; i < found; i += 64) {
      const bool own = i + lane < found;
      place(own, own ? bins[wave][i + lane] : 0, own ? rows[wave][i + lane] : 0);
    }
    return;
  }
  for (int i = 0; i < n; i += 64 * U) {
    read(i, w);
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const bool live = w[k] >= 0 && w[k] < A.v;
      const int t = live ? (int)w[k] : 0;
      const bool own = live && (t & mask) == mine;
      if (__ballot(own)) place(own, t >> shift, (int)(lo + i + k * 64 + lane));
    }
  }
}

struct SumArgs {
  const int *order, *keys, *live;
  const Range *ranges;
  const void *dy;
  void *dw;
  float *partial;
  long long rows, dys, dws, sum_blocks;
  int v, d, groups, bins, piece, accumulate;
  float scale;
  // LABELS (label_sums.h): of the rows; what each sum is added to; the scale's place
  const float *weights, *base, *scale_at;
  const int *slot;
  long long base_ld;
};

// slot: of the token in base
template <typename T, bool FAR, bool LABELS = false>
__device__ __forceinline__ void put_row(const SumArgs &A, int key, long long slot, int c, const float (&acc)[8]) {
  T *p = static_cast<T *>(A.dw) + key * A.dws + c;
  float x[8] = {};
  if constexpr (LABELS) {
    load_n<float, 8>(A.base + slot * A.base_ld + c, A.d - c, x);
    const float scale = *A.scale_at;
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = (x[k] + acc[k]) * scale;
    store_n<T, 8>(p, A.d - c, x);
    return;
  }
  if (A.accumulate) load_n<T, 8, FAR>(p, A.d - c, x);
#pragma unroll
  for (int k = 0; k < 8; ++k) x[k] = A.accumulate ? x[k] + acc[k] * A.scale : acc[k] * A.scale;
  store_n<T, 8, FAR>(p, A.d - c, x);
}

constexpr int kZeroRows = 16;        // rows of the table that a workgroup looks after for zeros

__device__ __forceinline__ Range range_of(const SumArgs &A, int key) {
  const int shift = 31 - __builtin_clz(A.groups);
  return A.ranges[(key & (A.groups - 1)) * A.bins + (key >> shift)];
}

// A piece takes the tokens that begin in it, to their ends: up to another piece's length behind its own.  Tokens with more rows than a
// piece are cut where the pieces are, and leave partial sums: slot 0 of a piece is the token that began before it, slot 1 the one that goes on.
template <typename T, int TPR, bool FAR, bool LABELS>
__global__ __launch_bounds__(256) void embed_sum_kernel(SumArgs A) {
  const int sub = threadIdx.x / TPR, c = (blockIdx.y * TPR + threadIdx.x % TPR) * 8;
  if (blockIdx.x >= A.sum_blocks) {
    __shared__ int counts[kZeroRows];
    const int v0 = (int)(blockIdx.x - A.sum_blocks) * kZeroRows;
    if (threadIdx.x < kZeroRows) counts[threadIdx.x] = v0 + (int)threadIdx.x < A.v ? range_of(A, v0 + threadIdx.x).count : 1;
    __syncthreads();
    if (c >= A.d) return;
    for (int k = sub; k < kZeroRows; k += 256 / TPR) {
      if (counts[k]) continue;
      const float zero[8] = {};
      store_n<T, 8, FAR>(static_cast<T *>(A.dw) + (v0 + k) * A.dws + c, A.d - c, zero);
    }
    return;
  }
  const int live = *A.live, piece = A.piece;
  const long long p = (long long)blockIdx.x * (256 / TPR) + sub, first = p * piece;
  if (first >= live || c >= A.d) return;
  const int *keys = A.keys + first, *order = A.order + first;
  const int left = live - first <= piece ? (int)(live - first) : piece + 1;
  int n = left < piece ? left : piece, i = 0;
  bool from_before = first > 0 && keys[-1] == keys[0], goes_on = n < left && keys[n] == keys[n - 1];
  if (from_before) {
    const Range r = range_of(A, keys[0]);
    if (r.count <= piece) {          // the piece before takes it
      i = (int)(r.start + r.count - first);
      if (i >= n) return;
      from_before = false;
    }
  }
  if (goes_on) {
    const Range r = range_of(A, keys[n - 1]);
    if (r.count <= piece) n = (int)(r.start + r.count - first), goes_on = false;
  }
  float acc[8] = {};
  bool head = true;                  // the sum is of the piece's first token
  int begin = i;                     // where the sum's token begins, if it does in this piece
  constexpr int U = 8;
  const T *dy = static_cast<const T *>(A.dy);
  for (; i < n; i += U) {
    typename VecOf<T, 8>::type x[U];
    int key[U + 1];
#pragma unroll
    for (int k = 0; k <= U; ++k) key[k] = keys[i + k < n ? i + k : n - 1];
    float weight[U];
    if constexpr (LABELS) {
#pragma unroll
      for (int k = 0; k < U; ++k) weight[k] = A.weights[order[i + k < n ? i + k : n - 1]];
    }
    if (c + 8 <= A.d) {
#pragma unroll
      for (int k = 0; k < U; ++k) x[k] = far_load<FAR, T, 8>(dy + order[i + k < n ? i + k : n - 1] * A.dys + c);
    } else {
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const T *row = dy + order[i + k < n ? i + k : n - 1] * A.dys + c;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[k][e] = c + e < A.d ? row[e] : T(0.f);
      }
    }
#pragma unroll
    for (int k = 0; k < U; ++k) {
      if (i + k >= n) break;
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] += LABELS ? weight[k] * static_cast<float>(x[k][e]) : static_cast<float>(x[k][e]);
      const bool last = i + k == n - 1;
      if (!last && key[k + 1] == key[k]) continue;
      const bool open_front = head && from_before, open_back = last && goes_on;
      if (open_front || open_back) store_n<float, 8>(A.partial + (p * 2 + (open_front ? 0 : 1)) * A.d + c, A.d - c, acc);
      else put_row<T, FAR, LABELS>(A, key[k], first + begin, c, acc);
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] = 0.f;
      head = false;
      begin = i + k + 1;
    }
  }
}

constexpr int kJoinPieces = 4;       // pieces a workgroup looks at for tokens that go on
constexpr int kJoinWaves = 8;

// A wave adds every eighth partial sum of a token, then the eight are added in order.
template <typename T, bool LABELS>
__global__ __launch_bounds__(64 * kJoinWaves) void embed_join_kernel(SumArgs A, long long pieces) {
  __shared__ float part[kJoinWaves][64][9];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, c = (blockIdx.y * 64 + lane) * 8;
  const int live = *A.live, piece = A.piece;
  // lane k looks at piece k: does a long token begin in it and go on?
  const long long mine = (long long)blockIdx.x * kJoinPieces + lane, end = (mine + 1) * piece;
  int key = 0;
  Range r{0, 0};
  if (lane < kJoinPieces && mine < pieces && end < live) key = A.keys[end - 1], r = range_of(A, key);
  const bool head = r.count > piece && r.start >= end - piece && r.start + (long long)r.count > end;
  unsigned long long heads = __ballot(head);
  while (heads) {
    const int k = __builtin_ctzll(heads);
    heads &= heads - 1;
    const int v = __shfl(key, k, 64), from = __shfl(r.start, k, 64);
    const long long p = (long long)blockIdx.x * kJoinPieces + k, last = ((long long)from + __shfl(r.count, k, 64) - 1) / piece;   // the piece that it ends in
    float acc[8] = {};
    if (c < A.d) {
      constexpr int U = 4;
      for (long long q = p + wave; q <= last; q += kJoinWaves * U) {
        float x[U][8];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const long long r = q + u * kJoinWaves;
          load_n<float, 8>(A.partial + (r * 2 + (r == p ? 1 : 0)) * A.d + c, r <= last ? A.d - c : 0, x[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int e = 0; e < 8; ++e) acc[e] += x[u][e];
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) part[wave][lane][e] = acc[e];
    __syncthreads();
    if (wave == 0 && c < A.d) {
#pragma unroll
      for (int w = 1; w < kJoinWaves; ++w)
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] += part[w][lane][e];
      put_row<T, false, LABELS>(A, v, from, c, acc);
    }
    __syncthreads();
  }
}

// Few rows, in one launch: a workgroup for each row and column tile looks for its token among all of them; the first row of a token adds all of its
// rows.  Other workgroups write the zeros.  Measured (bf16): 256 tokens of 30000 by 1024 10.6 us, in three launches 21; 256 times the same token by 8192, the
// worst there is, 23 us, in three launches 14.
constexpr int kFewRows = 256;

template <typename T, typename IT>
__global__ __launch_bounds__(256) void embed_few_kernel(SumArgs A, const IT *tokens) {
  __shared__ int list[kFewRows], before[4];
  __shared__ int there[kZeroRows];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, rows = (int)A.rows, c = (blockIdx.y * 256 + tid) * 8;
  const IT w = tid < rows ? tokens[tid] : IT(-1);
  const int token = w >= 0 && w < A.v ? (int)w : -1;
  if (blockIdx.x >= rows) {
    const int v0 = (int)(blockIdx.x - rows) * kZeroRows;
    if (tid < kZeroRows) there[tid] = v0 + tid >= A.v;
    __syncthreads();
    if (token >= v0 && token < v0 + kZeroRows) there[token - v0] = 1;
    __syncthreads();
    if (c >= A.d) return;
    for (int k = 0; k < kZeroRows; ++k) {
      const float zero[8] = {};
      if (!there[k]) store_n<T, 8>(static_cast<T *>(A.dw) + (v0 + k) * A.dws + c, A.d - c, zero);
    }
    return;
  }
  const int row = blockIdx.x;
  const IT x = tokens[row];
  if (!(x >= 0 && x < A.v)) return;
  const bool same = token == (int)x;
  const unsigned long long all = __ballot(same);
  if (lane == 0) before[wave] = __popcll(all);
  __syncthreads();
  int at = __popcll(all & ((1ull << lane) - 1)), n = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (k < wave) at += before[k];
    n += before[k];
  }
  if (same) list[at] = tid;
  __syncthreads();
  if (list[0] != row || c >= A.d) return;
  float acc[8] = {};
  constexpr int U = 16;
  const T *dy = static_cast<const T *>(A.dy);
  for (int i = 0; i < n; i += U) {
    typename VecOf<T, 8>::type y[U];
    if (c + 8 <= A.d) {
#pragma unroll
      for (int k = 0; k < U; ++k) y[k] = far_load<false, T, 8>(dy + list[i + k < n ? i + k : n - 1] * A.dys + c);
    } else {
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const T *from = dy + list[i + k < n ? i + k : n - 1] * A.dys + c;
#pragma unroll
        for (int e = 0; e < 8; ++e) y[k][e] = c + e < A.d ? from[e] : T(0.f);
      }
    }
#pragma unroll
    for (int k = 0; k < U; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] += i + k < n ? static_cast<float>(y[k][e]) : 0.f;
  }
  put_row<T, false>(A, (int)x, 0, c, acc);
}

// Sums by label of up to kFewLabels rows, in one launch: a workgroup for each row and 512 columns; the first row of a label adds all of its rows, each wave every eighth.
constexpr int kLabelWaves = 8;

template <typename T, typename IT>
__global__ __launch_bounds__(64 * kLabelWaves) void label_few_kernel(SumArgs A, const IT *labels) {
  constexpr int W = kLabelWaves, STEPS = kFewLabels / (64 * W), U = 8;
  __shared__ int list[kFewLabels], count[W];
  __shared__ float part[W][64][9];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, rows = (int)A.rows, row = blockIdx.x, c = (blockIdx.y * 64 + lane) * 8;
  const IT x = labels[row];
  if (!(x >= 0 && x < A.v) || A.slot[x] != row) return;
  // a wave looks through its share of the labels, from this row's on
  const int steps = (rows - row + 64 * W - 1) / (64 * W), from = row + wave * steps * 64;
  unsigned long long same[STEPS];
  int mine = 0;
#pragma unroll
  for (int k = 0; k < STEPS; ++k) {
    const int i = from + k * 64 + lane;
    same[k] = __ballot(k < steps && i < rows && labels[i < rows ? i : rows - 1] == x);
    mine += __popcll(same[k]);
  }
  if (lane == 0) count[wave] = mine;
  __syncthreads();
  int at = 0, n = 0;
#pragma unroll
  for (int k = 0; k < W; ++k) {
    if (k < wave) at += count[k];
    n += count[k];
  }
#pragma unroll
  for (int k = 0; k < STEPS; ++k) {
    if (same[k] >> lane & 1) list[at + __popcll(same[k] & ((1ull << lane) - 1))] = from + k * 64 + lane;
    at += __popcll(same[k]);
  }
  __syncthreads();
  float acc[8] = {};
  const T *h = static_cast<const T *>(A.dy);
  for (int i = wave; i < n && c < A.d; i += W * U) {
    typename VecOf<T, 8>::type y[U];
    float weight[U];
#pragma unroll
    for (int k = 0; k < U; ++k) weight[k] = A.weights[list[i + W * k < n ? i + W * k : n - 1]];
    if (c + 8 <= A.d) {
#pragma unroll
      for (int k = 0; k < U; ++k) y[k] = far_load<false, T, 8>(h + list[i + W * k < n ? i + W * k : n - 1] * A.dys + c);
    } else {
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const T *r = h + list[i + W * k < n ? i + W * k : n - 1] * A.dys + c;
#pragma unroll
        for (int e = 0; e < 8; ++e) y[k][e] = c + e < A.d ? r[e] : T(0.f);
      }
    }
#pragma unroll
    for (int k = 0; k < U; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] += i + W * k < n ? weight[k] * static_cast<float>(y[k][e]) : 0.f;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) part[wave][lane][e] = acc[e];
  __syncthreads();
  if (wave || c >= A.d) return;
  const int most = n < W ? n : W;
  for (int k = 1; k < most; ++k)
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] += part[k][lane][e];
  put_row<T, false, true>(A, (int)x, row, c, acc);
}

inline int row_threads(int d) {
  int t = 8;
  while (t < 256 && t * 8 < d) t *= 2;
  return t;
}

template <typename T, typename IT>
hipError_t launch_fwd(const FwdArgs &A, hipStream_t st) {
  const int tpr = row_threads(A.d);
  const int groups = 256 / tpr;
  const bool many = cdiv64(A.rows, groups) >= 8192;      // four rows a group still fill the chip
  const bool far = many && (double)A.rows * A.d * sizeof(T) > kLastLevelCache;
  const unsigned grid = (unsigned)cdiv64(A.rows, groups * (many ? 4 : 1));
#define FWD(N)                                                                      \
  case N:                                                                           \
    if (far) embed_fwd_kernel<T, IT, N, 4, true><<<grid, 256, 0, st>>>(A);          \
    else if (many) embed_fwd_kernel<T, IT, N, 4, false><<<grid, 256, 0, st>>>(A);   \
    else embed_fwd_kernel<T, IT, N, 1, false><<<grid, 256, 0, st>>>(A);             \
    break;
  switch (tpr) { FWD(8) FWD(16) FWD(32) FWD(64) FWD(128) FWD(256) }
#undef FWD
  return hipGetLastError();
}

template <typename T, bool LABELS = false>
hipError_t launch_sum(SumArgs A, const Plan &p, hipStream_t st) {
  const int tpr = row_threads(A.d);
  A.sum_blocks = cdiv64(p.pieces, 256 / tpr);
  const long long zero_blocks = A.accumulate ? 0 : cdiv64(A.v, kZeroRows);
  const dim3 grid((unsigned)(A.sum_blocks + zero_blocks), (A.d + tpr * 8 - 1) / (tpr * 8));
  const bool far = ((double)A.rows + (A.accumulate ? 0 : A.v)) * A.d * sizeof(T) > kLastLevelCache;
#define SUM(N)                                                                  \
  case N:                                                                       \
    if (far) embed_sum_kernel<T, N, true, LABELS><<<grid, 256, 0, st>>>(A);     \
    else embed_sum_kernel<T, N, false, LABELS><<<grid, 256, 0, st>>>(A);        \
    break;
  switch (tpr) { SUM(8) SUM(16) SUM(32) SUM(64) SUM(128) SUM(256) }
#undef SUM
  if (const hipError_t e = hipGetLastError()) return e;
  if (p.pieces > 1) embed_join_kernel<T, LABELS><<<dim3((unsigned)cdiv64(p.pieces, kJoinPieces), (A.d + 511) / 512), 64 * kJoinWaves, 0, st>>>(A, p.pieces);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_few(const SumArgs &A, const void *tokens, bool wide, hipStream_t st) {
  const dim3 grid((unsigned)(A.rows + (A.accumulate ? 0 : cdiv64(A.v, kZeroRows))), (A.d + 2047) / 2048);
  if (wide) embed_few_kernel<T, long long><<<grid, 256, 0, st>>>(A, static_cast<const long long *>(tokens));
  else embed_few_kernel<T, int><<<grid, 256, 0, st>>>(A, static_cast<const int *>(tokens));
  return hipGetLastError();
}

inline bool misaligned(const void *p, int size) { return (reinterpret_cast<uintptr_t>(p) & (size - 1)) != 0; }

pbkd_status check_embed(long long rows, int vocab, int d, int dtype, int index_dtype) {
  if (rows < 0 || vocab < 1 || d < 1) return set_error(PBKD_ESHAPE, "embed: %lld tokens, a table of %d rows of %d", rows, vocab, d);
  if (rows > kMaxRows || vocab > kMaxVocab || d > kMaxD)
    return set_error(PBKD_EUNSUPPORTED, "embed: %lld tokens, a table of %d rows of %d, at most %d of %d", rows, vocab, d, kMaxVocab, kMaxD);
  if (dtype != PBKD_F32 && dtype != PBKD_BF16 && dtype != PBKD_F16) return set_error(PBKD_EINVAL, "embed: dtype %d", dtype);
  if (index_dtype != PBKD_I32 && index_dtype != PBKD_I64) return set_error(PBKD_EINVAL, "embed: index_dtype %d", index_dtype);
  return PBKD_OK;
}

}  // namespace

size_t label_sums_bytes(int n, int vocab, int d) { return n <= kFewLabels ? 0 : make_plan(n, vocab, d).bytes; }

hipError_t launch_label_sort(const LabelSums &q, char *workspace, hipStream_t st) {
  const Plan p = make_plan(q.n, q.vocab, q.d);
  const SortArgs S{q.labels, reinterpret_cast<int *>(workspace + p.order), reinterpret_cast<int *>(workspace + p.keys), reinterpret_cast<int *>(workspace + p.live),
                   reinterpret_cast<Range *>(workspace + p.ranges), q.n, q.vocab, p.groups, p.bins, q.slot};
  if (q.wide) embed_sort_kernel<long long><<<p.groups, kSortThreads, 0, st>>>(S);
  else embed_sort_kernel<int><<<p.groups, kSortThreads, 0, st>>>(S);
  return hipGetLastError();
}

hipError_t launch_label_sums(const LabelSums &q, char *workspace, hipStream_t st) {
  const Plan p = make_plan(q.n, q.vocab, q.d);
  // as with a gradient that is added to another, no zeros are written
  const SumArgs A{reinterpret_cast<int *>(workspace + p.order), reinterpret_cast<int *>(workspace + p.keys), reinterpret_cast<int *>(workspace + p.live),
                  reinterpret_cast<Range *>(workspace + p.ranges), q.rows, q.out, reinterpret_cast<float *>(workspace + p.partial), q.n, q.stride, q.out_stride, 0,
                  q.vocab, q.d, p.groups, p.bins, p.piece, 1, 1.f, q.weights, q.base, q.scale, q.slot, q.base_ld};
  if (q.n > kFewLabels) return q.dtype == PBKD_BF16 ? launch_sum<bf16, true>(A, p, st) : launch_sum<f16, true>(A, p, st);
  const dim3 grid(q.n, (q.d + 511) / 512);
  const int *narrow = static_cast<const int *>(q.labels);
  const long long *wide = static_cast<const long long *>(q.labels);
  if (q.dtype == PBKD_BF16) {
    if (q.wide) label_few_kernel<bf16><<<grid, 64 * kLabelWaves, 0, st>>>(A, wide);
    else label_few_kernel<bf16><<<grid, 64 * kLabelWaves, 0, st>>>(A, narrow);
  } else {
    if (q.wide) label_few_kernel<f16><<<grid, 64 * kLabelWaves, 0, st>>>(A, wide);
    else label_few_kernel<f16><<<grid, 64 * kLabelWaves, 0, st>>>(A, narrow);
  }
  return hipGetLastError();
}

}  // namespace pbkd

using namespace pbkd;

extern "C" {

pbkd_status pbkd_embed_forward(const pbkd_embed_desc *q, void *hip_stream) {
  if (!q) return set_error(PBKD_EINVAL, "embed: null descriptor");
  if (const pbkd_status s = check_embed(q->rows, q->vocab, q->d, q->dtype, q->index_dtype)) return s;
  if (q->rows == 0) return PBKD_OK;
  if (!q->tokens_dev || !q->weight_dev || !q->y_dev) return set_error(PBKD_EINVAL, "embed: null tensor");
  const int size = q->dtype == PBKD_F32 ? 4 : 2;
  if (misaligned(q->tokens_dev, q->index_dtype == PBKD_I64 ? 8 : 4) || misaligned(q->weight_dev, size) || misaligned(q->y_dev, size))
    return set_error(PBKD_EINVAL, "embed: a tensor is not aligned to its elements");
  if (q->weight_stride < 0) return set_error(PBKD_EINVAL, "embed: negative stride");
  if (q->rows > 1 && q->y_stride < q->d) return set_error(PBKD_ESHAPE, "embed: rows of y overlap");
  FwdArgs A{q->tokens_dev, q->weight_dev, q->y_dev, q->rows, q->weight_stride, q->y_stride, q->vocab, q->d, q->scale};
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  const bool wide = q->index_dtype == PBKD_I64;
  switch (q->dtype) {
    case PBKD_F32: SEQ_HIPCHK((wide ? launch_fwd<float, long long>(A, st) : launch_fwd<float, int>(A, st))); break;
    case PBKD_BF16: SEQ_HIPCHK((wide ? launch_fwd<bf16, long long>(A, st) : launch_fwd<bf16, int>(A, st))); break;
    default: SEQ_HIPCHK((wide ? launch_fwd<f16, long long>(A, st) : launch_fwd<f16, int>(A, st))); break;
  }
  return PBKD_OK;
}

size_t pbkd_embed_workspace_bytes(long long rows, int vocab, int d) {
  if (rows < 0 || vocab < 1 || d < 1 || rows > kMaxRows || vocab > kMaxVocab || d > kMaxD) return 0;
  return make_plan(rows, vocab, d).bytes;
}

pbkd_status pbkd_embed_backward(const pbkd_embed_grad_desc *q, void *hip_stream) {
  if (!q) return set_error(PBKD_EINVAL, "embed: null descriptor");
  if (const pbkd_status s = check_embed(q->rows, q->vocab, q->d, q->dtype, q->index_dtype)) return s;
  if (!q->dweight_dev || (q->rows && (!q->tokens_dev || !q->dy_dev))) return set_error(PBKD_EINVAL, "embed: null tensor");
  const int size = q->dtype == PBKD_F32 ? 4 : 2;
  if (misaligned(q->tokens_dev, q->index_dtype == PBKD_I64 ? 8 : 4) || misaligned(q->dweight_dev, size) || misaligned(q->dy_dev, size))
    return set_error(PBKD_EINVAL, "embed: a tensor is not aligned to its elements");
  if (q->dy_stride < 0) return set_error(PBKD_EINVAL, "embed: negative stride");
  if (q->vocab > 1 && q->dweight_stride < q->d) return set_error(PBKD_ESHAPE, "embed: rows of dweight overlap");
  if (!q->workspace_dev || misaligned(q->workspace_dev, 256)) return set_error(PBKD_ENOMEM, "embed: the workspace must be 256-byte aligned");
  const Plan p = make_plan(q->rows, q->vocab, q->d);
  if (q->workspace_bytes < p.bytes) return set_error(PBKD_ENOMEM, "embed: workspace of %zu bytes is smaller than the %zu needed", q->workspace_bytes, p.bytes);
  if (q->rows == 0 && q->accumulate) return PBKD_OK;
  char *ws = static_cast<char *>(q->workspace_dev);
  int *order = reinterpret_cast<int *>(ws + p.order), *keys = reinterpret_cast<int *>(ws + p.keys), *live = reinterpret_cast<int *>(ws + p.live);
  Range *ranges = reinterpret_cast<Range *>(ws + p.ranges);
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  const SumArgs A{order, keys, live, ranges, q->dy_dev, q->dweight_dev, reinterpret_cast<float *>(ws + p.partial), q->rows, q->dy_stride, q->dweight_stride, 0,
                  q->vocab, q->d, p.groups, p.bins, p.piece, q->accumulate != 0, q->scale, nullptr, nullptr, nullptr, nullptr, 0};
  if (q->rows <= kFewRows) {
    const bool wide = q->index_dtype == PBKD_I64;
    switch (q->dtype) {
      case PBKD_F32: SEQ_HIPCHK(launch_few<float>(A, q->tokens_dev, wide, st)); break;
      case PBKD_BF16: SEQ_HIPCHK(launch_few<bf16>(A, q->tokens_dev, wide, st)); break;
      default: SEQ_HIPCHK(launch_few<f16>(A, q->tokens_dev, wide, st)); break;
    }
    return PBKD_OK;
  }
  const SortArgs S{q->tokens_dev, order, keys, live, ranges, (int)q->rows, q->vocab, p.groups, p.bins, nullptr};
  if (q->index_dtype == PBKD_I64) embed_sort_kernel<long long><<<p.groups, kSortThreads, 0, st>>>(S);
  else embed_sort_kernel<int><<<p.groups, kSortThreads, 0, st>>>(S);
  SEQ_HIPCHK(hipGetLastError());
  switch (q->dtype) {
    case PBKD_F32: SEQ_HIPCHK(launch_sum<float>(A, p, st)); break;
    case PBKD_BF16: SEQ_HIPCHK(launch_sum<bf16>(A, p, st)); break;
    default: SEQ_HIPCHK(launch_sum<f16>(A, p, st)); break;
  }
  return PBKD_OK;
}

}  // extern "C"
