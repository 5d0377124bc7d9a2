// Softmax cross entropy over a large vocabulary from the activations in front of the last product, with the gradients of both.
//
//   z = h W^T,  lse_n = log sum_v exp z_nv,  loss_n = lse_n - z_{n,label},  dz_nv = g_n (exp(z_nv - lse_n) - [v = label_n]),  dh = dz W,  dW = dz^T h
//
// Bound by its products of matrices: 2 N V d operations for the losses, and 6 N V d for the gradients, because z is not kept but formed
// again, piece of the vocabulary by piece.  The first pass leaves a maximum and a sum of every tile's rows; they give lse.  In the
// second a piece's dz comes out of the product once, n by v: dh reads it along v with W as it lies, dW along n with a copy of h's other layout, by the
// transposing reads of head_gemm.h.
//
// Measured (bf16): 8192 rows by 4096 over 131072 27.8 to 28.1 ms, 1250 to 1270 TFLOP/s over the four products; 4096 by 2048 over 65536 3.82 ms, 1150; losses of 32 rows by 2048 over 65536 53 us, W at 5.4 TB/s; 500 by 515 over 1013 fp32 71 us in nine launches.
//
// dz is rounded to the operands' type, but not where a row has its label: there it is nearly the row's weight, most of both gradients, and rounding it would be
// an error of the size that rounding the gradients has anyway (against 64 bits 0.0024 instead of 0.0017).  These numbers, one a row, stay in fp32, and dz is zero there: head_finish
// adds the label's row of W to dh, and the dW of places that are labels is kept in fp32 until label_sums.h has added their rows of h.  Small calls keep all of dz in two
// terms.  dz is formed with row weights times a power of two that puts the largest between 2^13 and 2^14: fp16 keeps probabilities in steps of 2^-24 / 2^13 of it.  fp32 is kept
// in three bf16 terms.
#include <type_traits>

#include "head_gemm.h"
#include "label_sums.h"

namespace pbkd {
namespace {

using namespace head;

constexpr int kMaxRows = 1 << 21, kMaxVocab = 1 << 22, kMaxD = 65536;
// dz is kept in two terms for so few rows, whose products wait for W anyway, and for calls of up to so many products (rows x vocabulary x width), where two more terms
// take less than another launch: 1000 x 1000 x 512 bf16 43 instead of 50 us, 80 x 20000 x 512 68 instead of 66, 2000 x 8192 x 1024 285 instead of 235.
constexpr int kFewRows = 64;
constexpr double kTwoTermsUpTo = 8e8;
// From here on (rows x vocabulary x width) fp32 logits come from pairs of fp16 terms, three products instead of six of triples: 4096 x 32768 x 1024 with
// gradients 7.10 -> 6.16 ms (4.7 since dz is written once), losses alone 1.46 -> 0.93 ms (0.79 since).  Below, looking for the largest numbers costs more than it saves: 500 x 1013 x 515 73 -> 90 us.
constexpr double kPairsFrom = 1e10;
constexpr double kPieceBytes = 600e6;        // dz of a piece: with 300 MB 8192 x 131072 x 4096 27.9 instead of 27.8 ms, with 150 28.4

inline int up64(long long n) { return (int)((n + 63) / 64 * 64); }
inline long long up4(int n) { return ((long long)n + 3) / 4 * 4; }        // rows of fp32 that begin at multiples of 16 bytes

// ------------------------------------------------------------------------------------------------------ small kernels
struct RowArgs {
  const void *labels;
  const float *g;
  float *gs, *scale;       // scale: 2^-s, what results are multiplied with
  int rows, v;
};

// Row weights times 2^s, 0 where there is no label.
template <typename IT>
__global__ __launch_bounds__(1024) void head_rows_kernel(RowArgs A) {
  __shared__ float red[16];
  const int tid = threadIdx.x;
  const IT *labels = static_cast<const IT *>(A.labels);
  float top = 0.f;
  for (int i = tid; i < A.rows; i += 1024) {
    const IT w = labels[i];
    const float g = w >= 0 && w < A.v ? (A.g ? A.g[i] : 1.f) : 0.f;
    if (fabsf(g) < __builtin_inff()) top = fmaxf(top, fabsf(g));
  }
  top = wave64_max(top);
  if ((tid & 63) == 0) red[tid >> 6] = top;
  __syncthreads();
  for (int k = 0; k < 16; ++k) top = fmaxf(top, red[k]);
  int e = top > 0.f ? 14 - __builtin_amdgcn_frexp_expf(top) : 0;       // top < 2^(14 - e): dz stays below 2^15
  e = e < 100 ? e : 100;
  const float s = ldexpf(1.f, e);
  for (int i = tid; i < A.rows; i += 1024) {
    const IT w = labels[i];
    A.gs[i] = w >= 0 && w < A.v ? (A.g ? A.g[i] : 1.f) * s : 0.f;
  }
  if (tid == 0) *A.scale = ldexpf(1.f, -e);
}

struct LayArgs {
  const void *src;
  long long stride;        // elements between the source's rows
  char *rows_dst, *cols_dst;                    // null: not wanted
  long long rows_ld, rows_plane, cols_ld, cols_plane;    // bytes
  char *pairs_dst;         // of fp32: like rows_dst, in two fp16 terms of the number times scale_of(top)
  const unsigned *top;
  int top_step;            // 1: a scale for each row
  const void *labels;      // rows without a label become zeros in cols_dst; null: none do
  int wide, vocab;
  int rows, cols, cols_fill, rows_fill;         // of the source; zeros behind the ends up to *_fill
};

// slot[0 .. vocab-1] <- -1.
struct ClearArgs {
  int *slot;               // null: none
  int vocab;
};

// The two layouts that a product reads along k: rows_dst[row][..] = src[row][..] and cols_dst[col][..] = src[..][col], in planes.  Tiles of 64 x 64.
template <typename T, typename E, int PLANES>
__global__ __launch_bounds__(256) void head_lay_kernel(LayArgs A, ClearArgs C) {
  __shared__ E tile[PLANES][64][66];
  if (C.slot)
    for (int v = (blockIdx.y * gridDim.x + blockIdx.x) * 256 + threadIdx.x; v < C.vocab; v += gridDim.x * gridDim.y * 256) C.slot[v] = -1;
  const int tid = threadIdx.x, r0 = blockIdx.x * 64, c0 = blockIdx.y * 64;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int r = k * 32 + tid / 8, c = tid % 8 * 8, row = r0 + r;
    float x[8] = {};
    if (row < A.rows) load_n<T, 8>(static_cast<const T *>(A.src) + row * A.stride + c0 + c, A.cols - c0 - c, x);
    if constexpr (sizeof(T) == 4) {
      if (A.pairs_dst && row < A.rows && c0 + c < A.cols_fill) {
        const float scale = scale_of(A.top[row * A.top_step]);
        f16 y[2][8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[0][e] = static_cast<f16>(x[e] * scale), y[1][e] = static_cast<f16>(x[e] * scale - static_cast<float>(y[0][e]));
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          uintx4 w;
          __builtin_memcpy(&w, y[p], 16);
          *reinterpret_cast<uintx4 *>(A.pairs_dst + p * A.rows_plane + row * A.rows_ld + (c0 + c) * 2) = w;
        }
      }
      if (!A.rows_dst && !A.cols_dst) continue;
    }
    const bool live = row < A.rows && (!A.labels || label_of(A.labels, A.wide, A.vocab, row) >= 0);
#pragma unroll
    for (int p = 0; p < PLANES; ++p) {
      E y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = static_cast<E>(x[e]), x[e] -= static_cast<float>(y[e]);
      if (A.rows_dst && row < A.rows && c0 + c < A.cols_fill) {
        uintx4 w;
        __builtin_memcpy(&w, y, 16);
        *reinterpret_cast<uintx4 *>(A.rows_dst + p * A.rows_plane + row * A.rows_ld + (c0 + c) * 2) = w;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) tile[p][c + e][r] = live ? y[e] : static_cast<E>(0.f);
    }
  }
  if (!A.cols_dst) return;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int c = k * 32 + tid / 8, r = tid % 8 * 8;
    if (c0 + c >= A.cols || r0 + r >= A.rows_fill) continue;
#pragma unroll
    for (int p = 0; p < PLANES; ++p) {
      E y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = tile[p][c][r + e];
      uintx4 w;
      __builtin_memcpy(&w, y, 16);
      *reinterpret_cast<uintx4 *>(A.cols_dst + p * A.cols_plane + (c0 + c) * A.cols_ld + (r0 + r) * 2) = w;
    }
  }
}

// Bits of the largest finite magnitude of a matrix, or of each of its rows: as integers they compare like the numbers.  h is scaled row by row, so that no
// row has to do with another.
__global__ void head_clear_kernel(unsigned *top) {
  if (threadIdx.x == 0) *top = 0;
}

template <bool ROWS>
__global__ __launch_bounds__(256) void head_top_kernel(const float *src, long long stride, int rows, int cols, unsigned *top) {
  __shared__ float red[4];
  float most = 0.f;
  for (int r = blockIdx.x; r < rows; r += gridDim.x)
    for (int c = threadIdx.x * 8; c < cols; c += 256 * 8) {
      float x[8];
      load_n<float, 8>(src + r * stride + c, cols - c, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) most = fabsf(x[e]) < __builtin_inff() ? fmaxf(most, fabsf(x[e])) : most;
    }
  most = wave64_max(most);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = most;
  __syncthreads();
  if (threadIdx.x) return;
  const unsigned bits = __builtin_bit_cast(unsigned, fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])));
  if (ROWS) top[blockIdx.x] = bits;
  else atomicMax(top, bits);
}

// A workgroup joins a row's pairs, in an order that only their number decides.  at_place, if wanted: dz where the row has its label; slot: the first row with a label.
__global__ __launch_bounds__(256) void head_lse_kernel(const float *part, int parts, int stride, const void *labels, int wide, int vocab, const float *at_label, float *lse,
                                                       float *lse_out, float *loss, const float *g, float *at_place, int *slot) {
  __shared__ float red[2][4];
  const int n = blockIdx.x, tid = threadIdx.x, wave = tid >> 6;
  const int label = label_of(labels, wide, vocab, n);
  const float z = at_label[n], weight = at_place ? g[n] : 0.f;
  int before = 0;
  if (slot && label >= 0)
    for (int k = tid; k < n; k += 256) before |= label_of(labels, wide, vocab, k) == label;
  const float *p = part + (long long)n * stride * 2;
  float top = -__builtin_inff(), sum = 0.f;
  for (int k = tid; k < parts; k += 256) {
    const float m = p[2 * k], s = p[2 * k + 1], most = fmaxf(top, m), ref = most == -__builtin_inff() ? 0.f : most;
    sum = sum * expf(top - ref) + s * expf(m - ref);
    top = most;
  }
  const float most = wave64_max(top), ref = most == -__builtin_inff() ? 0.f : most;
  sum = wave64_sum(sum * expf(top - ref));
  if ((tid & 63) == 0) red[0][wave] = most, red[1][wave] = sum;
  if (slot) before = __syncthreads_or(before);
  else __syncthreads();
  if (tid) return;
  top = fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
  const float base = top == -__builtin_inff() ? 0.f : top;
  sum = 0.f;
  for (int k = 0; k < 4; ++k) sum += red[1][k] * expf(red[0][k] - base);
  const float x = top + logf(sum);
  lse[n] = x;
  if (lse_out) lse_out[n] = x;
  loss[n] = label >= 0 ? x - z : 0.f;
  if (!at_place) return;
  at_place[n] = label >= 0 ? weight * expm1f(z - x) : 0.f;
  if (slot && label >= 0 && !before) slot[label] = n;
}

// What dz is at the rows' labels, where that is not among the products: null, or a number for each row.
template <typename T>
struct AtLabel {
  const float *dz;
  const T *weight;
  long long stride;
  const void *labels;
  int wide, vocab;
};

// out[n][m] = scale * (sum over the splits, and the label's part): eight numbers a thread.  With many splits GROUPS threads share them, and their sums are added in order.
template <typename T, int GROUPS>
__global__ __launch_bounds__(256) void head_finish_kernel(const float *sum, int splits, int rows, int cols, const float *scale, T *out, long long stride, AtLabel<T> at) {
  constexpr int LANES = 256 / GROUPS;
  __shared__ float part[GROUPS][LANES][9];
  const int per = (cols + 7) / 8, lane = threadIdx.x % LANES, g = threadIdx.x / LANES;
  const long long i = (long long)blockIdx.x * LANES + lane, row = i / per;
  const int c = (int)(i - row * per) * 8, left = i < (long long)rows * per ? cols - c : 0;
  float x[8] = {};
  for (int k = g; k < splits; k += GROUPS) {
    float y[8];
    load_n<float, 8>(sum + ((long long)k * rows + row) * cols + c, left, y);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] += y[e];
  }
  if constexpr (GROUPS > 1) {
#pragma unroll
    for (int e = 0; e < 8; ++e) part[g][lane][e] = x[e];
    __syncthreads();
    if (g) return;
#pragma unroll
    for (int k = 1; k < GROUPS; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] += part[k][lane][e];
  }
  if (at.dz && left > 0) {
    const int label = label_of(at.labels, at.wide, at.vocab, row);
    if (label >= 0) {
      const float dz = at.dz[row];
      float y[8];
      load_n<T, 8>(at.weight + label * at.stride + c, left, y);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] += dz * y[e];
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] *= *scale;
  store_n<T, 8>(out + row * stride + c, left, x);
}

// ---------------------------------------------------------------------------------------------------------- the plan
// Tiles of a product: the largest of which there are enough for the chip's 256 compute units (with the sum over k in parts, where it
// may be), narrow ones for few rows of n.
struct Shape {
  int tm, tn;
};
constexpr Shape kShapes[6] = {{256, 256}, {128, 128}, {64, 64}, {128, 64}, {128, 32}, {128, 128}};
constexpr int kFull = 192;           // tiles that count as enough
constexpr int kShortSum = 4;         // slices of a sum that is over before the next tile's operands are there

inline long long tiles_of(int shape, long long m, long long n) { return cdiv64(m, kShapes[shape].tm) * cdiv64(n, kShapes[shape].tn); }

// slices: of the sum over k, 0 where it cannot be cut.  A part has eight slices at least.
inline int splits_of(int shape, long long m, long long n, int slices) {
  long long s = 256 / tiles_of(shape, m, n);
  s = s > slices / 8 ? slices / 8 : s;
  return s < 1 ? 1 : (int)s;
}

inline int pick_shape(long long m, long long n, int slices = 0) {
  const int narrow = n <= 32 ? 4 : n <= 64 ? 3 : 0;
  if (narrow) return tiles_of(narrow, m, n) * splits_of(narrow, m, n, slices) >= kFull ? narrow : 2;
  for (int shape = 0; shape < 2; ++shape)
    if (tiles_of(shape, m, n) * splits_of(shape, m, n, slices) >= kFull) return shape;
  return 2;
}

struct Plan {
  int d_pad, n_pad, piece, pieces, planes, dz_planes, parts, first_shape, sum_shape, splits;
  bool pack_h, pack_w, pairs, by_label;
  Planes logits, grads;
  size_t gs, scale, tops, lse, at_label, part, h, ht, w, wpairs, dz, sum, at_place, slot, base, labels, bytes;
};

bool direct(const void *p, long long stride, int d, int dtype) {
  return dtype != PBKD_F32 && d % 64 == 0 && stride % 8 == 0 && stride <= 1 << 20 && (reinterpret_cast<uintptr_t>(p) & 15) == 0;
}

// pack_*: whether the operands have to be laid out (the workspace is counted as if they had).  in_place: a gradient lies where its tensor does, which the last
// launches read where dz is not zero at the labels.
Plan make_plan(int rows, int vocab, int d, int dtype, bool gradients, bool pack_h, bool pack_w, bool in_place) {
  Plan p{};
  const bool f32 = dtype == PBKD_F32;
  p.pairs = f32 && (double)rows * vocab * d >= kPairsFrom;
  p.logits = p.pairs ? kPairs : f32 ? kTriples : kOne;         // products of planes for the logits, and for the gradients
  p.planes = f32 ? 3 : 1, p.dz_planes = f32 ? 3 : rows <= kFewRows || (double)rows * vocab * d <= kTwoTermsUpTo || in_place ? 2 : 1;
  p.grads = f32 ? kTriples : p.dz_planes == 2 ? kTwoOfB : kOne;
  p.by_label = gradients && p.dz_planes == 1;
  p.d_pad = up64(d), p.n_pad = up64(rows > 0 ? rows : 1);
  p.pack_h = pack_h, p.pack_w = pack_w;
  // A piece's tiles of 256 x 256 fill whole rounds of the chip where that leaves pieces of a sensible size: 16 rows of tiles, 16 columns.
  const double most = kPieceBytes / (gradients ? 2.0 * p.dz_planes * p.n_pad : 2.0 * p.d_pad);
  long long unit = cdiv64(rows, 256);
  unit = (unit & -unit) < 256 ? 256 / (unit & -unit) * 256 : 256;
  if (unit > most / 2) unit = 256;
  long long piece = (long long)(most / unit) * unit;
  piece = piece < 1024 ? 1024 : piece;
  const int n = (int)cdiv64(vocab, piece);
  p.piece = (int)(cdiv64(cdiv64(vocab, n), unit) * unit);
  if (vocab <= p.piece) p.piece = (int)(cdiv64(vocab, 256) * 256);
  if (!gradients && !pack_w) p.piece = vocab;
  p.pieces = (int)cdiv64(vocab, p.piece);
  p.first_shape = pick_shape(p.piece, rows);
  // dh: few tiles, a long sum
  const int slices = up64(p.piece < vocab ? p.piece : vocab) / 64 * p.grads.terms;
  p.sum_shape = pick_shape(d, rows, slices);
  p.splits = splits_of(p.sum_shape, d, rows, slices);
  p.parts = (int)cdiv64(vocab, kShapes[p.first_shape].tm) + p.pieces;
  size_t at = 0;
  auto put = [&](size_t n) {
    const size_t here = at;
    at += (n + 255) / 256 * 256;
    return here;
  };
  const size_t R = rows, e = 2 * p.planes;
  p.gs = put(R * 4), p.scale = put(4), p.tops = put(p.pairs ? (R + 1) * 4 : 0), p.lse = put(R * 4), p.at_label = put(R * 4);
  p.part = put(R * p.parts * 8);
  // pairs: h as pairs only, W both ways
  p.h = put(pack_h ? R * p.d_pad * (p.pairs ? 4 : e) : 0);
  p.w = put(pack_w && (gradients || !p.pairs) ? (size_t)p.piece * p.d_pad * e : 0);
  p.wpairs = put(p.pairs ? (size_t)p.piece * p.d_pad * 4 : 0);
  if (gradients) {
    p.ht = put((size_t)d * p.n_pad * e);
    p.dz = put(R * p.piece * 2 * p.dz_planes);
    p.sum = put((size_t)p.splits * R * d * 4);
    if (p.by_label) p.at_place = put(R * 4), p.slot = put((size_t)vocab * 4), p.base = put(R * up4(d) * 4), p.labels = put(label_sums_bytes(rows, vocab, d));
  }
  p.bytes = at + 256;
  return p;
}

// --------------------------------------------------------------------------------------------------------- the launches
template <typename E, typename OutT, int EPI, int PLANES>
hipError_t launch_gemm(GemmArgs G, int shape, hipStream_t st) {
  const Shape &s = kShapes[shape];
  constexpr bool TA = EPI == kSum, TB = EPI == kOut;       // dh reads W as it lies, dW reads dz
  G.tiles_m = (int)cdiv64(G.m, s.tm), G.tiles_n = (int)cdiv64(G.n, s.tn);
  const dim3 grid(G.tiles_m * G.tiles_n, G.splits);
  switch (shape) {
    case 0:
      if constexpr (PLANES != 2) gemm_kernel<E, OutT, 256, 256, 2, 2, 2, EPI, PLANES, TA, TB><<<grid, 256, 0, st>>>(G);
      break;                         // dz in two planes takes smaller tiles
    case 1: gemm_kernel<E, OutT, 128, 128, 2, 2, 4, EPI, PLANES, TA, TB><<<grid, 256, 0, st>>>(G); break;
    case 2: gemm_kernel<E, OutT, 64, 64, 2, 2, 4, EPI, PLANES, TA, TB><<<grid, 256, 0, st>>>(G); break;
    case 3: gemm_kernel<E, OutT, 128, 64, 4, 1, 3, EPI, PLANES, TA, TB><<<grid, 256, 0, st>>>(G); break;
    case 4: gemm_kernel<E, OutT, 128, 32, 4, 1, 4, EPI, PLANES, TA, TB><<<grid, 256, 0, st>>>(G); break;
    default:                         // a short sum: two workgroups to a compute unit, one stores while the other begins
      if constexpr (EPI == kOut) gemm_kernel<E, OutT, 128, 128, 2, 2, 2, EPI, PLANES, TA, TB><<<grid, 256, 0, st>>>(G);
  }
  return hipGetLastError();
}

template <typename T, typename E, int PLANES>
hipError_t run(const pbkd_head_loss_desc &q, const Plan &p, hipStream_t st) {
  constexpr int es = sizeof(T);
  char *ws = static_cast<char *>(q.workspace_dev);
  const int rows = (int)q.rows, V = q.vocab, d = q.d;
  const bool gradients = q.dh_dev != nullptr;
  auto floats = [&](size_t at) { return reinterpret_cast<float *>(ws + at); };
  const int wide = q.index_dtype == PBKD_I64;
  auto lay = [&](LayArgs L, ClearArgs clear = {}) {
    L.wide = wide, L.vocab = V;
    const int r = L.cols_dst ? L.rows_fill : L.rows, c = L.rows_dst || L.pairs_dst ? L.cols_fill : L.cols;
    head_lay_kernel<T, E, PLANES><<<dim3((r + 63) / 64, (c + 63) / 64), 256, 0, st>>>(L, clear);
  };
  const bool sorted = rows > kFewLabels;
  const LabelSums sums{q.h_dev, q.h_stride, q.labels_dev, wide != 0, q.dtype, rows, V, d, floats(p.at_place), p.by_label ? reinterpret_cast<int *>(ws + p.slot) : nullptr,
                       floats(p.base), up4(d), floats(p.scale), q.dweight_dev, q.dweight_stride};
  if (gradients) {
    const RowArgs R{q.labels_dev, q.row_weight_dev, floats(p.gs), floats(p.scale), rows, V};
    if (wide) head_rows_kernel<long long><<<1, 1024, 0, st>>>(R);
    else head_rows_kernel<int><<<1, 1024, 0, st>>>(R);
  }
  constexpr bool F32 = es == 4;
  unsigned *tops = reinterpret_cast<unsigned *>(ws + p.tops);         // W's, and each row's of h
  if constexpr (F32) if (p.pairs) {
    head_clear_kernel<<<1, 64, 0, st>>>(tops);
    head_top_kernel<false><<<V < 2048 ? V : 2048, 256, 0, st>>>(static_cast<const float *>(q.weight_dev), q.weight_stride, V, d, tops);
    head_top_kernel<true><<<rows, 256, 0, st>>>(static_cast<const float *>(q.h_dev), q.h_stride, rows, d, tops + 1);
  }
  Operand H{static_cast<const char *>(q.h_dev), q.h_stride * es, 0, rows};
  if (p.pack_h || gradients) {
    LayArgs L{q.h_dev, q.h_stride, p.pack_h && !p.pairs ? ws + p.h : nullptr, gradients ? ws + p.ht : nullptr, p.d_pad * 2, (long long)rows * p.d_pad * 2, p.n_pad * 2,
              (long long)d * p.n_pad * 2, p.pairs ? ws + p.h : nullptr, tops + 1, 1, q.labels_dev, 0, 0, rows, d, p.d_pad, p.n_pad};
    lay(L, ClearArgs{sorted ? nullptr : sums.slot, V});
    if (p.pack_h) H = Operand{ws + p.h, L.rows_ld, L.rows_plane, rows};
  }
  // Rows v0 .. v0 + n of W for the logits, as they lie or laid out (a piece that is the whole vocabulary is laid out once); fp32: and for h's gradient.
  auto weight = [&](int v0, int n, bool now) {
    const T *w = static_cast<const T *>(q.weight_dev) + v0 * q.weight_stride;
    if (!p.pack_w) return Operand{reinterpret_cast<const char *>(w), q.weight_stride * es, 0, n, d};
    LayArgs L{w, q.weight_stride, gradients || !p.pairs ? ws + p.w : nullptr, nullptr, p.d_pad * 2, (long long)p.piece * p.d_pad * 2, 0, 0, p.pairs ? ws + p.wpairs : nullptr, tops, 0,
              nullptr, 0, 0, n, d, p.d_pad, 0};
    if (now) lay(L);
    return Operand{ws + (p.pairs ? p.wpairs : p.w), L.rows_ld, L.rows_plane, n, p.d_pad};
  };
  GemmArgs G{};
  G.b = H, G.kblocks = p.d_pad / 64, G.planes = p.logits, G.tops = p.pairs ? tops : nullptr, G.splits = 1;
  G.labels = q.labels_dev, G.wide = wide, G.vocab = V, G.lse = floats(p.lse), G.g = floats(p.gs), G.part = floats(p.part), G.at_label = floats(p.at_label);
  G.n = rows;
  int parts = 0;
  const bool whole = !p.pack_w;                       // W as it lies: one product over the whole vocabulary
  for (int v0 = 0; v0 < V; v0 += whole ? V : p.piece) {
    const int n = whole || V - v0 < p.piece ? V - v0 : p.piece;
    G.a = weight(v0, n, true), G.m = n, G.v0 = v0, G.parts = p.parts, G.part0 = parts;
    hipError_t e = hipSuccess;
    if constexpr (F32) e = p.pairs ? launch_gemm<f16, E, kStats, 1>(G, p.first_shape, st) : launch_gemm<E, E, kStats, 1>(G, p.first_shape, st);
    else e = launch_gemm<E, E, kStats, 1>(G, p.first_shape, st);
    if (e) return e;
    parts += (int)cdiv64(n, kShapes[p.first_shape].tm);
  }
  head_lse_kernel<<<rows, 256, 0, st>>>(floats(p.part), parts, p.parts, q.labels_dev, wide, V, floats(p.at_label), floats(p.lse), q.lse_dev, q.loss_dev,
                                        floats(p.gs), p.by_label ? floats(p.at_place) : nullptr, sorted ? nullptr : sums.slot);
  if (!gradients) return hipGetLastError();
  if (p.by_label && sorted)
    if (const hipError_t e = launch_label_sort(sums, ws + p.labels, st)) return e;
  G.slot = sums.slot;

  for (int v0 = 0; v0 < V; v0 += p.piece) {
    const int n = V - v0 < p.piece ? V - v0 : p.piece, n64 = up64(n);
    // dz of this piece
    G.a = weight(v0, n, p.pieces > 1), G.m = n, G.v0 = v0;
    G.dz = ws + p.dz, G.dz_ld = p.piece * 2, G.dz_plane = (long long)rows * p.piece * 2;
    G.m_pad = n64;
    hipError_t e = hipSuccess;
    if constexpr (F32) e = p.pairs ? launch_gemm<f16, E, kDz, PLANES>(G, p.first_shape, st) : launch_gemm<E, E, kDz, PLANES>(G, p.first_shape, st);
    else e = p.dz_planes == 2 ? launch_gemm<E, E, kDz, 2>(G, p.first_shape == 0 ? 1 : p.first_shape, st) : launch_gemm<E, E, kDz, 1>(G, p.first_shape, st);
    if (e) return e;
    GemmArgs D{};
    D.planes = p.grads, D.scale = floats(p.scale);
    D.a = G.a, D.m = d, D.n = rows;
    if (p.pairs) D.a.p = ws + p.w;                       // laid out alike, in three terms
    D.b = Operand{G.dz, G.dz_ld, G.dz_plane, rows, n64};
    D.kblocks = n64 / 64, D.splits = p.splits, D.sum = floats(p.sum), D.out_ld = d, D.add = v0 > 0;
    if (const hipError_t e = launch_gemm<E, T, kSum, 1>(D, p.sum_shape, st)) return e;
    D.a = Operand{ws + p.ht, p.n_pad * 2, (long long)d * p.n_pad * 2, d, 0}, D.n = n;      // and dz as it lies
    D.kblocks = p.n_pad / 64, D.splits = 1, D.v0 = v0, D.slot = sums.slot, D.base = floats(p.base), D.base_ld = sums.base_ld;
    D.out = static_cast<T *>(q.dweight_dev) + v0 * q.dweight_stride, D.out_ld = q.dweight_stride;
    D.whole_rows = es == 2 && d % 8 == 0 && q.dweight_stride % 8 == 0 && (reinterpret_cast<uintptr_t>(q.dweight_dev) & 15) == 0;
    const int shape = pick_shape(d, n);
    if (const hipError_t e = launch_gemm<E, T, kOut, 1>(D, shape == 0 && D.kblocks * D.planes.terms <= kShortSum ? 5 : shape, st)) return e;
  }
  const long long eights = (long long)rows * ((d + 7) / 8);
  T *dh = static_cast<T *>(q.dh_dev);
  const AtLabel<T> at{p.by_label ? floats(p.at_place) : nullptr, static_cast<const T *>(q.weight_dev), q.weight_stride, q.labels_dev, wide, V};
  if (p.splits >= 8) head_finish_kernel<T, 8><<<(unsigned)cdiv64(eights, 32), 256, 0, st>>>(floats(p.sum), p.splits, rows, d, floats(p.scale), dh, q.dh_stride, at);
  else head_finish_kernel<T, 1><<<(unsigned)cdiv64(eights, 256), 256, 0, st>>>(floats(p.sum), p.splits, rows, d, floats(p.scale), dh, q.dh_stride, at);
  if (const hipError_t e = hipGetLastError()) return e;
  return p.by_label ? launch_label_sums(sums, ws + p.labels, st) : hipSuccess;
}

inline bool misaligned(const void *p, int size) { return (reinterpret_cast<uintptr_t>(p) & (size - 1)) != 0; }

// Whether two matrices of rows x d share memory.
inline bool meet(const void *a, long long a_stride, const void *b, long long b_stride, long long rows, int d, int size) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + ((rows - 1) * b_stride + d) * size && y < x + ((rows - 1) * a_stride + d) * size;
}

inline bool supported(long long rows, int vocab, int d) { return rows <= kMaxRows && vocab <= kMaxVocab && d <= kMaxD; }

// dweight of a batch without rows
template <typename T>
__global__ __launch_bounds__(256) void head_zero_kernel(T *out, int rows, int cols, long long stride) {
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < (long long)rows * cols; i += (long long)gridDim.x * 256) out[i / cols * stride + i % cols] = T(0.f);
}

}  // namespace
}  // namespace pbkd

using namespace pbkd;

extern "C" {

size_t pbkd_head_loss_workspace_bytes(long long rows, int vocab, int d, int dtype, int gradients) {
  if (rows < 0 || vocab < 1 || d < 1 || !supported(rows, vocab, d) || (dtype != PBKD_F32 && dtype != PBKD_BF16 && dtype != PBKD_F16)) return 0;
  // laid out or not, in place or not: what the addresses and strides of a call decide
  size_t most = 0;
  for (int k = 0; k < 4; ++k) {
    const size_t n = make_plan((int)rows, vocab, d, dtype, gradients != 0, true, k & 1, k & 2).bytes;
    most = n > most ? n : most;
  }
  return most;
}

pbkd_status pbkd_head_loss(const pbkd_head_loss_desc *q, void *hip_stream) {
  if (!q) return set_error(PBKD_EINVAL, "head_loss: null descriptor");
  if (q->rows < 0 || q->vocab < 1 || q->d < 1) return set_error(PBKD_ESHAPE, "head_loss: %lld rows, a weight of %d rows of %d", q->rows, q->vocab, q->d);
  if (!supported(q->rows, q->vocab, q->d))
    return set_error(PBKD_EUNSUPPORTED, "head_loss: %lld rows, a weight of %d rows of %d, at most %d, %d of %d", q->rows, q->vocab, q->d, kMaxRows, kMaxVocab, kMaxD);
  if (q->dtype != PBKD_F32 && q->dtype != PBKD_BF16 && q->dtype != PBKD_F16) return set_error(PBKD_EINVAL, "head_loss: dtype %d", q->dtype);
  if (q->index_dtype != PBKD_I32 && q->index_dtype != PBKD_I64) return set_error(PBKD_EINVAL, "head_loss: index_dtype %d", q->index_dtype);
  if ((q->dh_dev != nullptr) != (q->dweight_dev != nullptr) && q->rows) return set_error(PBKD_EINVAL, "head_loss: dh and dweight come together");
  if (q->rows && (!q->h_dev || !q->weight_dev || !q->labels_dev || !q->loss_dev)) return set_error(PBKD_EINVAL, "head_loss: null tensor");
  const int size = q->dtype == PBKD_F32 ? 4 : 2;
  if (misaligned(q->h_dev, size) || misaligned(q->weight_dev, size) || misaligned(q->dh_dev, size) || misaligned(q->dweight_dev, size) ||
      misaligned(q->labels_dev, q->index_dtype == PBKD_I64 ? 8 : 4) || misaligned(q->row_weight_dev, 4) || misaligned(q->loss_dev, 4) || misaligned(q->lse_dev, 4))
    return set_error(PBKD_EINVAL, "head_loss: a tensor is not aligned to its elements");
  if (q->h_stride < 0 || q->weight_stride < 0) return set_error(PBKD_EINVAL, "head_loss: negative stride");
  if (q->dh_dev && ((q->rows > 1 && q->dh_stride < q->d) || (q->vocab > 1 && q->dweight_stride < q->d)))
    return set_error(PBKD_ESHAPE, "head_loss: rows of an output overlap");
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (q->rows == 0) {
    if (!q->dweight_dev) return PBKD_OK;
    if (size == 4) head_zero_kernel<float><<<1024, 256, 0, st>>>(static_cast<float *>(q->dweight_dev), q->vocab, q->d, q->dweight_stride);
    else head_zero_kernel<bf16><<<1024, 256, 0, st>>>(static_cast<bf16 *>(q->dweight_dev), q->vocab, q->d, q->dweight_stride);
    SEQ_HIPCHK(hipGetLastError());
    return PBKD_OK;
  }
  if (!q->workspace_dev || misaligned(q->workspace_dev, 256)) return set_error(PBKD_ENOMEM, "head_loss: the workspace must be 256-byte aligned");
  const size_t need = pbkd_head_loss_workspace_bytes(q->rows, q->vocab, q->d, q->dtype, q->dh_dev != nullptr);
  if (q->workspace_bytes < need) return set_error(PBKD_ENOMEM, "head_loss: workspace of %zu bytes is smaller than the %zu needed", q->workspace_bytes, need);
  const Plan p = make_plan((int)q->rows, q->vocab, q->d, q->dtype, q->dh_dev != nullptr, !direct(q->h_dev, q->h_stride, q->d, q->dtype),
                           !direct(q->weight_dev, q->weight_stride, q->d, q->dtype),
                           q->dh_dev && (meet(q->h_dev, q->h_stride, q->dh_dev, q->dh_stride, q->rows, q->d, size) ||
                                         meet(q->weight_dev, q->weight_stride, q->dweight_dev, q->dweight_stride, q->vocab, q->d, size)));
  switch (q->dtype) {
    case PBKD_F32: SEQ_HIPCHK((run<float, bf16, 3>(*q, p, st))); break;
    case PBKD_BF16: SEQ_HIPCHK((run<bf16, bf16, 1>(*q, p, st))); break;
    default: SEQ_HIPCHK((run<f16, f16, 1>(*q, p, st))); break;
  }
  return PBKD_OK;
}

}  // extern "C"
