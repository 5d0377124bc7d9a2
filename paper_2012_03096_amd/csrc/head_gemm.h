// The matrix product under the vocabulary loss, and its three uses.
//
//   C[m][n] = sum over k of A[m][k] B[n][k],   k contiguous (of A, as it suits: m contiguous), k a multiple of 64, 16-bit types, fp32 sums
//
// A workgroup forms a tile of TM x TN.  Slices of 64 k of both operands go from memory straight into LDS, STAGES of them at a time: one is
// multiplied while the others are on their way.  A slice's row is 128 bytes, eight pieces of 16; a row's pieces are swapped by bits of its number, so that
// the 16 rows that an MFMA's lanes read at once lie in different banks.  A wave's rows of A are dealt to its MFMA tiles so that
// a lane ends with 16 * MT consecutive m of one n: results leave in wide stores, and a softmax over m needs one exchange between lanes.
// An operand A with m contiguous is staged row of k by row of k and read by the transposing LDS read: in each group of 16 lanes, lane s gives
// the address of four m of the k that is s / 4 from the first, and lane i receives the four k of the i-th m.
//
// fp32 operands come in planes of 16-bit terms, and the product is the sum of the plane products that matter.  Where the numbers' relative size to the
// tensor's largest is all that counts (logits), two fp16 terms of x 2^s, s such that the largest lies near 2^14: what is left out is below
// 2^-20 of |a||b| and 2^-38 of the largest; three products.  Where small numbers count by themselves (gradients of rare tokens), three
// bf16 terms (x = x1 + x2 + x3 exactly, left out: 2^-24 of |a||b|); six products.  A slice's plane products follow each other: each plane is read from
// memory but once.
//
// The large tile reads (128 + 128) rows of 128 bytes from LDS a wave and slice for 64 MFMAs of 32 cycles: 1024 cycles of LDS beside 2048 of MFMA.  Eight waves of 128 x 64
// would read half as much again.  Measured: 16384 x 4096 results, k = 8192, bf16 787 to 820 us, 1340 to 1396 TFLOP/s.
#pragma once
#include <type_traits>

#include "seq_common.h"
#include "split_bf16.h"

namespace pbkd {
namespace head {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef float floatx4 __attribute__((ext_vector_type(4)));

struct Operand {
  const char *p;
  long long ld, plane;     // bytes between rows, between planes
  int rows;
  int cols;                // where k is not contiguous: numbers that a row (of one k) has
};

enum { kStats, kDz, kOut, kSum };    // what becomes of a tile

// Planes of A and B in each product, two bits each from the lowest on.
struct Planes {
  int terms, a, b;
};
constexpr Planes kOne = {1, 0, 0}, kTwoOfB = {2, 0, 0 | 1 << 2}, kPairs = {3, 0 | 0 << 2 | 1 << 4, 0 | 1 << 2 | 0 << 4},
                 kTriples = {6, 0 << 0 | 0 << 2 | 0 << 4 | 1 << 6 | 1 << 8 | 2 << 10, 0 << 0 | 1 << 2 | 2 << 4 | 0 << 6 | 1 << 8 | 0 << 10};

struct GemmArgs {
  Operand a, b;
  int m, n;                        // of the result
  int kblocks;                     // slices of 64 in a plane
  Planes planes;
  const unsigned *tops;            // kStats, kDz: bits of the largest numbers by which A, and each row of B, was scaled; null: they were not
  int tiles_m, tiles_n, splits;    // splits: parts of the sum over k, kSum only
  // kStats, kDz: m is a place in the vocabulary, n a row of h
  const void *labels;              // of 32 or 64 bits; outside 0..vocab-1: none
  int wide, vocab;
  const float *lse, *g;            // g: 0 where there is no label
  float *part, *at_label;          // kStats: [n][parts] pairs (maximum, sum)
  int parts, part0, v0;            // v0: place of the piece's first row of A
  char *dz;                        // [n][m]
  long long dz_ld, dz_plane;
  int m_pad;                       // dz is written up to here: zeros behind the end
  // null, or by place a row of base, -1 where no row has the place as its label.  kDz: dz is zero where a row has its label.  kOut: n is a place too, from v0 on; the results of
  // those with a slot go to base [slot][m] as well, neither scaled nor rounded
  const int *slot;
  float *base;
  long long base_ld;
  // kOut: out[n][m]; kSum: sum[split][n][m]
  void *out;
  long long out_ld;                // elements
  int whole_rows;                  // kOut: m is a multiple of 8, rows begin at multiples of 16 bytes
  const float *scale;
  float *sum;
  int add;
};

// Row n's label, -1 for none.
__device__ __forceinline__ int label_of(const void *labels, int wide, int vocab, long long n) {
  const long long w = wide ? static_cast<const long long *>(labels)[n] : static_cast<const int *>(labels)[n];
  return w >= 0 && w < vocab ? (int)w : -1;
}

typedef short shortx4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ uintx2 read_turned(const char *p) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_bit_cast(uintx2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) shortx4 *)p));
#else
  return uintx2{};
#endif
}

template <typename E>
__device__ __forceinline__ floatx16 mma(uintx4 a, uintx4 b, floatx16 c) {
  if constexpr (__is_same(E, f16)) return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

constexpr float kLog2e = 1.4426950408889634f;

// The power of two that brings numbers of at most `top` (its bits) below 2^14: its exponent, and itself.
__device__ __forceinline__ int exponent_of(unsigned bits) {
  const float top = __builtin_bit_cast(float, bits);
  const int e = top > 0.f ? 14 - __builtin_amdgcn_frexp_expf(top) : 0;
  return e < 126 ? e : 126;          // e >= 14 - 128
}
__device__ __forceinline__ float scale_of(unsigned bits) { return ldexpf(1.f, exponent_of(bits)); }

// What sums of products of numbers scaled by two such powers are multiplied with.  The two together may pass fp32's range (0.3 beside 1e-32: 2^133).  The
// unit stays a number that sums, minus infinity and zero can be multiplied with, also times log2 e: below 2^-126 no logit is above d 2^-97, which
// is zero to a softmax; above 2^126 products of the largest numbers pass fp32, and logits of zero stay zero.
__device__ __forceinline__ float unit_of(int a, int b) {
  const int e = -(a + b);
  return ldexpf(1.f, e < 126 ? e > -126 ? e : -126 : 126);
}

// OutT: the type of kOut's result, and of dz.  PLANES: of dz (2: 16-bit types in two terms; 3: fp32 in three bf16 terms).  TURN_A: A has m contiguous; TURN_B: B has n contiguous.
template <typename E, typename OutT, int TM, int TN, int WM, int WN, int STAGES, int EPI, int PLANES, bool TURN_A, bool TURN_B>
__global__ __launch_bounds__(64 * WM * WN, 1) void gemm_kernel(GemmArgs G) {
  constexpr int THREADS = 64 * WM * WN, MT = TM / WM / 32, NT = TN / WN / 32;
  constexpr int RA = TM * 8 / THREADS, RB = TN * 8 / THREADS, ROWS = THREADS / 8;     // rounds of loads, rows a round
  static_assert(RA * THREADS == TM * 8 && RB * THREADS == TN * 8, "whole rounds");
  // objects of their own: the compiler then knows that a read of one does not wait for loads into another
  constexpr int SLICE = (TM + TN) * 128;
  __shared__ __attribute__((aligned(1024))) char s0[SLICE], s1[SLICE], s2[STAGES > 2 ? SLICE : 16], s3[STAGES > 3 ? SLICE : 16];
  char *const stage[4] = {s0, s1, s2, s3};
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave % WM, wn = wave / WM;

  // neighbouring tiles meet in one die's L2: bands of 8 tiles of m, n inside a band
  int tile = xcd_contiguous(blockIdx.x, G.tiles_m * G.tiles_n);
  const int band = 8 * G.tiles_n, b0 = tile / band, in_band = G.tiles_m - b0 * 8 < 8 ? G.tiles_m - b0 * 8 : 8;
  tile -= b0 * band;
  const int m0 = (b0 * 8 + tile % in_band) * TM, n0 = tile / in_band * TN;

  auto swz_a = [](int r) { return (r >> 1 & 3) | (r / (16 * MT) & 1) << 2; };
  auto swz_b = [](int r) { return r >> 1 & 7; };
  // of a row of k: the four that a group of lanes reads at once lie in different banks
  auto swz_tb = [](int r) { return TN >= 128 ? (r & 3) << 2 : TN == 64 ? (r & 2) << 1 : 0; };
  auto swz_t = [](int r) { return MT == 4 ? (r & 3) << 1 : MT == 2 ? (r & 1) << 1 | (r & 2) << 2 : TM == 64 ? (r & 2) << 1 : (r & 3) << 2; };
  unsigned va[RA], vb[RB];
  {
    const int slot = tid & 7, r0 = tid >> 3;
#pragma unroll
    for (int i = 0; i < RA; ++i) {
      if constexpr (TURN_A) {
        const int at = (i * THREADS + tid) * 16, r = at / (TM * 2), left = G.a.cols / 8 - 1 - m0 / 8;
        const int piece = (at % (TM * 2) / 16) ^ swz_t(r);
        va[i] = (unsigned)(r * (int)G.a.ld + (piece < left ? piece : left) * 16);          // m behind the end: the last again
      } else {
        const int r = i * ROWS + r0, row = m0 + r < G.a.rows ? r : G.a.rows - 1 - m0;      // rows behind the last: the last again
        va[i] = (unsigned)(row * (int)G.a.ld + (slot ^ swz_a(r)) * 16);
      }
    }
#pragma unroll
    for (int i = 0; i < RB; ++i) {
      if constexpr (TURN_B) {
        const int at = (i * THREADS + tid) * 16, r = at / (TN * 2), left = G.b.cols / 8 - 1 - n0 / 8;
        const int piece = (at % (TN * 2) / 16) ^ swz_tb(r);
        vb[i] = (unsigned)(r * (int)G.b.ld + (piece < left ? piece : left) * 16);
      } else {
        const int r = i * ROWS + r0, row = n0 + r < G.b.rows ? r : G.b.rows - 1 - n0;
        vb[i] = (unsigned)(row * (int)G.b.ld + (slot ^ swz_b(r)) * 16);
      }
    }
  }
  const char *pa = G.a.p + (TURN_A ? m0 * 2 : m0 * G.a.ld), *pb = G.b.p + (TURN_B ? n0 * 2 : n0 * G.b.ld);
  const int rows_a = G.a.rows - m0 < TM ? G.a.rows - m0 : TM, rows_b = G.b.rows - n0 < TN ? G.b.rows - n0 : TN;
  const int bytes_a = (rows_a - 1) * (int)G.a.ld + G.kblocks * 128;
  const int bytes_b = (rows_b - 1) * (int)G.b.ld + G.kblocks * 128;

  // this workgroup's slices
  const int total = G.kblocks * G.planes.terms, per = (total + G.splits - 1) / G.splits;
  const int first = blockIdx.y * per, last = first + per < total ? first + per : total;
  int kb = first / G.planes.terms, term = first - kb * G.planes.terms;
  // Narrow tiles read A, once, from memory: each begins at another k, or all would ask the few channels that hold one k of rows a power of two apart.
  // Large tiles share what they read with the others on their die: the dies begin at different k.
  if (!TURN_A && G.splits == 1) kb = (int)(TN <= 64 ? (unsigned)(m0 / TM) * 7u % (unsigned)G.kblocks : (blockIdx.x & 7) * (unsigned)G.kblocks >> 3);
  auto load = [&](char *s) {
    const int qa = G.planes.a >> 2 * term & 3, qb = G.planes.b >> 2 * term & 3;
    // rows of k that an operand has here; what lies behind them reads as zeros
    const int ka = G.a.rows - kb * 64 < 64 ? G.a.rows - kb * 64 : 64, kbb = G.b.rows - kb * 64 < 64 ? G.b.rows - kb * 64 : 64;
    const char *fa = pa + qa * G.a.plane + (TURN_A ? kb * 64 * G.a.ld : 0), *fb = pb + qb * G.b.plane + (TURN_B ? kb * 64 * G.b.ld : 0);
    const __amdgpu_buffer_rsrc_t ra = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(fa), 0, TURN_A ? (ka - 1) * (int)G.a.ld + (G.a.cols - m0) * 2 : bytes_a, 0x00020000);
    const __amdgpu_buffer_rsrc_t rb = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(fb), 0, TURN_B ? (kbb - 1) * (int)G.b.ld + (G.b.cols - n0) * 2 : bytes_b, 0x00020000);
    char *d = s + wave * 1024;
#pragma unroll
    for (int i = 0; i < RA; ++i) load16_to_lds(ra, d + i * THREADS * 16, va[i], TURN_A ? 0 : kb * 128);
#pragma unroll
    for (int i = 0; i < RB; ++i) load16_to_lds(rb, d + TM * 128 + i * THREADS * 16, vb[i], TURN_B ? 0 : kb * 128);
    if (++term == G.planes.terms) term = 0, kb = kb + 1 == G.kblocks ? 0 : kb + 1;
  };

  floatx16 acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
  floatx16 second = acc[0][0];       // of a wave with one MFMA tile: products into one sum alone would wait for each other
  const int r32 = lane & 31, h = lane >> 5;
  // a lane's results: n = n1 + 32 j, m = m1 .. m1 + 16 MT - 1 (tile i: sixteen of them)
  const int m1 = m0 + wm * (MT * 32) + h * (16 * MT), n1 = n0 + wn * (NT * 32) + r32;
  // Read ahead of the sum, which may be short (128 x 131072 x 8192: dW 726 us, without 791).  The largest tile has no registers for that, and no short sums.
  constexpr bool EARLY = EPI == kOut && MT * NT < 16;
  int slot[NT];
  auto read_slots = [&] {
#pragma unroll
    for (int j = 0; j < NT; ++j) slot[j] = G.slot && n1 + 32 * j < G.n ? G.slot[G.v0 + n1 + 32 * j] : -1;
  };
  if (EARLY) read_slots();
  // MFMA row 8 a + 4 b + c of tile i is the wave's row b * 16 MT + 16 i + 4 a + c: a lane then holds 16 MT rows in order
  const int row_a = wm * (MT * 32) + (r32 >> 2 & 1) * (16 * MT) + (r32 >> 3) * 4 + (r32 & 3), row_b = wn * (NT * 32) + r32;
  const int sa = swz_a(row_a), sb = swz_b(row_b);       // rows 16 i and 32 j further on are swapped alike

  // where a lane's four m of tile i begin, of the k that is lane % 16 / 4 behind k (8 more for the upper half of the lanes)
  const int turn_k = (lane >> 2 & 3) + 8 * h, turn_m = wm * (MT * 32) + (lane & 1) * (16 * MT) + (lane >> 4 & 1) * 8 + (lane >> 1 & 1) * 4;
  auto turned = [&](int k, int i) {
    const int r = k + turn_k, m = turn_m + 16 * i;
    return r * (TM * 2) + ((m >> 3) ^ swz_t(turn_k)) * 16 + (m & 7) * 2;         // k is a multiple of four: it does not change the swap
  };
  // and its four n of tile j
  auto turned_b = [&](int k, int j) {
    const int r = k + turn_k, n = wn * (NT * 32) + (lane >> 4 & 1) * 16 + (lane & 3) * 4 + 32 * j;
    return TM * 128 + r * (TN * 2) + ((n >> 3) ^ swz_tb(turn_k)) * 16 + (n & 7) * 2;
  };
  // Operands of half a slice (two MFMA steps) wait in registers while the half before is multiplied.
  struct Half {
    uintx4 a[2][MT], b[2][NT];
  };
  auto fetch = [&](Half &f, const char *s, int half) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int c = half * 4 + u * 2 + h;
      if constexpr (TURN_B) {
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          const uintx2 lo = read_turned(s + turned_b(half * 32 + u * 16, j)), hi = read_turned(s + turned_b(half * 32 + u * 16 + 4, j));
          f.b[u][j] = uintx4{lo[0], lo[1], hi[0], hi[1]};
        }
      } else {
#pragma unroll
        for (int j = 0; j < NT; ++j) f.b[u][j] = *reinterpret_cast<const uintx4 *>(s + TM * 128 + (row_b + 32 * j) * 128 + (c ^ sb) * 16);
      }
      if constexpr (TURN_A) {
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          const uintx2 lo = read_turned(s + turned(half * 32 + u * 16, i)), hi = read_turned(s + turned(half * 32 + u * 16 + 4, i));
          f.a[u][i] = uintx4{lo[0], lo[1], hi[0], hi[1]};
        }
      } else {
#pragma unroll
        for (int i = 0; i < MT; ++i) f.a[u][i] = *reinterpret_cast<const uintx4 *>(s + (row_a + 16 * i) * 128 + (c ^ sa) * 16);
      }
    }
  };
  constexpr int READS = 2 * ((TURN_A ? 2 : 1) * MT + (TURN_B ? 2 : 1) * NT);
  auto multiply = [&](const Half &f) {
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          floatx16 &to = MT * NT == 1 && u ? second : acc[i][j];
          to = mma<E>(f.a[u][i], f.b[u][j], to);
        }
  };
  // All but the last `later` slices that this wave loads have landed in LDS, and then everybody's; everybody has read what it needs of the
  // slice before.  The waits are written out: a barrier alone does not wait for loads into LDS.
  auto arrived = [&](auto later) {
    constexpr int n = decltype(later)::value * (RA + RB);
    static_assert(n < 64, "vmcnt has six bits");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt((n & 15) | 0x70 | (n >> 4) << 14);       // vmcnt(n), lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
  };
  // The first half of a slice is in registers.  Behind the barrier the slice after it has arrived, and this one's place is free.
  Half f0, f1;
  auto step = [&](char *now, const char *next, bool more, bool ahead, auto later) {
    fetch(f1, now, 1);
    multiply(f0);
    // the reads first, one between two products, so that they are back before the barrier
#pragma unroll
    for (int i = 0; i < READS; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    }
    arrived(later);
    if (ahead) load(now);
    if (more) fetch(f0, next, 0);
    multiply(f1);
#pragma unroll
    for (int i = 0; i < READS; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x010, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  // Small tiles have too few products in half a slice to hide a read behind: a whole slice waits in registers (500 x 1013 x 515 fp32 75.5 -> 72.5 us, 2113 x 192 x
  // 888 116 -> 109; narrow tiles wait for memory and gain nothing).
  auto step_whole = [&](Half (&now)[2], Half (&then)[2], char *place, const char *next, bool more, bool ahead, auto later) {
    if (more) arrived(later);
    if (ahead) load(place);
    if (more) fetch(then[0], next, 0), fetch(then[1], next, 1);
    multiply(now[0]);
    multiply(now[1]);
    constexpr int PRODUCTS = 4 * MT * NT;
#pragma unroll
    for (int i = 0; i < PRODUCTS; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x010, (RA + RB + PRODUCTS - 1) / PRODUCTS, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, (2 * READS + PRODUCTS - 1) / PRODUCTS, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  if (first < last) {
#pragma unroll
    for (int i = 0; i < STAGES; ++i)
      if (first + i < last) load(stage[i]);
    if (first + STAGES <= last) arrived(std::integral_constant<int, STAGES - 1>());
    else arrived(std::integral_constant<int, 0>());
    int k = first;
    if constexpr (STAGES == 4 && TM == TN) {
      constexpr int U = STAGES;
      Half r[2][2];
      fetch(r[0][0], s0, 0), fetch(r[0][1], s0, 1);
      for (; k + U + STAGES - 1 < last; k += U) {
#pragma unroll
        for (int i = 0; i < U; ++i) step_whole(r[i & 1], r[~i & 1], stage[i % STAGES], stage[(i + 1) % STAGES], true, true, std::integral_constant<int, STAGES - 2>());
      }
      for (; k < last; k += U) {
#pragma unroll
        for (int i = 0; i < U; ++i)
          if (k + i < last)
            step_whole(r[i & 1], r[~i & 1], stage[i % STAGES], stage[(i + 1) % STAGES], k + i + 1 < last, k + i + STAGES < last, std::integral_constant<int, 0>());
      }
    } else {
      fetch(f0, s0, 0);
      for (; k + 2 * STAGES - 1 < last; k += STAGES) {
#pragma unroll
        for (int i = 0; i < STAGES; ++i) step(stage[i], stage[(i + 1) % STAGES], true, true, std::integral_constant<int, STAGES - 2>());
      }
      for (; k < last; k += STAGES) {
#pragma unroll
        for (int i = 0; i < STAGES; ++i)
          if (k + i < last) step(stage[i], stage[(i + 1) % STAGES], k + i + 1 < last, k + i + STAGES < last, std::integral_constant<int, 0>());
      }
    }
  }

  if (MT * NT == 1) {
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[0][0][e] += second[e];
  }

  // what belongs to a lane's rows of n, read together: rows behind the end read the last one's
  int label[NT];
  if constexpr (EPI == kStats || EPI == kDz) {
    if (G.wide) {
      long long w[NT];
#pragma unroll
      for (int j = 0; j < NT; ++j) w[j] = static_cast<const long long *>(G.labels)[n1 + 32 * j < G.n ? n1 + 32 * j : G.n - 1];
#pragma unroll
      for (int j = 0; j < NT; ++j) label[j] = w[j] >= 0 && w[j] < G.vocab && n1 + 32 * j < G.n ? (int)w[j] : -1;
    } else {
      int w[NT];
#pragma unroll
      for (int j = 0; j < NT; ++j) w[j] = static_cast<const int *>(G.labels)[n1 + 32 * j < G.n ? n1 + 32 * j : G.n - 1];
#pragma unroll
      for (int j = 0; j < NT; ++j) label[j] = w[j] >= 0 && w[j] < G.vocab && n1 + 32 * j < G.n ? w[j] : -1;
    }
  }
  const bool edge = m0 + TM > G.m;                  // the vocabulary ends in this tile
  float unit[NT];                                   // of the results
  if constexpr (EPI == kStats || EPI == kDz) {
#pragma unroll
    for (int j = 0; j < NT; ++j) unit[j] = 1.f;
    if (G.tops) {
      const int a = exponent_of(G.tops[0]);
#pragma unroll
      for (int j = 0; j < NT; ++j) unit[j] = unit_of(a, exponent_of(G.tops[1 + (n1 + 32 * j < G.n ? n1 + 32 * j : G.n - 1)]));
    }
  }
  if constexpr (EPI == kStats) {
    float *red = reinterpret_cast<float *>(s0);        // [WM][TN] pairs, once everybody is done with the slices
    __syncthreads();
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const int n = n1 + 32 * j, at = label[j] - G.v0 - m1;
      if (at >= 0 && at < 16 * MT) {                     // few lanes have their label here
        float mine = 0.f;
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (at == 16 * i + e) mine = acc[i][j][e];
        G.at_label[n] = mine * unit[j];
      }
      if (edge) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (m1 + 16 * i + e >= G.m) acc[i][j][e] = -__builtin_inff();
      }
      const float unit2 = unit[j] * kLog2e;
      float top = -__builtin_inff(), sum = 0.f;
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) top = fmaxf(top, acc[i][j][e]);
      top = fmaxf(top, __shfl_xor(top, 32, 64));
      const float ref = top == -__builtin_inff() ? 0.f : top * unit2;
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) sum += __builtin_amdgcn_exp2f(fmaf(acc[i][j][e], unit2, -ref));
      sum += __shfl_xor(sum, 32, 64);
      if (h == 0) red[(wm * TN + n - n0) * 2] = top * unit[j], red[(wm * TN + n - n0) * 2 + 1] = sum;
    }
    __syncthreads();
    for (int n = tid; n < TN && n0 + n < G.n; n += THREADS) {
      float top = -__builtin_inff(), sum = 0.f;
#pragma unroll
      for (int k = 0; k < WM; ++k) top = fmaxf(top, red[(k * TN + n) * 2]);
      const float ref = top == -__builtin_inff() ? 0.f : top;
#pragma unroll
      for (int k = 0; k < WM; ++k) sum += red[(k * TN + n) * 2 + 1] * __expf(red[(k * TN + n) * 2] - ref);
      float *p = G.part + ((long long)(n0 + n) * G.parts + G.part0 + m0 / TM) * 2;
      p[0] = top, p[1] = sum;
    }
  } else if constexpr (EPI == kDz) {
    float lse[NT], g[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) lse[j] = G.lse[n1 + 32 * j < G.n ? n1 + 32 * j : G.n - 1] * kLog2e, g[j] = G.g[n1 + 32 * j < G.n ? n1 + 32 * j : G.n - 1];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const int at = label[j] - G.v0 - m1;
      const float unit2 = unit[j] * kLog2e;
      const bool live = label[j] >= 0, hit = live && at >= 0 && at < 16 * MT;
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][j][e] = g[j] * __builtin_amdgcn_exp2f(fmaf(acc[i][j][e], unit2, -lse[j]));
      if (__any(hit)) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (at == 16 * i + e) acc[i][j][e] = G.slot ? 0.f : acc[i][j][e] - g[j];
      }
      if (__any(!live) || edge) {                        // zeros, whatever the logits are
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (!live || m1 + 16 * i + e >= G.m) acc[i][j][e] = 0.f;
      }
    }
    // dz leaves through the wave's own part of LDS, in whole rows: a lane's own results would go out in pieces of 16 bytes.
    constexpr int BYTES = 32 * MT * 32 * NT * 2, FIT = SLICE / BYTES;
    static_assert(FIT * 2 >= WM * WN, "the waves' tiles fit into two stages");
    char *own = (wave < FIT ? s0 : s1) + (wave < FIT ? wave : wave - FIT) * BYTES;
    __syncthreads();
    const int wave_m = m0 + wm * (MT * 32), wave_n = n0 + wn * (NT * 32);
#pragma unroll 1
    for (int k = 0; k < PLANES; ++k) {
      // a word has two m of one n, in their order: word(j, 8 i + e) is of tile i
      auto word_of = [&](int j, int w) {
        const OutT y[2] = {static_cast<OutT>(acc[w / 8][j][w % 8 * 2]), static_cast<OutT>(acc[w / 8][j][w % 8 * 2 + 1])};
        unsigned x;
        __builtin_memcpy(&x, y, 4);
        return x;
      };
      // rows of n: 4 MT pieces of 16 bytes, swapped by the row's number
      constexpr int PM = 4 * MT;
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        if (PLANES > 1) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 2 * MT; ++i) {
          const int row = 32 * j + r32, piece = (h * 2 * MT + i) ^ (row & (PM - 1));
          *reinterpret_cast<uintx4 *>(own + row * (PM * 16) + piece * 16) =
              uintx4{word_of(j, 4 * i), word_of(j, 4 * i + 1), word_of(j, 4 * i + 2), word_of(j, 4 * i + 3)};
        }
        if (PLANES > 1)                // what this plane leaves to the next
#pragma unroll
          for (int i = 0; i < MT; ++i) {
            __builtin_amdgcn_sched_barrier(0);
            asm volatile("" : "+a"(acc[i][j]));          // rounded once more, or all the rounded values are kept and spill
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] -= static_cast<float>(static_cast<OutT>(acc[i][j][e]));
          }
      }
      asm volatile("" ::: "memory");
#pragma unroll
      for (int t = 0; t < 32 * NT * PM / 64; ++t) {
        const int row = t * (64 / PM) + lane / PM, piece = lane % PM;
        const uintx4 w = *reinterpret_cast<const uintx4 *>(own + row * (PM * 16) + (piece ^ (row & (PM - 1))) * 16);
        const int n = wave_n + row, m = wave_m + piece * 8;
        if (n < G.n && m < G.m_pad) *reinterpret_cast<uintx4 *>(G.dz + k * G.dz_plane + n * G.dz_ld + m * 2) = w;
      }
      asm volatile("" ::: "memory");
    }
  } else {
    float scale = 1.f;
    if (EPI == kOut) scale = *G.scale;
    if constexpr (EPI == kOut && sizeof(OutT) == 2) {
      if (G.slot) {
        if (!EARLY) read_slots();
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          __builtin_amdgcn_sched_barrier(0);
          if (slot[j] >= 0) {          // up to the row's end in steps of 16 bytes: base's rows are that long
            float *p = G.base + slot[j] * G.base_ld + m1;
#pragma unroll
            for (int i = 0; i < 4 * MT; ++i) {
              const floatx16 &x = acc[i / 4][j];
              const int e = i % 4 * 4;
              if (m1 + 4 * i < G.m) *reinterpret_cast<floatx4 *>(p + 4 * i) = floatx4{x[e], x[e + 1], x[e + 2], x[e + 3]};
            }
          }
#pragma unroll
          for (int i = 0; i < MT; ++i) asm volatile("" : "+a"(acc[i][j]));      // stays where it is, or the copies spill
        }
      }
      if (G.whole_rows) {              // 16-byte steps: the results leave in whole rows, as dz does
        constexpr int BYTES = 32 * MT * 32 * NT * 2, FIT = SLICE / BYTES, PM = 4 * MT;
        char *own = (wave < FIT ? s0 : s1) + (wave < FIT ? wave : wave - FIT) * BYTES;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int i = 0; i < 2 * MT; ++i) {
            const int row = 32 * j + r32, piece = (h * 2 * MT + i) ^ (row & (PM - 1));
            OutT y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = static_cast<OutT>(acc[i / 2][j][i % 2 * 8 + e] * scale);
            uintx4 w;
            __builtin_memcpy(&w, y, 16);
            *reinterpret_cast<uintx4 *>(own + row * (PM * 16) + piece * 16) = w;
          }
        asm volatile("" ::: "memory");
#pragma unroll
        for (int t = 0; t < 32 * NT * PM / 64; ++t) {
          const int row = t * (64 / PM) + lane / PM, piece = lane % PM;
          const uintx4 w = *reinterpret_cast<const uintx4 *>(own + row * (PM * 16) + (piece ^ (row & (PM - 1))) * 16);
          const int n = n0 + wn * (NT * 32) + row, m = m0 + wm * (MT * 32) + piece * 8;
          if (n < G.n && m < G.m) *reinterpret_cast<uintx4 *>(static_cast<char *>(G.out) + (n * G.out_ld + m) * 2) = w;
        }
        return;
      }
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const int n = n1 + 32 * j;
      if (n >= G.n) continue;
#pragma unroll
      for (int i = 0; i < 2 * MT; ++i) {
        const int m = m1 + 8 * i, left = G.m - m;
        if (left <= 0) break;
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = acc[i / 2][j][i % 2 * 8 + e] * scale;
        if constexpr (EPI == kOut) {
          store_n<OutT, 8>(static_cast<OutT *>(G.out) + n * G.out_ld + m, left, x);
        } else {
          float *p = G.sum + ((long long)blockIdx.y * G.n + n) * G.out_ld + m;
          if (G.add) {
            float y[8];
            load_n<float, 8>(p, left, y);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] += y[e];
          }
          store_n<float, 8>(p, left, x);
        }
      }
    }
  }
}

}  // namespace head
}  // namespace pbkd
