// Gated linear recurrence over time, channel by channel, forward, backward and for single tokens:
//
//   x = gate + bias,  a = 1/(1+e^-x),  z = 1/(1+e^x) = 1 - a,  h_t = a_t h_{t-1} + z_t u_t,  y_t = h_t silu(o_t)
//
// A step is the affine map h -> a h + b (b = z u), maps compose as (A1,B1) then (A2,B2) = (A2 A1, A2 B1 + B2), so a
// range of tokens is one pair (A, B) a channel and time can be cut into pieces.  Backward, with c_t = dy_t silu(o_t):
//
//   dh_t = c_t + e_t,  e_{t-1} = a_t dh_t   (the same composition from the last token on),
//   du = z dh, dgate = dh (h_{t-1} - u) a z, do = dy h silu'(o)
//
// A tile is kSlice channels by a number of tokens: a thread holds L consecutive tokens of two channels, half a wave next to
// each other a row of kSlice channels, the half waves of a workgroup (of four waves mostly) follow each other in time.  Each thread folds its
// tokens, the half waves' pairs are joined by an exchange between the halves and through LDS, and the tokens are gone through
// again from the registers: each tensor is read once.  Tiles of all times run at once and hand the state on (below).
//
// Bound by memory, then by the wait for the state.  A row of a tile is 128 bytes of a 16-bit type (a slice of 128 channels in workgroups of
// 512 threads reads better alone, but half as many tiles fit at a time: 8x4096x2048 324 us against 288).
// Measured (bf16, with the output gate): 1x65536x1280 forward 128 us, 5.2 TB/s; 8x4096x2048
// forward and backward 288 us, 5.1 TB/s (forward 105, backward 182, the rest clears words and sums the bias gradient); fp32
// 7x1000x515, padded, 46 us; one token of 64 sequences of 2048 channels 3.6 us, which is a launch's own length.  One workgroup going
// through a chain alone took 8.8 ms for the first of these.
#include "seq_common.h"

#include <initializer_list>
#include <type_traits>

namespace pbkd {
namespace {

constexpr int kSlice = 64;          // channels of a tile: 128 bytes of a 16-bit type
constexpr int kFwdL = 16;           // tokens of a thread, forward: a tile of four waves has 8 times as many (8: 1x65536x1280 182 us, then 143)
constexpr int kBwdL = 8;            // backward: more is held per token
constexpr int kMostSteps = 64;      // tokens that may be taken one after the other
constexpr int kSaved = 8 * kBwdL;   // the forward pass saves the state in front of every backward tile of four waves

struct FwdArgs {
  const void *u, *g, *o;
  const float *bias;
  const int *lengths;
  const float *h0;
  float *hT;
  void *y;
  float *saved;
  unsigned long long *work;
  long long len, ub, us, gb, gs, ob, os, yb, ys;
  int batch, D, slices, tiles;
};

struct BwdArgs {
  const void *u, *g, *o, *dy;
  const float *bias;
  const int *lengths;
  const float *saved, *dhT;
  void *du, *dg, *dou;
  float *dbias_partial, *dh0;
  unsigned long long *work;
  long long len, ub, us, gb, gs, ob, os, yb, ys, dub, dus, dgb, dgs, dob, dos;
  int batch, D, slices, tiles;
};

constexpr float kLog2e = 1.44269504088896340736f;

// sigmoid(x) and sigmoid(-x), both from e = exp(-|x|), so that neither is a difference from 1.  The larger is good to a few units of its last place;
// the smaller one's relative error grows with |x|, whose product with log2 e is rounded before exp2: 4 units of the last place up to
// |x| = 4, 15 up to 17, 62 at 80 (times 2^-24).
__device__ __forceinline__ void sigmoids(float x, float &a, float &z) {
  const float e = __builtin_amdgcn_exp2f(-kLog2e * fabsf(x)), r = __builtin_amdgcn_rcpf(1.f + e), s = e * r;
  a = x >= 0.f ? r : s;
  z = x >= 0.f ? s : r;
}
// sigmoid(x) far: exp(-x) may be infinite
__device__ __forceinline__ float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * x)); }

// The two channels of a lane.  A row's last lane may have only one (D is odd): it reads the last two and moves its own to the front.
// Lanes beyond the row read its last channels again, and nothing of them is written.
struct Lane {
  int c;        // first channel that is read
  int n;        // channels that exist: 2, 1 or 0
  bool odd;     // a lane of the workgroup has only one
};
// How a workgroup's lanes take their channels: all two by two; a lane may have one; the row has no two.
enum { PAIRS, ODD, SINGLE };
__device__ __forceinline__ Lane lane_of(int slice, int D) {
  Lane q;
  const int c0 = slice * kSlice + (threadIdx.x & 31) * 2, last = D > 2 ? D - 2 : 0;
  q.odd = (D & 1) && slice * kSlice + kSlice > D;
  q.n = D - c0 < 2 ? (D - c0 < 0 ? 0 : D - c0) : 2;
  q.c = c0 < last ? c0 : last;
  return q;
}
template <typename T>
using Raw = typename VecOf<T, 2>::type;
// FAR: see far_load; and no cache line has another tile's channels too, or the line's second reader would fetch it again
// (7x1000x515 in fp32, forward and backward, with it: 64 us, without: 56; 8x4096x2048, whose tiles are alone with theirs: 305, without: 319).
template <typename T, int HOW, bool FAR>
__device__ __forceinline__ Raw<T> raw2(const T *p, const Lane &q) {
  Raw<T> r;
  if (HOW == SINGLE) {
    r[0] = r[1] = *p;
  } else {
    r = far_load<FAR, T, 2>(p);
    if (HOW == ODD) r[0] = q.n == 1 ? r[1] : r[0];
  }
  return r;
}
// lanes without channels do not come here
template <typename T, int HOW, bool FAR>
__device__ __forceinline__ void put2(T *p, const Lane &q, const float (&v)[2]) {
  if (HOW != PAIRS && q.n == 1) {
    p[HOW == SINGLE ? 0 : 1] = static_cast<T>(v[0]);      // its place was moved with its reads
  } else {
    Raw<T> r;
    r[0] = static_cast<T>(v[0]), r[1] = static_cast<T>(v[1]);
    far_store<FAR, T, 2>(r, p);
  }
}
// fp32 rows of channels, by the lane's own place
template <int HOW>
__device__ __forceinline__ void floats2(const float *p, const Lane &q, float (&v)[2]) {
  const Raw<float> r = raw2<float, HOW, false>(p + q.c, q);
  v[0] = r[0], v[1] = r[1];
}
template <int HOW>
__device__ __forceinline__ void put_floats2(float *p, const Lane &q, const float (&v)[2]) {
  if (q.n > 0) put2<float, HOW, false>(p + q.c, q, v);
}

// Places of a thread's L tokens in one tensor: a base that its wave shares, and each token's own 32-bit distance from it, which
// the loads and stores take as they are.  In tiles that are not WHOLE a token behind the last is moved to the last.
constexpr long long kMaxStride = 1LL << 25;      // elements between tokens: 2 * kFwdL of them, in bytes, below 2^32
template <typename T, int L, bool WHOLE>
struct Place {
  char *base;
  unsigned stride, mine;    // bytes; WHOLE: the distance of the first token; else: of the channels far
  int token, last;          // the thread's first token and the sequence's last, counted from the base's
  __device__ __forceinline__ Place(const void *p, long long batch_at, long long stride_, int t0, int slice, const Lane &q, long long T_) {
    const int w0 = t0 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * 2 * L, at = WHOLE || w0 < T_ ? w0 : (int)T_ - 1;
    stride = (unsigned)stride_ * (unsigned)sizeof(T);
    const int c0 = slice > 0 ? slice * kSlice - 2 : 0;      // a slice's only lane may read from the channel in front
    base = const_cast<char *>(static_cast<const char *>(p)) + (batch_at + at * stride_ + c0) * (long long)sizeof(T);
    token = threadIdx.x & 32 ? L : 0, last = (int)T_ - 1 - at;
    mine = (unsigned)(q.c - c0) * (unsigned)sizeof(T);
    if (WHOLE) mine += (unsigned)token * stride;
  }
  __device__ __forceinline__ T *at(int i) const {
    return reinterpret_cast<T *>(base + (WHOLE ? mine + i * stride : mine + (unsigned)(token + i < last ? token + i : last) * stride));
  }
};

__device__ __forceinline__ int length_of(const int *lengths, int b, long long len) {
  if (!lengths) return (int)len;
  const long long n = lengths[b];
  return (int)(n < 0 ? 0 : n > len ? len : n);
}

// How tiles that follow each other in time hand on the state.  The tiles of one sequence and slice are a chain, cut into
// segments of kSeg.  Every tile publishes its own pair (A, B), which needs nothing of the tiles in front of it; it then folds
// the pairs of its segment's earlier tiles, and the last tile of a segment also publishes the state behind it, so that only
// one tile in kSeg waits for one before.  All folds have a fixed order: results do not depend on who was first.
//
// A tile's place in its chain comes from the chain's counter, and it waits for nothing but tiles with smaller numbers: they were
// taken by workgroups that run already, so every wait ends.
//
// A pair travels in one 64-bit word, written and read whole at the scope of the device (the eight dies' L2 caches do not see each
// other's writes otherwise): 0 is "not there yet", B below, A with its sign bit set above (A, a product of sigmoids, has
// none of its own).  The words are cleared by a kernel in front.
constexpr int kSeg = 8;      // forward with 4, 8 and 16, us: 1x131072x64 82, 53, 46; 1x65536x1280 131, 130, 140; 8x4096x2048 108, 108, 168

__device__ __forceinline__ void put_word(unsigned long long *p, float low, unsigned high) {
  __hip_atomic_store(p, (unsigned long long)high << 32 | __builtin_bit_cast(unsigned, low), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ unsigned long long peek_word(const unsigned long long *p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// All lanes of the wave come here together and leave together: lanes that wait under a mask of their own are where the compiler, short
// of registers, was seen to copy others' under that mask.
__device__ __forceinline__ unsigned long long await_word(const unsigned long long *p, unsigned long long v) {
  while (__any(v == 0)) {
    __builtin_amdgcn_s_sleep(1);
    v = peek_word(p);
  }
  return v;
}
__device__ __forceinline__ unsigned pair_high(float A) { return (A == A ? __builtin_bit_cast(unsigned, A) : 0x7FC00000u) | 0x80000000u; }
__device__ __forceinline__ float low_of(unsigned long long v) { return __builtin_bit_cast(float, (unsigned)v); }
__device__ __forceinline__ float high_of(unsigned long long v) { return __builtin_bit_cast(float, (unsigned)(v >> 32) & 0x7FFFFFFFu); }

struct Chain {
  unsigned long long *pairs, *states;     // [tiles][kSlice], [segments][kSlice]
};
// As many workgroups for each chain as it has tiles, those of one time step next to each other; a die takes neighbouring slices, so
// that what it reads at a time are whole rows, which spread over all channels of its L2 (one slice in eight meets a quarter of
// them at row lengths that are multiples of 4 KB: 8x4096x2048 forward and backward 381 us, this way 337 us).
__device__ __forceinline__ int chain_of_workgroup(unsigned n, unsigned chains) { return xcd_contiguous(n % chains, chains); }

// The words of a chain: its counter (a line of its own), its pairs, its states.
constexpr int kCounter = 16;
inline __host__ __device__ long long words_of_chain(long long tiles) { return kCounter + (tiles + (tiles + kSeg - 1) / kSeg) * kSlice; }
__device__ __forceinline__ Chain chain_of(unsigned long long *work, int chain, int tiles) {
  unsigned long long *p = work + chain * words_of_chain(tiles);
  return {p + kCounter, p + kCounter + (long long)tiles * kSlice};
}

// The first wave does this, a lane for each channel.  look_early reads the words of the segment's earlier tiles and the state in
// front of the segment, which are mostly there by then, while the tile's own data are on their way; look_back waits for those
// that were not and returns the state in front of the tile.  The last tile of a segment passes the state behind it on as soon as it
// knows the one in front: one addition and one product lie between them.  Only the chain's first tile reads the state in
// front of the chain (`first`), and its pair is the constant map to the state behind it: the last tile, which may write over the
// initial state, thereby has every reader of it behind itself.
// EARLY of the pairs' words are read early.  Seven cost registers for as long as the tile's data are on their way, and tiles of eight waves
// have the fewest: with three 1x65536x1280 backward takes 237 us instead of 254, 1x65536x4096 728 instead of 778.
// With four waves all of them are: 8x2048x2047 forward and backward 193 us, with three 197.  Neither choice keeps every kernel out of
// scratch memory.  The compiler reports registers spilled in the gated kernels of 16-bit types: forward with four waves 18 past the caches and 30
// (bf16) or 27 (f16) within, with eight 16, 25 and 29; backward with eight waves within the caches 32 and 18.  All others spill none.
constexpr int early_words(int waves) { return waves == 8 ? 3 : kSeg - 1; }
template <int EARLY>
struct Words {
  unsigned long long v[EARLY], state;
};
template <int EARLY>
__device__ __forceinline__ Words<EARLY> look_early(const Chain &q, int pos) {
  const int ch = threadIdx.x & 63, seg = pos / kSeg, in = pos % kSeg;
  const unsigned long long *p = q.pairs + (long long)seg * kSeg * kSlice + ch;
  Words<EARLY> k;
#pragma unroll
  for (int j = 0; j < EARLY; ++j) k.v[j] = j < in ? peek_word(p + j * kSlice) : 1;
  k.state = seg > 0 ? peek_word(q.states + (long long)(seg - 1) * kSlice + ch) : 1;
  return k;
}
// At, Bt: the tile's own pair
template <int EARLY>
__device__ __forceinline__ float look_back(const Chain &q, int pos, bool last, float At, float Bt, float first, const Words<EARLY> &k) {
  const int ch = threadIdx.x & 63, seg = pos / kSeg, in = pos % kSeg;
  const unsigned long long *p = q.pairs + (long long)seg * kSeg * kSlice + ch;
  unsigned long long late[kSeg - 1];
#pragma unroll
  for (int j = EARLY; j < kSeg - 1; ++j) late[j] = j < in ? peek_word(p + j * kSlice) : 1;
  float A = 1.f, B = 0.f;
#pragma unroll
  for (int j = 0; j < kSeg - 1; ++j) {
    if (j < in) {
      const unsigned long long v = await_word(p + j * kSlice, j < EARLY ? k.v[j < EARLY ? j : 0] : late[j]);
      const float A2 = high_of(v);
      B = fmaf(A2, B, low_of(v));
      A *= A2;
    }
  }
  const float A2 = At * A, B2 = fmaf(At, B, Bt);
  const float at = seg > 0 ? low_of(await_word(q.states + (long long)(seg - 1) * kSlice + ch, k.state)) : pos == 0 ? first : 0.f;
  if (in == kSeg - 1 && !last) put_word(q.states + (long long)seg * kSlice + ch, fmaf(A2, at, B2), 1u);
  return fmaf(A, at, B);
}
__device__ __forceinline__ void publish_pair(const Chain &q, int pos, float A, float B, float first) {
  put_word(q.pairs + (long long)pos * kSlice + (threadIdx.x & 63), pos == 0 ? fmaf(A, first, B) : B, pair_high(pos == 0 ? 0.f : A));
}

// 9 MB (8x4096x2048 backward) in 5.8 us, most of it one kernel waiting for another.
__global__ __launch_bounds__(256) void clear_words_kernel(unsigned long long *p, long long n) {
  typedef unsigned long long u2 __attribute__((ext_vector_type(2)));
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n / 2; i += (long long)gridDim.x * 256) reinterpret_cast<u2 *>(p)[i] = u2{0, 0};
}

// What a workgroup shares.
template <int W>
struct alignas(16) Shared {
  float2 tot[W][kSlice], back[W][kSlice];      // each wave's pair, forward and backward in time
  float2 part[W][kSlice];                      // what lies between the tile's start (the chain's way) and each wave's
  float h[W][kSlice];                          // backward: the state in front of each wave
  float at[kSlice];
  unsigned number;
};

// A chain of one tile has no words, nor are they cleared for it.
__device__ __forceinline__ int place_in_chain(unsigned long long *work, int chain, int tiles, unsigned &number) {
  if (tiles == 1) return 0;
  if (threadIdx.x == 0) number = (unsigned)atomicAdd(work + chain * words_of_chain(tiles), 1ull);
  __syncthreads();
  return __builtin_amdgcn_readfirstlane(number);
}

// The pairs of two channels next to each other, and the state behind them.
__device__ __forceinline__ void apply_pairs(const float2 *p, float (&h)[2]) {
  const float4 v = *reinterpret_cast<const float4 *>(p);
  h[0] = fmaf(v.x, h[0], v.y), h[1] = fmaf(v.z, h[1], v.w);
}

// What was computed from r before is not kept for later, it is computed again: registers are what limits the waves of a compute unit.
template <typename R>
__device__ __forceinline__ R forget(R r) {
  using Bits = std::conditional_t<sizeof(R) == 4, unsigned, unsigned long long>;
  Bits b = __builtin_bit_cast(Bits, r);
  asm("" : "+v"(b));
  return __builtin_bit_cast(R, b);
}

__device__ __forceinline__ float other_half(float v) { return __shfl_xor(v, 32, 64); }

// WHOLE: all tokens of the tile are the sequence's own: no place is moved, nothing is masked.
template <typename T, bool GATED, bool WHOLE, int HOW, bool FAR, int W>
__device__ __forceinline__ void fwd_tile(const FwdArgs &P, Shared<W> &S, int tile, int chain, const Lane &q, int len) {
  constexpr int L = kFwdL, TILE = 2 * W * L;
  const int slice = chain % P.slices, b = chain / P.slices;
  const Chain links = chain_of(P.work, chain, P.tiles);
  const int cl = (threadIdx.x & 31) * 2, grp = threadIdx.x >> 5, wave = threadIdx.x >> 6;
  const bool upper = threadIdx.x & 32;
  const int t0 = tile * TILE, tk = t0 + grp * L, first = t0 + __builtin_amdgcn_readfirstlane(wave) * 2 * L;      // the wave's first token
  const Place<T, L, WHOLE> u(P.u, b * P.ub, P.us, t0, slice, q, P.len), g(P.g, b * P.gb, P.gs, t0, slice, q, P.len);
  const Place<T, L, WHOLE> o(P.o, b * P.ob, P.os, t0, slice, q, P.len), y(P.y, b * P.yb, P.ys, t0, slice, q, P.len);
  // reads come back in order: what is needed first goes first
  float bias[2] = {0.f, 0.f};
  if (P.bias) floats2<HOW>(P.bias, q, bias);
  Raw<T> ur[L], gr[L], orr[L];
  if (WHOLE || first < len) {
#pragma unroll
    for (int i = 0; i < L; ++i) gr[i] = raw2<T, HOW, FAR>(g.at(i), q), ur[i] = raw2<T, HOW, FAR>(u.at(i), q);
    if (GATED) {
#pragma unroll
      for (int i = 0; i < L; ++i) orr[i] = raw2<T, HOW, FAR>(o.at(i), q);
    }
  } else {                   // behind the sequence: nothing to read, only zeros to write (in the sequence's tokens) and the state to pass on
#pragma unroll
    for (int i = 0; i < L; ++i) gr[i] = ur[i] = orr[i] = Raw<T>{};
  }
  Words<early_words(W)> words;
  if (wave == 0) words = look_early<early_words(W)>(links, tile);
  float a[L][2], bb[L][2], A[2] = {1.f, 1.f}, B[2] = {0.f, 0.f}, Ae[2], Be[2];
#pragma unroll
  for (int i = 0; i < L; ++i) {
    const bool live = WHOLE || tk + i < len;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      float z;
      sigmoids(static_cast<float>(gr[i][k]) + bias[k], a[i][k], z);
      bb[i][k] = live ? z * static_cast<float>(ur[i][k]) : 0.f;
      a[i][k] = live ? a[i][k] : 1.f;
      B[k] = fmaf(a[i][k], B[k], bb[i][k]);
      A[k] *= a[i][k];
    }
  }
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const float A1 = other_half(A[k]), B1 = other_half(B[k]);
    Ae[k] = upper ? A1 : 1.f, Be[k] = upper ? B1 : 0.f;
    if (upper) S.tot[wave][cl + k] = make_float2(A[k] * A1, fmaf(A[k], B1, B[k]));
  }
  __syncthreads();
  const int ch = threadIdx.x & 63, c = slice * kSlice + ch;
  if (wave == 0) {
    float At = 1.f, Bt = 0.f, first = 0.f;                 // the whole tile's pair, channel ch
#pragma unroll
    for (int w = 0; w < W; ++w) Bt = fmaf(S.tot[w][ch].x, Bt, S.tot[w][ch].y), At *= S.tot[w][ch].x;
    if (tile == 0 && P.h0) first = P.h0[(long long)b * P.D + (c < P.D ? c : P.D - 1)];
    if (tile + 1 < P.tiles) publish_pair(links, tile, At, Bt, first);
    S.at[ch] = look_back(links, tile, tile + 1 == P.tiles, At, Bt, first, words);
  } else if (wave == 1) {
    float2 v = make_float2(1.f, 0.f);
#pragma unroll
    for (int w = 0; w < W; ++w) {
      S.part[w][ch] = v;
      v = make_float2(v.x * S.tot[w][ch].x, fmaf(S.tot[w][ch].x, v.y, S.tot[w][ch].y));
    }
  }
  __syncthreads();
  float h[2] = {S.at[cl], S.at[cl + 1]};
  apply_pairs(&S.part[wave][cl], h);
#pragma unroll
  for (int k = 0; k < 2; ++k) h[k] = fmaf(Ae[k], h[k], Be[k]);
  if (P.saved && (grp * L) % kSaved == 0 && tk < P.len)
    put_floats2<HOW>(P.saved + (b * ((P.len + kSaved - 1) / kSaved) + tk / kSaved) * P.D, q, h);
  if (q.n == 0) return;
#pragma unroll
  for (int i = 0; i < L; ++i) {
    float out[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      h[k] = fmaf(a[i][k], h[k], bb[i][k]);
      out[k] = h[k];
      if (GATED) {
        const float ov = static_cast<float>(orr[i][k]);
        out[k] *= ov * sigmoid(ov);
      }
      out[k] = WHOLE || tk + i < len ? out[k] : 0.f;
    }
    if (WHOLE || tk + i < P.len) put2<T, HOW, FAR>(y.at(i), q, out);
  }
  if (P.hT && tile + 1 == P.tiles && grp == 2 * W - 1) put_floats2<HOW>(P.hT + (long long)b * P.D, q, h);
}

template <typename T, bool GATED, bool FAR, int W>
__global__ __launch_bounds__(64 * W, sizeof(T) == 4 ? 3 : 4) void recurrence_fwd_kernel(FwdArgs P) {
  __shared__ Shared<W> S;
  const int chain = chain_of_workgroup(blockIdx.x, P.batch * P.slices);
  const int tile = place_in_chain(P.work, chain, P.tiles, S.number);
  const Lane q = lane_of(chain % P.slices, P.D);
  const int len = length_of(P.lengths, chain / P.slices, P.len);
  if (FAR) {                 // rows are whole cache lines
    if ((tile + 1) * (2LL * W * kFwdL) > len) fwd_tile<T, GATED, false, PAIRS, FAR, W>(P, S, tile, chain, q, len);
    else fwd_tile<T, GATED, true, PAIRS, FAR, W>(P, S, tile, chain, q, len);
  } else if (P.D == 1) {
    fwd_tile<T, GATED, false, SINGLE, false, W>(P, S, tile, chain, q, len);
  } else if ((tile + 1) * (2LL * W * kFwdL) > len) {
    fwd_tile<T, GATED, false, ODD, false, W>(P, S, tile, chain, q, len);
  } else if (q.odd) {
    fwd_tile<T, GATED, true, ODD, false, W>(P, S, tile, chain, q, len);
  } else {
    fwd_tile<T, GATED, true, PAIRS, false, W>(P, S, tile, chain, q, len);
  }
}

// A tile of W waves, which share three roles between them.
template <typename T, bool GATED, bool WHOLE, int HOW, bool FAR, int W>
__device__ __forceinline__ void bwd_tile(const BwdArgs &P, Shared<W> &S, int pos, int chain, const Lane &q, int len) {
  constexpr int L = kBwdL, TILE = 2 * W * L;
  const auto mine = [](int role) { return W == 1 || (int)(threadIdx.x >> 6) == role % W; };
  const int slice = chain % P.slices, b = chain / P.slices;
  const int tile = P.tiles - 1 - pos;       // the chain starts at the last tile
  const Chain links = chain_of(P.work, chain, P.tiles);
  const int cl = (threadIdx.x & 31) * 2, grp = threadIdx.x >> 5, wave = threadIdx.x >> 6;
  const bool upper = threadIdx.x & 32;
  const int t0 = tile * TILE, tk = t0 + grp * L, first = t0 + __builtin_amdgcn_readfirstlane(wave) * 2 * L;      // the wave's first token
  const Place<T, L, WHOLE> u(P.u, b * P.ub, P.us, t0, slice, q, P.len), g(P.g, b * P.gb, P.gs, t0, slice, q, P.len);
  const Place<T, L, WHOLE> o(P.o, b * P.ob, P.os, t0, slice, q, P.len), dy(P.dy, b * P.yb, P.ys, t0, slice, q, P.len);
  float bias[2] = {0.f, 0.f}, db[2] = {0.f, 0.f}, saved = 0.f;
  if (P.bias) floats2<HOW>(P.bias, q, bias);
  Raw<T> ur[L], gr[L], orr[L], yr[L];
  if (WHOLE || first < len) {
#pragma unroll
    for (int i = 0; i < L; ++i) gr[i] = raw2<T, HOW, FAR>(g.at(i), q), ur[i] = raw2<T, HOW, FAR>(u.at(i), q);
#pragma unroll
    for (int i = L - 1; i >= 0; --i) {
      yr[i] = raw2<T, HOW, FAR>(dy.at(i), q);
      if (GATED) orr[i] = raw2<T, HOW, FAR>(o.at(i), q);
    }
  } else {
#pragma unroll
    for (int i = 0; i < L; ++i) gr[i] = ur[i] = orr[i] = yr[i] = Raw<T>{};
  }
  const int ch = threadIdx.x & 63, cc = slice * kSlice + ch;
  if (mine(2)) saved = P.saved[(b * ((P.len + kSaved - 1) / kSaved) + t0 / kSaved) * P.D + (cc < P.D ? cc : P.D - 1)];
  Words<early_words(W)> words;
  if (wave == 0) words = look_early<early_words(W)>(links, pos);
  if (!WHOLE) {
#pragma unroll
    for (int i = 0; i < L; ++i)
      if (tk + i >= len) {
        ur[i][0] = ur[i][1] = yr[i][0] = yr[i][1] = T(0.f);
        if (GATED) orr[i][0] = orr[i][1] = T(0.f);
      }
  }
  float a[L][2], z[L][2], hb[L][2], sg[L][2];
  float A[2] = {1.f, 1.f}, B[2] = {0.f, 0.f}, Br[2] = {0.f, 0.f}, Ae[2], Be[2], Ax[2], Bx[2];
#pragma unroll
  for (int i = 0; i < L; ++i) {
    const bool live = WHOLE || tk + i < len;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      sigmoids(static_cast<float>(gr[i][k]) + bias[k], a[i][k], z[i][k]);
      if (!live) a[i][k] = 1.f, z[i][k] = 0.f;
      B[k] = fmaf(a[i][k], B[k], z[i][k] * static_cast<float>(ur[i][k]));
      A[k] *= a[i][k];
    }
  }
#pragma unroll
  for (int i = L - 1; i >= 0; --i)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const float ov = GATED ? static_cast<float>(orr[i][k]) : 0.f, yv = static_cast<float>(yr[i][k]);
      sg[i][k] = GATED ? sigmoid(ov) : 1.f;
      const float c = GATED ? yv * (ov * sg[i][k]) : yv;
      Br[k] = i == L - 1 ? c : fmaf(a[i + 1 < L ? i + 1 : i][k], Br[k], c);      // dh
    }
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    Br[k] *= a[0][k];
    const float A1 = other_half(A[k]), B1 = other_half(B[k]), R1 = other_half(Br[k]);
    Ae[k] = upper ? A1 : 1.f, Be[k] = upper ? B1 : 0.f;
    Ax[k] = upper ? 1.f : A1, Bx[k] = upper ? 0.f : R1;
    if (upper) S.tot[wave][cl + k] = make_float2(A[k] * A1, fmaf(A[k], B1, B[k]));
    else S.back[wave][cl + k] = make_float2(A[k] * A1, fmaf(A[k], R1, Br[k]));
  }
  __syncthreads();
  if (mine(0)) {
    float At = 1.f, Bt = 0.f, first = 0.f;
#pragma unroll
    for (int w = W - 1; w >= 0; --w) Bt = fmaf(S.back[w][ch].x, Bt, S.back[w][ch].y), At *= S.back[w][ch].x;
    if (pos == 0 && P.dhT) first = P.dhT[(long long)b * P.D + (cc < P.D ? cc : P.D - 1)];
    if (tile > 0) publish_pair(links, pos, At, Bt, first);
    S.at[ch] = look_back(links, pos, tile == 0, At, Bt, first, words);
  }
  if (mine(1)) {
    float2 v = make_float2(1.f, 0.f);
#pragma unroll
    for (int w = W - 1; w >= 0; --w) {
      S.part[w][ch] = v;
      v = make_float2(v.x * S.back[w][ch].x, fmaf(S.back[w][ch].x, v.y, S.back[w][ch].y));
    }
  }
  if (mine(2)) {
    float v = saved;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      S.h[w][ch] = v;
      v = fmaf(S.tot[w][ch].x, v, S.tot[w][ch].y);
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < L; ++i) {
    ur[i] = forget(ur[i]), yr[i] = forget(yr[i]);
    if (GATED) orr[i] = forget(orr[i]);
  }
  float h[2] = {S.h[wave][cl], S.h[wave][cl + 1]}, e[2] = {S.at[cl], S.at[cl + 1]};
  apply_pairs(&S.part[wave][cl], e);
#pragma unroll
  for (int k = 0; k < 2; ++k) h[k] = fmaf(Ae[k], h[k], Be[k]), e[k] = fmaf(Ax[k], e[k], Bx[k]);
#pragma unroll
  for (int i = 0; i < L; ++i)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      hb[i][k] = h[k];
      h[k] = fmaf(a[i][k], h[k], z[i][k] * static_cast<float>(ur[i][k]));
    }
  const Place<T, L, WHOLE> du(P.du, b * P.dub, P.dus, t0, slice, q, P.len), dgp(P.dg, b * P.dgb, P.dgs, t0, slice, q, P.len);
  const Place<T, L, WHOLE> dop(P.dou, b * P.dob, P.dos, t0, slice, q, P.len);
  if (q.n > 0) {
    float dh[2];
#pragma unroll
    for (int i = L - 1; i >= 0; --i) {
      float dv[2], dg[2], dou[2];
      const bool live = WHOLE || tk + i < len;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const float s = sg[i][k], yv = static_cast<float>(yr[i][k]), ov = GATED ? static_cast<float>(orr[i][k]) : 0.f, t = ov * s;
        const float hi = i + 1 < L ? hb[i + 1 < L ? i + 1 : i][k] : h[k], in = i == L - 1 ? e[k] : a[i + 1 < L ? i + 1 : i][k] * dh[k];
        dh[k] = GATED ? fmaf(yv, t, in) : yv + in;
        dv[k] = live ? z[i][k] * dh[k] : 0.f;
        dg[k] = live ? (hb[i][k] - static_cast<float>(ur[i][k])) * a[i][k] * dv[k] : 0.f;
        if (GATED) dou[k] = live ? yv * hi * fmaf(t, 1.f - s, s) : 0.f;
        db[k] += dg[k];
      }
      if (WHOLE || tk + i < P.len) {
        put2<T, HOW, FAR>(du.at(i), q, dv);
        put2<T, HOW, FAR>(dgp.at(i), q, dg);
        if (GATED) put2<T, HOW, FAR>(dop.at(i), q, dou);
      }
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) e[k] = a[0][k] * dh[k];
  }
  if (P.dh0 && tile == 0 && grp == 0) put_floats2<HOW>(P.dh0 + (long long)b * P.D, q, e);
  if (P.dbias_partial) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const float v = db[k] + other_half(db[k]);
      if (!upper) S.h[wave][cl + k] = v;        // each wave's own, which only it read
    }
    __syncthreads();
    if (wave == 0 && cc < P.D) {
      float v = S.h[0][ch];
#pragma unroll
      for (int w = 1; w < W; ++w) v += S.h[w][ch];
      P.dbias_partial[((long long)b * P.tiles + tile) * P.D + cc] = v;
    }
  }
}

template <typename T, bool GATED, bool FAR, int W>
__global__ __launch_bounds__(64 * W, W == 8 ? 4 : sizeof(T) == 4 ? 2 : 3) void recurrence_bwd_kernel(BwdArgs P) {
  __shared__ Shared<W> S;
  const int chain = chain_of_workgroup(blockIdx.x, P.batch * P.slices);
  const int pos = place_in_chain(P.work, chain, P.tiles, S.number);
  const Lane q = lane_of(chain % P.slices, P.D);
  const int len = length_of(P.lengths, chain / P.slices, P.len);
  if (FAR) {                 // rows are whole cache lines
    if ((P.tiles - pos) * (2LL * W * kBwdL) > len) bwd_tile<T, GATED, false, PAIRS, FAR, W>(P, S, pos, chain, q, len);
    else bwd_tile<T, GATED, true, PAIRS, FAR, W>(P, S, pos, chain, q, len);
  } else if (P.D == 1) {
    bwd_tile<T, GATED, false, SINGLE, false, W>(P, S, pos, chain, q, len);
  } else if ((P.tiles - pos) * (2LL * W * kBwdL) > len) {
    bwd_tile<T, GATED, false, ODD, false, W>(P, S, pos, chain, q, len);
  } else if (q.odd) {
    bwd_tile<T, GATED, true, ODD, false, W>(P, S, pos, chain, q, len);
  } else {
    bwd_tile<T, GATED, true, PAIRS, false, W>(P, S, pos, chain, q, len);
  }
}

// One thread takes four channels of a sequence through its tokens, one after the other: single tokens and short pieces, for which a
// tile of 128 tokens would be mostly empty.  Bound by latency, with many sequences by memory (256x24x4096 31 us, 6.6 TB/s out of the
// last-level cache).  Measured in us, steps against tiles (bf16, with the output gate):
//   tokens         16            24            32            48            64
//   1x1280      4.7 /  6.8    6.3 /  6.7    7.9 /  6.7   11.1 /  6.8   14.4 /  6.9
//   32x2048        -          6.8 /  9.0    8.5 /  8.9   11.9 / 10.1   15.6 / 11.3
//   64x2048     5.5 / 15.0    7.3 / 15.4    9.3 / 16.1   15.7 / 20.3   19.9 / 22.8
//   256x4096   21.6 / 97.5   30.6 / 98.3   40.3 /  131   84.5 /  161    113 /  172
// All of these have channels in fours.  Otherwise the last thread of a sequence goes token by token, three reads after another, which was
// not measured against tiles.
constexpr int kFewChains = 128, kLongChain = 8192;
constexpr int kFewSteps = 24, kManyThreads = 32768;
constexpr int kAhead = 8;      // tokens on their way together (4: 5.0 against 4.7 us for 1x16x1280)
template <typename T, bool GATED>
__global__ __launch_bounds__(64) void recurrence_step_kernel(FwdArgs P) {
  using Four = typename VecOf<T, 4>::type;
  const int quads = (P.D + 3) / 4;
  const long long id = (long long)blockIdx.x * 64 + threadIdx.x;
  const int b = (int)(id / quads), c = (int)(id % quads) * 4, n = P.D - c < 4 ? P.D - c : 4;
  if (b >= P.batch) return;
  const int len = length_of(P.lengths, b, P.len);
  const T *u = static_cast<const T *>(P.u) + b * P.ub + c, *g = static_cast<const T *>(P.g) + b * P.gb + c, *o = static_cast<const T *>(P.o) + b * P.ob + c;
  T *y = static_cast<T *>(P.y) + b * P.yb + c;
  float h[4] = {0.f, 0.f, 0.f, 0.f}, bias[4] = {0.f, 0.f, 0.f, 0.f};
  if (P.h0) load_n<float, 4>(P.h0 + (long long)b * P.D + c, n, h);
  if (P.bias) load_n<float, 4>(P.bias + c, n, bias);
  auto token = [&](const float (&uv)[4], const float (&gv)[4], const float (&ov)[4], float (&out)[4]) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      float a, z;
      sigmoids(gv[k] + bias[k], a, z);
      h[k] = fmaf(a, h[k], z * uv[k]);
      out[k] = h[k];
      if (GATED) out[k] *= ov[k] * sigmoid(ov[k]);
    }
  };
  if (P.saved) store_n<float, 4>(P.saved + (long long)b * P.D + c, n, h);
  static_assert(kMostSteps <= kSaved, "one saved state");
  // kAhead tokens from t on; those behind the last are the last again and not used
  auto tokens = [&](auto whole, int t) {
    constexpr int N = kAhead;
    Four ur[N], gr[N], orr[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int at = whole.value || t + i < len ? t + i : len - 1;
      gr[i] = far_load<false, T, 4>(g + at * P.gs), ur[i] = far_load<false, T, 4>(u + at * P.us);
      if (GATED) orr[i] = far_load<false, T, 4>(o + at * P.os);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (!whole.value && t + i >= len) return;
      float uv[4], gv[4], ov[4] = {}, out[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) uv[k] = static_cast<float>(ur[i][k]), gv[k] = static_cast<float>(gr[i][k]), ov[k] = GATED ? static_cast<float>(orr[i][k]) : 0.f;
      token(uv, gv, ov, out);
      store_n<T, 4>(y + (t + i) * P.ys, 4, out);
    }
  };
  int t = 0;
  if (n == 4) {
    for (; t + kAhead <= len; t += kAhead) tokens(std::true_type{}, t);
    if (t + 1 < len) tokens(std::false_type{}, t), t = len;
  }
  for (; t < P.len; ++t) {
    float out[4] = {0.f, 0.f, 0.f, 0.f};
    if (t < len) {
      float uv[4], gv[4], ov[4] = {};
      load_n<T, 4>(g + t * P.gs, n, gv);
      load_n<T, 4>(u + t * P.us, n, uv);
      if (GATED) load_n<T, 4>(o + t * P.os, n, ov);
      token(uv, gv, ov, out);
    }
    store_n<T, 4>(y + t * P.ys, n, out);
  }
  if (P.hT) store_n<float, 4>(P.hT + (long long)b * P.D + c, n, h);
}

// The states' gradient of sequences without tokens.
__global__ __launch_bounds__(256) void copy_or_zero_kernel(const float *from, float *to, long long n) {
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  if (i < n) to[i] = from ? from[i] : 0.f;
}

void clear_words(unsigned long long *p, long long n, hipStream_t st) {
  const long long blocks = cdiv64(n, 512);
  clear_words_kernel<<<(unsigned)(blocks < 2048 ? blocks : 2048), 256, 0, st>>>(p, n);
}

// Whether a tile's rows in this tensor are whole cache lines.
inline bool lines(const void *p, long long batch_stride, long long stride, int size) {
  return ((reinterpret_cast<uintptr_t>(p) | (uintptr_t)(batch_stride * size) | (uintptr_t)(stride * size)) & 127) == 0;
}

// Whether tiles have eight waves.  A chain hands its state from segment to segment, about 0.75 us each (1x131072x64: 128 segments in 94 us, 64
// in 53); few long chains are bound by that, and tiles of twice the tokens halve it.  Many chains hide it, and want small workgroups.  Measured in us, four / eight waves (bf16 with the output gate):
//                     chains  forward     backward                           chains  forward     backward
//   1x131072x64          1     94 /  53   156 /  88      8x8192x512            64     63 /  59   115 / 104
//   1x65536x1280        20    147 / 128   282 / 237      4x16384x1280          80    137 / 127   264 / 237
//   1x16384x1280        20   47.3 / 47.8 79.7 / 69.5     8x8192x1280          160    134 / 131   252 / 245
//   1x65536x4096        64    428 / 396   799 / 724      8x8192x2048          256    193 / 200
// fp32 stays with four: its registers leave a compute unit one workgroup of eight waves, 1x65536x1280 forward 244 / 249.  Fewer or shorter
// chains would gain there too, 1x65536x320 79.5 / 73.4 and 1x1024x1280 16.8 / 15.8; no rule has been measured that parts the two.
inline bool tall_tiles(int batch, long long len, int slices, int size) { return size == 2 && (long long)batch * slices <= kFewChains && len >= kLongChain; }

template <typename T>
hipError_t launch_fwd(FwdArgs A, hipStream_t st) {
  const long long threads = (long long)A.batch * ((A.D + 3) / 4);
  if (A.len <= kFewSteps || (A.len <= kMostSteps && threads >= kManyThreads)) {
    const unsigned blocks = (unsigned)cdiv64(threads, 64);
    if (A.o) recurrence_step_kernel<T, true><<<blocks, 64, 0, st>>>(A);
    else recurrence_step_kernel<T, false><<<blocks, 64, 0, st>>>(A);
  } else {
    const int size = sizeof(T);
    const bool far = (double)A.batch * A.len * A.D * size * (A.o ? 4 : 3) > kLastLevelCache && A.D * size % 128 == 0 && lines(A.u, A.ub, A.us, size) && lines(A.g, A.gb, A.gs, size) && (!A.o || lines(A.o, A.ob, A.os, size));
    const int waves = tall_tiles(A.batch, A.len, A.slices, size) ? 8 : 4;
    A.tiles = (int)cdiv64(A.len, 2 * waves * kFwdL);
    const unsigned grid = (unsigned)A.batch * A.slices * A.tiles;
    if (A.tiles > 1) clear_words(A.work, (long long)A.batch * A.slices * words_of_chain(A.tiles), st);
    if constexpr (sizeof(T) == 2) {
      if (waves == 8) {
        if (A.o && far) recurrence_fwd_kernel<T, true, true, 8><<<grid, 512, 0, st>>>(A);
        else if (A.o) recurrence_fwd_kernel<T, true, false, 8><<<grid, 512, 0, st>>>(A);
        else if (far) recurrence_fwd_kernel<T, false, true, 8><<<grid, 512, 0, st>>>(A);
        else recurrence_fwd_kernel<T, false, false, 8><<<grid, 512, 0, st>>>(A);
        return hipGetLastError();
      }
    }
    if (A.o && far) recurrence_fwd_kernel<T, true, true, 4><<<grid, 256, 0, st>>>(A);
    else if (A.o) recurrence_fwd_kernel<T, true, false, 4><<<grid, 256, 0, st>>>(A);
    else if (far) recurrence_fwd_kernel<T, false, true, 4><<<grid, 256, 0, st>>>(A);
    else recurrence_fwd_kernel<T, false, false, 4><<<grid, 256, 0, st>>>(A);
  }
  return hipGetLastError();
}

// Short sequences take tiles of fewer waves, of which more fit on a compute unit.  Measured in us, four waves against one (16 tokens) or two
// (32): bf16 with the output gate, 1x16x1280 6.3 / 4.5, 64x16x2048 19.4 / 7.5, 256x16x4096 127 / 38;
// 1x32x1280 6.4 / 4.7, 64x32x2048 21.7 / 14.1, 256x32x4096 109 / 101, 256x17x4096 137 / 77.
inline int bwd_waves(int batch, long long len, int slices, int size) {
  return len <= 2 * kBwdL ? 1 : len <= 4 * kBwdL ? 2 : tall_tiles(batch, len, slices, size) ? 8 : 4;
}
inline long long bwd_tiles(int batch, long long len, int channels, int size) { return cdiv64(len, 2 * bwd_waves(batch, len, cdiv(channels, kSlice), size) * kBwdL); }

template <typename T>
hipError_t launch_bwd(const BwdArgs &A, hipStream_t st) {
  const unsigned grid = (unsigned)A.batch * A.slices * A.tiles;
  const int size = sizeof(T);
  const bool far = (double)A.batch * A.len * A.D * size * (A.o ? 7 : 5) > kLastLevelCache && A.D * size % 128 == 0 && lines(A.u, A.ub, A.us, size) && lines(A.g, A.gb, A.gs, size) && lines(A.dy, A.yb, A.ys, size) &&
                     (!A.o || lines(A.o, A.ob, A.os, size));
  if (A.tiles > 1) clear_words(A.work, (long long)A.batch * A.slices * words_of_chain(A.tiles), st);
  const int waves = bwd_waves(A.batch, A.len, A.slices, size);
  if (A.o && waves == 1) recurrence_bwd_kernel<T, true, false, 1><<<grid, 64, 0, st>>>(A);
  else if (waves == 1) recurrence_bwd_kernel<T, false, false, 1><<<grid, 64, 0, st>>>(A);
  else if (A.o && waves == 2) recurrence_bwd_kernel<T, true, false, 2><<<grid, 128, 0, st>>>(A);
  else if (waves == 2) recurrence_bwd_kernel<T, false, false, 2><<<grid, 128, 0, st>>>(A);
  else if (waves == 8) {
    if constexpr (sizeof(T) == 2) {
      if (A.o && far) recurrence_bwd_kernel<T, true, true, 8><<<grid, 512, 0, st>>>(A);
      else if (A.o) recurrence_bwd_kernel<T, true, false, 8><<<grid, 512, 0, st>>>(A);
      else if (far) recurrence_bwd_kernel<T, false, true, 8><<<grid, 512, 0, st>>>(A);
      else recurrence_bwd_kernel<T, false, false, 8><<<grid, 512, 0, st>>>(A);
    }
  } else if (A.o && far) recurrence_bwd_kernel<T, true, true, 4><<<grid, 256, 0, st>>>(A);
  else if (A.o) recurrence_bwd_kernel<T, true, false, 4><<<grid, 256, 0, st>>>(A);
  else if (far) recurrence_bwd_kernel<T, false, true, 4><<<grid, 256, 0, st>>>(A);
  else recurrence_bwd_kernel<T, false, false, 4><<<grid, 256, 0, st>>>(A);
  return hipGetLastError();
}

inline bool off(const void *p, int size) { return (reinterpret_cast<uintptr_t>(p) & (size - 1)) != 0; }

inline bool sizes_ok(int batch, long long len, int channels) {
  if (batch < 0 || len < 0 || channels < 1 || (long long)batch * channels > 0x7fffffffLL || len > 0x7fffffffLL) return false;
  const long long chains = (long long)batch * cdiv(channels, kSlice);
  return chains <= (1LL << 22) && chains * cdiv64(len, kSaved) <= (1LL << 22);     // a launch's threads must stay below 2^32
}

// The workspace: the chains' words (the backward pass has the more and shorter tiles), then the bias gradient's partials, one row for
// each backward tile of a sequence, and what their sums need.
inline size_t work_bytes(int batch, long long len, int channels) {
  return (size_t)batch * cdiv(channels, kSlice) * words_of_chain(cdiv64(len, kSaved)) * 8;
}
inline size_t partial_floats(int batch, long long len, int channels) { return (size_t)batch * cdiv64(len, kSaved) * channels; }

pbkd_status check_sizes(int batch, long long len, int channels, int dtype) {
  if (batch < 0 || len < 0 || channels < 1) return set_error(PBKD_ESHAPE, "recurrence: [%d, %lld, %d]", batch, len, channels);
  if (!sizes_ok(batch, len, channels)) return set_error(PBKD_EUNSUPPORTED, "recurrence: [%d, %lld, %d] is too large", batch, len, channels);
  if (dtype != PBKD_F32 && dtype != PBKD_BF16 && dtype != PBKD_F16) return set_error(PBKD_EINVAL, "recurrence: dtype %d", dtype);
  return PBKD_OK;
}

// Whether the strides between tokens are what the tiles take (a single token has none).
inline bool strides_ok(long long len, std::initializer_list<long long> strides) {
  for (long long s : strides)
    if (len > 1 && s > kMaxStride) return false;
  return true;
}

// Whether an output's rows are apart from each other, sequences in front of tokens or tokens in front of sequences.
inline bool apart(int batch, long long len, int D, long long bs, long long ts) {
  if (bs < 0 || ts < 0) return false;
  if (len > 1 && ts < D) return false;
  if (batch > 1 && bs < D) return false;
  if (batch > 1 && len > 1 && bs < (len - 1) * ts + D && ts < (batch - 1) * bs + D) return false;
  return true;
}

pbkd_status forward(const pbkd_recurrence_desc *q, bool step, void *hip_stream) {
  if (!q) return set_error(PBKD_EINVAL, "recurrence: null descriptor");
  const long long len = step ? 1 : q->len;
  if (const pbkd_status s = check_sizes(q->batch, len, q->channels, q->dtype)) return s;
  if (step && (!q->state_dev || !q->state_out_dev)) return set_error(PBKD_EINVAL, "recurrence: a step needs the state and where it goes");
  const int size = q->dtype == PBKD_F32 ? 4 : 2;
  const bool any = q->batch > 0 && len > 0;
  if (any && (!q->u_dev || !q->gate_dev || !q->y_dev)) return set_error(PBKD_EINVAL, "recurrence: null tensor");
  if (off(q->u_dev, size) || off(q->gate_dev, size) || off(q->out_gate_dev, size) || off(q->y_dev, size) || off(q->bias_dev, 4) || off(q->lengths_dev, 4) ||
      off(q->state_dev, 4) || off(q->state_out_dev, 4))
    return set_error(PBKD_EINVAL, "recurrence: a tensor is not aligned to its elements");
  if (q->u_stride < 0 || q->u_batch_stride < 0 || q->gate_stride < 0 || q->gate_batch_stride < 0 || q->out_gate_stride < 0 || q->out_gate_batch_stride < 0)
    return set_error(PBKD_EINVAL, "recurrence: negative stride");
  if (!strides_ok(len, {q->u_stride, q->gate_stride, q->out_gate_stride, q->y_stride})) return set_error(PBKD_EUNSUPPORTED, "recurrence: tokens more than 2^25 elements apart");
  if (any && !apart(q->batch, len, q->channels, q->y_batch_stride, q->y_stride)) return set_error(PBKD_ESHAPE, "recurrence: rows of y overlap");
  if (!step && q->saved_dev) {
    if (off(q->saved_dev, 4)) return set_error(PBKD_EINVAL, "recurrence: a tensor is not aligned to its elements");
    if (q->saved_bytes < pbkd_recurrence_saved_bytes(q->batch, len, q->channels))
      return set_error(PBKD_ENOMEM, "recurrence: saved_dev of %zu bytes is smaller than the %zu needed", q->saved_bytes, pbkd_recurrence_saved_bytes(q->batch, len, q->channels));
  }
  if (!step) {
    if (!q->workspace_dev || off(q->workspace_dev, 256)) return set_error(PBKD_ENOMEM, "recurrence: the workspace must be 256-byte aligned");
    if (q->workspace_bytes < pbkd_recurrence_workspace_bytes(q->batch, len, q->channels))
      return set_error(PBKD_ENOMEM, "recurrence: workspace of %zu bytes is smaller than the %zu needed", q->workspace_bytes,
                       pbkd_recurrence_workspace_bytes(q->batch, len, q->channels));
  }
  if (q->batch == 0) return PBKD_OK;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (len == 0) {
    const long long n = (long long)q->batch * q->channels;
    if (q->state_out_dev) copy_or_zero_kernel<<<(unsigned)cdiv64(n, 256), 256, 0, st>>>(q->state_dev, q->state_out_dev, n);
    SEQ_HIPCHK(hipGetLastError());
    return PBKD_OK;
  }
  FwdArgs A{q->u_dev, q->gate_dev, q->out_gate_dev, q->bias_dev, q->lengths_dev, q->state_dev, q->state_out_dev, q->y_dev,
            step ? nullptr : static_cast<float *>(q->saved_dev), static_cast<unsigned long long *>(q->workspace_dev), len, q->u_batch_stride, q->u_stride, q->gate_batch_stride, q->gate_stride,
            q->out_gate_batch_stride, q->out_gate_stride, q->y_batch_stride, q->y_stride, q->batch, q->channels, cdiv(q->channels, kSlice),
            (int)cdiv64(len, 8 * kFwdL)};
  switch (q->dtype) {
    case PBKD_F32: SEQ_HIPCHK(launch_fwd<float>(A, st)); break;
    case PBKD_BF16: SEQ_HIPCHK(launch_fwd<bf16>(A, st)); break;
    default: SEQ_HIPCHK(launch_fwd<f16>(A, st)); break;
  }
  return PBKD_OK;
}

}  // namespace
}  // namespace pbkd

using namespace pbkd;

extern "C" {

size_t pbkd_recurrence_saved_bytes(int batch, long long len, int channels) {
  if (!sizes_ok(batch, len, channels)) return 0;
  return (size_t)batch * cdiv64(len, kSaved) * channels * sizeof(float) + 256;
}

size_t pbkd_recurrence_workspace_bytes(int batch, long long len, int channels) {
  if (!sizes_ok(batch, len, channels)) return 0;
  return work_bytes(batch, len, channels) + partial_floats(batch, len, channels) * sizeof(float) +
         colsum_scratch_floats((long long)batch * cdiv64(len, kSaved), channels) * sizeof(float) + 256;
}

pbkd_status pbkd_recurrence_forward(const pbkd_recurrence_desc *desc, void *hip_stream) { return forward(desc, false, hip_stream); }

pbkd_status pbkd_recurrence_step(const pbkd_recurrence_desc *desc, void *hip_stream) { return forward(desc, true, hip_stream); }

pbkd_status pbkd_recurrence_backward(const pbkd_recurrence_grad_desc *q, void *hip_stream) {
  if (!q) return set_error(PBKD_EINVAL, "recurrence: null descriptor");
  if (const pbkd_status s = check_sizes(q->batch, q->len, q->channels, q->dtype)) return s;
  const int size = q->dtype == PBKD_F32 ? 4 : 2;
  const bool any = q->batch > 0 && q->len > 0;
  if (any && (!q->u_dev || !q->gate_dev || !q->dy_dev || !q->du_dev || !q->dgate_dev || !q->saved_dev)) return set_error(PBKD_EINVAL, "recurrence: null tensor");
  if ((q->out_gate_dev != nullptr) != (q->dout_gate_dev != nullptr)) return set_error(PBKD_EINVAL, "recurrence: out_gate and dout_gate come together");
  if (off(q->u_dev, size) || off(q->gate_dev, size) || off(q->out_gate_dev, size) || off(q->dy_dev, size) || off(q->du_dev, size) || off(q->dgate_dev, size) ||
      off(q->dout_gate_dev, size) || off(q->bias_dev, 4) || off(q->lengths_dev, 4) || off(q->dstate_out_dev, 4) || off(q->dbias_dev, 4) || off(q->dstate_dev, 4))
    return set_error(PBKD_EINVAL, "recurrence: a tensor is not aligned to its elements");
  if (q->u_stride < 0 || q->u_batch_stride < 0 || q->gate_stride < 0 || q->gate_batch_stride < 0 || q->out_gate_stride < 0 || q->out_gate_batch_stride < 0 ||
      q->dy_stride < 0 || q->dy_batch_stride < 0)
    return set_error(PBKD_EINVAL, "recurrence: negative stride");
  if (!strides_ok(q->len, {q->u_stride, q->gate_stride, q->out_gate_stride, q->dy_stride, q->du_stride, q->dgate_stride, q->dout_gate_stride}))
    return set_error(PBKD_EUNSUPPORTED, "recurrence: tokens more than 2^25 elements apart");
  if (any && (!apart(q->batch, q->len, q->channels, q->du_batch_stride, q->du_stride) || !apart(q->batch, q->len, q->channels, q->dgate_batch_stride, q->dgate_stride) ||
              (q->dout_gate_dev && !apart(q->batch, q->len, q->channels, q->dout_gate_batch_stride, q->dout_gate_stride))))
    return set_error(PBKD_ESHAPE, "recurrence: rows of a gradient overlap");
  if (any && (off(q->saved_dev, 4) || q->saved_bytes < pbkd_recurrence_saved_bytes(q->batch, q->len, q->channels)))
    return set_error(PBKD_ENOMEM, "recurrence: saved_dev is misaligned or smaller than the %zu bytes needed", pbkd_recurrence_saved_bytes(q->batch, q->len, q->channels));
  if (!q->workspace_dev || off(q->workspace_dev, 256)) return set_error(PBKD_ENOMEM, "recurrence: the workspace must be 256-byte aligned");
  if (q->workspace_bytes < pbkd_recurrence_workspace_bytes(q->batch, q->len, q->channels))
    return set_error(PBKD_ENOMEM, "recurrence: workspace of %zu bytes is smaller than the %zu needed", q->workspace_bytes,
                     pbkd_recurrence_workspace_bytes(q->batch, q->len, q->channels));
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  float *partial = reinterpret_cast<float *>(static_cast<char *>(q->workspace_dev) + work_bytes(q->batch, q->len, q->channels));
  const long long tiles = bwd_tiles(q->batch, q->len, q->channels, size);
  if (any) {
    BwdArgs A{q->u_dev, q->gate_dev, q->out_gate_dev, q->dy_dev, q->bias_dev, q->lengths_dev, static_cast<const float *>(q->saved_dev), q->dstate_out_dev,
              q->du_dev, q->dgate_dev, q->dout_gate_dev, q->dbias_dev ? partial : nullptr, q->dstate_dev, static_cast<unsigned long long *>(q->workspace_dev), q->len, q->u_batch_stride, q->u_stride,
              q->gate_batch_stride, q->gate_stride, q->out_gate_batch_stride, q->out_gate_stride, q->dy_batch_stride, q->dy_stride,
              q->du_batch_stride, q->du_stride, q->dgate_batch_stride, q->dgate_stride, q->dout_gate_batch_stride, q->dout_gate_stride,
              q->batch, q->channels, cdiv(q->channels, kSlice), (int)tiles};
    switch (q->dtype) {
      case PBKD_F32: SEQ_HIPCHK(launch_bwd<float>(A, st)); break;
      case PBKD_BF16: SEQ_HIPCHK(launch_bwd<bf16>(A, st)); break;
      default: SEQ_HIPCHK(launch_bwd<f16>(A, st)); break;
    }
  } else if (q->batch > 0 && q->dstate_dev) {
    const long long n = (long long)q->batch * q->channels;
    copy_or_zero_kernel<<<(unsigned)cdiv64(n, 256), 256, 0, st>>>(q->dstate_out_dev, q->dstate_dev, n);
    SEQ_HIPCHK(hipGetLastError());
  }
  if (q->dbias_dev) SEQ_HIPCHK(launch_colsum(partial, any ? q->batch * tiles : 0, q->channels, partial + partial_floats(q->batch, q->len, q->channels), q->dbias_dev, st));
  return PBKD_OK;
}

}  // extern "C"
