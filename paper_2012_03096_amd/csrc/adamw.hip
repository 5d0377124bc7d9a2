// AdamW over many tensors at once, states in 32 or in 8 bits.
//
//   m <- b1 m + (1-b1) g,  v <- b2 v + (1-b2) g^2,  p <- p (1 - lr wd) - (lr/bc1) m / (sqrt(v)/sqrt(bc2) + eps)
//
// One launch takes up to kTensors tensors, whose descriptors travel in the kernel's arguments: nothing has to be copied to
// the device first.  So do the step's own numbers, for which reason a call is refused while its stream is captured.  A workgroup owns a chunk of elements of one tensor, found by a
// search over the tensors' first chunks; four consecutive elements go to a lane, so that a wave's 256 are just one block of
// the 8-bit states and its maximum is a reduction over the wave.
//
// Bound by memory: 67M fp32 parameters with 32-bit states 303 us, 6.2 TB/s; 201M fp32 parameters, bf16 gradients and copies,
// 8-bit states 541 us, 6.0 TB/s.  Smaller calls are bound by the last-level cache and their arithmetic (6M bf16 parameters, 8-bit
// states, 18.0 us), eight tensors of a convolutional block by the host (9.2 us, the kernel takes 5.0).
#include "seq_common.h"

namespace pbkd {
namespace {

constexpr int kBlock = 256;                    // elements that share a scale
// Elements of a workgroup: four waves, of a block each in every round.  Calls that go past the caches are long enough for four rounds;
// others have too few workgroups then (6M bf16 parameters 17.6 against 18.4 us, 201M 553 against 542 us).
constexpr int rounds_of(bool far) { return far ? 4 : 2; }
constexpr int chunk_of(bool far) { return 4 * rounds_of(far) * kBlock; }
constexpr int kTensors = 40;                   // descriptors of a launch: 72 bytes each, below the 4 KB of a kernel's arguments

struct Tensor {
  void *p;
  const void *g;
  void *m, *v;
  float *ms, *vs;
  void *copy;
  long long n;
  unsigned first;                              // of the elements' numbers, for the random numbers
  float decay;                                 // 1 - lr * weight decay
};
struct Launch {
  Tensor t[kTensors];
  unsigned chunk0[kTensors + 1];               // first chunk of each tensor
  unsigned char kind[kTensors];                // parameter type + 2 * gradient type
  int tensors;
  unsigned seed;
  float b1, c1, b2, c2, eps, gscale, step, root;   // c = 1 - b, step = lr / bc1, root = 1 / sqrt(bc2)
};
static_assert(sizeof(Launch) <= 4000, "kernel arguments");

// A random number for each element: multiplications and xor-shifts of its number and the seed.  The shifts and the two factors of
// element_hash are those published with C. Wellons' search for 32-bit mixing functions ("hash prospector"); kMul is a prime next to
// 2^32 over the golden ratio.
constexpr unsigned kMul = 0x9E3779B1u;
__device__ __forceinline__ unsigned element_hash(unsigned x) {       // x = number * kMul + seed * 0x632BE5AB
  x = (x ^ (x >> 16)) * 0x21F0AAADu;
  x = (x ^ (x >> 15)) * 0x735A2D97u;
  return x ^ (x >> 15);
}

// x in [0, 448] to one of the two neighbouring e4m3 values, by 20 random bits; above zero stays above zero.  In the
// normal range the lower 20 of the float's 23 mantissa bits are cut after the addition; below 2^-6, where the grid is 2^-9, so
// they are with 2^-6 added.
__device__ __forceinline__ float random_e4m3(float x, unsigned up) {
  const float base = x < 0x1p-6f ? 0x1p-6f : 0.f;
  const float r = __builtin_bit_cast(float, (__builtin_bit_cast(unsigned, x + base) + up) & ~0xFFFFFu) - base;
  return x > 0.f ? fmaxf(r, 0x1p-9f) : x;      // a NaN stays one: the sum above may carry out of its mantissa
}

// the maximum of numbers >= 0 over a wave, uniform: within the rows of 16 lanes, then row by row into lane 63
__device__ __forceinline__ float wave_top(float v) {
  v = fmaxf(v, dpp_mov<0x111>(v));      // row_shr:1, 2, 4, 8
  v = fmaxf(v, dpp_mov<0x112>(v));
  v = fmaxf(v, dpp_mov<0x114>(v));
  v = fmaxf(v, dpp_mov<0x118>(v));
  v = fmaxf(v, dpp_mov<0x142>(v));      // row_bcast:15, 31
  v = fmaxf(v, dpp_mov<0x143>(v));
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}

// 1/x to a unit of its last place and its residual put right once; x below 2^126, or the result would be below fp32's normal range
__device__ __forceinline__ float reciprocal(float x) {
  const float r = __builtin_amdgcn_rcpf(x);
  return fmaf(fmaf(-x, r, 1.f), r, r);
}

// A block with an infinite value has its scale from the others, and NaN in that place: 8 bits hold no infinity, and an infinite scale
// would lose the block's other 255 values.
__device__ __forceinline__ float finite_or_nan(float x) { return fabsf(x) < __builtin_inff() ? x : __builtin_nanf(""); }

// The root and the quotient of the update in 8-bit kernels, whose arithmetic takes as long as their memory: the hardware's
// approximations with the residual put right once, within 0.6 units of the last place (random rounding of a bf16 parameter
// looks at bits far below its own).  Squares below 2^-126 have the root zero.
__device__ __forceinline__ float root_of(float v) {
  const float s = __builtin_amdgcn_sqrtf(v), r = fmaf(fmaf(-s, s, v), 0.5f * __builtin_amdgcn_rsqf(v), s);
  return __builtin_amdgcn_classf(v, 0x100) ? r : s;      // positive and normal: not zero, infinite or NaN
}
__device__ __forceinline__ float quotient(float a, float b) {
  const float r = __builtin_amdgcn_rcpf(b), q = a * r;
  return __builtin_amdgcn_div_fixupf(fmaf(fmaf(-q, b, a), r, q), b, a);      // zeros and infinities: the residual above is NaN
}

// a b + c d with every product and the sum rounded.  What ends in 8 bits, or in bf16 by a random number, takes its steps as the formula
// has them: a value near the middle between two codes is then coded the same however the steps were computed, on the host or one
// operation a kernel.  Fused, 700 of 201M codes were others; 6M bf16 parameters took 17.4 instead of 18.4 us, 201M 542 either way.
__device__ __forceinline__ float sum_of_products(float a, float b, float c, float d) {
#pragma clang fp contract(off)
  return a * b + c * d;
}

// WHOLE: all of the chunk's elements exist.
template <typename P, typename G, bool EIGHT, bool FAR, bool WHOLE, int kRounds>
__device__ __forceinline__ void adamw_chunk(const Launch &L, const Tensor &t, long long chunk) {
  constexpr int kChunk = 4 * kRounds * kBlock;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float p[kRounds][4], g[kRounds][4], m[kRounds][4], v[kRounds][4];
  const long long base = chunk * kChunk + wave * (kRounds * kBlock) + lane * 4, left = t.n - base;
  using Codes = typename VecOf<unsigned char, 4>::type;
#pragma unroll
  for (int k = 0; k < kRounds; ++k) {
    const long long e = base + k * kBlock;
    const int n = WHOLE || left - k * kBlock >= 4 ? 4 : left - k * kBlock > 0 ? (int)(left - k * kBlock) : 0;
    load_n<P, 4, FAR>(static_cast<const P *>(t.p) + e, n, p[k]);
    load_n<G, 4, FAR>(static_cast<const G *>(t.g) + e, n, g[k]);
    if (!EIGHT) {
      load_n<float, 4, FAR>(static_cast<const float *>(t.m) + e, n, m[k]);
      load_n<float, 4, FAR>(static_cast<const float *>(t.v) + e, n, v[k]);
    } else {
      unsigned mc = 0, vc = 0;
      const unsigned char *mp = static_cast<const unsigned char *>(t.m) + e, *vp = static_cast<const unsigned char *>(t.v) + e;
      if (n == 4) {
        mc = __builtin_bit_cast(unsigned, far_load<FAR, unsigned char, 4>(mp)), vc = __builtin_bit_cast(unsigned, far_load<FAR, unsigned char, 4>(vp));
      } else {
        for (int i = 0; i < n; ++i) mc |= (unsigned)mp[i] << (8 * i), vc |= (unsigned)vp[i] << (8 * i);
      }
      const float sm = n > 0 ? t.ms[e / kBlock] : 0.f, sv = n > 0 ? t.vs[e / kBlock] : 0.f;
      const auto m01 = __builtin_amdgcn_cvt_pk_f32_fp8(mc, false), m23 = __builtin_amdgcn_cvt_pk_f32_fp8(mc, true);
      const auto v01 = __builtin_amdgcn_cvt_pk_f32_fp8(vc, false), v23 = __builtin_amdgcn_cvt_pk_f32_fp8(vc, true);
      m[k][0] = m01[0] * sm, m[k][1] = m01[1] * sm, m[k][2] = m23[0] * sm, m[k][3] = m23[1] * sm;
      v[k][0] = v01[0] * sv, v[k][1] = v01[1] * sv, v[k][2] = v23[0] * sv, v[k][3] = v23[1] * sv;
    }
  }
  const unsigned number = (t.first + (unsigned)base) * kMul + L.seed * 0x632BE5ABu;
#pragma unroll
  for (int k = 0; k < kRounds; ++k) {
    const long long e = base + k * kBlock;
    const int n = WHOLE || left - k * kBlock >= 4 ? 4 : left - k * kBlock > 0 ? (int)(left - k * kBlock) : 0;
    float root[4];
    unsigned noise[4];
    float mtop = 0.f, vtop = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float gr = g[k][i] * L.gscale, square = EIGHT ? v[k][i] * v[k][i] : v[k][i];
      m[k][i] = sum_of_products(m[k][i], L.b1, gr, L.c1);
      v[k][i] = sum_of_products(square, L.b2, gr * gr, L.c2);
      root[i] = EIGHT ? root_of(v[k][i]) : sqrtf(v[k][i]);
      const float below = sum_of_products(root[i], L.root, L.eps, 1.f);
      const float q = sum_of_products(p[k][i], t.decay, EIGHT ? quotient(m[k][i], below) : m[k][i] / below, -L.step);
      if (EIGHT || sizeof(P) == 2) noise[i] = element_hash(number + (k * kBlock + i) * kMul);
      if (sizeof(P) == 2) {
        // to one of the two neighbours, by 16 random bits; infinities and NaN stay what they are
        const unsigned b = __builtin_bit_cast(unsigned, q);
        const unsigned r = (b & 0x7F800000u) == 0x7F800000u ? b : (b + (noise[i] & 0xFFFFu)) & ~0xFFFFu;
        p[k][i] = __builtin_bit_cast(float, r);
      } else {
        p[k][i] = q;
      }
      mtop = fmaxf(mtop, fabsf(m[k][i]));
      vtop = fmaxf(vtop, root[i]);
    }
    store_n<P, 4, FAR>(static_cast<P *>(t.p) + e, n, p[k]);
    if (sizeof(P) == 4 && t.copy) store_n<bf16, 4, FAR>(static_cast<bf16 *>(t.copy) + e, n, p[k]);
    if (!EIGHT) {
      store_n<float, 4, FAR>(static_cast<float *>(t.m) + e, n, m[k]);
      store_n<float, 4, FAR>(static_cast<float *>(t.v) + e, n, v[k]);
    } else {
      mtop = fmaxf(wave_top(mtop), 0x1p-100f), vtop = fmaxf(wave_top(vtop), 0x1p-100f);
      float mi = reciprocal(mtop) * 448.f, vi = reciprocal(vtop) * 448.f;
      if (fmaxf(mtop, vtop) >= 0x1p126f) {     // the same for the whole wave
        mtop = vtop = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) m[k][i] = finite_or_nan(m[k][i]), root[i] = finite_or_nan(root[i]), mtop = fmaxf(mtop, fabsf(m[k][i])), vtop = fmaxf(vtop, root[i]);
        mtop = fmaxf(wave_top(mtop), 0x1p-100f), vtop = fmaxf(wave_top(vtop), 0x1p-100f);
        mi = 448.f / mtop, vi = 448.f / vtop;
      }
      float r[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        m[k][i] *= mi;
        const float x = root[i] * vi;
        r[i] = random_e4m3(x > 448.f ? 448.f : x, noise[i] >> 12);
      }
      const unsigned mc = pack_e4m3(m[k][0], m[k][1], m[k][2], m[k][3]), vc = pack_e4m3(r[0], r[1], r[2], r[3]);
      unsigned char *mp = static_cast<unsigned char *>(t.m) + e, *vp = static_cast<unsigned char *>(t.v) + e;
      if (n == 4) {
        far_store<FAR, unsigned char, 4>(__builtin_bit_cast(Codes, mc), mp), far_store<FAR, unsigned char, 4>(__builtin_bit_cast(Codes, vc), vp);
      } else {
        for (int i = 0; i < n; ++i) mp[i] = (unsigned char)(mc >> (8 * i)), vp[i] = (unsigned char)(vc >> (8 * i));
      }
      if (lane == 0 && n > 0) t.ms[e / kBlock] = mtop * (1.f / 448.f), t.vs[e / kBlock] = vtop * (1.f / 448.f);
    }
  }
}

template <typename P, typename G, bool EIGHT, bool FAR>
__device__ __forceinline__ void adamw_piece(const Launch &L, const Tensor &t, long long chunk) {
  constexpr int kRounds = rounds_of(FAR);
  if ((chunk + 1) * chunk_of(FAR) <= t.n) adamw_chunk<P, G, EIGHT, FAR, true, kRounds>(L, t, chunk);
  else adamw_chunk<P, G, EIGHT, false, false, kRounds>(L, t, chunk);
}

// Six waves a SIMD are worth 3 % with 32-bit states, and cost the 8-bit kernel on much data 2 % (201M parameters 551 against 544 us): it has five,
// whatever its registers would allow.
template <bool EIGHT, bool FAR>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(EIGHT ? 5 : 6, EIGHT && FAR ? 5 : 8))) void adamw_kernel(Launch L) {
  int lo = 0, hi = L.tensors - 1;              // the last tensor that starts at or before this chunk
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (L.chunk0[mid] <= blockIdx.x) lo = mid;
    else hi = mid - 1;
  }
  const Tensor &t = L.t[lo];
  const long long chunk = blockIdx.x - L.chunk0[lo];
  switch (L.kind[lo]) {
    case 0: adamw_piece<float, float, EIGHT, FAR>(L, t, chunk); break;
    case 1: adamw_piece<bf16, float, EIGHT, FAR>(L, t, chunk); break;
    case 2: adamw_piece<float, bf16, EIGHT, FAR>(L, t, chunk); break;
    case 3: adamw_piece<bf16, bf16, EIGHT, FAR>(L, t, chunk); break;
    case 4: adamw_piece<float, f16, EIGHT, FAR>(L, t, chunk); break;
    default: adamw_piece<bf16, f16, EIGHT, FAR>(L, t, chunk); break;
  }
}

inline bool off(const void *p, int size) { return (reinterpret_cast<uintptr_t>(p) & (size - 1)) != 0; }

}  // namespace
}  // namespace pbkd

using namespace pbkd;

extern "C" pbkd_status pbkd_adamw_step(int n_tensors, const pbkd_adamw_tensor *tensors, const pbkd_adamw_args *a, void *hip_stream) {
  if (n_tensors < 0 || (n_tensors > 0 && !tensors) || !a) return set_error(PBKD_EINVAL, "adamw: bad argument");
  if (a->state_bits != 32 && a->state_bits != 8) return set_error(PBKD_EINVAL, "adamw: state_bits must be 32 or 8");
  if (a->step < 1) return set_error(PBKD_EINVAL, "adamw: step counts from 1");
  if (!(a->beta1 >= 0. && a->beta1 < 1. && a->beta2 >= 0. && a->beta2 < 1.)) return set_error(PBKD_EINVAL, "adamw: beta1 and beta2 must be in [0,1)");
  if (!(a->eps >= 0.) || !(a->lr >= 0.) || !(a->grad_scale == a->grad_scale)) return set_error(PBKD_EINVAL, "adamw: lr and eps must not be negative, nor grad_scale NaN");
  const bool eight = a->state_bits == 8;
  double bytes = 0.;                           // of the whole call
  for (int i = 0; i < n_tensors; ++i) {        // all of them before the first launch
    const pbkd_adamw_tensor &t = tensors[i];
    if (t.n < 0) return set_error(PBKD_ESHAPE, "adamw: tensor %d has %lld elements", i, t.n);
    if (t.n > (1LL << 34)) return set_error(PBKD_EUNSUPPORTED, "adamw: tensor %d has %lld elements, at most 2^34", i, t.n);
    if (t.param_dtype != PBKD_F32 && t.param_dtype != PBKD_BF16) return set_error(PBKD_EINVAL, "adamw: tensor %d: param_dtype must be PBKD_F32 or PBKD_BF16", i);
    if (t.grad_dtype != PBKD_F32 && t.grad_dtype != PBKD_BF16 && t.grad_dtype != PBKD_F16) return set_error(PBKD_EINVAL, "adamw: tensor %d: grad_dtype %d", i, t.grad_dtype);
    if (t.copy_dev && t.param_dtype != PBKD_F32) return set_error(PBKD_EINVAL, "adamw: tensor %d: a bf16 copy needs fp32 parameters", i);
    if (!(t.weight_decay >= 0.f)) return set_error(PBKD_EINVAL, "adamw: tensor %d: weight_decay must not be negative", i);
    if (t.n == 0) continue;
    if (!t.param_dev || !t.grad_dev || !t.m_dev || !t.v_dev || (eight && (!t.m_scale_dev || !t.v_scale_dev)))
      return set_error(PBKD_EINVAL, "adamw: tensor %d: null pointer", i);
    if (off(t.param_dev, t.param_dtype == PBKD_F32 ? 4 : 2) || off(t.grad_dev, t.grad_dtype == PBKD_F32 ? 4 : 2) || off(t.copy_dev, 2) ||
        (!eight && (off(t.m_dev, 4) || off(t.v_dev, 4))) || (eight && (off(t.m_scale_dev, 4) || off(t.v_scale_dev, 4))))
      return set_error(PBKD_EINVAL, "adamw: tensor %d is not aligned to its elements", i);
    bytes += (double)t.n * ((t.param_dtype == PBKD_F32 ? 8 : 4) + (t.grad_dtype == PBKD_F32 ? 4 : 2) + (eight ? 4 : 16) + (t.copy_dev ? 2 : 0));
  }
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (bytes > 0. && st) {                      // the null stream cannot be captured
    hipStreamCaptureStatus capture;
    SEQ_HIPCHK(hipStreamIsCapturing(st, &capture));
    if (capture != hipStreamCaptureStatusNone)
      return set_error(PBKD_EUNSUPPORTED, "adamw: a captured step would repeat its bias corrections, learning rate and random numbers; capture what is around it");
  }
  const bool far = bytes > kLastLevelCache;
  Launch L;
  L.seed = a->seed;
  L.b1 = (float)a->beta1, L.c1 = (float)(1. - a->beta1), L.b2 = (float)a->beta2, L.c2 = (float)(1. - a->beta2);
  L.eps = (float)a->eps, L.gscale = (float)a->grad_scale;
  L.step = (float)(a->lr / (1. - pow(a->beta1, (double)a->step)));
  L.root = (float)(1. / sqrt(1. - pow(a->beta2, (double)a->step)));
  L.tensors = 0, L.chunk0[0] = 0;
  auto flush = [&]() -> hipError_t {
    if (L.tensors == 0) return hipSuccess;
    const unsigned grid = L.chunk0[L.tensors];
    if (eight && far) adamw_kernel<true, true><<<grid, 256, 0, st>>>(L);
    else if (eight) adamw_kernel<true, false><<<grid, 256, 0, st>>>(L);
    else if (far) adamw_kernel<false, true><<<grid, 256, 0, st>>>(L);
    else adamw_kernel<false, false><<<grid, 256, 0, st>>>(L);
    L.tensors = 0, L.chunk0[0] = 0;
    return hipGetLastError();
  };
  for (int i = 0; i < n_tensors; ++i) {
    const pbkd_adamw_tensor &t = tensors[i];
    const long long chunks = cdiv64(t.n, chunk_of(far));   // at most 2^22 (what is not far is small); a launch's threads must stay below 2^32
    if (chunks == 0) continue;
    if (L.tensors == kTensors || L.chunk0[L.tensors] + chunks > (1LL << 23)) SEQ_HIPCHK(flush());
    const int k = L.tensors++;
    L.t[k] = Tensor{t.param_dev, t.grad_dev, t.m_dev, t.v_dev, t.m_scale_dev, t.v_scale_dev, t.copy_dev, t.n, (unsigned)t.first,
                    (float)(1. - a->lr * (double)t.weight_decay)};
    L.kind[k] = (unsigned char)((t.param_dtype == PBKD_BF16) + 2 * (t.grad_dtype == PBKD_F32 ? 0 : t.grad_dtype == PBKD_BF16 ? 1 : 2));
    L.chunk0[k + 1] = L.chunk0[k] + (unsigned)chunks;
  }
  SEQ_HIPCHK(flush());
  return PBKD_OK;
}
