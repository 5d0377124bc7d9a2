// Shared by the kernels of the sequence operators (rmsnorm.hip, recurrence.hip, adamw.hip): element types, vector
// loads and stores at any alignment, reductions over a wave, and the error text of the C entry points.
#pragma once
#include "../../include/pbkd.h"
#include "pbkd_internal.h"

namespace pbkd {

// Sets the calling thread's error text and returns `status` (pbkd_runtime.hip).
pbkd_status set_error(pbkd_status status, const char *fmt, ...);

#define SEQ_HIPCHK(expr)                                                                       \
  do {                                                                                         \
    hipError_t e_ = (expr);                                                                    \
    if (e_ != hipSuccess) return set_error(PBKD_EHIP, "%s: %s", #expr, hipGetErrorString(e_)); \
  } while (0)

constexpr double kLastLevelCache = 256e6;      // bytes

inline long long cdiv64(long long a, long long b) { return (a + b - 1) / b; }

// Column sums of partial[rows][cols] into out[cols], in a fixed order (rmsnorm.hip).  scratch: colsum_scratch_floats()
// floats behind which nothing is needed; it may not overlap partial.
size_t colsum_scratch_floats(long long rows, int cols);
hipError_t launch_colsum(const float *partial, long long rows, int cols, float *scratch, float *out, hipStream_t st);

using bf16 = __bf16;
using f16 = _Float16;

#if defined(__HIPCC__)
// Vectors of N elements that are only as aligned as one element: gfx950 moves them in 4- to 16-byte accesses at any
// address, so odd row lengths and shifted views take the same instructions as aligned ones (a vector across two cache
// lines costs the second line's access).
template <typename T, int N>
struct VecOf {
  typedef T type __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};

// Accesses with FAR go past the caches.  It is for calls that move more than the last-level cache holds, none of which can be
// there from the call before or for the call behind (measured on 67M parameters, 1.9 GB: 347 -> 303 us; but on 100 MB that come
// again and again, 29 -> 36 us).
template <bool FAR, typename T, int N>
__device__ __forceinline__ typename VecOf<T, N>::type far_load(const T *p) {
  if (FAR) return __builtin_nontemporal_load(reinterpret_cast<const typename VecOf<T, N>::type *>(p));
  return *reinterpret_cast<const typename VecOf<T, N>::type *>(p);
}
template <bool FAR, typename T, int N>
__device__ __forceinline__ void far_store(typename VecOf<T, N>::type v, T *p) {
  if (FAR) __builtin_nontemporal_store(v, reinterpret_cast<typename VecOf<T, N>::type *>(p));
  else *reinterpret_cast<typename VecOf<T, N>::type *>(p) = v;
}

// n of the N elements exist (n <= 0: none); the others come back as zero and are not read.
template <typename T, int N, bool FAR = false>
__device__ __forceinline__ void load_n(const T *p, int n, float (&v)[N]) {
  if (n >= N) {
    const typename VecOf<T, N>::type r = far_load<FAR, T, N>(p);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = static_cast<float>(r[i]);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = i < n ? static_cast<float>(p[i]) : 0.f;
  }
}

// Rounds to nearest (even).  n as above: only existing elements are written.
template <typename T, int N, bool FAR = false>
__device__ __forceinline__ void store_n(T *p, int n, const float (&v)[N]) {
  if (n >= N) {
    typename VecOf<T, N>::type r;
#pragma unroll
    for (int i = 0; i < N; ++i) r[i] = static_cast<T>(v[i]);
    far_store<FAR, T, N>(r, p);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < n) p[i] = static_cast<T>(v[i]);
  }
}

// Four floats to four e4m3 codes (nearest even); the caller keeps them within +-448.  NaN becomes the code of NaN.
__device__ __forceinline__ unsigned pack_e4m3(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return static_cast<unsigned>(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true));
}

// every lane receives the maximum over its wave (fmaxf: a NaN counts as absent)
__device__ __forceinline__ float wave64_max(float v) {
  v = fmaxf(v, dpp_mov<0xB1>(v));
  v = fmaxf(v, dpp_mov<0x4E>(v));
  v = fmaxf(v, dpp_mov<0x141>(v));
  v = fmaxf(v, dpp_mov<0x140>(v));
  v = fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_ds_swizzle(__builtin_bit_cast(int, v), 0x401F)));
  return fmaxf(v, __shfl_xor(v, 32, 64));
}
#endif

}  // namespace pbkd
