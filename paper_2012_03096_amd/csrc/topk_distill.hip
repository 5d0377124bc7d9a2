// Distillation from a teacher's top logits: loss and, in the same call, the gradient of the student's logits.
//
//   q = softmax(t / T) over the known pairs,  p = softmax(z / T) over the vocabulary
//   loss = T^2 sum_j q_j (log q_j - z_j / T + lse),  dz_v = g T (p_v - sum of the q_j whose place is v)
//
// Bound by memory: a workgroup takes a row, reads it once for its maximum and sum (one pass, the sum rescaled when the maximum
// grows) and once more for the gradient, when it comes from the caches.  The pairs wait in LDS; their places' gradients
// are written last, each by the first pair that names the place.
#include "seq_common.h"

namespace pbkd {
namespace {

constexpr int kMaxTop = 1024;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct Args {
  const void *z, *t, *at;
  const float *g;
  float *loss;
  void *dz;
  long long rows, zs, ds;
  int v, top;
  float inv_t, temperature;
};

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// m, s of one part of a row (s relative to 2^m) joined with another's; m is -inf where nothing was seen.
__device__ __forceinline__ void join(float &m, float &s, float m2, float s2) {
  const float top = fmaxf(m, m2);
  const float ref = top == -__builtin_inff() ? 0.f : top;
  s = s * exp2_fast(m - ref) + s2 * exp2_fast(m2 - ref);
  m = top;
}

template <typename T, typename TT, typename IT, int THREADS, bool FAR>
__global__ __launch_bounds__(THREADS) void topk_distill_kernel(Args A) {
  constexpr int W = THREADS / 64;
  __shared__ int place[kMaxTop];
  __shared__ float share[kMaxTop];
  __shared__ float red[4][W];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, v = A.v, top = A.top;
  const long long row = blockIdx.x;
  const T *z = static_cast<const T *>(A.z) + row * A.zs;
  const float c = A.inv_t * kLog2e;            // logits in units of log 2, over T

  // the row's maximum and sum
  float m = -__builtin_inff(), s = 0.f;
  for (int i = tid * 8; i < v; i += THREADS * 8) {
    float x[8];
    if (i + 8 <= v) load_n<T, 8>(z + i, 8, x);
    else {
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = i + k < v ? static_cast<float>(z[i + k]) : -__builtin_inff();
    }
    float most = m;
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] *= c, most = fmaxf(most, x[k]);
    const float ref = most == -__builtin_inff() ? 0.f : most;
    s *= exp2_fast(m - ref);
#pragma unroll
    for (int k = 0; k < 8; ++k) s += exp2_fast(x[k] - ref);
    m = most;
  }
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) {
    const float m2 = __shfl_xor(m, k, 64), s2 = __shfl_xor(s, k, 64);
    join(m, s, m2, s2);
  }

  // the pairs: which are known, and their logits' maximum
  const TT *t = static_cast<const TT *>(A.t) + row * top;
  const IT *at = static_cast<const IT *>(A.at) + row * top;
  float tm = -__builtin_inff();
  for (int j = tid; j < top; j += THREADS) {
    const IT w = at[j];
    float x = static_cast<float>(t[j]) * A.inv_t;
    const bool known = w >= 0 && w < v && x > -__builtin_inff();
    place[j] = known ? static_cast<int>(w) : -1;
    share[j] = x = known ? x : -__builtin_inff();
    tm = fmaxf(tm, x);
  }
  tm = wave64_max(tm);
  if (lane == 0) red[0][wave] = m, red[1][wave] = s, red[2][wave] = tm;
  __syncthreads();
  m = red[0][0], s = red[1][0], tm = red[2][0];
#pragma unroll
  for (int k = 1; k < W; ++k) join(m, s, red[0][k], red[1][k]), tm = fmaxf(tm, red[2][k]);
  const bool some = tm > -__builtin_inff();
  const float lse = (m + __builtin_amdgcn_logf(s)) * kLn2;
  float qs = 0.f;
  for (int j = tid; j < top; j += THREADS)
    if (place[j] >= 0) qs += expf(share[j] - tm);
  qs = wave64_sum(qs);
  if (lane == 0) red[3][wave] = qs;
  __syncthreads();
  qs = red[3][0];
#pragma unroll
  for (int k = 1; k < W; ++k) qs += red[3][k];
  const float log_qs = logf(qs), inv_qs = 1.f / qs;

  // loss, and each pair's share.  The student's logits there are read before anything is written: dz may be z
  constexpr int PER = kMaxTop / THREADS;
  float mine[PER];
  float far = 0.f;
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int j = k * THREADS + tid;
    mine[k] = 0.f;
    if (j < top) {
      const int w = place[j];
      float q = 0.f;
      if (w >= 0) {
        const float x = share[j] - tm;
        q = expf(x) * inv_qs;
        const float zj = static_cast<float>(z[w]);
        mine[k] = zj * c;
        if (q > 0.f) far += q * (x - log_qs - zj * A.inv_t + lse);
      }
      share[j] = q;
    }
  }
  far = wave64_sum(far);
  __syncthreads();
  if (lane == 0) red[0][wave] = far;
  __syncthreads();
  if (tid == 0) {
    far = red[0][0];
    for (int k = 1; k < W; ++k) far += red[0][k];
    A.loss[row] = some ? far * A.temperature * A.temperature : 0.f;
  }
  if (!A.dz) return;

  T *dz = static_cast<T *>(A.dz) + row * A.ds;
  const float g = (A.g ? A.g[row] : 1.f) * A.temperature;
  const float shift = m == -__builtin_inff() ? __builtin_nanf("") : m, scale = g / s;
  for (int i = tid * 8; i < v; i += THREADS * 8) {
    float x[8];
    load_n<T, 8>(z + i, v - i, x);
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = some ? exp2_fast(x[k] * c - shift) * scale : 0.f;
    store_n<T, 8, FAR>(dz + i, v - i, x);
  }
  __syncthreads();
  if (!some) return;
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int j = k * THREADS + tid;
    if (j >= top || place[j] < 0) continue;
    const int w = place[j];
    float q = 0.f;
    bool first = true;
    for (int i = 0; i < top; ++i)
      if (place[i] == w) q += share[i], first &= i >= j;
    if (first) dz[w] = static_cast<T>(exp2_fast(mine[k] - shift) * scale - g * q);
  }
}

template <typename T, typename TT, typename IT>
hipError_t launch(const Args &A, hipStream_t st) {
  const bool far = A.dz && (double)A.rows * A.v * sizeof(T) > kLastLevelCache;
  const unsigned grid = (unsigned)A.rows;
  if (A.v <= 8192) topk_distill_kernel<T, TT, IT, 256, false><<<grid, 256, 0, st>>>(A);
  else if (far) topk_distill_kernel<T, TT, IT, 1024, true><<<grid, 1024, 0, st>>>(A);
  else topk_distill_kernel<T, TT, IT, 1024, false><<<grid, 1024, 0, st>>>(A);
  return hipGetLastError();
}

template <typename T, typename TT>
hipError_t launch_index(const Args &A, bool wide, hipStream_t st) {
  return wide ? launch<T, TT, long long>(A, st) : launch<T, TT, int>(A, st);
}

template <typename T>
hipError_t launch_teacher(const Args &A, int teacher, bool wide, hipStream_t st) {
  return teacher == PBKD_F32 ? launch_index<T, float>(A, wide, st) : teacher == PBKD_BF16 ? launch_index<T, bf16>(A, wide, st) : launch_index<T, f16>(A, wide, st);
}

inline bool misaligned(const void *p, int size) { return (reinterpret_cast<uintptr_t>(p) & (size - 1)) != 0; }

}  // namespace
}  // namespace pbkd

using namespace pbkd;

extern "C" pbkd_status pbkd_topk_distill(const pbkd_topk_distill_desc *q, void *hip_stream) {
  if (!q) return set_error(PBKD_EINVAL, "topk_distill: null descriptor");
  if (q->rows < 0 || q->vocab < 1 || q->top < 1) return set_error(PBKD_ESHAPE, "topk_distill: %lld rows of %d logits, %d of the teacher's", q->rows, q->vocab, q->top);
  if (q->top > kMaxTop) return set_error(PBKD_EUNSUPPORTED, "topk_distill: %d of the teacher's logits, at most %d", q->top, kMaxTop);
  if (q->rows > 1 << 21) return set_error(PBKD_EUNSUPPORTED, "topk_distill: %lld rows", q->rows);
  for (int dtype : {q->dtype, q->teacher_dtype})
    if (dtype != PBKD_F32 && dtype != PBKD_BF16 && dtype != PBKD_F16) return set_error(PBKD_EINVAL, "topk_distill: dtype %d", dtype);
  if (q->index_dtype != PBKD_I32 && q->index_dtype != PBKD_I64) return set_error(PBKD_EINVAL, "topk_distill: index_dtype %d", q->index_dtype);
  if (!(q->temperature > 0.f) || !(1.f / q->temperature > 0.f) || !(1.f / q->temperature < __builtin_inff()))
    return set_error(PBKD_EINVAL, "topk_distill: the temperature must be above zero, and finite as its inverse");
  if (q->rows == 0) return PBKD_OK;
  if (!q->logits_dev || !q->teacher_dev || !q->at_dev || !q->loss_dev) return set_error(PBKD_EINVAL, "topk_distill: null tensor");
  const int size = q->dtype == PBKD_F32 ? 4 : 2;
  if (misaligned(q->logits_dev, size) || misaligned(q->dlogits_dev, size) || misaligned(q->teacher_dev, q->teacher_dtype == PBKD_F32 ? 4 : 2) ||
      misaligned(q->at_dev, q->index_dtype == PBKD_I64 ? 8 : 4) || misaligned(q->row_weight_dev, 4) || misaligned(q->loss_dev, 4))
    return set_error(PBKD_EINVAL, "topk_distill: a tensor is not aligned to its elements");
  if (q->logits_stride < 0) return set_error(PBKD_EINVAL, "topk_distill: negative stride");
  if (q->rows > 1 && q->dlogits_dev && q->dlogits_stride < q->vocab) return set_error(PBKD_ESHAPE, "topk_distill: rows of dlogits overlap");
  if (q->dlogits_dev == q->logits_dev && q->rows > 1 && q->dlogits_stride != q->logits_stride)
    return set_error(PBKD_EINVAL, "topk_distill: dlogits in the logits' place needs their stride");
  Args A{q->logits_dev, q->teacher_dev, q->at_dev, q->row_weight_dev, q->loss_dev, q->dlogits_dev, q->rows, q->logits_stride, q->dlogits_stride,
         q->vocab, q->top, 1.f / q->temperature, q->temperature};
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  const bool wide = q->index_dtype == PBKD_I64;
  switch (q->dtype) {
    case PBKD_F32: SEQ_HIPCHK(launch_teacher<float>(A, q->teacher_dtype, wide, st)); break;
    case PBKD_BF16: SEQ_HIPCHK(launch_teacher<bf16>(A, q->teacher_dtype, wide, st)); break;
    default: SEQ_HIPCHK(launch_teacher<f16>(A, q->teacher_dtype, wide, st)); break;
  }
  return PBKD_OK;
}
