// Distillation from a teacher's top logits: loss and, in the same call, the gradient of the student's logits.
//
//   q = softmax(t / T) over the known pairs,  p = softmax(z / T) over the vocabulary
//   loss = T^2 sum_j q_j (log q_j - z_j / T + lse),  dz_v = g T (p_v - sum of the q_j whose place is v)
//
// Bound by memory: a workgroup takes a row, reads it once for its maximum and sum (one pass, the sum rescaled when the maximum
// grows) and once more for the gradient: the first 64 KB from LDS, where they were left, the rest from the caches.  The pairs' places get their
// gradients last, each from the first pair that names it.
//
// Measured: 8192 rows of 65536 bf16 with the gradient 407 us (5.3 TB/s of each number read and written once; without LDS 475, a row in registers 624: one workgroup
// a compute unit); 4095 rows of 131071 fp16, losses 178 us, 6.0 TB/s; 1023 rows of 50021 fp32 100 us (32 bytes a thread and access instead of 16: 113).
#include "seq_common.h"
#include "split_bf16.h"

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

// Vectors of 16 bytes a thread works on at a time, the next ones on their way.
constexpr int kAhead = 4;

template <typename T, typename TT, typename IT, int THREADS, bool GRADIENT, bool FAR>
__global__ __launch_bounds__(THREADS, THREADS == 1024 ? 8 : 4) void topk_distill_kernel(Args A) {
  constexpr int W = THREADS / 64, PER = kMaxTop / THREADS, N = 16 / sizeof(T), HELD = kAhead, STEP = HELD * THREADS * N;
  typedef typename VecOf<T, N>::type Vec;
  __shared__ int place[kMaxTop];
  __shared__ float share[kMaxTop];
  __shared__ float red[4][W];
  __shared__ unsigned seen[256];               // a bit for each place that a pair names
  __shared__ int twice;
  __shared__ Vec kept[GRADIENT ? HELD : 1][GRADIENT ? THREADS : 1];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, v = A.v, top = A.top;
  const long long row = blockIdx.x;
  const T *const z = static_cast<const T *>(A.z) + row * A.zs;
  // A 16-bit row that begins between two words is taken from the number before it on (the row before's last, or what lies between rows), which gets no
  // weight: its vectors then begin with words (4095 rows of 131071 fp16, loss only: 207 us by reads between words, 178 so).
  const int par = sizeof(T) == 2 ? static_cast<int>(row * A.zs & 1) : 0, n = v + par;
  const T *const zz = z - par;
  const float c = A.inv_t * kLog2e;            // logits in units of log 2, over T

  // whether a place is named twice is looked up where rows are short (in long ones it hides, and 28 registers would spill)
  constexpr bool LOOK = GRADIENT && THREADS < 1024;
  if (LOOK && tid < 256) seen[tid] = 0;
  if (LOOK && tid == 0) twice = 0;
  // the pairs are read first, then the student's logits there: dz may be z, and nothing is written before
  const TT *t = static_cast<const TT *>(A.t) + row * top;
  const IT *at = static_cast<const IT *>(A.at) + row * top;
  float mine[PER], logit[PER];
  int w[PER];
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int j = k * THREADS + tid;
    const IT x = j < top ? at[j] : IT(-1);
    logit[k] = j < top ? static_cast<float>(t[j]) * A.inv_t : -__builtin_inff();
    w[k] = x >= 0 && x < v && logit[k] > -__builtin_inff() ? static_cast<int>(x) : -1;
  }

  Vec held[HELD];
  // the row's maximum, times c and rounded, and its sum relative to just that number: a batch's maximum first, one rescaling a batch, by exactly 1
  // where the maximum stays.  (From the exact product, a rescaling would be off by what the product was rounded by, every batch: rows of 2^21 with one
  // logit of 500 had a log-sum off by 2e-3.)
  float m = -__builtin_inff(), s = 0.f;
  auto raise = [&](float most) {
    const float before = m;
    m = fmaxf(m, most * c);
    const float ref = m == -__builtin_inff() ? 0.f : m;
    s *= exp2_fast(before - ref);
    return ref;
  };
  auto take = [&](const Vec (&raw)[HELD]) {
    float most = -__builtin_inff();
#pragma unroll
    for (int k = 0; k < HELD; ++k)
#pragma unroll
      for (int e = 0; e < N; ++e) most = fmaxf(most, static_cast<float>(raw[k][e]));
    const float ref = raise(most);
#pragma unroll
    for (int k = 0; k < HELD; ++k) {
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < N; ++e) sum += exp2_fast(fmaf(static_cast<float>(raw[k][e]), c, -ref));
      s += sum;
    }
  };
  Vec next[HELD];
  constexpr int ONE = THREADS * N;
  const int full = n / STEP * STEP;              // the batches that the row fills
  auto fetch = [&](int base) {
#pragma unroll
    for (int k = 0; k < HELD; ++k) next[k] = far_load<FAR && !GRADIENT, T, N>(zz + base + k * ONE + tid * N);
  };
  // What is left goes one vector a thread at a time (all at once they would not fit into the registers).  A thread at the row's end, or behind it, reads
  // the row's last logits, and those that are another thread's get no weight: reads behind branches, one after the other, cost 9 us a row.
  auto fetch_one = [&](int base) {
    const int i = base + tid * N;
    if (n >= N) next[0] = far_load<FAR && !GRADIENT, T, N>(zz + (i + N <= n ? i : n - N));
    else
#pragma unroll
      for (int e = 0; e < N; ++e) next[0][e] = zz[e < n ? e : n - 1];
  };
  auto mask = [&](int i, float (&x)[N]) {
    const int at = i + N <= n ? i : n >= N ? n - N : 0;
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (at + e < i || at + e >= n || at + e < par) x[e] = -__builtin_inff();
  };
  if (full) fetch(0);
  else fetch_one(0);
#pragma unroll
  for (int k = 0; k < PER; ++k) mine[k] = w[k] >= 0 ? static_cast<float>(z[w[k]]) : 0.f;
  for (int base = 0; base < full; base += STEP) {
#pragma unroll
    for (int k = 0; k < HELD; ++k) held[k] = next[k];
    if (base + STEP < full) fetch(base + STEP);
    else if (full < n) fetch_one(full);
    if (sizeof(T) == 2 && base == 0 && par && tid == 0) {
      const T none = static_cast<T>(-__builtin_inff());
      unsigned short bits;
      __builtin_memcpy(&bits, &none, 2);
      uintx4 words = __builtin_bit_cast(uintx4, held[0]);
      words[0] = (words[0] & 0xffff0000u) | bits;
      held[0] = __builtin_bit_cast(Vec, words);
    }
    if (GRADIENT && base == 0) {
#pragma unroll
      for (int k = 0; k < HELD; ++k) kept[k][tid] = held[k];
    }
    take(held);
  }
  for (int base = full; base < n; base += ONE) {
    float x[N], most = -__builtin_inff();
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = static_cast<float>(next[0][e]);
    if (base + ONE < n) fetch_one(base + ONE);
    mask(base + tid * N, x);
#pragma unroll
    for (int e = 0; e < N; ++e) most = fmaxf(most, x[e]);
    const float ref = raise(most);
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < N; ++e) sum += exp2_fast(fmaf(x[e], c, -ref));
    s += sum;
  }
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) {
    const float m2 = __shfl_xor(m, k, 64), s2 = __shfl_xor(s, k, 64);
    join(m, s, m2, s2);
  }

  float tm = -__builtin_inff();
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    if (w[k] < 0) logit[k] = -__builtin_inff();
    tm = fmaxf(tm, logit[k]);
  }
  tm = wave64_max(tm);
  if (lane == 0) red[0][wave] = m, red[1][wave] = s, red[2][wave] = tm;
  __syncthreads();
  m = red[0][0], s = 0.f, tm = red[2][0];
#pragma unroll
  for (int k = 1; k < W; ++k) m = fmaxf(m, red[0][k]), tm = fmaxf(tm, red[2][k]);
  const float base = m == -__builtin_inff() ? 0.f : m;
#pragma unroll
  for (int k = 0; k < W; ++k) s += red[1][k] * exp2_fast(red[0][k] - base);
  const bool some = tm > -__builtin_inff();
  const float lse = (m + __builtin_amdgcn_logf(s)) * kLn2;
  // Places beyond 8192 may share a bit and count as named twice: looking through all pairs for each pair costs 2 us of a row with 235 (12149 rows of 744 fp16
  // 172 us, so 50).
  if (LOOK) {
#pragma unroll
    for (int k = 0; k < PER; ++k)
      if (w[k] >= 0) {
        const int bit = (w[k] ^ w[k] >> 13) & 8191;
        if (atomicOr(&seen[bit >> 5], 1u << (bit & 31)) >> (bit & 31) & 1) twice = 1;
      }
  }
  float qs = 0.f;
#pragma unroll
  for (int k = 0; k < PER; ++k)
    if (w[k] >= 0) qs += expf(logit[k] - tm);
  qs = wave64_sum(qs);
  if (lane == 0) red[3][wave] = qs;
  __syncthreads();
  qs = red[3][0];
#pragma unroll
  for (int k = 1; k < W; ++k) qs += red[3][k];
  const float log_qs = logf(qs), inv_qs = 1.f / qs;

  // loss, and each pair's share
  float far = 0.f;
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int j = k * THREADS + tid;
    float q = 0.f;
    if (w[k] >= 0) {
      const float x = logit[k] - tm;
      q = expf(x) * inv_qs;
      if (q > 0.f) far += q * (x - log_qs - mine[k] * A.inv_t + lse);
    }
    if (j < top) place[j] = w[k], share[j] = q;
  }
  far = wave64_sum(far);
  if (lane == 0) red[2][wave] = far;           // its readers of before are behind the barrier of qs
  __syncthreads();
  if (tid == 0) {
    far = red[2][0];
    for (int k = 1; k < W; ++k) far += red[2][k];
    A.loss[row] = some ? far * A.temperature * A.temperature : 0.f;
  }
  if (!GRADIENT) return;

  T *const dz = static_cast<T *>(A.dz) + row * A.ds, *const dd = dz - par;
  if (!some) {
    const float zero[N] = {};
    for (int i = tid * N; i < v; i += ONE) store_n<T, N>(dz + i, v - i, zero);
    return;
  }
  const float g = (A.g ? A.g[row] : 1.f) * A.temperature;
  const float shift = m == -__builtin_inff() ? __builtin_nanf("") : m, scale = g / s;
  auto give = [&](const Vec &raw, int i) {
    float x[N];
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = exp2_fast(fmaf(static_cast<float>(raw[e]), c, -shift)) * scale;
    if (par && i == 0) {             // but not in front of the row
#pragma unroll
      for (int e = 1; e < N; ++e) dd[e] = static_cast<T>(x[e]);
    } else {
      store_n<T, N, FAR>(dd + i, N, x);
    }
  };
  if (STEP < full) fetch(STEP);
  else if (full < n) fetch_one(full);
  if (full) {
#pragma unroll
    for (int k = 0; k < HELD; ++k) give(kept[k][tid], k * ONE + tid * N);
  }
  for (int base = STEP; base < full; base += STEP) {
#pragma unroll
    for (int k = 0; k < HELD; ++k) held[k] = next[k];
    if (base + STEP < full) fetch(base + STEP);
    else if (full < n) fetch_one(full);
#pragma unroll
    for (int k = 0; k < HELD; ++k) give(held[k], base + k * ONE + tid * N);
  }
  for (int base = full; base < n; base += ONE) {
    const int i = base + tid * N;
    float x[N];
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = exp2_fast(fmaf(static_cast<float>(next[0][e]), c, -shift)) * scale;
    if (base + ONE < n) fetch_one(base + ONE);
    if (i + N <= n && !(par && i == 0)) {
      store_n<T, N, FAR>(dd + i, N, x);
    } else {
      const int at = i + N <= n ? i : n >= N ? n - N : 0;
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (at + e >= i && at + e < n && at + e >= par) dd[at + e] = static_cast<T>(x[e]);
    }
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    if (w[k] < 0) continue;
    const int j = k * THREADS + tid;
    float q = 0.f;
    bool first = true;
    if (LOOK && !twice) q = share[j];
    else
      for (int i = 0; i < top; ++i)
        if (place[i] == w[k]) q += share[i], first &= i >= j;
    if (first) dz[w[k]] = static_cast<T>(exp2_fast(fmaf(mine[k], c, -shift)) * scale - g * q);
  }
}

template <typename T, typename TT, typename IT>
hipError_t launch(const Args &A, hipStream_t st) {
  const unsigned grid = (unsigned)A.rows;
  const bool far = (double)A.rows * A.v * sizeof(T) > kLastLevelCache;      // of what nobody reads again
#define DISTILL(THREADS, GRADIENT)                                                                       \
  {                                                                                                      \
    if (far) topk_distill_kernel<T, TT, IT, THREADS, GRADIENT, true><<<grid, THREADS, 0, st>>>(A);       \
    else topk_distill_kernel<T, TT, IT, THREADS, GRADIENT, false><<<grid, THREADS, 0, st>>>(A);          \
    return hipGetLastError();                                                                            \
  }
  if (A.v <= 8192) {
    if (A.dz) DISTILL(256, true)
    DISTILL(256, false)
  }
  if constexpr (sizeof(T) == 2)
    if (A.v <= 16384) {
      if (A.dz) DISTILL(512, true)
      DISTILL(512, false)
    }
  if (A.dz) DISTILL(1024, true)
  DISTILL(1024, false)
#undef DISTILL
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
  if (q->rows > 1 << 21 || q->vocab > 1 << 30) return set_error(PBKD_EUNSUPPORTED, "topk_distill: %lld rows of %d logits", q->rows, q->vocab);
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
