// Root-mean-square norm with the residual's addition, forward (output in the activations' type or in 8 bits with row
// scales) and backward, and the column sums that finish weight gradients of the sequence operators.
//
//   forward    s = x + residual, r = 1/sqrt(mean s^2 + eps), y = s r w
//   backward   g = dy w, dx = r (g - s r mean(g s r)) + dtotal, dweight = sum over rows of dy s r
//
// Both are bound by memory: a row is read once into registers (eight elements a lane and item, 16 bytes of a 16-bit type),
// its sums are taken in fp32 over a wave or a workgroup, and the outputs are formed from the registers.
//
// Measured (bf16, with the residual): 16383 rows of 4096 to 8 bits 79 us, 5.9 TB/s; 32768 rows of 2048 forward and backward
// 179 us, 6.0 TB/s, what a large sum of two tensors reaches on this card; 16 rows of 2048 to 8 bits 3.4 us, which is a launch's own length.
#include "seq_common.h"

namespace pbkd {
namespace {

constexpr int kMaxD = 16384;         // 1024 threads x 2 items x 8 elements: four items spill in the backward kernel

// Threads to a row: eight elements each as long as that goes.  Measured (bf16): 16383 rows of 4096 forward to e4m3, 512 threads
// 86 us, 256 threads with 16 elements 97 us, 64 with 64 elements 130 us; 32768 rows of 2048 backward, 256 threads 126 us, 64 with
// 32 elements 167 us: more waves with fewer registers keep more reads on their way, which is worth the barrier in the sums.
inline int row_threads(int d) { return d <= 512 ? 64 : d <= 1024 ? 128 : d <= 2048 ? 256 : d <= 4096 ? 512 : 1024; }

// Workgroups of the backward kernel: two waves for each SIMD, with the next row on its way (four: 203 against 198 us for 32768 rows of
// 2048 forward and backward, and twice the partials).  Each leaves one row of weight-gradient partials.
constexpr int kBwdThreads = 128 * 1024;
inline int bwd_groups(long long rows, int d) {
  const int tpr = row_threads(d);
  const long long groups = tpr == 64 ? cdiv64(rows, 4) : rows;
  const int most = kBwdThreads / (tpr == 64 ? 256 : tpr);
  return (int)(groups < most ? groups : most);
}

struct FwdArgs {
  const void *x, *res;
  const float *w;
  void *total, *y;
  float *scale;
  long long rows, xs, rs, ts, ys;
  int d;
  float eps;
};

struct BwdArgs {
  const void *total, *dy, *dtotal;
  const float *w;
  void *dx;
  float *partial;
  long long rows, ts, ys, gs, xs;
  int d;
  float eps;
};

template <typename T>
using Raw = typename VecOf<T, 8>::type;

// Sum (or maximum) over the TPR threads of a row, known to all of them.  `slot` holds one float per wave; callers alternate
// between two of them, so that the barrier inside also keeps a slot's readers ahead of its next writers.
template <int TPR, bool MAX>
__device__ __forceinline__ float row_reduce(float v, float *slot) {
  v = MAX ? wave64_max(v) : wave64_sum(v);
  if (TPR == 64) return v;
  constexpr int W = TPR / 64;
  if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = v;
  __syncthreads();
  float t = slot[0];
#pragma unroll
  for (int k = 1; k < W; ++k) t = MAX ? fmaxf(t, slot[k]) : t + slot[k];
  return t;
}

// TPR threads take a row, at most 4096 workgroups go through the rows: the weight is read once by each, and its registers live on.
template <typename T, int TPR, int ITEMS, bool FP8, bool FAR>
__global__ __launch_bounds__(TPR == 64 ? 256 : TPR) void rmsnorm_fwd_kernel(FwdArgs A) {
  constexpr int RPB = TPR == 64 ? 4 : 1;             // rows a workgroup works on at a time
  __shared__ float red[4][16];
  const int lane = threadIdx.x % TPR, d = A.d;
  float w[ITEMS][8];
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    const int c = (k * TPR + lane) * 8;
    load_n<float, 8>(A.w + c, d - c, w[k]);
  }
  int flip = 0;
  for (long long row = (long long)blockIdx.x * RPB + threadIdx.x / TPR; row < A.rows; row += (long long)gridDim.x * RPB, flip ^= 2) {
    float s[ITEMS][8];
    const T *x = static_cast<const T *>(A.x) + row * A.xs;
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      const int c = (k * TPR + lane) * 8;
      load_n<T, 8, FAR>(x + c, d - c, s[k]);
    }
    if (A.res) {
      const T *r = static_cast<const T *>(A.res) + row * A.rs;
#pragma unroll
      for (int k = 0; k < ITEMS; ++k) {
        const int c = (k * TPR + lane) * 8;
        float q[8];
        load_n<T, 8, FAR>(r + c, d - c, q);
#pragma unroll
        for (int i = 0; i < 8; ++i) s[k][i] += q[i];
      }
    }
    float ss = 0.f;
#pragma unroll
    for (int k = 0; k < ITEMS; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = fmaf(s[k][i], s[k][i], ss);
    ss = row_reduce<TPR, false>(ss, red[flip]);
    const float rms = sqrtf(ss / d + A.eps), r = 1.f / rms;
    const bool mend = r > 0.f && r < __builtin_inff();
    if (A.total) {
      T *t = static_cast<T *>(A.total) + row * A.ts;
#pragma unroll
      for (int k = 0; k < ITEMS; ++k) {
        const int c = (k * TPR + lane) * 8;
        store_n<T, 8, FAR>(t + c, d - c, s[k]);
      }
    }
#pragma unroll
    for (int k = 0; k < ITEMS; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        // s / rms to its last place: the product's remainder is put right.  Each step is rounded as the formula has it, so that a code in the
        // middle between two falls as it does where the steps are operations of their own: of 435 codes in 759M that are not the nearest to
        // the exact ones 375 are theirs too; s w over its own maximum, two roundings less, has 312, but other ones
        float q = s[k][i] * r;
        q = mend ? fmaf(fmaf(-q, rms, s[k][i]), r, q) : q;
        s[k][i] = q * w[k][i];
      }
    if (FP8) {
      float top = 0x1p-100f;
#pragma unroll
      for (int k = 0; k < ITEMS; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(s[k][i]));
      top = row_reduce<TPR, true>(top, red[flip + 1]);
      const float inv = 1.f / top * 448.f;   // |y| inv exceeds 448 by rounding only, far below where e4m3 would overflow
      if (lane == 0) A.scale[row] = top * (1.f / 448.f);
      unsigned char *y = static_cast<unsigned char *>(A.y) + row * A.ys;
#pragma unroll
      for (int k = 0; k < ITEMS; ++k) {
        const int c = (k * TPR + lane) * 8;
        unsigned q[2];
        q[0] = pack_e4m3(s[k][0] * inv, s[k][1] * inv, s[k][2] * inv, s[k][3] * inv);
        q[1] = pack_e4m3(s[k][4] * inv, s[k][5] * inv, s[k][6] * inv, s[k][7] * inv);
        if (c + 8 <= d) {
          far_store<FAR, unsigned char, 8>(__builtin_bit_cast(Raw<unsigned char>, q), y + c);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (c + i < d) y[c + i] = static_cast<unsigned char>(q[i >> 2] >> (8 * (i & 3)));
        }
      }
    } else {
      T *y = static_cast<T *>(A.y) + row * A.ys;
#pragma unroll
      for (int k = 0; k < ITEMS; ++k) {
        const int c = (k * TPR + lane) * 8;
        store_n<T, 8, FAR>(y + c, d - c, s[k]);
      }
    }
  }
}

template <bool FAR, typename T>
__device__ __forceinline__ Raw<T> raw_n(const T *p, int n) {
  Raw<T> r;
  if (n >= 8) {
    r = far_load<FAR, T, 8>(p);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = i < n ? p[i] : T(0.f);
  }
  return r;
}

// A workgroup goes through its rows with the weight gradient of its own columns in registers, the next row on its way while it
// works on one, and leaves one row of partials; with a wave to a row its four waves' sums are joined through LDS first.
template <typename T, int TPR, int ITEMS, bool FAR>
__global__ __launch_bounds__(TPR == 64 ? 256 : TPR) void rmsnorm_bwd_kernel(BwdArgs A) {
  constexpr int RPB = TPR == 64 ? 4 : 1;
  constexpr bool AHEAD = ITEMS == 1;      // with two items the next row does not fit in the registers
  __shared__ float red[4][16];
  __shared__ float join[RPB > 1 ? (RPB - 1) * TPR * ITEMS * 8 : 1];
  const int lane = threadIdx.x % TPR, sub = threadIdx.x / TPR, d = A.d;
  const T *tp = static_cast<const T *>(A.total), *yp = static_cast<const T *>(A.dy), *gp = static_cast<const T *>(A.dtotal);
  T *xp = static_cast<T *>(A.dx);
  float dw[ITEMS][8] = {}, w[ITEMS][8];
  Raw<T> s[ITEMS], y[ITEMS], g[ITEMS];
  long long row = (long long)blockIdx.x * RPB + sub;
  const long long step = (long long)gridDim.x * RPB;
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    const int c = (k * TPR + lane) * 8;
    load_n<float, 8>(A.w + c, d - c, w[k]);
    if (AHEAD && row < A.rows) {
      s[k] = raw_n<FAR>(tp + row * A.ts + c, d - c), y[k] = raw_n<FAR>(yp + row * A.ys + c, d - c);
      if (A.dtotal) g[k] = raw_n<FAR>(gp + row * A.gs + c, d - c);
    }
  }
  int flip = 0;
  for (; row < A.rows; row += step, flip ^= 2) {
    float sv[ITEMS][8], yv[ITEMS][8], ss = 0.f, gs = 0.f;
    Raw<T> gr[ITEMS];
    const long long next = row + step;
    if (!AHEAD) {
#pragma unroll
      for (int k = 0; k < ITEMS; ++k) {
        const int c = (k * TPR + lane) * 8;
        s[k] = raw_n<FAR>(tp + row * A.ts + c, d - c), y[k] = raw_n<FAR>(yp + row * A.ys + c, d - c);
        if (A.dtotal) g[k] = raw_n<FAR>(gp + row * A.gs + c, d - c);
      }
    }
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      const int c = (k * TPR + lane) * 8;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        sv[k][i] = static_cast<float>(s[k][i]), yv[k][i] = static_cast<float>(y[k][i]);
        ss = fmaf(sv[k][i], sv[k][i], ss);
        gs = fmaf(yv[k][i] * w[k][i], sv[k][i], gs);
      }
      gr[k] = g[k];
      if (AHEAD && next < A.rows) {
        s[k] = raw_n<FAR>(tp + next * A.ts + c, d - c), y[k] = raw_n<FAR>(yp + next * A.ys + c, d - c);
        if (A.dtotal) g[k] = raw_n<FAR>(gp + next * A.gs + c, d - c);
      }
    }
    ss = row_reduce<TPR, false>(ss, red[flip]);
    gs = row_reduce<TPR, false>(gs, red[flip + 1]);
    const float r = 1.f / sqrtf(ss / d + A.eps), mean = gs * r / d;
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      const int c = (k * TPR + lane) * 8;
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float xh = sv[k][i] * r;
        v[i] = r * (yv[k][i] * w[k][i] - xh * mean);
        if (A.dtotal) v[i] += static_cast<float>(gr[k][i]);
        dw[k][i] = fmaf(yv[k][i], xh, dw[k][i]);
      }
      store_n<T, 8, FAR>(xp + row * A.xs + c, d - c, v);
    }
  }
  if (RPB > 1) {
    if (sub > 0) {
#pragma unroll
      for (int k = 0; k < ITEMS; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) join[((sub - 1) * ITEMS * 8 + k * 8 + i) * TPR + lane] = dw[k][i];
    }
    __syncthreads();
    if (sub > 0) return;
#pragma unroll
    for (int j = 0; j < RPB - 1; ++j)
#pragma unroll
      for (int k = 0; k < ITEMS; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[k][i] += join[(j * ITEMS * 8 + k * 8 + i) * TPR + lane];
  }
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    const int c = (k * TPR + lane) * 8;
    store_n<float, 8>(A.partial + (long long)blockIdx.x * d + c, d - c, dw[k]);
  }
}

// out[slab][c] = sum of the slab's rows of partial[rows][cols]: 16 columns a workgroup, a slab's rows over 64 groups of 16
// threads, which are joined in order.  rows == 0 writes zeros.  Bound by its launch and two round trips to memory: 512 rows of 2048
// (4 MB, out of the last-level cache) 5.1 us.
__global__ __launch_bounds__(1024) void colsum_kernel(const float *partial, long long rows, int cols, int per_slab, float *out) {
  __shared__ float part[64][17];
  const int lane = threadIdx.x & 15, g = threadIdx.x >> 4, c = blockIdx.x * 16 + lane;
  const long long lo = (long long)blockIdx.y * per_slab, hi = lo + per_slab < rows ? lo + per_slab : rows;
  float v = 0.f;
  if (c < cols) {
#pragma unroll 16
    for (long long r = lo + g; r < hi; r += 64) v += partial[r * cols + c];
  }
  part[g][lane] = v;
  __syncthreads();
  if (g < 8) {
#pragma unroll
    for (int k = 1; k < 8; ++k) v += part[g + 8 * k][lane];
    part[g][lane] = v;       // only this thread reads or writes it here
  }
  __syncthreads();
  if (g == 0 && c < cols) {
#pragma unroll
    for (int k = 1; k < 8; ++k) v += part[k][lane];
    out[(long long)blockIdx.y * cols + c] = v;
  }
}

constexpr int kSlab = 2048;
static_assert(kBwdThreads / 128 <= kSlab, "the norm's partials are summed in one pass, without scratch");

template <typename T, bool FP8>
hipError_t launch_fwd(const FwdArgs &A, hipStream_t st) {
  const int d = A.d;
  const bool far = (double)A.rows * d * (sizeof(T) * (1 + (A.res != nullptr) + (A.total != nullptr)) + (FP8 ? 1 : sizeof(T))) > kLastLevelCache;
#define FWD(TPR, ITEMS)                                                                                              \
  {                                                                                                                  \
    const long long groups = cdiv64(A.rows, TPR == 64 ? 4 : 1);                                                      \
    const unsigned grid = (unsigned)(groups < 4096 ? groups : 4096), threads = TPR == 64 ? 256 : TPR;                 \
    if (far) rmsnorm_fwd_kernel<T, TPR, ITEMS, FP8, true><<<grid, threads, 0, st>>>(A);                               \
    else rmsnorm_fwd_kernel<T, TPR, ITEMS, FP8, false><<<grid, threads, 0, st>>>(A);                                  \
  }
  switch (row_threads(d)) {
    case 64: FWD(64, 1) break;
    case 128: FWD(128, 1) break;
    case 256: FWD(256, 1) break;
    case 512: FWD(512, 1) break;
    default:
      if (d <= 8192) FWD(1024, 1)
      else FWD(1024, 2)
  }
#undef FWD
  return hipGetLastError();
}

template <typename T>
hipError_t launch_bwd(const BwdArgs &A, int groups, hipStream_t st) {
  const int d = A.d;
  const bool far = (double)A.rows * d * sizeof(T) * (3 + (A.dtotal != nullptr)) > kLastLevelCache;
#define BWD(TPR, ITEMS)                                                                             \
  {                                                                                                 \
    const unsigned threads = TPR == 64 ? 256 : TPR;                                                 \
    if (far) rmsnorm_bwd_kernel<T, TPR, ITEMS, true><<<groups, threads, 0, st>>>(A);                \
    else rmsnorm_bwd_kernel<T, TPR, ITEMS, false><<<groups, threads, 0, st>>>(A);                   \
  }
  switch (row_threads(d)) {
    case 64: BWD(64, 1) break;
    case 128: BWD(128, 1) break;
    case 256: BWD(256, 1) break;
    case 512: BWD(512, 1) break;
    default:
      if (d <= 8192) BWD(1024, 1)
      else BWD(1024, 2)
  }
#undef BWD
  return hipGetLastError();
}

pbkd_status check_rows(long long rows, int d, int dtype, float eps) {
  if (rows < 0 || d < 1) return set_error(PBKD_ESHAPE, "rmsnorm: %lld rows of %d elements", rows, d);
  if (d > kMaxD) return set_error(PBKD_EUNSUPPORTED, "rmsnorm: rows of %d elements, at most %d", d, kMaxD);
  if (dtype != PBKD_F32 && dtype != PBKD_BF16 && dtype != PBKD_F16) return set_error(PBKD_EINVAL, "rmsnorm: dtype %d", dtype);
  if (!(eps >= 0.f)) return set_error(PBKD_EINVAL, "rmsnorm: eps must not be negative");
  return PBKD_OK;
}

inline bool misaligned(const void *p, int size) { return (reinterpret_cast<uintptr_t>(p) & (size - 1)) != 0; }

}  // namespace

size_t colsum_scratch_floats(long long rows, int cols) { return rows > kSlab ? (size_t)cdiv64(rows, kSlab) * cols + colsum_scratch_floats(cdiv64(rows, kSlab), cols) : 0; }

hipError_t launch_colsum(const float *partial, long long rows, int cols, float *scratch, float *out, hipStream_t st) {
  while (rows > kSlab) {
    const long long slabs = cdiv64(rows, kSlab);
    colsum_kernel<<<dim3((cols + 15) / 16, (unsigned)slabs), 1024, 0, st>>>(partial, rows, cols, kSlab, scratch);
    partial = scratch, scratch += slabs * cols, rows = slabs;
  }
  colsum_kernel<<<dim3((cols + 15) / 16, 1), 1024, 0, st>>>(partial, rows, cols, kSlab, out);
  return hipGetLastError();
}

}  // namespace pbkd

using namespace pbkd;

extern "C" {

pbkd_status pbkd_rmsnorm_forward(const pbkd_rmsnorm_desc *q, void *hip_stream) {
  if (!q) return set_error(PBKD_EINVAL, "rmsnorm: null descriptor");
  if (const pbkd_status s = check_rows(q->rows, q->d, q->dtype, q->eps)) return s;
  const bool fp8 = q->y_dtype == PBKD_E4M3;
  if (!fp8 && q->y_dtype != q->dtype) return set_error(PBKD_EINVAL, "rmsnorm: y_dtype must be dtype or PBKD_E4M3");
  if (q->rows == 0) return PBKD_OK;
  if (!q->x_dev || !q->weight_dev || !q->y_dev || (fp8 && !q->scale_dev)) return set_error(PBKD_EINVAL, "rmsnorm: null tensor");
  const int size = q->dtype == PBKD_F32 ? 4 : 2;
  if (misaligned(q->x_dev, size) || misaligned(q->residual_dev, size) || misaligned(q->total_dev, size) || misaligned(q->y_dev, fp8 ? 1 : size) ||
      misaligned(q->weight_dev, 4) || misaligned(q->scale_dev, 4))
    return set_error(PBKD_EINVAL, "rmsnorm: a tensor is not aligned to its elements");
  if (q->x_stride < 0 || q->residual_stride < 0) return set_error(PBKD_EINVAL, "rmsnorm: negative stride");
  if (q->rows > 1 && (q->y_stride < q->d || (q->total_dev && q->total_stride < q->d)))
    return set_error(PBKD_ESHAPE, "rmsnorm: rows of an output overlap");
  if (q->total_dev && q->total_dev == q->y_dev) return set_error(PBKD_EINVAL, "rmsnorm: total and y are the same tensor");
  FwdArgs A{q->x_dev, q->residual_dev, q->weight_dev, q->total_dev, q->y_dev, q->scale_dev, q->rows, q->x_stride, q->residual_stride, q->total_stride,
            q->y_stride, q->d, q->eps};
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  switch (q->dtype) {
    case PBKD_F32: SEQ_HIPCHK((fp8 ? launch_fwd<float, true>(A, st) : launch_fwd<float, false>(A, st))); break;
    case PBKD_BF16: SEQ_HIPCHK((fp8 ? launch_fwd<bf16, true>(A, st) : launch_fwd<bf16, false>(A, st))); break;
    default: SEQ_HIPCHK((fp8 ? launch_fwd<f16, true>(A, st) : launch_fwd<f16, false>(A, st))); break;
  }
  return PBKD_OK;
}

size_t pbkd_rmsnorm_workspace_bytes(long long rows, int d) {
  if (rows < 0 || d < 1 || d > kMaxD) return 0;
  const size_t n = (size_t)bwd_groups(rows, d) * d * sizeof(float);
  return (n + 255) / 256 * 256 + 256;
}

pbkd_status pbkd_rmsnorm_backward(const pbkd_rmsnorm_grad_desc *q, void *hip_stream) {
  if (!q) return set_error(PBKD_EINVAL, "rmsnorm: null descriptor");
  if (const pbkd_status s = check_rows(q->rows, q->d, q->dtype, q->eps)) return s;
  if (!q->dweight_dev || !q->weight_dev || (q->rows && (!q->total_dev || !q->dy_dev || !q->dx_dev))) return set_error(PBKD_EINVAL, "rmsnorm: null tensor");
  const int size = q->dtype == PBKD_F32 ? 4 : 2;
  if (misaligned(q->total_dev, size) || misaligned(q->dy_dev, size) || misaligned(q->dtotal_dev, size) || misaligned(q->dx_dev, size) ||
      misaligned(q->weight_dev, 4) || misaligned(q->dweight_dev, 4))
    return set_error(PBKD_EINVAL, "rmsnorm: a tensor is not aligned to its elements");
  if (q->total_stride < 0 || q->dy_stride < 0 || q->dtotal_stride < 0) return set_error(PBKD_EINVAL, "rmsnorm: negative stride");
  if (q->rows > 1 && q->dx_stride < q->d) return set_error(PBKD_ESHAPE, "rmsnorm: rows of an output overlap");
  if (!q->workspace_dev || misaligned(q->workspace_dev, 256)) return set_error(PBKD_ENOMEM, "rmsnorm: the workspace must be 256-byte aligned");
  if (q->workspace_bytes < pbkd_rmsnorm_workspace_bytes(q->rows, q->d))
    return set_error(PBKD_ENOMEM, "rmsnorm: workspace of %zu bytes is smaller than the %zu needed", q->workspace_bytes, pbkd_rmsnorm_workspace_bytes(q->rows, q->d));
  float *partial = static_cast<float *>(q->workspace_dev);
  const int groups = bwd_groups(q->rows, q->d);
  BwdArgs A{q->total_dev, q->dy_dev, q->dtotal_dev, q->weight_dev, q->dx_dev, partial, q->rows, q->total_stride, q->dy_stride, q->dtotal_stride,
            q->dx_stride, q->d, q->eps};
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (groups > 0) {
    switch (q->dtype) {
      case PBKD_F32: SEQ_HIPCHK(launch_bwd<float>(A, groups, st)); break;
      case PBKD_BF16: SEQ_HIPCHK(launch_bwd<bf16>(A, groups, st)); break;
      default: SEQ_HIPCHK(launch_bwd<f16>(A, groups, st)); break;
    }
  }
  SEQ_HIPCHK(launch_colsum(partial, groups, q->d, nullptr, q->dweight_dev, st));     // at most kSlab rows: no scratch
  return PBKD_OK;
}

}  // extern "C"
