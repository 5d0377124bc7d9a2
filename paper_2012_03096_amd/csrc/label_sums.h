// Sums of rows by their label, each with a weight (embed.hip: the embedding's gradient for the vocabulary loss).
//
//   out_v = scale * (base_{slot_v} + sum over n with label_n = v of weight_n row_n), rounded once, for the labels v that occur; the other rows of out stay as they are
#pragma once
#include <cstddef>

#include <hip/hip_runtime.h>

namespace pbkd {

struct LabelSums {
  const void *rows;          // [n, d], of dtype PBKD_BF16 or PBKD_F16, strided
  long long stride;
  const void *labels;        // [n], of 32 or 64 bits; those outside 0..vocab-1 name nothing
  bool wide;
  int dtype, n, vocab, d;
  const float *weights;      // [n]
  int *slot;                 // [vocab]: which row of base is a label's, -1 for those that do not occur
  const float *base;         // [n, base_ld]
  long long base_ld;
  const float *scale;
  void *out;                 // [vocab, d], strided
  long long out_stride;
};

// Up to here one launch finds a label's rows among all, and slot is the caller's to give: the first row that has the label.  Beyond, rows are sorted first, and
// launch_label_sort() writes slot.  Measured (bf16, with the call around it): 1500 rows of 8192 x 1024 210 us, sorted 215; 2048 of 2000 x 512 77, 87; 2000 of 50000 x 2048 1653, 1636.
constexpr int kFewLabels = 2048;

size_t label_sums_bytes(int n, int vocab, int d);
// workspace: label_sums_bytes(), 256-byte aligned, the same for both
hipError_t launch_label_sort(const LabelSums &q, char *workspace, hipStream_t st);
hipError_t launch_label_sums(const LabelSums &q, char *workspace, hipStream_t st);

}  // namespace pbkd
