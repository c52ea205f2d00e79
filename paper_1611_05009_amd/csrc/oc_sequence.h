// Arguments of the row operators' kernels (norm, label log probabilities,
// gradient clipping), shared with the C entry points.
#pragma once
#include "oc_internal.h"

namespace oci {

// Element types (the header's OC_F32 ... values).
constexpr int kF32 = 0, kF16 = 1, kBF16 = 2, kF8 = 3;

// f(a value of the element type).
template <class F>
hipError_t by_type(int dtype, F f) {
  if (dtype == kF32) return f(float());
  if (dtype == kF16) return f(_Float16());
  return f(__bf16());
}

inline bool ok16(const void* p) { return ((uintptr_t)p & 15) == 0; }

struct NormArgs {
  const void *x, *residual;  // [rows][c]; residual may be null
  const float* weight;       // [c]
  int64_t rows;
  int c;
  float eps;
  void* sum;                 // [rows][c]: output of the forward pass (may be null), input of the gradient
  void* y;
  float* scale;              // [rows], 8-bit output only
  const void *dy, *dsum;     // gradient; dsum may be null
  void* dx;
  float* part;               // [norm_back_groups][c], or null
  int lanes;                 // set by the launch
};

constexpr int kNormMaxWidth = 32768;
int norm_back_groups(int64_t rows, int c);
hipError_t launch_rms_norm(NormArgs a, int x_type, int sum_type, int y_type, hipStream_t s);
hipError_t launch_rms_norm_back(NormArgs a, int sum_type, int y_type, float* dweight, hipStream_t s);

struct LabelArgs {
  const void* logits;        // [rows][classes]
  const int32_t* labels;     // [rows], outside [0, classes): none
  int64_t rows;
  int classes, top;
  float *logprob, *lse, *entropy;  // [rows]
  float* top_logprob;        // [rows][top]
  int32_t* top_label;
  // Long rows in parts: [rows][parts](3) statistics, [rows][parts][top] lists
  int parts, per;
  float *part_stat, *part_val;
  int* part_idx;
  // Gradient: lse and entropy are inputs
  const float *dlogprob, *dentropy;
  void* dlogits;
  int lanes;                 // set by the launch
};

constexpr int kMostTop = 32;
int label_parts(int64_t rows, int classes);
hipError_t launch_labels(LabelArgs a, int dtype, hipStream_t s);
hipError_t launch_labels_back(LabelArgs a, int dtype, hipStream_t s);

// Tensors of one launch of the gradient clipping, in its argument block.
constexpr int kClipBatch = 96;
struct ClipBatch {
  const void* in[kClipBatch];
  void* out[kClipBatch];
  int64_t count[kClipBatch];
  uint32_t first[kClipBatch + 1];  // first chunk of each tensor
  uint8_t type[kClipBatch];
  int n;
};
constexpr int64_t kClipChunk = 16384;   // elements of a workgroup's chunk
constexpr int kClipParts = 1024;        // workgroups, and partial sums, of a launch at most
hipError_t launch_square_sums(const ClipBatch& b, double* parts, int groups, hipStream_t s);
hipError_t launch_clip(const ClipBatch& b, const double* parts, int n_parts, float max_norm, float* norm, int groups,
                       hipStream_t s);

}  // namespace oci
