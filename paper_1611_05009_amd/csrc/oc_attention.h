// Arguments of the attention kernels, shared with the C entry points.
#pragma once
#include "oc_sequence.h"

namespace oci {

struct AttnArgs {
  const void *q, *k, *v;                 // [n_q][heads][dim], [n_k][kv_heads][dim] by strides
  int64_t q_row, q_head, k_row, k_head, v_row, v_head;  // strides in elements
  const int64_t *q_off, *k_off, *k_len;  // device; null: one sequence / whole key ranges
  int n_seq;
  int64_t n_q, n_k;
  int heads, kv_heads, dim;
  int group;                             // heads / kv_heads, and its division
  uint32_t div_mul;
  int div_shift;
  float scale;
  int causal;
  void* out;                             // [n_q][heads][dim]
  float* lse;                            // [n_q][heads]
  // Split keys (forward, dq: parts [n_split][n_q][heads](...)) or rows
  // (dk and dv: parts [n_split][2][n_k][kv_heads][dim])
  int n_split;
  float *part, *part_lse;
  // Backward
  const void* dout;                      // [n_q][heads][dim]
  float *delta, *lse2;                   // [n_q][heads] scratch
  void *dq, *dk, *dv;                    // contiguous, as out / the keys
};

// Fills group and its division from heads and kv_heads.
void attention_set_group(AttnArgs* a);
// Parts into which the keys of each row tile are split.
int attention_splits(int64_t n_q, int64_t n_k, int n_seq, int heads, int kv_heads, int dtype,
                     bool causal);
hipError_t launch_attention(const AttnArgs& a, int dtype, hipStream_t s);
// Parts of the gradients' kernels and the bytes that these take.
struct AttnParts {
  int dq, dkv;
  size_t bytes;
};
AttnParts attention_back_parts(int64_t n_q, int64_t n_k, int n_seq, int heads, int kv_heads, int dim,
                               int dtype, bool causal);
hipError_t launch_attention_backward(AttnArgs a, int dtype, hipStream_t s);

}  // namespace oci
