// Internal interface of the top-logits kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dppo {

struct TopArgs {
  const void* logits;  // row t at logits + t * ld
  int64_t ld;
  int32_t T, V, k;
  int32_t parts;       // workgroups per row
  float l2e;           // log2(e) / temperature
  double t2e;          // the same in 64 bits, for far rows
  float* values;       // [T, k]
  int32_t* ids;        // [T, k]
  float* lse;          // [T]
  uint64_t* cand;      // parts > 1: [T, parts, k] composites, best first, 0 where a part has none
  float* part;         // parts > 1: [T, parts, 2] (n, s) of the parts' sums of exponentials
};

// Workgroups per row for the k largest of T rows of V entries of es bytes.
int top_parts(int64_t T, int64_t V, int es, int k);
hipError_t launch_top_logits(const TopArgs& a, bool bf16, hipStream_t st);

}  // namespace dppo
