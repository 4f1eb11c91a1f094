// Internal interface of the distillation kernels.
#pragma once

#include "loss_stage.h"

namespace dppo {

// The row arguments (logits, dlogits, mask, token scale, flags, stats, scale; loss_tok is the
// per-token loss) and the teacher's record.
struct DistillArgs : RowArgs {
  const float* values;    // [T, k]
  const int32_t* tokens;  // [T, k], -1: empty
  const float* tlse;      // [T] the teacher's log-sum-exp, NULL: the record is renormalised
  int32_t k;
  float l2e;              // log2(e) / temperature, as the kernels use it on the student's logits
  double t2e;             // the same in 64 bits, for the record's values
  double inv_tau;
};

// Longest batch whose tokens every workgroup counts by itself; a kernel ahead counts longer ones. With
// and without it, bf16 and k = 16: 22 and 25 us at T = 1024, V = 1500, 27 and 26 at T = 4096; 250 and 208
// us at T = 65536; 1610 and 1516 us at T = 65536, V = 30000.
constexpr int64_t kDistillCountT = 4096;

hipError_t launch_distill(const DistillArgs& a, bool bf16, hipStream_t st);
// The loss and the counters from the rows' kl and flags (T = 0: zeros).
hipError_t launch_distill_sum(const DistillArgs& a, float* loss, hipStream_t st);

}  // namespace dppo
