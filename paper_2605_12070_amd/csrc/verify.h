// Internal interface of the draft verification kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dppo {

// A row's normaliser: p(v) = 2^((z[v] - m) t2e - log2s). The two are kept apart: their sum would lose
// log2s beside a far maximum.
struct VerifyNorm {
  double m, log2s;
};

// What a sequence draws its last token from.
struct VerifyDraw {
  VerifyNorm p, q;
  int32_t pos;           // accepted drafts: the position drawn at
  int32_t mode;          // a VerifyMode
};
enum VerifyMode {
  kDrawBad = 0,          // a row or an id that cannot be evaluated
  kDrawTarget = 1,       // r = p: every draft accepted
  kDrawResidual = 2,     // r = max(p - q, 0)
  kDrawWithout = 3,      // r = p without the drafted token (drafts without a distribution)
};

struct VerifyArgs {
  const void* target;
  const void* draft;     // NULL: drafts without a distribution
  int64_t target_seq, target_row, draft_seq, draft_row;
  int32_t B, D, V;
  const int64_t* ids;
  const int32_t* num;    // NULL: D
  const float* u;
  const float* u_new;
  double t2e;            // log2(e) / temperature
  int32_t* accepted;
  int64_t* tokens;
  float* logp;
  int32_t parts;         // workgroups per row of the statistics
  int32_t draw_parts;    // workgroups per sequence of the draw's weights
  int32_t cells;         // weight sums per sequence
  double* stats;         // [D + 1, B, 2, parts, 2] (maximum, sum) of the rows' parts
  double* cell;          // [B, cells]
  VerifyDraw* draw;      // [B]
};

// Fills parts, draw_parts and cells, and returns the workspace's bytes; with a workspace, the
// pointers into it as well.
int64_t verify_layout(VerifyArgs& a, int es, bool with_draft, void* workspace);
hipError_t launch_verify(const VerifyArgs& a, bool bf16, hipStream_t st);

}  // namespace dppo
