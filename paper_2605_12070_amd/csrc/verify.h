// Internal interface of the draft verification kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dppo {

// A row's exact normaliser: p(v) = 2^((z[v] - m) t2e - log2s). The two are kept apart: their sum would
// lose log2s beside a far maximum.
struct VerifyNorm {
  double m, log2s;
};

// One part of a row's statistics: its sum of exponentials is about 2^n s (log2 units), its largest
// logit m.
struct VerifyPart {
  double n, s, m;
};

// What a sequence draws its last token from.
enum VerifyMode {
  kDrawBad = 0,          // a row or an id that cannot be evaluated
  kDrawTarget = 1,       // r = p: every draft accepted
  kDrawResidual = 2,     // r = max(p - q, 0)
  kDrawWithout = 3,      // r = p without the drafted token (drafts without a distribution)
};
struct VerifyDraw {
  // The weights' scales: p = 2^((z K + sp) / 64) up to a factor near 1 that the cells' sums correct,
  // q likewise with sq, times phi (sp and sq are integers; phi is what rounding them cost).
  double sp, sq, phi;
  VerifyNorm p, q;       // far rows: exact normalisers instead
  int32_t pos;           // accepted drafts: the position drawn at
  int32_t mode;          // a VerifyMode
  int32_t far;
};

// Sums over a cell of a row drawn from (written as four doubles in this order).
struct VerifyCell {
  double r;              // weights, with p and q as scaled
  double slope;          // q over the entries with a positive weight: d r / d (scale of q) = -slope
  double p, q;           // p and q
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
  VerifyPart* stats;     // [D + 1, B, 2, parts]
  VerifyCell* cell;      // [B, cells]
  VerifyDraw* draw;      // [B]
};

// Fills parts, draw_parts and cells, and returns the workspace's bytes; with a workspace, the
// pointers into it as well.
int64_t verify_layout(VerifyArgs& a, int es, bool with_draft, void* workspace);
hipError_t launch_verify(const VerifyArgs& a, bool bf16, hipStream_t st);

}  // namespace dppo
