// Internal interface of the log probabilities (k_score.hip).
#pragma once

#include "serve_common.h"

namespace palq {

struct ScoreArgs {
  const void *x;                   // logits, rows ld elements apart
  int64_t rows, ld;
  int32_t vocab;
  float scale;
  const int32_t *ids;              // [rows][given]
  int32_t given;
  float *out;                      // [rows][given]
  float *entropy;                  // [rows], nullable
  int32_t top;
  int32_t *top_ids;                // [rows][top]
  float *top_out;
  int32_t step;                    // logits of a wave's step
  int32_t splits, each;            // parts of a row, of four waves with `each` steps; 0: a row is one wave's
  float *part;                     // their results (score_work_bytes)
};

// Chooses the parts, and the device memory for them.
void score_plan(ScoreArgs &a, int cus);
size_t score_work_bytes(const ScoreArgs &a);
hipError_t launch_score(const ScoreArgs &a, int type, hipStream_t s);

}  // namespace palq
