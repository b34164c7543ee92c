// Launchers of a feed-forward block's products where they are small (products_few.cu), and when
// that is.
#pragma once

#include "dlm_internal.h"

namespace dlm {

// How a product runs, and its time as the plan has it.
struct FewPlan {
  int n, splits;  // rows of a tile, CTAs that share its K
  double us;
};

// The rows and splits that end first. rows: of the result (`matrices` results side by side);
// row_tiles: tiles across it; outer: both operands MN-major, tiles of whole 64s of rows. splits:
// these alone (0: any), or one where that is allowed too.
FewPlan plan_few(int64_t rows, int64_t row_tiles, int64_t kblocks, int matrices, bool outer, int splits = 0, bool or_one = false);
// The CTAs of launch_few_outer, those of the whole GPU at most where K is not split.
int64_t few_outer_ctas(int64_t rows, int64_t row_tiles, int matrices, const FewPlan& plan);

int launch_few_gated(const GatedArgs& a, const FewPlan& plan, cudaStream_t stream);
// out = act(x w^T + bias) + residual (turned: w's columns instead of its rows; up to two runs of K).
int launch_few_cols(const Matrix* x, const Matrix* w, int runs, bool turned, const Epilogue& ep, const FewPlan& plan,
                    cudaStream_t stream);
// out[i] = z[i]^T x for one or two matrices z of the same shape.
int launch_few_outer(const Matrix* z, const Matrix& x, const Matrix* out, int count, const FewPlan& plan, cudaStream_t stream);
// Both from z in one launch: dx = sum z[i] w[i] + what ep adds, dw[i] = z[i]^T x. The plan of dw
// has one split, or as many as that of dx.
int launch_few_gradients(const Matrix* z, const Matrix* w, int count, const Epilogue& ep, const FewPlan& x_plan, const Matrix& x,
                         const Matrix* dw, const FewPlan& w_plan, cudaStream_t stream);

}  // namespace dlm
