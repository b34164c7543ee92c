// The forms that a feed-forward block's products take, chosen by their sizes on the host alone, and the
// launchers of those where they are small (products_few.cu).
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

// A product on pairs of CTAs (product_kernel, tiles of `bn` columns), or a small one.
struct ProductPlan {
  bool pairs;
  int bn;       // pairs only
  FewPlan few;  // of the others
  double us;
};
// Pairs of CTAs that run at once on the current device: of a gated block, a projection, d x and dW.
struct ProductPairs {
  int gated, cols, turned, rows;
};
ProductPairs product_pairs();
// workers: pairs of CTAs that run at once; kblocks: K steps of 64, of all runs.
ProductPlan plan_gated(int64_t N, int64_t f, int64_t kblocks, int workers);
// A result of N x M (turned: by the weight's columns, d x).
ProductPlan plan_cols(int64_t N, int64_t M, int64_t kblocks, bool turned, int workers);
// dW = dz^T x, M x d, for `count` matrices dz.
ProductPlan plan_rows(int64_t M, int64_t d, int64_t kblocks, int count, int workers);
// Both gradients of N rows through weights of m x d: in one launch of small products, or each by itself.
struct GradientsPlan {
  bool together;
  ProductPlan x, w;
};
GradientsPlan plan_gradients(int64_t N, int64_t m, int64_t d, int count, int x_workers, int w_workers);

// How the columns of N x m are summed for the bias's gradient.
struct BiasSplit {
  int lanes;     // of eight columns, in a CTA's strip
  int64_t runs;  // of rows, whose sums are kept and added by a launch of their own where there are several
  int ranks;     // CTAs of a cluster that share a run
};
BiasSplit bias_split(int64_t N, int64_t m);

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
