"""Sizes for each form that the feed-forward block's products take, and the library's own word on
which one a size takes: the plans of csrc/products.h, called through a few lines of C++ that link the
built library.

A form is "pairs128" / "pairs256" (pairs of CTAs, tiles of 128 / 256 columns) or "few<n>/<s>" (single
CTAs, tiles of n rows, K split over s of them). Widths are odd multiples of 8 and rows odd numbers, so
that every last tile and the last step of K are ragged; sizes for pairs give some of them three
tiles and more, so that an accumulator is used again, except where a name ends in " few tiles"."""
import ctypes
import os
import subprocess

PROGRAM = r"""
#include "products.h"
using namespace dlm;
extern "C" {
static void put(const ProductPlan& p, int64_t* o) {
  o[0] = p.pairs;
  o[1] = p.pairs ? p.bn : p.few.n;
  o[2] = p.pairs ? 0 : p.few.splits;
}
void pairs(int32_t* o) {
  const ProductPairs p = product_pairs();
  o[0] = p.gated, o[1] = p.cols, o[2] = p.turned, o[3] = p.rows;
}
void gated(int64_t N, int64_t d, int64_t f, const int32_t* w, int64_t* o) { put(plan_gated(N, f, (d + 63) / 64, w[0]), o); }
void cols(int64_t N, int64_t k, int64_t m, const int32_t* w, int64_t* o) { put(plan_cols(N, m, (k + 63) / 64, false, w[1]), o); }
void gradients(int64_t N, int64_t k, int64_t m, int32_t count, const int32_t* w, int64_t* o) {
  const GradientsPlan g = plan_gradients(N, m, k, count, w[2], w[3]);
  o[0] = g.together;
  put(g.x, o + 1);
  put(g.w, o + 4);
}
void bias(int64_t N, int64_t m, int64_t* o) {
  const BiasSplit b = bias_split(N, m);
  o[0] = b.lanes, o[1] = b.runs, o[2] = b.ranks;
}
}
"""

# rows, width, inner width: x [N, d], weights [f, d]
GATED = [(2, 520, 2472, "few16/1"), (2, 1048, 2440, "few16/2"), (2, 2088, 1224, "few16/4"), (2, 4104, 72, "few16/8"),
         (17, 536, 5000, "few32/1"), (17, 1048, 2456, "few32/2"), (305, 2056, 72, "few32/4"), (17, 4328, 584, "few32/8"),
         (35, 520, 5192, "few64/1"), (1290, 1496, 72, "few64/2"), (618, 2072, 72, "few64/4"), (305, 4168, 72, "few64/8"),
         (65, 520, 9736, "few128/1"), (66, 72, 10248, "few128/1"), (1393, 2712, 72, "few128/4"),
         (13193, 72, 136, "pairs128"), (145, 552, 9896, "pairs128"), (523, 72, 8680, "pairs256"), (259, 536, 9752, "pairs256")]

# rows, width, output columns: x [N, k], weight [m, k]
COLS = [(2, 520, 5000, "few16/1"), (2, 1064, 5000, "few16/2"), (2, 2136, 2456, "few16/4"), (2, 4104, 72, "few16/8"),
        (17, 520, 9832, "few32/1"), (635, 1048, 136, "few32/2"), (311, 2072, 136, "few32/4"), (145, 4184, 136, "few32/8"),
        (33, 536, 9752, "few64/1"), (1238, 1496, 136, "few64/2"), (624, 2056, 136, "few64/4"), (309, 4248, 136, "few64/8"),
        (9781, 72, 136, "few128/1"), (9964, 520, 136, "few128/1"), (2498, 4072, 136, "few128/2"), (1233, 2696, 136, "few128/4"),
        (13283, 264, 264, "pairs128"), (13521, 520, 264, "pairs128"), (16227, 328, 552, "pairs256"), (17123, 520, 520, "pairs256")]

# weights, rows, width, inner width; one launch for both or not; dx's form, dW's
GRADIENTS = [
    (1, 2, 72, 392, "together", "few16/4", "few128/1"), (1, 2, 2120, 584, "together", "few16/2", "few128/1"),
    (1, 394, 72, 72, "together", "few16/2", "few64/2"), (1, 398, 72, 1160, "together", "few16/4", "few64/4"),
    (1, 1153, 72, 4952, "together", "few16/2", "few128/2"), (1, 67, 3864, 72, "together", "few32/1", "few128/1"),
    (1, 147, 136, 1816, "together", "few32/8", "few128/1"), (1, 740, 72, 2584, "together", "few32/4", "few128/4"),
    (1, 774, 72, 456, "together", "few64/8", "few64/8"), (1, 1243, 136, 72, "together", "few64/2", "few64/2"),
    (1, 515, 4264, 72, "together", "few128/1", "few128/1"), (1, 857, 648, 776, "together", "few128/2", "few128/2"),
    (1, 773, 264, 1672, "together", "few128/4", "few128/1"),
    (1, 201, 4904, 72, "apart", "few32/1", "few128/1"), (1, 3717, 72, 72, "apart", "few32/1", "few64/8"),
    (1, 580, 3528, 72, "apart", "few64/1", "few64/2"), (1, 1761, 1320, 72, "apart", "few128/1", "few64/4"),
    (1, 2795, 2456, 72, "apart", "few128/1", "few128/4"), (1, 13283, 264, 264, "apart", "pairs128", "few64/8"),
    (1, 2770, 3880, 264, "apart", "pairs128", "pairs128 few tiles"), (1, 16409, 520, 328, "apart", "pairs256", "few64/8"),
    (1, 3209, 296, 3480, "apart", "pairs128 few tiles", "pairs128 few tiles"),
    (1, 2697, 2056, 1064, "apart", "pairs256 few tiles", "pairs256 few tiles"),
    (1, 530, 4648, 2824, "apart", "pairs256 few tiles", "pairs256"),
    (1, 2945, 264, 6424, "apart", "few128/2", "pairs256 few tiles"),
    (2, 2, 72, 392, "together", "few16/8", "few128/1"), (2, 390, 72, 600, "together", "few16/4", "few64/4"),
    (2, 645, 72, 1304, "together", "few32/4", "few128/4"), (2, 129, 3944, 72, "together", "few128/2", "few128/1"),
    (2, 34, 5032, 856, "together", "few64/2", "few128/1"), (2, 780, 72, 200, "together", "few64/8", "few64/8"),
    (2, 837, 1224, 200, "together", "few128/2", "few128/2"), (2, 783, 264, 792, "together", "few128/4", "few128/1"),
    (2, 70, 2088, 7208, "together", "few128/8", "few128/1"),
    (2, 165, 5096, 72, "apart", "few32/1", "few128/1"), (2, 641, 4904, 72, "apart", "few128/1", "few128/1"),
    (2, 1541, 2584, 72, "apart", "few128/1", "few128/2"), (2, 9850, 136, 72, "apart", "few128/1", "few64/8"),
    (2, 12985, 264, 136, "apart", "pairs128", "few64/8"), (2, 2513, 2440, 200, "apart", "pairs128", "pairs128 few tiles"),
    (2, 4591, 5016, 72, "apart", "pairs256", "pairs256 few tiles"), (2, 577, 5256, 1160, "apart", "pairs256 few tiles", "pairs256"),
    (2, 2693, 2456, 392, "apart", "pairs256 few tiles", "pairs256 few tiles"),
    (2, 3225, 360, 1688, "apart", "pairs128 few tiles", "pairs128 few tiles")]

# rows, columns: lanes of a strip, runs, CTAs that share a run
BIAS = [(1, 8, (8, 1, 1)), (65, 72, (8, 1, 2)), (449, 136, (8, 1, 8)), (4101, 72, (8, 9, 8)), (38917, 40, (8, 76, 8)),
        (13165, 2312, (32, 60, 1)), (18817, 1560, (32, 43, 2)), (65601, 264, (32, 38, 8)), (131073, 136, (32, 76, 8))]

GB300_PAIRS = 76  # 152 SMs


def build(out_dir):
    """The program as a library."""
    from paper_2608_02625_gb300 import build as b
    src, out = os.path.join(out_dir, "plans.cpp"), os.path.join(out_dir, "plans.so")
    with open(src, "w") as f:
        f.write(PROGRAM)
    cuda = os.path.join(os.path.dirname(os.path.dirname(b.nvcc())), "include")
    r = subprocess.run([os.environ.get("CXX", "g++"), "-O1", "-shared", "-fPIC", "-std=c++17", "-I", b.INCLUDE, "-I", b.CSRC, "-I", cuda,
                        src, "-o", out, "-L" + b.PKG, "-ldlmrefine", "-Wl,-rpath," + b.PKG], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return ctypes.CDLL(out)


class Plans:
    """What the library would launch, with `pairs` pairs of CTAs (None: as many as the GPU has room for)."""

    def __init__(self, out_dir, pairs=None):
        self.lib = build(out_dir)
        self.pairs = (ctypes.c_int32 * 4)(*([pairs or 0] * 4))
        if pairs is None:
            self.lib.pairs(self.pairs)

    def _ask(self, name, *sizes):
        o = (ctypes.c_int64 * 7)()
        args = [ctypes.c_int32(s) if name == "gradients" and i == 3 else ctypes.c_int64(s) for i, s in enumerate(sizes)]
        getattr(self.lib, name)(*args, *([] if name == "bias" else [self.pairs]), o)
        return list(o)

    @staticmethod
    def _name(o):
        return f"pairs{o[1]}" if o[0] else f"few{o[1]}/{o[2]}"

    def _pairs_name(self, o, workers, tiles_of):
        return self._name(o) + (" few tiles" if o[0] and tiles_of(o[1]) <= 2 * workers else "")

    def gated(self, N, d, f):
        return self._pairs_name(self._ask("gated", N, d, f), self.pairs[0], lambda bn: -(-N // 256) * -(-2 * f // bn))

    def cols(self, N, k, m):
        return self._pairs_name(self._ask("cols", N, k, m), self.pairs[1], lambda bn: -(-m // 256) * -(-N // bn))

    def gradients(self, count, N, k, m):
        o = self._ask("gradients", N, k, m, count)
        return ("together" if o[0] else "apart",
                self._pairs_name(o[1:4], self.pairs[2], lambda bn: -(-k // 256) * -(-N // bn)),
                self._pairs_name(o[4:7], self.pairs[3], lambda bn: count * -(-m // 256) * -(-k // bn)))

    def bias(self, N, m):
        return tuple(self._ask("bias", N, m)[:3])
