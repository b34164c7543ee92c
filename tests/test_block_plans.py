"""The sizes that the feed-forward block's tests give to each of its kernels take those kernels
(host arithmetic of the library, with the pairs of CTAs that a GB300 has room for): a fit that moves a
size elsewhere fails here instead of leaving a kernel without a test."""
import os
import shutil

import pytest

import block_forms as F


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    from paper_2608_02625_gb300 import build
    if not shutil.which(os.environ.get("CXX", "g++")):
        pytest.skip("no host compiler")
    build.build()
    return F.Plans(str(tmp_path_factory.mktemp("plans")), F.GB300_PAIRS)


def test_gated(plans):
    assert [plans.gated(*c[:3]) for c in F.GATED] == [c[3] for c in F.GATED]


def test_projections(plans):
    assert [plans.cols(*c[:3]) for c in F.COLS] == [c[3] for c in F.COLS]


def test_gradients(plans):
    assert [plans.gradients(*c[:4]) for c in F.GRADIENTS] == [c[4:] for c in F.GRADIENTS]


def test_bias_gradients(plans):
    assert [plans.bias(*c[:2]) for c in F.BIAS] == [c[2] for c in F.BIAS]


def test_every_form_has_a_size():
    few = {f"few{n}/{s}" for n in (16, 32, 64) for s in (1, 2, 4, 8)}
    for cases in (F.GATED, F.COLS):
        assert few | {"few128/1", "few128/4", "pairs128", "pairs256"} <= {c[3] for c in cases}
    for count in (1, 2):
        x, w = ({c[k].replace(" few tiles", "") for c in F.GRADIENTS if c[0] == count} for k in (5, 6))
        assert {"pairs128", "pairs256", "few128/1", "few128/2", "few16/4"} <= x and {"pairs128", "pairs256", "few64/8", "few128/1", "few128/2"} <= w
        assert {c[4] for c in F.GRADIENTS if c[0] == count} == {"together", "apart"}
    assert {(c[2][0], c[2][1] > 1, c[2][2] > 1) for c in F.BIAS} >= {(8, False, True), (8, True, True), (32, True, False), (32, True, True)}


def test_runs_of_bias_sums_are_few(plans):
    """At most 76, eight CTAs each: what a column's sum is rounded."""
    for N in (1, 63, 64, 65, 1000, 4864, 16384, 131072, 2 ** 20, 2 ** 28):
        for m in (8, 64, 72, 256, 264, 1000, 2048, 8192, 2 ** 20):
            lanes, runs, ranks = plans.bias(N, m)
            assert lanes in (8, 32) and 1 <= runs <= 76 and ranks in (1, 2, 4, 8), (N, m, lanes, runs, ranks)
