"""Calls whose inputs are not finite everywhere, as after a step that diverged: the results are NaN, and the call takes no longer than it has to.
(Rows with values that are not finite are formed again where another segment's values may have reached them.  Rows that are so by
their own segment's doing were, too, in scalar steps.)"""
import pytest
import torch

from tests.test_gpu_rel_attention import Run, problem

pytestmark = pytest.mark.gpu
KINDS = [("bf16", 32), ("bf16", 64)]
# several images, one, few with many rows (clusters), segments of up to 128 and of up to 64 rows
SHAPES = [((24, 24), [400, 576, 300, 77, 512] * 3, 4), ((47, 83), [3901], 2), ((33, 40), [700, 300], 1), ((10, 10), [100, 60, 93, 70] * 8, 4),
          ((7, 7), [49] * 64, 6)]


def milliseconds(call, n=3):
    best = float("inf")
    for _ in range(n):
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record(); call(); b.record()
        torch.cuda.synchronize()
        best = min(best, a.elapsed_time(b))
    return best


@pytest.mark.parametrize("dtype,d", KINDS)
@pytest.mark.parametrize("grid,counts,H", SHAPES)
@pytest.mark.parametrize("what", ["everything", "v", "d_out", "a row of k in every segment"])
def test_time_of_calls_that_are_not_finite(dtype, d, grid, counts, H, what):
    run = Run(problem(dtype, d, H, *grid, counts, seed=1))
    C, Np = run.pr["C"], run.Np
    run.fwd(); run.bwd()
    finite = milliseconds(run.fwd), milliseconds(run.bwd)
    nan = float("nan")
    if what == "everything":
        run.qkv[:Np] = nan
        run.d_out[:Np] = nan
    elif what == "v":
        run.qkv[:Np, 2 * C:] = nan
    elif what == "d_out":
        run.d_out[:Np] = nan
    else:
        run.qkv[run.seg[:-1].long(), C:2 * C] = nan
    run.fwd(); run.bwd()
    times = milliseconds(run.fwd), milliseconds(run.bwd)
    print(what, grid, d, ["%.3f -> %.3f ms" % p for p in zip(finite, times)])
    if what != "d_out":
        assert torch.isnan(run.out[:Np]).all()
    qkv_nan = torch.isnan(run.dqkv[:Np])
    assert qkv_nan[:, :2 * C].all() and torch.isnan(run.dtable).all()
    assert qkv_nan[:, 2 * C:].all() == (what != "v")     # dV has P and dO in it, but not V
    assert what != "v" or torch.isfinite(run.dqkv[:Np, 2 * C:]).all()
    # a time, so with room: the work of a finite call, and as much again for what is found out row by row, three times over
    for t, f in zip(times, finite):
        assert t <= 6 * f + 0.1, (what, times, finite)
