"""The gradient of the table beside a large value: the sums are integers, scaled by a bound that holds for every row of a head, so a row of V far
above the others makes the unit coarse for everyone.  What is left has to be as good as a sum in fp32.

The second image has all of its tokens, the first those of even rows: offsets of an odd number of rows are the second image's
alone.  Its values, and what the kernels compute of them, are the same whatever the first image holds, so a difference between two calls
in these buckets comes from the sums:
  each of them  a pair is rounded to a unit of 2^-43 (fp32-FMA kernels: 2^-42 or finer) of a power of two of at most twice the bound
          2 max |dO| max |v|, and its item's sum, with up to 2^16 rows, to one of 2^-46: half a unit each, 2^-43 + 2^-46 < 2^-44 + 2^-42 of the bound a
          pair, in both calls.
  together  as good as fp32: 4 u = 2^-22 of the root mean square, of which 2 u are the roundings of the two results.  Half a unit for a
          thousand-fold V is 2^-46 2^10 of what the rows themselves need, which is 2^10 to 2^12 of a pair: 2^-24 of a pair, and of sums of many less.
(As multiples of 2^-30 of the bound they were off by 2^-31 of it a pair: up to 5e-4 of the root mean square.)
"""
import numpy as np
import pytest
import torch

from oracle import rel_sandwich as R
from tests.gpu_util import dev, host, round_to
from tests.test_gpu_rel_attention import Run, U, problem

pytestmark = pytest.mark.gpu

CASES = [("bf16", 32, 0), ("bf16", 64, 0), ("bf16", 64, 8), ("f32", 32, 0)]


def two_images(dtype, d, rows, cols, seg_len, seed):
    N = rows * cols
    pr = problem(dtype, d, 2, rows, cols, (N, N), seed=seed)
    even = np.arange(N) // cols % 2 == 0
    n0 = int(even.sum())
    take = np.concatenate((np.nonzero(even)[0], N + np.arange(N)))
    pr["idx"] = take.astype(np.int32)
    pr["qkv"], pr["d_out"] = pr["qkv"][take], pr["d_out"][take]
    pr["cu"] = np.array([0, n0, n0 + N], np.int32)
    seg = None
    if seg_len:   # parts of images
        cuts = sorted({0, n0, n0 + N} | set(range(0, n0, seg_len)) | set(range(n0, n0 + N, seg_len)))
        seg = np.array(cuts, np.int32)
    dy = np.arange((2 * rows - 1) * (2 * cols - 1)) // (2 * cols - 1) - (rows - 1)
    return pr, seg, n0, dy % 2 != 0


@pytest.mark.parametrize("dtype,d,flags", CASES)
# long segments (two passes), up to 128 rows to a tile, up to 64 rows (pairs), a few long ones (clusters), a table beyond shared memory
@pytest.mark.parametrize("rows,cols,seg_len", [(24, 24, 0), (12, 10, 0), (14, 14, 40), (40, 30, 0), (2, 20000, 300)])
@pytest.mark.parametrize("factor", [100.0, 1000.0])
def test_a_large_value_of_another_image_leaves_the_sums(dtype, d, flags, rows, cols, seg_len, factor):
    pr, seg, n0, odd = two_images(dtype, d, *((rows, cols) if rows > 2 else (2, cols)), seg_len, 3)
    if rows == 2:   # a long grid: the columns at the start of the rows
        keep = np.concatenate((np.arange(200), n0 + np.arange(200), n0 + cols + np.arange(200)))
        pr["idx"], pr["qkv"], pr["d_out"] = pr["idx"][keep], pr["qkv"][keep], pr["d_out"][keep]
        pr["cu"], seg, n0 = np.array([0, 200, 600], np.int32), None, 200
    C, H = pr["C"], pr["H"]
    got, run = [], None
    for f in (1.0, factor):
        q = dict(pr, qkv=pr["qkv"].copy())
        q["qkv"][n0 // 2, 2 * C:] = round_to(q["qkv"][n0 // 2, 2 * C:] * f, dtype)
        run = Run(q, flags, seg=seg)
        run.fwd(); run.bwd()
        torch.cuda.synchronize()
        assert run.status.item() == 0
        got.append((host(run.dtable)[odd], host(run.dqkv)[n0:]))
    assert np.array_equal(got[0][1], got[1][1])                 # the second image computes the same
    args = (pr["cu"] if seg is None else seg, pr["idx"], pr["rows"], pr["cols"], pr["bucket"], pr["table"], H)
    count = R.rel_bwd(q["qkv"], host(run.out)[:run.Np], host(run.lse)[:, :run.Np], pr["d_out"], *args)["count"][odd]
    norm = lambda a: np.sqrt((a.reshape(run.Np, H, d) ** 2).sum(2).max())
    bound = 2 * norm(q["qkv"][:, 2 * C:]) * norm(pr["d_out"])
    diff, want = np.abs(got[1][0] - got[0][0]), got[0][0]
    assert np.all(diff <= 2 * (2.0 ** -44 + 2.0 ** -42) * bound * count + 2 * U * np.abs(want))
    assert np.sqrt((diff ** 2).sum()) <= 4 * U * np.sqrt((want ** 2).sum()), np.sqrt((diff ** 2).sum() / (want ** 2).sum())
