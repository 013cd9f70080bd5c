"""Where the operators could go wrong for their size or their company: many heads, tables larger than shared memory, arrays beyond 4 GB, empty
batches, two calls at a time, infinities beside other segments."""
import numpy as np
import pytest
import torch

from oracle import rel_sandwich as R
from tests.gpu_util import dev, host, round_to
from tests.test_gpu_rel_attention import KINDS, Run, U, W, check, problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d,flags", KINDS)
@pytest.mark.parametrize("H", [40, 61])
def test_many_heads(dtype, d, flags, H):
    check(Run(problem(dtype, d, H, 7, 8, (56, 20, 3), seed=H), flags), flags)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_most_heads(dtype):
    """C = 8192 in heads of 32: 256 of them, more chunks to a row than threads to a CTA."""
    check(Run(problem(dtype, 32, 256, 3, 4, (12, 5), seed=1)))


@pytest.mark.parametrize("dtype,d,flags", KINDS)
@pytest.mark.parametrize("cols", [6000, 30000])
def test_tables_larger_than_shared_memory(dtype, d, flags, cols):
    """One long row of tokens: a table (and at 30 000 the bins, too) that shared memory does not hold."""
    check(Run(problem(dtype, d, 1, 1, cols, (300, 0, 130), seed=2), flags), flags)


@pytest.mark.parametrize("dtype,d,flags", KINDS)
def test_no_segments(dtype, d, flags):
    for counts in ((), (0, 0, 0)):
        pr = problem(dtype, d, 2, 3, 3, counts)
        run = Run(pr, flags, extra=1)
        run.fwd(); run.bwd()
        torch.cuda.synchronize()
        assert run.status.item() == 0 and bool((run.dtable == 0).all())
        assert bool((run.out == Run.GUARD).all()) and bool((run.dqkv == Run.GUARD).all())


@pytest.mark.parametrize("dtype,d,flags", KINDS)
def test_two_calls_at_a_time(dtype, d, flags):
    """Two problems on two streams, each with a workspace of its own, as often as it takes to run side by side."""
    runs = [Run(problem(dtype, d, 3, 14, 14, [(53 * i + 7 * s) % 190 + 1 for i in range(10)], seed=s), flags) for s in (0, 1)]
    names = ("out", "lse", "peak", "dqkv", "dtable")
    want = []
    for r in runs:
        r.fwd(); r.bwd()
        torch.cuda.synchronize()
        want.append({k: getattr(r, k).clone() for k in names})
    streams = [torch.cuda.Stream() for _ in runs]
    for _ in range(20):
        for r, st in zip(runs, streams):
            with torch.cuda.stream(st):
                r.fwd(); r.bwd()
    torch.cuda.synchronize()
    for r, w in zip(runs, want):
        assert r.status.item() == 0
        for k in names:
            assert torch.equal(getattr(r, k).nan_to_num(), w[k].nan_to_num()), k


@pytest.mark.parametrize("dtype,d,flags", KINDS)
@pytest.mark.parametrize("grid,counts", [((7, 9), (40, 30, 63)), ((9, 14), (100, 126, 20)), ((20, 20), (300, 20, 170))])
@pytest.mark.parametrize("what", ["q", "k", "v", "d_out"])
def test_values_that_are_not_finite_stay_in_their_segment(dtype, d, flags, grid, counts, what):
    """An infinity in the second segment: the others have the values of a call without it."""
    pr = problem(dtype, d, 2, *grid, counts, seed=5)
    clean = Run(pr, flags)
    clean.fwd(); clean.bwd()
    run = Run(pr, flags)
    row = counts[0] + 3
    if what == "d_out":
        run.d_out[row, 1] = float("inf")
    else:
        run.qkv[row, {"q": 0, "k": 1, "v": 2}[what] * pr["C"] + 1] = float("inf")
    run.fwd(); run.bwd()
    torch.cuda.synchronize()
    own = slice(counts[0], counts[0] + counts[1])
    other = [r for r in range(run.Np) if not own.start <= r < own.stop]
    for k in ("out", "dqkv"):
        a, b = host(getattr(run, k))[other], host(getattr(clean, k))[other]
        # rows that were formed again differ by the order of their sums and, on tensor cores, by roundings of P and dS to bf16
        tol = (4 * W if dtype == "bf16" else 64 * U) * np.abs(b).max()
        assert np.isfinite(a).all() and np.abs(a - b).max() <= tol, (k, np.abs(a - b).max() / tol)
    assert torch.isfinite(run.dtable[:, 1]).all()


@pytest.mark.parametrize("dtype,d,flags", KINDS)
@pytest.mark.parametrize("grid,counts", [((17, 16), (272,)), ((17, 16), (1, 200)), ((24, 25), (600, 3)), ((24, 25), (64, 65, 300)), ((33, 40), (1320,)),
                                         ((33, 40), (129, 1000)), ((33, 40), (0, 30, 0, 700))])
@pytest.mark.parametrize("H", [1, 3])
def test_few_long_segments(dtype, d, flags, grid, counts, H):
    """Few row tiles with many keys each: the keys of a tile are dealt to several CTAs, of which some may get none."""
    check(Run(problem(dtype, d, H, *grid, counts, seed=sum(counts) + H), flags), flags)


@pytest.mark.parametrize("dtype,d,flags", KINDS)
@pytest.mark.parametrize("what", ["q", "k", "v", "d_out"])
def test_infinities_in_one_of_few_long_segments(dtype, d, flags, what):
    pr = problem(dtype, d, 1, 33, 40, (700, 300), seed=5)
    clean, run = Run(pr, flags), Run(pr, flags)
    if what == "d_out":
        run.d_out[720, 1] = float("inf")
    else:
        run.qkv[720, {"q": 0, "k": 1, "v": 2}[what] * pr["C"] + 1] = float("inf")
    for r in (clean, run):
        r.fwd(); r.bwd()
    torch.cuda.synchronize()
    for k in ("out", "dqkv"):
        a, b = host(getattr(run, k))[:700], host(getattr(clean, k))[:700]
        tol = (4 * W if dtype == "bf16" else 64 * U) * np.abs(b).max()
        assert np.isfinite(a).all() and np.abs(a - b).max() <= tol, (k, np.abs(a - b).max() / tol)


@pytest.mark.parametrize("dtype,d,flags", KINDS)
@pytest.mark.parametrize("grid,counts,nb", [((33, 40), (700, 300), None), ((33, 40), (1320,), 7), ((7, 7), (49, 49, 30, 49), 5), ((14, 14), [150] * 12, 9)])
def test_reproducible_in_a_graph(dtype, d, flags, grid, counts, nb):
    """Split items, and sums by offset that are folded into few buckets: the same bits with every replay, and those of the call alone."""
    run = Run(problem(dtype, d, 2, *grid, counts, nb=nb, seed=3), flags)
    run.fwd(); run.bwd()
    torch.cuda.synchronize()
    want = [t.clone() for t in (run.dqkv, run.dtable)]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run.fwd(); run.bwd()
    for _ in range(5):
        run.ws.fill_(0x55)
        run.dqkv.fill_(Run.GUARD); run.dtable.fill_(5.0)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(run.dqkv, want[0]) and torch.equal(run.dtable, want[1])


def test_rows_beyond_four_gigabytes():
    """2^20 packed rows of 2 304 bf16 values: places past 2^31 elements and 2^32 bytes, in segments of 64."""
    from paper_2410_23608_b200 import binding as L
    B, rows, cols, C, H, d = 1024, 32, 32, 768, 24, 32
    N, Np = rows * cols, B * rows * cols
    g = torch.Generator(device="cuda").manual_seed(0)
    qkv = torch.empty(Np, 3 * C, dtype=torch.bfloat16, device="cuda")
    d_out = torch.empty(Np, C, dtype=torch.bfloat16, device="cuda")
    for t in (qkv, d_out):
        for part in t.split(1 << 17):
            part.copy_(torch.randn(part.shape, generator=g, device="cuda"))
    p = L.make_params(B, N, C, H, "bf16", capacity=Np)
    E = (2 * rows - 1) * (2 * cols - 1)
    bucket = torch.arange(E, dtype=torch.int32, device="cuda") % 50
    table = torch.randn(50, H, generator=g, device="cuda").bfloat16()
    rel = L.rel_bias(rows, cols, bucket, table)
    idx = torch.arange(Np, dtype=torch.int32, device="cuda")
    seg = torch.arange(0, Np + 1, 64, dtype=torch.int32, device="cuda")
    out, dqkv = torch.empty_like(d_out), torch.empty_like(qkv)
    lse, peak = (torch.empty(H, Np, device="cuda") for _ in range(2))
    dtable, status = torch.empty(50, H, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.empty(L.spa_rel_workspace_bytes(p, rel), dtype=torch.uint8, device="cuda")
    L.spa_packed_attention_rel_fwd(p, rel, qkv, seg, seg.numel() - 1, idx, out, lse, peak, ws, d_status=status)
    L.spa_packed_attention_rel_bwd(p, rel, qkv, out, lse, peak, d_out, seg, seg.numel() - 1, idx, dqkv, dtable, ws, d_status=status)
    torch.cuda.synchronize()
    assert status.item() == 0 and torch.isfinite(dtable).all()
    for first in (0, 1 << 19, Np - 128):
        sl, cu = slice(first, first + 128), np.array([0, 64, 128])
        args = (cu, idx[sl].cpu().numpy(), rows, cols, bucket.cpu().numpy(), host(table), H)
        f = R.rel_fwd(host(qkv[sl]), *args)
        assert np.all(np.abs(host(out[sl]) - f["out"]) <= (2 * W) * (f["mean_abs"] + np.abs(f["out"])))
        b = R.rel_bwd(host(qkv[sl]), host(out[sl]), host(lse[:, sl]), host(d_out[sl]), *args, p_err=1e-4, dot_err=40 * U, round_p=W)
        assert np.all(np.abs(host(dqkv[sl]) - b["dqkv"]) <= b["dqkv_tol"] + 2 * W * np.abs(b["dqkv"]) + 1e-30)


def test_norm_rows_beyond_four_gigabytes():
    from paper_2410_23608_b200 import binding as L
    B, N, C = 1, 262147, 8192
    p = L.make_params(B, N, C, 1, "bf16")
    x = torch.empty(N, C, dtype=torch.bfloat16, device="cuda")
    z = torch.empty_like(x)
    g = torch.Generator(device="cuda").manual_seed(0)
    for t in (x, z):
        for part in t.split(1 << 15):
            part.copy_(torch.randn(part.shape, generator=g, device="cuda"))
    y, n, stats = torch.empty_like(x), torch.empty_like(x), torch.empty(4, N, device="cuda")
    sw = L.sandwich("rms", "token", gate=z)
    L.spa_sandwich_norm(p, sw, x, z, None, y, n, stats)
    torch.cuda.synchronize()
    for r in (0, 131072, N - 1):
        xr, zr = host(x[r]), host(z[r])
        want = xr + zr * zr / np.sqrt((zr * zr).mean() + 1e-5)
        assert np.all(np.abs(host(y[r]) - want) <= 2 * W * np.abs(want) + 1e-5)
        want = want / np.sqrt((want * want).mean() + 1e-5)
        assert np.all(np.abs(host(n[r]) - want) <= 2 * W * np.abs(want) + 1e-5)
    dx, dz, dg = torch.empty_like(x), torch.empty_like(x), torch.empty(C, device="cuda")
    ws = torch.empty(L.spa_sandwich_workspace_bytes(p, sw), dtype=torch.uint8, device="cuda")
    L.spa_sandwich_norm_bwd(p, sw, None, x, None, z, None, stats, dx, dz, dg_post=dg, workspace=ws)
    torch.cuda.synchronize()
    assert torch.equal(dx[-1], x[-1]) and torch.isfinite(dz[-1]).all() and torch.isfinite(dg).all()
