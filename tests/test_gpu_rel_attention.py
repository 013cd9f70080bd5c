"""Attention with a learned relative position bias against the fp64 oracle: every segment length where tiles end, odd grids, few
and many buckets, masking entries, containers, shifted orders, both types and kernel families; rows behind the last one,
reproducibility, graphs, and what the device refuses.

Error bounds, componentwise, u = 2^-24 (fp32) and w = 2^-8 (a bf16 rounding), d the head dimension, n the segment's length:
  S       a dot product of d terms, scaled, plus a bias: (d + 4) u times the largest sum of absolute values, and where the exponential
          is taken in base 2, 3 u more of it for the factors log2 e.  P is off by twice that (its own and its sum's) and
          8 u + n u for the exponentials and the sum.
  out     P's error and n u times sum P |v|; tensor cores: P rounded to bf16 once, w sum P |v|; stored as bf16: w |out|.
  grads   oracle.rel_sandwich.rel_bwd adds up the same through dS; the table's sum in integers adds half a unit per pair.
"""
import numpy as np
import pytest
import torch

from oracle import rel_sandwich as R
from tests.gpu_util import dev, host, round_to

pytestmark = pytest.mark.gpu
U, W = 2.0 ** -24, 2.0 ** -8


def problem(dtype, d, H, rows, cols, counts, nb=None, seed=0, mask=0.0, std=1.0):
    rng = np.random.default_rng(seed)
    N, C, B = rows * cols, H * d, len(counts)
    cu = np.concatenate(([0], np.cumsum(counts))).astype(np.int32)
    idx = np.concatenate([b * N + np.sort(rng.choice(N, n, replace=False)) for b, n in enumerate(counts)] + [np.zeros(0, np.int64)]).astype(np.int32)
    E = (2 * rows - 1) * (2 * cols - 1)
    bucket = (np.arange(E) if nb is None else rng.integers(0, nb, E)).astype(np.int32)
    table = round_to(0.5 * rng.normal(size=(E if nb is None else nb, H)), dtype)
    table[rng.random(table.shape) < mask] = -np.inf
    r = lambda *s: round_to(std * rng.normal(size=s), dtype)
    return dict(dtype=dtype, d=d, H=H, rows=rows, cols=cols, B=B, N=N, C=C, cu=cu, idx=idx, bucket=bucket, table=table,
                qkv=r(int(cu[-1]), 3 * C), d_out=r(int(cu[-1]), C))


class Run:
    """The problem on the device, in buffers with `extra` rows behind the last one that hold a known value."""
    GUARD = 7.0

    def __init__(self, pr, flags=0, extra=5, seg=None, scale=0.0):
        from paper_2410_23608_b200 import binding as L
        self.L, self.pr = L, pr
        Np, C, H = int(pr["cu"][-1]), pr["C"], pr["H"]
        cap = min(max(Np + extra, 1), max(pr["B"], 1) * pr["N"])
        self.cap, self.Np = cap, Np
        T = torch.float32 if pr["dtype"] == "f32" else torch.bfloat16
        self.p = L.make_params(pr["B"], pr["N"], C, H, pr["dtype"], capacity=cap, flags=flags, softmax_scale=scale)
        full = lambda rows, cols_, dt=T: torch.full((rows, cols_), self.GUARD, dtype=dt, device="cuda")

        def padded(a, cols_):
            t = full(cap, cols_)
            t[:Np] = dev(a, pr["dtype"]).view(Np, cols_)
            return t
        self.qkv, self.d_out = padded(pr["qkv"], 3 * C), padded(pr["d_out"], C)
        self.out, self.dqkv = full(cap, C), full(cap, 3 * C)
        self.lse, self.peak = full(H, cap, torch.float32), full(H, cap, torch.float32)
        self.dtable = full(*pr["table"].shape, torch.float32)
        i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()
        self.seg = i32(pr["cu"] if seg is None else seg)
        self.idx = torch.full((cap,), 1 << 30, dtype=torch.int32, device="cuda")
        self.idx[:Np] = i32(pr["idx"])
        self.rel = L.rel_bias(pr["rows"], pr["cols"], i32(pr["bucket"]), dev(pr["table"], pr["dtype"]))
        self.ws = torch.full((L.spa_rel_workspace_bytes(self.p, self.rel),), 0xff, dtype=torch.uint8, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def fwd(self):
        self.L.spa_packed_attention_rel_fwd(self.p, self.rel, self.qkv, self.seg, self.seg.numel() - 1, self.idx, self.out, self.lse, self.peak,
                                            self.ws, d_status=self.status)

    def bwd(self, peak=True):
        self.L.spa_packed_attention_rel_bwd(self.p, self.rel, self.qkv, self.out, self.lse, self.peak if peak else None, self.d_out, self.seg,
                                            self.seg.numel() - 1, self.idx, self.dqkv, self.dtable, self.ws, d_status=self.status)


def check(run, flags=0, peak=True, seg=None, scale=None):
    pr, L = run.pr, run.L
    Np, C, H, d = run.Np, pr["C"], pr["H"], pr["d"]
    cu = pr["cu"] if seg is None else seg
    bf16, tc = pr["dtype"] == "bf16", pr["dtype"] == "bf16" and not flags & L.SPA_FLAG_SIMT_ONLY
    args = (cu, pr["idx"], pr["rows"], pr["cols"], pr["bucket"], pr["table"], H)
    run.fwd()
    torch.cuda.synchronize()
    assert run.status.item() == 0
    f = R.rel_fwd(pr["qkv"], *args, scale=scale)
    n = max([1] + list(np.diff(cu)))
    s_err = (d + 7) * U * f["s_abs"]
    p_err = 2 * s_err + (8 + n) * U
    store = W if bf16 else U
    got = host(run.out)
    tol = (p_err + (W if tc else 0) + n * U) * f["mean_abs"] + store * np.abs(f["out"]) + 1e-30
    assert np.all(np.abs(got[:Np] - f["out"]) <= tol * (1 + 1e-6)), np.max(np.abs(got[:Np] - f["out"]) / tol)
    assert np.all(got[Np:] == Run.GUARD)
    for name in ("lse", "peak"):
        g, ref = host(getattr(run, name)), f[name]
        assert np.array_equal(np.isinf(g[:, :Np]), np.isinf(ref)), name
        ok = ~np.isinf(ref)
        # a logarithm of the sum, and a maximum that is rounded with it
        tol = s_err + (8 + n) * U + 4 * U * (np.abs(ref[ok]) + f["s_abs"])
        assert np.all(np.abs(g[:, :Np][ok] - ref[ok]) <= tol), name
        assert np.all(g[:, Np:] == Run.GUARD), name
    # ---- backward, from the forward's own out and lse
    run.bwd(peak)
    torch.cuda.synchronize()
    assert run.status.item() == 0
    o, lse = got[:Np], host(run.lse)[:, :Np]
    lse_max = np.abs(np.where(np.isinf(lse), 0, lse)).max() if Np else 0.0
    kw = dict(p_err=s_err + (8 + 3 * lse_max) * U, dot_err=(d + 2) * U, round_p=W if tc else 0.0, scale=scale)
    b = R.rel_bwd(pr["qkv"], o, lse, pr["d_out"], *args, **kw)
    g = host(run.dqkv)
    tol = b["dqkv_tol"] + 2 * store * np.abs(b["dqkv"]) + 1e-30
    assert np.all(np.abs(g[:Np] - b["dqkv"]) <= tol), np.max(np.abs(g[:Np] - b["dqkv"]) / tol)
    assert np.all(g[Np:] == Run.GUARD)
    # the integer bins: half a unit per pair, of a power of two up to twice the bound 2 max |dO| max |v| (times the largest
    # probability, with peak): 2^-30 of the bound on tensor cores, 2^-42 otherwise
    half = 0.0
    if Np:
        v = pr["qkv"][:, 2 * C:].reshape(Np, H, d)
        bound = 2 * np.sqrt((v ** 2).sum(2).max()) * np.sqrt((pr["d_out"].reshape(Np, H, d) ** 2).sum(2).max())
        half = bound * (2.0 ** -30 if tc else 2.0 ** -42)
    tol = b["dtable_tol"] + half * b["count"] + 2 * U * np.abs(b["dtable"]) + 1e-30
    g = host(run.dtable)
    assert np.all(np.abs(g - b["dtable"]) <= tol), np.max(np.abs(g - b["dtable"]) / tol)


KINDS = [("f32", 32, 0), ("f32", 64, 0), ("bf16", 32, 0), ("bf16", 64, 0), ("bf16", 32, 8), ("bf16", 64, 8)]   # 8: SPA_FLAG_SIMT_ONLY


@pytest.mark.parametrize("dtype,d,flags", KINDS)
@pytest.mark.parametrize("counts", [(1,), (0, 0), (2, 0, 1), (33,), (64, 65, 63), (127, 1, 128, 129), (0, 200, 3, 190, 0), (255, 256, 257)])
def test_segment_lengths(dtype, d, flags, counts):
    run = Run(problem(dtype, d, 2, 15, 19, counts, seed=sum(counts)), flags)
    check(run, flags)


@pytest.mark.parametrize("dtype,d,flags", KINDS)
@pytest.mark.parametrize("rows,cols,nb", [(1, 1, None), (1, 7, None), (9, 1, 3), (7, 7, None), (7, 7, 1), (14, 14, 25), (3, 90, 11), (47, 83, 225)])
def test_grids_and_buckets(dtype, d, flags, rows, cols, nb):
    N = rows * cols
    counts = [max(1, N // 3) % 700, min(N, 50), 0, min(N, 300)]
    check(Run(problem(dtype, d, 3, rows, cols, counts, nb=nb, seed=rows), flags), flags)


@pytest.mark.parametrize("dtype,d,flags", KINDS)
def test_large_grid_with_a_bucket_for_every_offset(dtype, d, flags):
    check(Run(problem(dtype, d, 2, 50, 84, (300, 0, 17), seed=3), flags), flags)


@pytest.mark.parametrize("dtype,d,flags", KINDS)
@pytest.mark.parametrize("mask", [0.3, 0.97, 1.0])
def test_masking_entries_and_rows_without_a_key(dtype, d, flags, mask):
    pr = problem(dtype, d, 2, 9, 11, (99, 1, 40, 66), seed=int(100 * mask), mask=mask)
    f = R.rel_fwd(pr["qkv"], pr["cu"], pr["idx"], pr["rows"], pr["cols"], pr["bucket"], pr["table"], pr["H"])
    assert mask < 0.9 or np.isinf(f["lse"]).any()
    check(Run(pr, flags), flags)


@pytest.mark.parametrize("dtype,d,flags", KINDS)
def test_lowest_value_of_the_type_as_mask(dtype, d, flags):
    """A table entry of the type's lowest finite value: no weight beside other keys."""
    pr = problem(dtype, d, 1, 5, 5, (25, 12), seed=4)
    low = float(torch.finfo(torch.float32 if dtype == "f32" else torch.bfloat16).min)
    pr["table"][::3] = low
    run = Run(pr, flags)
    run.fwd()
    run.bwd()
    f = R.rel_fwd(pr["qkv"], pr["cu"], pr["idx"], 5, 5, pr["bucket"], pr["table"], 1)
    keep = (f["lse"][0] > -1e30)
    assert keep.sum() > 30 and run.status.item() == 0
    got = host(run.out)[:run.Np]
    assert np.isfinite(got).all() and torch.isfinite(run.dqkv).all()
    tol = (U * (d + 20) * 8 + (W if dtype == "bf16" else 0)) * f["mean_abs"] + (W if dtype == "bf16" else U) * np.abs(f["out"])
    assert np.all(np.abs(got - f["out"])[keep] <= 2 * tol[keep])


@pytest.mark.parametrize("dtype,d,flags", KINDS)
@pytest.mark.parametrize("low", [-1e9, "lowest"])
@pytest.mark.parametrize("grid,counts", [((9, 11), (99, 1, 40, 66)), ((14, 15), (210, 130))])
def test_entries_that_mask_without_being_infinite(dtype, d, flags, low, grid, counts):
    """What is below -1e6 masks as -inf does, where it is all that a row has, too: forward and backward as with -inf."""
    pr = problem(dtype, d, 2, *grid, counts, seed=4, mask=0.99)
    masked = np.isinf(pr["table"])
    run = Run(pr, flags)
    run.rel.tensors[1][torch.from_numpy(masked).cuda()] = torch.finfo(run.qkv.dtype).min if low == "lowest" else low
    check(run, flags)


@pytest.mark.parametrize("dtype,d,flags", KINDS)
@pytest.mark.parametrize("own", [False, True])
def test_rows_without_a_key_beside_infinities(dtype, d, flags, own):
    """They are zeros and have no gradient, whatever V is, in their segment or in one that shares their tile."""
    pr = problem(dtype, d, 1, 7, 9, (40, 30), seed=6)
    pr["table"][:] = -np.inf
    run = Run(pr, flags)
    run.qkv[5 if own else 45, 2 * pr["C"] + 3] = float("inf")
    run.fwd(); run.bwd()
    torch.cuda.synchronize()
    assert bool((run.out[:40] == 0).all()) and bool((run.lse[:, :40] == -float("inf")).all()) and bool((run.peak[:, :40] == 0).all())
    if not own:
        assert bool((run.dqkv[:40] == 0).all())


@pytest.mark.parametrize("dtype,d,flags", KINDS)
@pytest.mark.parametrize("v_std,d_std", [(1e-24, 1e12), (1e15, 1e-26)])
def test_table_gradient_of_values_whose_squares_vanish(dtype, d, flags, v_std, d_std):
    """The bound that the sums are scaled by is taken from squares: they may underflow, the bound may not."""
    pr = problem(dtype, d, 2, 7, 9, (40, 63, 30), nb=6, seed=7)
    C, H = pr["C"], pr["H"]
    pr["qkv"][:, 2 * C:] = round_to(pr["qkv"][:, 2 * C:] * v_std, dtype)
    pr["d_out"] = round_to(pr["d_out"] * d_std, dtype)
    run = Run(pr, flags)
    run.fwd(); run.bwd()
    torch.cuda.synchronize()
    args = (pr["cu"], pr["idx"], pr["rows"], pr["cols"], pr["bucket"], pr["table"], H)
    lse = host(run.lse)[:, :run.Np]
    s_err = (d + 7) * U * R.rel_fwd(pr["qkv"], *args)["s_abs"]
    b = R.rel_bwd(pr["qkv"], host(run.out)[:run.Np], lse, pr["d_out"], *args, p_err=s_err + (8 + 3 * np.abs(lse).max()) * U, dot_err=(d + 2) * U)
    # half a unit per pair, as elsewhere, of a bound for which neither norm is below 2^-63
    most = lambda x: max(2.0 ** -63, np.sqrt((x.reshape(run.Np, H, d) ** 2).sum(2).max()))
    half = 2 * most(pr["d_out"]) * most(pr["qkv"][:, 2 * C:]) * 2.0 ** -30
    g = host(run.dtable)
    tol = b["dtable_tol"] + half * b["count"] + 2 * U * np.abs(b["dtable"])
    assert np.all(np.abs(g - b["dtable"]) <= tol), np.max(np.abs(g - b["dtable"]) / tol)


@pytest.mark.parametrize("dtype,d,flags", KINDS)
def test_large_logits_and_the_moving_maximum(dtype, d, flags):
    pr = problem(dtype, d, 2, 16, 20, (320, 250), seed=8, std=3.0)
    pr["table"] = round_to(40.0 * np.linspace(-1, 1, pr["table"].size).reshape(pr["table"].shape), dtype)
    check(Run(pr, flags), flags)


@pytest.mark.parametrize("dtype,d,flags", KINDS)
def test_without_peak_and_with_a_scale(dtype, d, flags):
    pr = problem(dtype, d, 2, 7, 9, (63, 30), seed=9)
    check(Run(pr, flags, scale=0.05), flags, peak=False, scale=0.05)


@pytest.mark.parametrize("dtype,d,flags", KINDS)
@pytest.mark.parametrize("length", [1, 49, 130])
def test_containers_and_a_shifted_order(dtype, d, flags, length):
    """Segments that are parts of images, tokens in the order of a shifted map: positions do not ascend."""
    pr = problem(dtype, d, 2, 12, 13, (156, 77, 0, 140), seed=length)
    rng = np.random.default_rng(length)
    for lo, hi in zip(pr["cu"][:-1], pr["cu"][1:]):
        pr["idx"][lo:hi] = pr["idx"][lo:hi][rng.permutation(hi - lo)]
    cuts = sorted(set(pr["cu"].tolist()) | set(range(0, int(pr["cu"][-1]), length)))
    seg = np.array(cuts + [cuts[-1]] * 3, np.int32)          # padded with empty segments
    check(Run(pr, flags, seg=seg), flags, seg=seg)


@pytest.mark.parametrize("dtype,d,flags", KINDS)
def test_many_items_and_heads(dtype, d, flags):
    counts = [(37 * i) % 190 + 1 for i in range(24)]
    check(Run(problem(dtype, d, 12, 14, 14, counts, seed=1), flags), flags)


@pytest.mark.parametrize("dtype,d,flags", [k for k in KINDS if k[2] == 0])
def test_many_segments(dtype, d, flags):
    """More segments than are searched in shared memory."""
    counts = [(5 * i) % 7 for i in range(2300)]
    check(Run(problem(dtype, d, 1, 2, 3, [min(c, 6) for c in counts], seed=1), flags), flags)


@pytest.mark.parametrize("dtype,d,flags", KINDS)
def test_bitwise_reproducible_on_other_streams_and_in_a_graph(dtype, d, flags):
    run = Run(problem(dtype, d, 4, 14, 14, [(61 * i) % 180 + 10 for i in range(12)], nb=9, seed=2), flags)
    names = ("out", "lse", "peak", "dqkv", "dtable")
    run.fwd(); run.bwd()
    torch.cuda.synchronize()
    first = {k: getattr(run, k).clone() for k in names}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for k in names:
            getattr(run, k).fill_(3.0)
        run.fwd(); run.bwd()
    torch.cuda.synchronize()
    for k in names:
        assert torch.equal(getattr(run, k).view(-1)[:1], first[k].view(-1)[:1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run.fwd(); run.bwd()
    for _ in range(3):
        run.dtable.fill_(5.0)
        g.replay()
    torch.cuda.synchronize()
    for k in names:
        a, b = getattr(run, k), first[k]
        rows = slice(0, run.Np)
        assert torch.equal(a[:, rows] if k in ("lse", "peak") else a if k == "dtable" else a[rows],
                           b[:, rows] if k in ("lse", "peak") else b if k == "dtable" else b[rows]), k
    # new inputs under the same graph
    run.qkv.mul_(0.5)
    run.ws.fill_(0x55)
    g.replay()
    torch.cuda.synchronize()
    replayed = run.dtable.clone()
    run.fwd(); run.bwd()
    torch.cuda.synchronize()
    assert torch.equal(run.dtable, replayed)


@pytest.mark.parametrize("dtype,d,flags", KINDS)
@pytest.mark.parametrize("what", ["idx", "idx_negative", "bucket", "bucket_negative", "two_images", "twice"])
def test_what_the_device_refuses(dtype, d, flags, what):
    pr = problem(dtype, d, 2, 7, 9, (40, 30), nb=5, seed=9)
    seg = None
    if what.startswith("idx"):
        pr["idx"][11] = -1 if what.endswith("negative") else 2 * 63
    if what.startswith("bucket"):
        pr["bucket"][70] = -1 if what.endswith("negative") else 5
    if what == "two_images":
        seg = np.array([0, 55, 70], np.int32)
    if what == "twice":
        pr["idx"][11] = pr["idx"][10]
    run = Run(pr, flags, seg=seg)
    run.fwd()
    torch.cuda.synchronize()
    assert run.status.item() == (0 if what == "twice" else run.L.SPA_ERR_INVALID_ARG)
    run.status.zero_()
    run.out.zero_()
    run.lse.zero_()
    run.bwd()
    torch.cuda.synchronize()
    assert run.status.item() == run.L.SPA_ERR_INVALID_ARG
    # the rows behind the last one are as they were, and the next call is right
    assert bool((run.dqkv[run.Np:] == Run.GUARD).all())


@pytest.mark.parametrize("dtype,d,flags", KINDS)
def test_values_that_are_not_finite_show_in_the_table(dtype, d, flags):
    for name in ("q", "v", "d_out"):
        pr = problem(dtype, d, 2, 7, 9, (40, 30), nb=5, seed=9)
        run = Run(pr, flags)
        if name == "d_out":
            run.d_out[50, 3] = float("nan")
        else:
            run.qkv[50, (2 * pr["C"] if name == "v" else 0) + 3] = float("inf") if name == "v" else float("nan")
        run.fwd(); run.bwd()
        torch.cuda.synchronize()
        assert run.status.item() == 0
        assert torch.isnan(run.dtable[:, 0]).all() and torch.isfinite(run.dtable[:, 1]).all()
        # the other head, and the other image of the same head, keep their values
        assert torch.isfinite(run.out[:run.Np, pr["d"]:]).all()
        assert torch.isfinite(run.out[:40]).all() and torch.isfinite(run.dqkv[:40]).all()
