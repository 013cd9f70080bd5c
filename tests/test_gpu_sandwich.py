"""The norms around a block against the fp64 oracle: every row width where the kernels change, packed rows, all gates, absent parameters,
in-place calls, reproducibility and graphs.

Error bounds, u = 2^-24, w the half step of the stored type: a sum of C values in a thread's chain of at most 32 and a tree is off by
(32 + 16) u of the sum of absolute values; mean, deviation and normalised value together by K u of the row's largest normalised
value, K = 160 (mean 48, squares 2 * 48, root and products the rest).
"""
import numpy as np
import pytest
import torch

from oracle import rel_sandwich as R
from tests.gpu_util import dev, host, round_to

pytestmark = pytest.mark.gpu
U, K = 2.0 ** -24, 160


def problem(dtype, B, N, C, kind, gate_kind, keep=1.0, params=True, seed=0, shift=0.0):
    rng = np.random.default_rng(seed)
    r = lambda *s, std=1.0, mean=0.0: round_to(mean + std * rng.normal(size=s), dtype)
    T = B * N
    has = rng.random(T) < keep if keep < 1 else np.ones(T, bool)
    Z = max(1, int(has.sum()))
    row = np.full(T, -1, np.int32)
    row[has] = rng.permutation(int(has.sum())) if keep < 1 else np.arange(T)
    v = dict(x=r(T, C, mean=shift), z=r(Z, C, mean=shift), dn=r(T, C), dy=r(T, C))
    names = ("scale", "g_post", "b_post", "g_pre", "b_pre")
    v.update({k: r(C, std=0.3, mean=0.0 if k.startswith("b") else 1.0) for k in names})
    if not params:
        v.update(scale=np.ones(C), g_post=np.ones(C), g_pre=np.ones(C), b_post=np.zeros(C), b_pre=np.zeros(C))
    gate = {"none": None, "score": rng.normal(size=T).astype(np.float32).astype(np.float64), "image": r(B, C), "token": r(T, C)}[gate_kind]
    return dict(v, dtype=dtype, B=B, N=N, C=C, kind=kind, gate_kind=gate_kind, gate=gate, row=row, packed=keep < 1, params=params, names=names)


class Run:
    GUARD = 7.0

    def __init__(self, pr, eps=1e-5, extra=3):
        from paper_2410_23608_b200 import binding as L
        self.L, self.pr, self.eps = L, pr, eps
        dt, T, C = pr["dtype"], pr["B"] * pr["N"], pr["C"]
        Z = pr["z"].shape[0]
        cap = min(Z + extra, T) if pr["packed"] else T
        self.p = L.make_params(pr["B"], pr["N"], C, 1, dt, capacity=cap)
        ty = torch.float32 if dt == "f32" else torch.bfloat16
        e = lambda *s, t=ty: torch.full(s, self.GUARD, dtype=t, device="cuda")
        f = lambda *s: e(*s, t=torch.float32)
        self.x, self.dn, self.dy = (dev(pr[k], dt) for k in ("x", "dn", "dy"))
        self.z = e(cap, C)
        self.z[:Z] = dev(pr["z"], dt)
        self.row = torch.from_numpy(pr["row"]).cuda() if pr["packed"] else None
        self.par = {k: dev(pr[k], dt) if pr["params"] else None for k in pr["names"]}
        self.gate = None if pr["gate"] is None else dev(pr["gate"], "f32" if pr["gate_kind"] == "score" else dt)
        self.sw = L.sandwich(pr["kind"], pr["gate_kind"], gate=self.gate, eps=eps, **self.par)
        self.y, self.n, self.stats = e(T, C), e(T, C), f(4, T)
        self.dx, self.dz = e(T, C), e(cap, C)
        self.dgate = {"none": lambda: None, "score": lambda: f(T), "image": lambda: f(pr["B"], C), "token": lambda: e(T, C)}[pr["gate_kind"]]()
        self.grads = {"d" + k: f(C) for k in pr["names"]}
        self.ws = torch.full((L.spa_sandwich_workspace_bytes(self.p, self.sw),), 0xff, dtype=torch.uint8, device="cuda")

    def fwd(self):
        self.L.spa_sandwich_norm(self.p, self.sw, self.x, self.z, self.row, self.y, self.n, self.stats)

    def bwd(self, dn=True, dy=True):
        self.L.spa_sandwich_norm_bwd(self.p, self.sw, self.dn if dn else None, self.dy if dy else None, self.y, self.z, self.row, self.stats,
                                     self.dx, self.dz, dgate=self.dgate, workspace=self.ws, **self.grads)


def check(run, dn=True, dy=True):
    pr = run.pr
    w = 2.0 ** -8 if pr["dtype"] == "bf16" else U
    a = (pr["gate"], pr["gate_kind"], pr["scale"], pr["g_post"], pr["b_post"], pr["g_pre"])
    run.fwd()
    torch.cuda.synchronize()
    f = R.sandwich_fwd(pr["x"], pr["z"], pr["row"], *a, pr["b_pre"], pr["kind"], run.eps, pr["B"], pr["N"])
    branch = np.abs(f["y"] - pr["x"])
    scale_row = (np.abs(pr["x"]) + branch).max(1, keepdims=True)
    g = host(run.y)
    # branch: relative error K u of the largest of its factors
    big = (np.abs(pr["g_post"]).max() * np.sqrt(pr["C"]) + np.abs(pr["b_post"]).max()) * np.abs(pr["scale"]).max() * \
        (1.0 if pr["gate"] is None or pr["gate_kind"] == "score" else np.abs(pr["gate"]).max())
    err_y = K * U * np.minimum(big, 1e9) + 4 * U * scale_row
    zmean = np.abs(pr["z"]).max()
    r1 = np.where(f["stats"][1] > 0, f["stats"][1], 0)[:, None]
    err_y = err_y * (1 + 48 * zmean * r1 / max(1.0, np.sqrt(pr["C"])))      # the mean's rounding, seen through 1 / deviation
    assert np.all(np.abs(g - f["y"]) <= err_y + w * np.abs(f["y"])), np.max(np.abs(g - f["y"]) / (err_y + w * np.abs(f["y"])))
    unsel = pr["row"] < 0
    assert np.array_equal(g[unsel], pr["x"][unsel])
    m, r = f["stats"][2][:, None], f["stats"][3][:, None]
    vh = np.abs((f["y"] - m) * r)
    err_h = r * (err_y + 64 * U * np.abs(f["y"]).max(1, keepdims=True)) * (1 + vh) + K * U * (1 + vh)
    err_n = np.abs(pr["g_pre"]) * err_h + 4 * U * np.abs(pr["b_pre"]) + w * np.abs(f["n"])
    gn = host(run.n)
    assert np.all(np.abs(gn - f["n"]) <= err_n), np.max(np.abs(gn - f["n"]) / err_n)
    st = host(run.stats)
    assert np.array_equal(st[:2][:, unsel], np.zeros((2, int(unsel.sum()))))
    dev_rel = K * U + err_y.max(1) * f["stats"][3] * 2 + 64 * U * np.abs(f["y"]).max(1) * f["stats"][3]
    assert np.all(np.abs(st[3] - f["stats"][3]) <= dev_rel * f["stats"][3])
    # ---- backward from the forward's own y and statistics
    y, st64 = host(run.y), host(run.stats)
    zero = np.zeros_like(pr["dn"])
    b = R.sandwich_bwd(pr["dn"] if dn else zero, pr["dy"] if dy else zero, y, pr["z"], pr["row"], st64, *a, pr["kind"], pr["B"], pr["N"])
    run.bwd(dn, dy)
    torch.cuda.synchronize()
    # every element of a row's gradient is a difference of terms as large as the row's largest
    vh2 = np.abs((y - st64[2][:, None]) * st64[3][:, None])
    gmax = (np.abs(pr["dn"]) * np.abs(pr["g_pre"])).max(1, keepdims=True) * (1 if dn else 0)
    err_d = K * U * (st64[3][:, None] * gmax * (1 + vh2) * (1 + vh2.max(1, keepdims=True)) + np.abs(b["dx"]) + np.abs(pr["dy"]))
    g = host(run.dx)
    assert np.all(np.abs(g - b["dx"]) <= err_d + w * np.abs(b["dx"])), "dx"
    has = ~unsel
    gate = np.broadcast_to(R._gate(pr["gate"], pr["gate_kind"], pr["B"], pr["N"]), b["dx"].shape)
    fac = np.abs(gate * pr["scale"] * pr["g_post"])
    err_g = (err_d + K * U * np.abs(b["dx"])) * fac
    zh = np.zeros_like(b["dx"])
    zh[has] = np.abs((pr["z"][pr["row"][has]] - st64[0][has, None]) * st64[1][has, None])
    err_z = st64[1][:, None] * ((err_g + K * U * (np.abs(b["dx"]) * fac).max(1, keepdims=True)).max(1, keepdims=True) * (1 + zh) * (1 + zh.max(1, keepdims=True)))
    gz, ref = host(run.dz), b["dz"]
    rows = pr["row"][has]
    assert np.all(np.abs(gz[rows] - ref[rows]) <= err_z[has] + w * np.abs(ref[rows])), "dz"
    other = np.setdiff1d(np.arange(gz.shape[0]), rows)
    assert np.all(gz[other] == Run.GUARD)
    T = pr["B"] * pr["N"]
    rel = (K + T + 64) * U
    extra = dict(dscale=(err_d * np.abs(gate) * (np.abs(pr["g_post"]) * zh + np.abs(pr["b_post"])))[has].sum(0),
                 dg_post=(err_d * np.abs(gate * pr["scale"]) * zh)[has].sum(0), db_post=(err_d * np.abs(gate * pr["scale"]))[has].sum(0),
                 dg_pre=np.zeros(pr["C"]), db_pre=np.zeros(pr["C"]))
    # dscale, dg_post and dgate come from A = sum d gate zh and B = sum d gate: their errors go by the sums of absolute values
    for k in pr["names"]:
        g, t = host(run.grads["d" + k]), 3 * rel * b["abs"]["d" + k] + extra["d" + k] + 1e-30
        assert np.all(np.abs(g - b["d" + k]) <= t), ("d" + k, np.max(np.abs(g - b["d" + k]) / t))
    if pr["gate_kind"] != "none":
        g, t = host(run.dgate), b["abs"]["dgate_row"] * 3 * rel + (err_d * np.abs(pr["scale"]) * (np.abs(pr["g_post"]) * zh + np.abs(pr["b_post"])))
        if pr["gate_kind"] == "score":
            t = t.sum(1)
        elif pr["gate_kind"] == "image":
            t = t.reshape(pr["B"], pr["N"], -1).sum(1)
        else:
            t = t + w * np.abs(b["dgate"])
        assert np.all(np.abs(g - b["dgate"]) <= t + 1e-30), "dgate"


DTYPES = ["f32", "bf16"]
GATES = ["none", "score", "image", "token"]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("gate_kind", GATES)
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("chunks", [1, 31, 32, 33, 64, 65, 96, 97, 128, 129, 256, 257, 511, 512, 513, 1023, 1024])
def test_row_widths(dtype, gate_kind, kind, chunks):
    C = chunks * (4 if dtype == "f32" else 8)
    check(Run(problem(dtype, 3, 5, C, kind, gate_kind, keep=1.0 if chunks % 2 else 0.6, seed=chunks)))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("gate_kind", GATES)
@pytest.mark.parametrize("B,N", [(1, 1), (64, 1), (1, 700), (7, 197), (300, 3), (2, 1025)])
def test_batches(dtype, gate_kind, B, N):
    check(Run(problem(dtype, B, N, 96, "layer", gate_kind, keep=0.5, seed=B)))
    check(Run(problem(dtype, B, N, 96, "rms", gate_kind, seed=N)))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("gate_kind", GATES)
def test_absent_parameters_and_gradients(dtype, gate_kind):
    run = Run(problem(dtype, 3, 40, 128, "layer", gate_kind, params=False))
    check(run)
    check(run, dn=True, dy=False)
    check(run, dn=False, dy=True)
    whole = [t.clone() for t in (run.dx, run.dz)]
    for k in run.grads:
        run.grads[k] = None
    run.dgate = None
    run.bwd(dn=False)
    torch.cuda.synchronize()
    assert torch.equal(run.dx, whole[0]) and torch.equal(run.dz, whole[1])


@pytest.mark.parametrize("dtype", DTYPES)
def test_no_token_has_a_row(dtype):
    pr = problem(dtype, 2, 30, 64, "layer", "score", keep=0.5)
    pr["row"][:] = -1
    check(Run(pr))


@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_out_of_range_pass_x_on(dtype):
    pr = problem(dtype, 2, 30, 64, "layer", "token", keep=0.5)
    run = Run(pr)
    run.row[3], run.row[5] = run.p.capacity, 1 << 30
    run.fwd(); run.bwd()
    torch.cuda.synchronize()
    assert torch.equal(run.y[[3, 5]], run.x[[3, 5]]) and bool((run.dgate[[3, 5]] == 0).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shift", [30.0])
def test_a_mean_far_from_zero(dtype, shift):
    check(Run(problem(dtype, 2, 50, 256, "layer", "image", shift=shift)))


@pytest.mark.parametrize("dtype", DTYPES)
def test_constant_rows(dtype):
    """No deviation: 1 / sqrt(eps), and a normalised value of zero."""
    pr = problem(dtype, 1, 4, 64, "layer", "none")
    pr["z"][:] = 2.0
    run = Run(pr)
    run.fwd()
    torch.cuda.synchronize()
    y = pr["x"] + pr["scale"] * pr["b_post"]
    assert np.all(np.abs(host(run.y) - y) <= 2.0 ** -8 * np.abs(y) + 1e-5) and np.allclose(host(run.stats)[1], 1e-5 ** -0.5, rtol=1e-5)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("gate_kind", GATES)
def test_in_place_on_another_stream_and_in_a_graph(dtype, gate_kind):
    pr = problem(dtype, 4, 190, 384, "layer", gate_kind, keep=0.7)
    run = Run(pr)
    run.fwd(); run.bwd()
    torch.cuda.synchronize()
    outs = lambda r: [t.clone() for t in (r.y, r.n, r.stats, r.dx, r.dz, *r.grads.values()) + (() if r.dgate is None else (r.dgate,))]
    first = outs(run)
    again = Run(pr)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again.y = again.x                  # y over x, dx over dy
        again.dx = again.dy
        again.fwd(); again.bwd()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, outs(again)))
    g = torch.cuda.CUDAGraph()
    run.ws.fill_(0x55)
    with torch.cuda.graph(g):
        run.fwd(); run.bwd()
    for t in (run.y, run.n, run.dx):
        t.fill_(3.0)
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, outs(run)))


def test_inference_without_statistics_or_second_norm():
    run = Run(problem("bf16", 4, 50, 768, "rms", "image", keep=0.4))
    run.fwd()
    torch.cuda.synchronize()
    y, n = run.y.clone(), run.n.clone()
    run.y.zero_()
    run.L.spa_sandwich_norm(run.p, run.sw, run.x, run.z, run.row, run.y, None, None)
    torch.cuda.synchronize()
    assert torch.equal(run.y, y)
    run.n.zero_()
    run.L.spa_sandwich_norm(run.p, run.sw, run.x, run.z, run.row, run.y, run.n, None)
    torch.cuda.synchronize()
    assert torch.equal(run.n, n)


def test_empty_batch_clears_the_sums():
    from paper_2410_23608_b200 import binding as L
    p = L.make_params(0, 5, 64, 1, "f32", capacity=1)
    t = torch.ones(1, 64, device="cuda")
    sw = L.sandwich()
    grad = torch.ones(64, device="cuda")
    ws = torch.empty(max(256, L.spa_sandwich_workspace_bytes(p, sw)), dtype=torch.uint8, device="cuda")
    L.spa_sandwich_norm(p, sw, t, t, None, t, t, t)
    L.spa_sandwich_norm_bwd(p, sw, t, t, t, t, None, t, t, t, dscale=grad, workspace=ws)
    torch.cuda.synchronize()
    assert bool((grad == 0).all()) and bool((t == 1).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", [64, 768, 4096])
@pytest.mark.parametrize("what", ["score", "z"])
def test_values_that_are_not_finite_beside_the_selection(dtype, C, what):
    """Tokens without a row have scores that are NaN, rows of z that no token names are NaN: nothing changes."""
    pr = problem(dtype, 3, 45, C, "layer", "score", keep=0.5, seed=C)
    clean = Run(pr)
    clean.fwd(); clean.bwd()
    run = Run(pr)
    if what == "score":
        run.gate[torch.from_numpy(pr["row"] < 0).cuda()] = float("nan")
    else:
        run.z[pr["z"].shape[0]:] = float("nan")
    run.fwd(); run.bwd()
    torch.cuda.synchronize()
    for k in ("y", "n", "stats", "dx", "dz", "dgate"):
        assert torch.equal(getattr(run, k), getattr(clean, k)), k
    for k, g in run.grads.items():
        assert torch.equal(g, clean.grads[k]), k
