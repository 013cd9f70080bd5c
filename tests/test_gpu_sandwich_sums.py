"""Sums over the rows in the backward of the norms around a block.  A thread adds at most 256 rows of its CTA's share one after the other (each
addition off by u = 2^-24 of the sum of absolute values at most), the CTA its groups of threads (rows of more than 256 chunks: one
group), and the CTAs' lines are added in 64 bits and rounded once.  Rows that are all the same value make the roundings of a chain go one way."""
import numpy as np
import pytest
import torch

from tests.gpu_util import dev, host

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def fp32(rng, n):
    return (1.0 + rng.random(n)).astype(np.float32).astype(np.float64)


@pytest.mark.parametrize("gate_kind,N", [("none", 1), ("image", 2), ("image", 500)])
@pytest.mark.parametrize("T", [148, 1184, 300000])
def test_sums_over_rows(gate_kind, N, T):
    from paper_2410_23608_b200 import binding as L
    C, T = 1028, max(N, T // N * N)                        # 257 chunks: a row to a group, a group to a CTA
    rng = np.random.default_rng(T + N)
    dn, dy, g = fp32(rng, C), fp32(rng, C), fp32(rng, C)
    p = L.make_params(T // N, N, C, 1, "f32")
    rows = lambda v: dev(v, "f32").expand(T, C).contiguous()
    gate = dev(np.broadcast_to(g, (T // N, C)), "f32") if gate_kind == "image" else None
    sw = L.sandwich("rms", gate_kind, gate=gate)
    zero = torch.zeros(T, C, device="cuda")
    stats = torch.zeros(4, T, device="cuda")               # nothing goes through the norms
    dx, dz = torch.empty(T, C, device="cuda"), torch.empty(T, C, device="cuda")
    f = lambda *s: torch.empty(*s, device="cuda")
    db_pre, db_post, dgate = f(C), f(C), f(T // N, C) if gate_kind == "image" else None
    ws = torch.empty(L.spa_sandwich_workspace_bytes(p, sw), dtype=torch.uint8, device="cuda")
    L.spa_sandwich_norm_bwd(p, sw, rows(dn), rows(dy), zero, zero, None, stats, dx, dz, dgate=dgate, db_pre=db_pre, db_post=db_post, workspace=ws)
    torch.cuda.synchronize()
    chain = min(256, -(-T // 148))                         # 148 CTAs, or as many more as that takes
    want = T * dn
    assert np.all(np.abs(host(db_pre) - want) <= (chain + 1) * U * want), np.max(np.abs(host(db_pre) - want) / (U * want))
    want = T * dy * (g if gate_kind == "image" else 1.0)
    # with a gate per image: a sum of its rows in the CTA, a product, and a sum of the CTA's images
    images = 0 if gate_kind == "none" else 1 + chain // N + 2
    assert np.all(np.abs(host(db_post) - want) <= (chain + images + 1) * U * want), np.max(np.abs(host(db_post) - want) / (U * want))
    if dgate is not None:                                  # the branch is zero
        assert bool((dgate == 0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gate_kind", ["none", "image", "score"])
@pytest.mark.parametrize("chunks", [1, 32, 33, 96, 129, 256, 257, 513, 1024])
@pytest.mark.parametrize("B,N", [(2, 1025), (41, 50)])
def test_every_row_is_in_the_sums_once(dtype, gate_kind, chunks, B, N):
    """2 050 rows of positive values, a bound that a row left out or taken twice is far beyond: a share of 14 rows, at most 14 additions of rows, 12 of
    groups, with a gate per image those of the images of a share, and the result's rounding."""
    from paper_2410_23608_b200 import binding as L
    T, C = B * N, chunks * (4 if dtype == "f32" else 8)
    g = torch.Generator(device="cuda").manual_seed(chunks)
    ty = torch.float32 if dtype == "f32" else torch.bfloat16
    new = lambda *s: (1.0 + torch.rand(*s, generator=g, device="cuda")).to(ty)
    dn, dy, zero = new(T, C), new(T, C), torch.zeros(T, C, dtype=ty, device="cuda")
    row = torch.full((T,), -1, dtype=torch.int32, device="cuda")
    has = torch.rand(T, generator=g, device="cuda") < 0.7
    row[has] = torch.randperm(int(has.sum()), generator=g, device="cuda").int()
    gate = {"none": None, "image": new(B, C), "score": torch.zeros(T, device="cuda")}[gate_kind]
    p = L.make_params(B, N, C, 1, dtype, capacity=T)
    sw = L.sandwich("layer", gate_kind, gate=gate)
    f = lambda *s: torch.empty(*s, device="cuda")
    dgate = {"none": lambda: None, "image": lambda: f(B, C), "score": lambda: f(T)}[gate_kind]()
    db_pre, db_post = f(C), f(C)
    ws = torch.empty(L.spa_sandwich_workspace_bytes(p, sw), dtype=torch.uint8, device="cuda")
    L.spa_sandwich_norm_bwd(p, sw, dn, dy, zero, zero, row, torch.zeros(4, T, device="cuda"), torch.empty_like(dy), torch.empty_like(dy), dgate=dgate,
                            db_pre=db_pre, db_post=db_post, workspace=ws)
    torch.cuda.synchronize()
    tol = (14 + 12 + 2) * U
    want = host(dn).sum(0)
    assert np.all(np.abs(host(db_pre) - want) <= tol * want)
    w = {"none": 1.0, "image": None, "score": 0.5}[gate_kind]
    w = np.repeat(host(gate), N, 0) if w is None else w      # sigmoid(0) is 1 / 2
    want = (host(dy) * w)[has.cpu().numpy()].sum(0)
    assert np.all(np.abs(host(db_post) - want) <= (tol + 4 * U) * want)
