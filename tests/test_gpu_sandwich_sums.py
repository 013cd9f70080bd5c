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
