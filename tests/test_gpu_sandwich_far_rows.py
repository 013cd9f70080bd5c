"""Rows of the norms around a block whose mean is far from zero.

Where mean and variance are whole numbers, of 2^k values, both are exact in fp32: a normalised value has the rounding of 1 / deviation (rsqrtf:
2 units in the last place, 4 u) and of one product, and a row's sums in the backward those of 64 terms.  (Normalised as v r - m r, with m r rounded,
they were off by up to half a unit of m r: 2^-24 times the mean in deviations.)"""
import numpy as np
import pytest
import torch

from tests.gpu_util import dev, host

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("C", [64, 256, 1024, 4096])
@pytest.mark.parametrize("N", [1, 37])
def test_rows_far_from_zero(C, N):
    from paper_2410_23608_b200 import binding as L
    rng = np.random.default_rng(C)
    sign = np.stack([rng.permutation(np.repeat([1.0, -1.0], C // 2)) for _ in range(N)])
    z, x = 4096.0 + 3.0 * sign, np.zeros((N, C))
    p = L.make_params(1, N, C, 1, "f32")
    big = 65536.0
    b_post = np.full(C, big)                               # y = 65536 +- 1, and a little
    sw = L.sandwich("layer", "none", b_post=dev(b_post, "f32"), eps=0.0)
    e = lambda *s: torch.empty(*s, device="cuda")
    y, y2, n, stats = e(N, C), e(N, C), e(N, C), e(4, N)
    L.spa_sandwich_norm(p, sw, dev(x, "f32"), dev(z, "f32"), None, y, n, stats)
    L.spa_sandwich_norm(p, L.sandwich("layer", "none", eps=0.0), dev(x, "f32"), dev(z, "f32"), None, y2, n, stats)
    torch.cuda.synchronize()
    assert np.all(np.abs(host(y2) - sign) <= 8 * U), np.max(np.abs(host(y2) - sign)) / U
    # the norm behind the sum, of y as it is rounded there: to a unit of 2^-7
    assert np.all(np.abs(host(y) - (big + sign)) <= 2.0 ** -8 + 8 * U)
    # backward: dz of the branch alone, from y = 2 sign + 12288, whose statistics are exact too
    yb = 12288.0 + 3.0 * sign
    third = float(np.float32(1.0 / 3.0))
    st = np.stack((np.full(N, 4096.0), np.full(N, third), np.full(N, 12288.0), np.full(N, third)))
    d = rng.integers(-8, 9, (N, C)).astype(np.float64)
    dx, dz, dg_pre, dg_post = e(N, C), e(N, C), e(C), e(C)
    ws = torch.empty(L.spa_sandwich_workspace_bytes(p, sw), dtype=torch.uint8, device="cuda")
    plain = L.sandwich("layer", "none", eps=0.0)
    L.spa_sandwich_norm_bwd(p, plain, dev(d, "f32"), None, dev(yb, "f32"), dev(z, "f32"), None, dev(st, "f32"), dx, dz, dg_pre=dg_pre, dg_post=dg_post,
                            workspace=ws)
    torch.cuda.synchronize()
    h = sign * 3.0 * third                                 # (v - m) / deviation: a product of 3 and the stored third
    through = lambda g: third * (g - g.mean(1, keepdims=True) - h * (g * h).mean(1, keepdims=True))
    gx = through(d)
    gz = through(gx)
    top = np.abs(d).max()
    # a row's two sums: a chain of at most 32 terms and a tree of at most 16 steps, of terms of at most `top`; a few products
    assert np.all(np.abs(host(dx) - gx) <= (2 * (48 + 8)) * U * top), np.max(np.abs(host(dx) - gx)) / (U * top)
    assert np.all(np.abs(host(dz) - gz) <= (4 * (48 + 8)) * U * top), np.max(np.abs(host(dz) - gz)) / (U * top)
    rows = min(N, 256) + 16                                # rows one after the other, and groups
    assert np.all(np.abs(host(dg_pre) - (d * h).sum(0)) <= (rows + 4) * U * np.abs(d * h).sum(0))
    assert np.all(np.abs(host(dg_post) - (gx * h).sum(0)) <= (rows + 4) * U * np.abs(gx * h).sum(0) + N * 2 * (48 + 8) * U * top)
