"""The operators as a block uses them: LayerNorm, selection and packing, QKV, attention with the relative position bias, projection, and the
norms around the sum with the selection's scores as gate; then all the way back.  Against the same block in torch's fp64 autograd.

Error bounds: fp32 1e-4 of the largest value, the package's bound for chains.  bf16: a rounding is off by at most 2^-8 of the value, its
root mean square by 2^-8 / sqrt(3); the longest way (packed rows, qkv, P, attention, z, y; dz, its product, dS, dqkv, dx and two weights
beside them) has 13, which may add up."""
import numpy as np
import pytest
import torch

from tests.gpu_util import dev, host, round_to

pytestmark = pytest.mark.gpu
EPS = 1e-5


def problem(dtype, seed=0):
    rng = np.random.default_rng(seed)
    B, rows, cols, C, H = 3, 9, 11, 128, 4
    N, E = rows * cols, (2 * rows - 1) * (2 * cols - 1)
    r = lambda *s, std=1.0, mean=0.0: round_to(mean + std * rng.normal(size=s), dtype)
    mask = rng.random((B, N)) < np.array([0.6, 0.2, 0.9])[:, None]
    nb = 40
    return dict(B=B, N=N, rows=rows, cols=cols, C=C, H=H, nb=nb, mask=mask, bucket=rng.integers(0, nb, E).astype(np.int32), scores=rng.normal(size=B * N),
                x=r(B * N, C), g1=r(C, std=0.1, mean=1.0), be1=r(C, std=0.1), W_qkv=r(3 * C, C, std=C ** -0.5), b_qkv=r(3 * C, std=0.1),
                W_o=r(C, C, std=C ** -0.5), b_o=r(C, std=0.1), table=r(nb, H), scale=r(C, std=0.2, mean=0.5), g_post=r(C, std=0.1, mean=1.0),
                b_post=r(C, std=0.1), g_pre=r(C, std=0.1, mean=1.0), b_pre=r(C, std=0.1), dn=r(B * N, C), dy=r(B * N, C))


def reference(pr):
    t = {k: torch.tensor(v, dtype=torch.float64, requires_grad=True) for k, v in pr.items()
         if isinstance(v, np.ndarray) and k not in ("mask", "bucket", "dn", "dy")}
    B, N, C, H, cols, rows = (pr[k] for k in ("B", "N", "C", "H", "cols", "rows"))
    ln = lambda v: (v - v.mean(1, keepdim=True)) / (v.var(1, unbiased=False, keepdim=True) + EPS).sqrt()
    a = ln(t["x"]) * t["g1"] + t["be1"]
    z = torch.zeros(B * N, C, dtype=torch.float64)
    parts = []
    for b in range(B):
        sel = np.nonzero(pr["mask"][b])[0]
        y, x = torch.tensor(sel // cols), torch.tensor(sel % cols)
        off = (y[:, None] - y[None] + rows - 1) * (2 * cols - 1) + x[:, None] - x[None] + cols - 1
        bias = t["table"][torch.tensor(pr["bucket"], dtype=torch.long)[off]].permute(2, 0, 1)
        qkv = (a[b * N + sel] @ t["W_qkv"].T + t["b_qkv"]).view(len(sel), 3, H, C // H).permute(1, 2, 0, 3)
        P = torch.softmax(qkv[0] @ qkv[1].transpose(1, 2) * (C // H) ** -0.5 + bias, 2)
        parts.append((P @ qkv[2]).transpose(0, 1).reshape(len(sel), C) @ t["W_o"].T + t["b_o"])
    has = torch.tensor(pr["mask"].reshape(-1))
    z = torch.zeros(B * N, C, dtype=torch.float64).masked_scatter(has[:, None].expand(-1, C), torch.cat(parts))
    branch = t["scale"] * torch.sigmoid(t["scores"])[:, None] * (t["g_post"] * ln(torch.cat(parts)) + t["b_post"])[torch.cumsum(has, 0).clamp(min=1) - 1]
    y = t["x"] + torch.where(has[:, None], branch, torch.zeros_like(z))
    n = t["g_pre"] * ln(y) + t["b_pre"]
    ((n * torch.tensor(pr["dn"])).sum() + (y * torch.tensor(pr["dy"])).sum()).backward()
    return y.detach().numpy(), n.detach().numpy(), {k: v.grad.numpy() for k, v in t.items() if v.grad is not None}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_block_forward_and_backward(dtype):
    from paper_2410_23608_b200 import binding as L
    pr = problem(dtype)
    B, N, C, H = (pr[k] for k in ("B", "N", "C", "H"))
    Np = int(pr["mask"].sum())
    p = L.make_params(B, N, C, H, dtype, capacity=B * N)
    T = torch.float32 if dtype == "f32" else torch.bfloat16
    e = lambda *s, t=T: torch.full(s, 3.0, dtype=t, device="cuda")
    f = lambda *s: e(*s, t=torch.float32)
    i = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")
    d = {k: dev(v, dtype) for k, v in pr.items() if isinstance(v, np.ndarray) and k not in ("mask", "bucket", "scores")}
    scores = dev(pr["scores"], "f32")
    mask = torch.from_numpy(pr["mask"].astype(np.uint8).reshape(-1)).cuda()
    cap, status = B * N, i(1)
    a, m1, r1 = e(cap, C), f(cap), f(cap)
    xp, idx, inv, cu = e(cap, C), i(cap), i(cap), i(B + 1)
    qkv, ao, z, y, n = e(cap, 3 * C), e(cap, C), e(cap, C), e(cap, C), e(cap, C)
    lse, peak, stats = f(H, cap), f(H, cap), f(4, cap)
    rel = L.rel_bias(pr["rows"], pr["cols"], torch.from_numpy(pr["bucket"]).cuda(), d["table"])
    sw = L.sandwich("layer", "score", gate=scores, eps=EPS, **{k: d[k] for k in ("scale", "g_post", "b_post", "g_pre", "b_pre")})
    ws = torch.empty(max(256, L.spa_workspace_bytes(p), L.spa_train_workspace_bytes(p), L.spa_rel_workspace_bytes(p, rel),
                         L.spa_sandwich_workspace_bytes(p, sw)), dtype=torch.uint8, device="cuda")
    # ---- forward
    L.spa_layer_norm(p, d["x"], d["g1"], d["be1"], EPS, a, m1, r1)
    L.spa_select_pack(p, a, mask, None, xp, idx, inv, cu, d_status=status)
    L.spa_packed_qkv(p, xp, d["W_qkv"], d["b_qkv"], cu, qkv, d_status=status)
    L.spa_packed_attention_rel_fwd(p, rel, qkv, cu, B, idx, ao, lse, peak, ws, d_status=status)
    L.spa_packed_proj(p, ao, d["W_o"], d["b_o"], cu, z, d_status=status)
    L.spa_sandwich_norm(p, sw, d["x"], z, inv, y, n, stats)
    # ---- backward
    dx_sum, dz, d_ao, dqkv, dxp, da, dx = e(cap, C), e(cap, C), e(cap, C), e(cap, 3 * C), e(cap, C), e(cap, C), e(cap, C)
    g = {k: f(*pr[k].shape) for k in ("scale", "g_post", "b_post", "g_pre", "b_pre", "W_qkv", "b_qkv", "W_o", "b_o", "table", "g1", "be1", "scores")}
    L.spa_sandwich_norm_bwd(p, sw, d["dn"], d["dy"], y, z, inv, stats, dx_sum, dz, dgate=g["scores"], dscale=g["scale"], dg_post=g["g_post"],
                            db_post=g["b_post"], dg_pre=g["g_pre"], db_pre=g["b_pre"], workspace=ws)
    L.spa_packed_linear_bwd(p, ao, d["W_o"], dz, C, C, cu, d_ao, g["W_o"], g["b_o"], workspace=ws, d_status=status)
    L.spa_packed_attention_rel_bwd(p, rel, qkv, ao, lse, peak, d_ao, cu, B, idx, dqkv, g["table"], ws, d_status=status)
    L.spa_packed_linear_bwd(p, xp, d["W_qkv"], dqkv, C, 3 * C, cu, dxp, g["W_qkv"], g["b_qkv"], workspace=ws, d_status=status)
    da.zero_()
    L.spa_select_pack_bwd(p, dxp, None, idx, cu, da)
    L.spa_layer_norm_bwd(p, da, d["x"], d["g1"], m1, r1, dx_sum, dx, g["g1"], g["be1"], ws)
    torch.cuda.synchronize()
    assert status.item() == 0 and cu.cpu().numpy()[-1] == Np
    ref_y, ref_n, ref = reference(pr)
    got = dict({k: host(v) for k, v in g.items()}, x=host(dx), y=host(y), n=host(n))
    for k, want in dict(ref, y=ref_y, n=ref_n).items():
        if dtype == "f32":
            assert np.abs(got[k] - want).max() <= 1e-4 * max(1.0, np.abs(want).max()), (k, np.abs(got[k] - want).max())
        else:
            rms = np.sqrt(((got[k] - want) ** 2).mean() / (want ** 2).mean())
            assert rms <= 13 * 2.0 ** -8 / np.sqrt(3), (k, rms)
