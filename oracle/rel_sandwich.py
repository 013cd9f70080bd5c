"""fp64 oracle of the attention with a learned relative position bias and of the norms around a block, forward and backward.

Test infrastructure only, written from the formulas: numpy float64, one segment after the other, `@` the only library step.
Beside the values the attention functions return what error bounds are made of (sums of absolute values).
"""
import numpy as np


def offsets(idx, rows, cols):
    """off(i, j) of every pair of the tokens idx (flat positions b * rows * cols + n)."""
    n = np.asarray(idx, np.int64) % (rows * cols)
    y, x = n // cols, n % cols
    return (y[:, None] - y[None, :] + rows - 1) * (2 * cols - 1) + (x[:, None] - x[None, :] + cols - 1)


def rel_fwd(qkv, cu, idx, rows, cols, bucket, table, H, scale=None):
    Np, C = int(cu[-1]), qkv.shape[1] // 3
    d = C // H
    scale = d ** -0.5 if scale is None else scale
    out, mean_abs = np.zeros((Np, C)), np.zeros((Np, C))
    lse, peak = np.full((H, Np), -np.inf), np.zeros((H, Np))
    s_abs = 0.0
    for lo, hi in zip(cu[:-1], cu[1:]):
        if hi == lo:
            continue
        off = offsets(idx[lo:hi], rows, cols)
        for h in range(H):
            q, k, v = (qkv[lo:hi, w * C + h * d:w * C + (h + 1) * d] for w in range(3))
            b = table[bucket[off], h]
            S = q @ k.T * scale + b
            s_abs = max(s_abs, float((np.abs(q) @ np.abs(k).T * scale + np.abs(np.where(np.isinf(b), 0, b))).max()))
            m = S.max(1)
            ok = m > -np.inf
            e = np.exp(S - np.where(ok, m, 0.0)[:, None])
            l = e.sum(1)
            P = e / np.where(ok, l, 1.0)[:, None]
            out[lo:hi, h * d:(h + 1) * d] = P @ v
            mean_abs[lo:hi, h * d:(h + 1) * d] = P @ np.abs(v)
            lse[h, lo:hi] = np.where(ok, m + np.log(np.where(ok, l, 1.0)), -np.inf)
            peak[h, lo:hi] = np.where(ok, -np.log(np.where(ok, l, 1.0)), 0.0)
    return dict(out=out, lse=lse, peak=peak, mean_abs=mean_abs, s_abs=s_abs)


def rel_bwd(qkv, out, lse, d_out, cu, idx, rows, cols, bucket, table, H, scale=None, p_err=0.0, dot_err=0.0, round_p=0.0):
    """Gradients, and under the same names with "_tol" a bound on the error of a computation whose probabilities are off by p_err and
    whose dot products by dot_err of their absolute sums, and that rounds P and dS by round_p before the products that use them."""
    Np, C = int(cu[-1]), qkv.shape[1] // 3
    d = C // H
    scale = d ** -0.5 if scale is None else scale
    r = {k: np.zeros((Np, 3 * C)) for k in ("dqkv", "dqkv_tol")}
    r.update({k: np.zeros(table.shape) for k in ("dtable", "dtable_tol", "count")})
    for lo, hi in zip(cu[:-1], cu[1:]):
        if hi == lo:
            continue
        off = offsets(idx[lo:hi], rows, cols)
        b = bucket[off]
        for h in range(H):
            cols_of = [slice(w * C + h * d, w * C + (h + 1) * d) for w in range(3)]
            q, k, v = (qkv[lo:hi, c] for c in cols_of)
            o, do = out[lo:hi, h * d:(h + 1) * d], d_out[lo:hi, h * d:(h + 1) * d]
            S = q @ k.T * scale + table[b, h]
            lrow = lse[h, lo:hi]
            ok = lrow > -np.inf
            P = np.where(ok[:, None], np.exp(S - np.where(ok, lrow, 0.0)[:, None]), 0.0)
            D = (do * o).sum(1)
            dP = do @ v.T
            dS = P * (dP - D[:, None])
            E = P * (p_err * np.abs(dP - D[:, None]) + dot_err * (np.abs(do) @ np.abs(v).T + (np.abs(do) * np.abs(o)).sum(1)[:, None]))
            E2 = E + (round_p + (hi - lo) * 2.0 ** -24) * np.abs(dS)
            P2 = P * (p_err + round_p + (hi - lo) * 2.0 ** -24)
            for c, g, t in zip(cols_of, (scale * dS @ k, scale * dS.T @ q, P.T @ do),
                               (scale * E2 @ np.abs(k), scale * E2.T @ np.abs(q), P2.T @ np.abs(do))):
                r["dqkv"][lo:hi, c], r["dqkv_tol"][lo:hi, c] = g, t
            np.add.at(r["dtable"][:, h], b, dS)
            np.add.at(r["dtable_tol"][:, h], b, E)
            np.add.at(r["count"][:, h], b, 1.0)
    return r


def _stats(v, kind, eps):
    m = v.mean(1) if kind == "layer" else np.zeros(v.shape[0])
    return m, 1.0 / np.sqrt(((v - m[:, None]) ** 2).mean(1) + eps)


def _gate(gate, gate_kind, B, N):
    if gate_kind == "none":
        return np.ones((B * N, 1))
    if gate_kind == "score":
        return (1.0 / (1.0 + np.exp(-gate)))[:, None]
    return np.repeat(gate, N, 0) if gate_kind == "image" else gate


def sandwich_fwd(x, z, row, gate, gate_kind, scale, g_post, b_post, g_pre, b_pre, kind, eps, B, N):
    """x [B N, C]; row [B N] the row of z of every token or -1; all parameters given."""
    has = row >= 0
    m1, r1 = np.zeros(B * N), np.zeros(B * N)
    y = x.copy()
    if has.any():
        v = z[row[has]]
        m1[has], r1[has] = _stats(v, kind, eps)
        zh = (v - m1[has, None]) * r1[has, None]
        y[has] += scale * _gate(gate, gate_kind, B, N)[has if gate_kind != "none" else slice(0, int(has.sum()))] * (g_post * zh + b_post)
    m2, r2 = _stats(y, kind, eps)
    return dict(y=y, n=g_pre * (y - m2[:, None]) * r2[:, None] + b_pre, stats=np.stack((m1, r1, m2, r2)))


def _through_norm(g, vh, r, kind):
    out = g - vh * (g * vh).mean(1, keepdims=True)
    if kind == "layer":
        out = out - g.mean(1, keepdims=True)
    return out * r[:, None]


def sandwich_bwd(dn, dy, y, z, row, stats, gate, gate_kind, scale, g_post, b_post, g_pre, kind, B, N):
    m1, r1, m2, r2 = stats
    has = row >= 0
    yh = (y - m2[:, None]) * r2[:, None]
    d = dy + _through_norm(dn * g_pre, yh, r2, kind)
    w = np.broadcast_to(_gate(gate, gate_kind, B, N), d.shape)
    zh = np.zeros_like(d)
    zh[has] = (z[row[has]] - m1[has, None]) * r1[has, None]
    a = np.where(has[:, None], g_post * zh + b_post, 0.0)
    da = np.where(has[:, None], d * w * scale, 0.0)
    dz = np.zeros_like(z)
    dz[row[has]] = _through_norm((da * g_post)[has], zh[has], r1[has], kind)
    dg = d * scale * a
    r = dict(dx=d, dz=dz, dscale=(d * w * a).sum(0), dg_post=(da * zh).sum(0), db_post=da.sum(0), dg_pre=(dn * yh).sum(0), db_pre=dn.sum(0))
    if gate_kind == "score":
        r["dgate"] = dg.sum(1) * w[:, 0] * (1 - w[:, 0])
    elif gate_kind == "image":
        r["dgate"] = dg.reshape(B, N, -1).sum(1)
    elif gate_kind == "token":
        r["dgate"] = dg
    # sums of absolute values, which errors of the sums over rows go by
    ad = np.abs(d) * np.abs(w)
    r["abs"] = dict(dscale=(ad * (np.abs(g_post * zh) + np.abs(b_post)) * has[:, None]).sum(0), dg_post=(ad * np.abs(scale * zh) * has[:, None]).sum(0),
                    db_post=(ad * np.abs(scale) * has[:, None]).sum(0), dg_pre=np.abs(dn * yh).sum(0), db_pre=np.abs(dn).sum(0),
                    dgate_row=(np.abs(d * scale) * (np.abs(g_post * zh) + np.abs(b_post)) * has[:, None]))
    return r
