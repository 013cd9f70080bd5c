"""Attention with a learned relative position bias, and the norms around a block: measurable cases.

Two operators, each in both directions:

  rel    attention of packed tokens inside their segments with a learned bias per head and bucket of the relative grid
         position.  Keys of a case: direction "forward" or "backward", dtype, B images of rows x cols tokens, C channels, H
         heads, keep_lo .. keep_hi the images' fractions of selected tokens (spread evenly), axis the buckets per axis
         (logarithmic in the distance; 0: a bucket for every offset).
  norm   y = x + scale * gate * norm(z), n = norm(y).  Keys: direction, dtype, B images of N tokens, C channels, kind "layer" or
         "rms", gate "none", "score", "image" or "token", keep: 1 with a row of z for every token, else the fraction of
         tokens that have one (z is packed then).

The plain forms compute in 32 bits from elementary torch operations and round once; the table's gradient, a sum over up to
millions of pairs, is summed in 64.  `exact` is the definition in 64 bits, segment after segment.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-6
_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _rel(name, direction, dtype, B, rows, cols, C, H, keep_lo, keep_hi, axis):
    c = dict(op="rel", direction=direction, dtype=dtype, B=B, rows=rows, cols=cols, C=C, H=H, keep_lo=keep_lo, keep_hi=keep_hi, axis=axis)
    return dict(c, name=name) if name else c


def _norm(name, direction, dtype, B, N, C, kind, gate, keep):
    c = dict(op="norm", direction=direction, dtype=dtype, B=B, N=N, C=C, kind=kind, gate=gate, keep=keep)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one photo while a user waits: launches and latency
        _rel("rel_one_image", "forward", "bf16", 1, 14, 14, 384, 6, 0.35, 0.65, 9),
        # detection inference on a batch of frames: long segments, a table over a large grid, an odd grid
        _rel("rel_frames", "forward", "bf16", 8, 47, 83, 256, 8, 0.10, 0.50, 15),
        # classification inference in a large batch
        _rel("rel_vit_b", "forward", "bf16", 128, 14, 14, 768, 12, 0.05, 0.70, 0),
        # fp32 inference, where bf16 is not wanted
        _rel("rel_vit_s_f32", "forward", "f32", 16, 14, 14, 384, 6, 0.20, 0.80, 9),
        # a first experiment or a numerical check in fp32
        _rel("rel_tiny_f32_train", "backward", "f32", 4, 14, 14, 96, 3, 0.10, 0.50, 0),
        # windows of 7 x 7 as a hierarchical backbone trains them: all tokens, one bucket for every offset
        _rel("rel_windows_train", "backward", "bf16", 512, 7, 7, 384, 12, 1.0, 1.0, 0),
        # large images, half selected on average
        _rel("rel_vit_b16_384_train", "backward", "bf16", 32, 24, 24, 768, 12, 0.10, 0.90, 0),
        # the tokens of a step of 64 requests, each with its own gate
        _norm("norm_tokens", "forward", "bf16", 64, 1, 1024, "rms", "image", 1),
        # detection inference: the attention's packed rows joined to the feature map, gated by the selection's score
        _norm("norm_packed", "forward", "bf16", 16, 4200, 256, "layer", "score", 0.3),
        # an fp32 experiment
        _norm("norm_f32_train", "backward", "f32", 16, 196, 384, "layer", "image", 1),
        # training of a conditioned block: a gate per image
        _norm("norm_image_train", "backward", "bf16", 32, 576, 768, "layer", "image", 1),
        # wide rows, a gate for every element
        _norm("norm_wide_train", "backward", "bf16", 8, 1023, 4096, "rms", "token", 1),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Single images to large batches, windows to detection grids; single tokens to feature maps, narrow to wide rows."""
    direction = rng.choice(("forward", "backward"))
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    while True:
        if rng.random() < 0.6:
            side = _log_int(rng, 3, 50)
            rows, cols = side, max(2, int(round(side * rng.uniform(0.8, 1.7))))
            d = rng.choice((32, 64))
            H = _log_int(rng, 1, 12)
            lo = rng.uniform(0.02, 0.6)
            hi = 1.0 if rng.random() < 0.2 else min(1.0, lo + rng.uniform(0.05, 0.6))
            lo = 1.0 if rng.random() < 0.1 else lo
            c = _rel("", direction, dtype, _log_int(rng, 1, 512), rows, cols, H * d, H, round(lo, 3), round(max(lo, hi), 3),
                     rng.choice((0, 0, 5, 9, 15)))
            if rows * cols <= 4200 and c["B"] * rows * cols <= 1 << 19 and _cost(c) <= _COST_MAX[dtype]:
                return c
        else:
            C = 8 * _log_int(rng, 8, 512)
            N = _log_int(rng, 1, 4200)
            c = _norm("", direction, dtype, _log_int(rng, 1, 128), N, C, rng.choice(("layer", "rms")),
                      rng.choice(("none", "score", "image", "token")), 1 if rng.random() < 0.6 else round(rng.uniform(0.05, 0.95), 3))
            if c["B"] * N <= 1 << 19 and _cost(c) <= _COST_MAX["norm"]:
                return c


# ---------------------------------------------------------------------------------------------------- work
def _counts(c):
    """Selected tokens of each image, before the seed permutes the images."""
    B, N = c["B"], c["rows"] * c["cols"]
    return [max(1, min(N, int(round(N * (c["keep_lo"] + (c["keep_hi"] - c["keep_lo"]) * (b + 0.5) / B))))) for b in range(B)]


def _packed_rows(c):
    return c["B"] * c["N"] if c["keep"] == 1 else max(1, int(round(c["keep"] * c["B"] * c["N"])))


def work(case):
    """Inputs read once, outputs written once; two operations per multiply-add of the attention's products (two forward, five
    backward), ten or twenty per element of the norms."""
    c = case
    es = 4 if c["dtype"] == "f32" else 2
    if c["op"] == "rel":
        n = _counts(c)
        rows, pairs, C, H = sum(n), sum(k * k for k in n), c["C"], c["H"]
        offsets = (2 * c["rows"] - 1) * (2 * c["cols"] - 1)
        table = (c["axis"] ** 2 if c["axis"] else offsets) * H
        small = 4 * offsets + 4 * rows + es * table
        if c["direction"] == "forward":
            return {"bytes": 4 * rows * C * es + 8 * rows * H + small, "flops": 4 * C * pairs}
        return {"bytes": 8 * rows * C * es + 8 * rows * H + small + 4 * table, "flops": 10 * C * pairs}
    T, Z, C = c["B"] * c["N"], _packed_rows(c), c["C"]
    gate = {"none": 0, "score": 4 * T, "image": c["B"] * C * es, "token": T * C * es}[c["gate"]]
    rowmap = 0 if c["keep"] == 1 else 4 * T
    if c["direction"] == "forward":
        return {"bytes": (3 * T + Z) * C * es + gate + rowmap + 16 * T + 5 * C * es, "flops": 10 * C * (T + Z)}
    dgate = {"none": 0, "score": 4 * T, "image": 4 * c["B"] * C, "token": T * C * es}[c["gate"]]
    return {"bytes": (4 * T + 2 * Z) * C * es + gate + dgate + rowmap + 16 * T + 5 * C * (es + 4), "flops": 20 * C * (T + Z)}


def _cost(c):
    w = work(c)
    return w["bytes"] / 5e12 + w["flops"] / (2e13 if c["dtype"] == "f32" else 3e14)


_COST_MAX = {"bf16": max(_cost(c) for c in listed() if c["op"] == "rel"), "f32": 1e-3,
             "norm": max(_cost(c) for c in listed() if c["op"] == "norm")}
_COST_MAX["f32"] = min(_COST_MAX["f32"], max(_cost(c) for c in listed()))


# ---------------------------------------------------------------------------------------------------- inputs
def _axis_bucket(n, axis):
    """Bucket of every distance -(n-1) .. n-1 along one axis: the small ones exactly, the others by their logarithm."""
    half = axis // 2
    exact = max(1, half // 2)
    out = []
    for d in range(-(n - 1), n):
        a = abs(d)
        if a > exact:
            a = min(half, exact + int(math.log(a / exact) / math.log(max(n, exact + 2) / exact) * (half - exact)) + 1)
        out.append(half + (a if d > 0 else -a))
    return out


def _buckets(c):
    R, K, axis = c["rows"], c["cols"], c["axis"]
    if axis == 0:
        return torch.arange((2 * R - 1) * (2 * K - 1), dtype=torch.int32), (2 * R - 1) * (2 * K - 1)
    by, bx = torch.tensor(_axis_bucket(R, axis)), torch.tensor(_axis_bucket(K, axis))
    return (by[:, None] * axis + bx[None, :]).reshape(-1).to(torch.int32), axis * axis


def _select(c, gen, dev):
    """Flat indices of the selected tokens, ascending: per image those nearest to one to four random centres."""
    B, R, K = c["B"], c["rows"], c["cols"]
    n = torch.tensor(_counts(c), device=dev)[torch.randperm(B, generator=gen, device=dev)]
    cy = torch.rand(B, 4, 1, generator=gen, device=dev) * R
    cx = torch.rand(B, 4, 1, generator=gen, device=dev) * K
    off = torch.arange(4, device=dev)[None, :, None] > torch.randint(0, 4, (B, 1, 1), generator=gen, device=dev)
    yy = (torch.arange(R * K, device=dev) // K + 0.5)[None, None]
    xx = (torch.arange(R * K, device=dev) % K + 0.5)[None, None]
    dist = torch.where(off, torch.inf, (yy - cy) ** 2 + (xx - cx) ** 2).amin(1)
    rank = dist.argsort(dim=1, stable=True).argsort(dim=1)
    idx = (rank < n[:, None]).reshape(-1).nonzero()[:, 0].to(torch.int32)
    return idx, n


def prepare(case, seed):
    c, dev = dict(case), "cuda"
    T = _TYPES[c["dtype"]]
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed))

    def normal(*shape, std=1.0, mean=0.0):
        return torch.randn(*shape, generator=gen, device=dev).mul_(std).add_(mean).to(T)

    s = dict(case=c)
    if c["op"] == "rel":
        C, H = c["C"], c["H"]
        s["idx"], n = _select(c, gen, dev)
        cu = torch.zeros(c["B"] + 1, dtype=torch.int32, device=dev)
        cu[1:] = n.cumsum(0)
        s["cu"], s["lens"] = cu, n.tolist()
        rows = sum(s["lens"])
        bucket, nb = _buckets(c)
        s["bucket"], s["table"] = bucket.to(dev), normal(nb, H, std=0.5)
        s["qkv"] = normal(rows, 3 * C)
        if c["direction"] == "backward":
            s["d_out"] = normal(rows, C)
            o, s["lse"], s["peak"] = _rel_forward(s)
            s["out"] = o.to(T)
    else:
        B, N, C = c["B"], c["N"], c["C"]
        Z = _packed_rows(c)
        s["x"], s["z"] = normal(B * N, C), normal(Z, C, std=0.7, mean=0.1)
        s["row"] = None
        if c["keep"] != 1:
            pick = torch.randperm(B * N, generator=gen, device=dev)[:Z].sort()[0]
            s["row"] = torch.full((B * N,), -1, dtype=torch.int32, device=dev)
            s["row"][pick] = torch.arange(Z, dtype=torch.int32, device=dev)
        s["gate"] = {"none": lambda: None, "score": lambda: torch.randn(B * N, generator=gen, device=dev),
                     "image": lambda: normal(B, C, std=0.3, mean=0.5), "token": lambda: normal(B * N, C, std=0.3, mean=0.5)}[c["gate"]]()
        s["scale"] = normal(C, std=0.1, mean=0.3)
        s["g_post"], s["g_pre"] = normal(C, std=0.05, mean=1.0), normal(C, std=0.05, mean=1.0)
        s["b_post"], s["b_pre"] = (normal(C, std=0.02), normal(C, std=0.02)) if c["kind"] == "layer" else (None, None)
        if c["direction"] == "backward":
            y, _, s["stats"] = _norm_forward(s)
            s["y"] = y.to(T)
            s["dn"], s["dy"] = normal(B * N, C), normal(B * N, C)
    if own:
        _prepare_own(s)
    return s


def _prepare_own(s):
    """The buffers that a user's program allocates once."""
    from paper_2410_23608_b200 import binding as L
    c, dev, T = s["case"], "cuda", _TYPES[s["case"]["dtype"]]
    e = lambda *shape, dt=T: torch.empty(*shape, dtype=dt, device=dev)
    f32 = torch.float32
    s["status"] = torch.zeros(1, dtype=torch.int32, device=dev)
    if c["op"] == "rel":
        rows, C, H = s["qkv"].shape[0], c["C"], c["H"]
        s["p"] = L.make_params(c["B"], c["rows"] * c["cols"], C, H, c["dtype"], capacity=rows)
        s["rel"] = L.rel_bias(c["rows"], c["cols"], s["bucket"], s["table"])
        s["ws"] = e(L.spa_rel_workspace_bytes(s["p"], s["rel"]), dt=torch.uint8)
        if c["direction"] == "forward":
            s["o_out"], s["o_lse"], s["o_peak"] = e(rows, C), e(H, rows, dt=f32), e(H, rows, dt=f32)
        else:
            s["o_dqkv"], s["o_dtable"] = e(rows, 3 * C), e(*s["table"].shape, dt=f32)
        return
    B, N, C = c["B"], c["N"], c["C"]
    s["p"] = L.make_params(B, N, C, 1, c["dtype"], capacity=s["z"].shape[0])
    s["sw"] = L.sandwich(kind=c["kind"], gate_kind=c["gate"], eps=EPS, **{k: s[k] for k in ("gate", "scale", "g_post", "b_post", "g_pre", "b_pre")})
    if c["direction"] == "forward":
        s["o_y"], s["o_n"], s["o_stats"] = e(B * N, C), e(B * N, C), e(4, B * N, dt=f32)
        return
    s["ws"] = e(max(256, L.spa_sandwich_workspace_bytes(s["p"], s["sw"])), dt=torch.uint8)
    s["o_dx"], s["o_dz"] = e(B * N, C), e(*s["z"].shape)
    s["o_dgate"] = {"none": lambda: None, "score": lambda: e(B * N, dt=f32), "image": lambda: e(B, C, dt=f32),
                    "token": lambda: e(B * N, C)}[c["gate"]]()
    for k in ("dscale", "dg_post", "dg_pre"):
        s["o_" + k] = e(C, dt=f32)
    for k in ("db_post", "db_pre"):
        s["o_" + k] = e(C, dt=f32) if c["kind"] == "layer" else None


# ---------------------------------------------------------------------------------------------------- plain forms
def _groups(s, limit=1 << 26):
    """Segments in groups of similar length, padded: (first rows [S], lengths [S], longest)."""
    H, lens = s["case"]["H"], s["lens"]
    start = [0]
    for k in lens:
        start.append(start[-1] + k)
    order = sorted(range(len(lens)), key=lambda b: lens[b])
    i = 0
    while i < len(order):
        j = i + 1
        while j < len(order) and (j + 1 - i) * lens[order[j]] ** 2 * H <= limit and lens[order[j]] <= 1.25 * lens[order[i]] + 16:
            j += 1
        g = order[i:j]
        yield [start[b] for b in g], [lens[b] for b in g], lens[order[j - 1]]
        i = j


def _pairs(s, first, lens, L):
    """What a group of segments has in common in both directions: row numbers, which of them are there, offsets, S."""
    c, qkv = s["case"], s["qkv"]
    dev, H, C, K = qkv.device, c["H"], c["C"], c["cols"]
    at = torch.arange(L, device=dev)[None] + torch.tensor(first, device=dev)[:, None]
    there = torch.arange(L, device=dev)[None] < torch.tensor(lens, device=dev)[:, None]
    at = torch.where(there, at, torch.tensor(first, device=dev)[:, None])
    n = s["idx"].long()[at] % (c["rows"] * K)
    p = n // K * (2 * K - 1) + n % K
    off = p[:, :, None] - p[:, None, :] + (c["rows"] - 1) * (2 * K - 1) + K - 1
    q, k, v = (qkv[at][..., w * C:(w + 1) * C].float().unflatten(-1, (H, C // H)).transpose(1, 2) for w in range(3))
    bias = s["table"].float()[s["bucket"].long()].t()[:, off].transpose(0, 1)
    S = (q @ k.transpose(2, 3)) * (C // H) ** -0.5 + bias
    S = S.masked_fill(~there[:, None, None, :], -torch.inf)
    return at, there, off, q, k, v, S


def _rel_forward(s):
    c, qkv = s["case"], s["qkv"]
    o = torch.zeros(qkv.shape[0], c["C"], device=qkv.device)
    lse = torch.zeros(c["H"], qkv.shape[0], device=qkv.device)
    peak = torch.zeros_like(lse)
    for first, lens, L in _groups(s):
        at, there, _, _, _, v, S = _pairs(s, first, lens, L)
        m = S.amax(3, keepdim=True)
        e = (S - m).exp()
        l = e.sum(3, keepdim=True)
        out = (e @ v / l).transpose(1, 2).flatten(2)
        o[at[there]] = out[there]
        lse[:, at[there]] = (m + l.log())[..., 0].transpose(1, 2)[there].t()
        peak[:, at[there]] = -l.log()[..., 0].transpose(1, 2)[there].t()
    return o, lse, peak


def _rel_backward(s):
    c, qkv = s["case"], s["qkv"]
    H, C, scale = c["H"], c["C"], (c["C"] // c["H"]) ** -0.5
    dqkv = torch.zeros(qkv.shape, device=qkv.device)
    bins = torch.zeros(H, s["bucket"].numel(), dtype=torch.float64, device=qkv.device)
    D = (s["d_out"].float() * s["out"].float()).unflatten(1, (H, C // H)).sum(2)
    for first, lens, L in _groups(s):
        at, there, off, q, k, v, S = _pairs(s, first, lens, L)
        do = s["d_out"][at].float().unflatten(-1, (H, C // H)).transpose(1, 2)
        P = (S - s["lse"].t()[at].transpose(1, 2)[..., None]).exp().masked_fill(~there[:, None, :, None], 0.0)
        dS = P * (do @ v.transpose(2, 3) - D[at].transpose(1, 2)[..., None])
        parts = ((dS @ k) * scale, (dS.transpose(2, 3) @ q) * scale, P.transpose(2, 3) @ do)
        dqkv[at[there]] = torch.cat([w.transpose(1, 2).flatten(2) for w in parts], 2)[there]
        for h in range(H):
            bins[h].index_add_(0, off.reshape(-1), dS[:, h].reshape(-1).double())
    dtable = torch.zeros(s["table"].shape, dtype=torch.float64, device=qkv.device)
    dtable.index_add_(0, s["bucket"].long(), bins.t().contiguous())
    return dqkv, dtable.float()


def _normalise(v, kind):
    if kind == "layer":
        m = v.mean(1)
        r = ((v - m[:, None]) ** 2).mean(1).add(EPS).rsqrt()
    else:
        m = torch.zeros(v.shape[0], device=v.device)
        r = (v * v).mean(1).add(EPS).rsqrt()
    return m, r


def _gate(s):
    """The gate of every token, [T, C] or [T, 1], and 1 without one."""
    c = s["case"]
    if c["gate"] == "none":
        return torch.ones(1, 1, device=s["z"].device)
    g = s["gate"].float()
    if c["gate"] == "score":
        return (1.0 / (1.0 + (-g).exp()))[:, None]
    return g.repeat_interleave(c["N"], 0) if c["gate"] == "image" else g


def _z_rows(s):
    """z of every token (zero where there is none) and which tokens have a row."""
    if s["row"] is None:
        return s["z"].float(), None
    has = s["row"] >= 0
    return torch.where(has[:, None], s["z"].float()[s["row"].clamp(min=0).long()], 0.0), has


def _norm_forward(s):
    kind = s["case"]["kind"]
    z, has = _z_rows(s)
    m1, r1 = _normalise(z, kind)
    a = (z - m1[:, None]) * r1[:, None] * s["g_post"].float()
    if s["b_post"] is not None:
        a = a + s["b_post"].float()
    a = a * s["scale"].float() * _gate(s)
    if has is not None:
        a, m1, r1 = torch.where(has[:, None], a, 0.0), torch.where(has, m1, 0.0), torch.where(has, r1, 0.0)
    y = s["x"].float() + a
    m2, r2 = _normalise(y, kind)
    n = (y - m2[:, None]) * r2[:, None] * s["g_pre"].float()
    if s["b_pre"] is not None:
        n = n + s["b_pre"].float()
    return y, n, torch.stack((m1, r1, m2, r2))


def _norm_grad(g, vh, r, kind):
    m2 = (g * vh).mean(1, keepdim=True)
    m1 = g.mean(1, keepdim=True) if kind == "layer" else 0.0
    return (g - m1 - vh * m2) * r[:, None]


def _norm_backward(s):
    c, kind = s["case"], s["case"]["kind"]
    m1, r1, m2, r2 = s["stats"]
    dn, y = s["dn"].float(), s["y"].float()
    yh = (y - m2[:, None]) * r2[:, None]
    out = {"dg_pre": (dn * yh).double().sum(0).float(), "db_pre": dn.double().sum(0).float()}
    dx = s["dy"].float() + _norm_grad(dn * s["g_pre"].float(), yh, r2, kind)
    z, has = _z_rows(s)
    zh = (z - m1[:, None]) * r1[:, None]
    d = dx if has is None else torch.where(has[:, None], dx, 0.0)
    a = zh * s["g_post"].float()
    if s["b_post"] is not None:
        a = a + s["b_post"].float()
    gate, scale = _gate(s), s["scale"].float()
    out["dscale"] = (d * gate * a).double().sum(0).float()
    dgate = d * scale * a
    da = d * gate * scale
    out["dg_post"], out["db_post"] = (da * zh).double().sum(0).float(), da.double().sum(0).float()
    dz = _norm_grad(da * s["g_post"].float(), zh, r1, kind)
    out["dx"], out["dz"] = dx, dz if has is None else dz[has]
    if c["gate"] == "score":
        out["dgate"] = (dgate.sum(1, keepdim=True) * gate * (1.0 - gate))[:, 0]
    elif c["gate"] == "image":
        out["dgate"] = dgate.view(c["B"], c["N"], -1).double().sum(1).float()
    elif c["gate"] == "token":
        out["dgate"] = dgate
    if kind == "rms":
        del out["db_pre"], out["db_post"]
    T = s["z"].dtype
    for k in ("dx", "dz") + (("dgate",) if c["gate"] == "token" else ()):
        out[k] = out[k].to(T)
    return out


def run(state):
    s = state
    c, T = s["case"], _TYPES[s["case"]["dtype"]]
    if own:
        return _run_own(s)
    if c["op"] == "rel":
        if c["direction"] == "forward":
            o, lse, peak = _rel_forward(s)
            return {"out": o.to(T), "lse": lse, "peak": peak}
        dqkv, dtable = _rel_backward(s)
        return {"dqkv": dqkv.to(T), "dtable": dtable}
    if c["direction"] == "forward":
        y, n, stats = _norm_forward(s)
        return {"y": y.to(T), "n": n.to(T), "stats": stats}
    return _norm_backward(s)


def _run_own(s):
    from paper_2410_23608_b200 import binding as L
    c = s["case"]
    if c["op"] == "rel":
        if c["direction"] == "forward":
            L.spa_packed_attention_rel_fwd(s["p"], s["rel"], s["qkv"], s["cu"], c["B"], s["idx"], s["o_out"], s["o_lse"], s["o_peak"], s["ws"],
                                           d_status=s["status"])
            return {"out": s["o_out"], "lse": s["o_lse"], "peak": s["o_peak"]}
        L.spa_packed_attention_rel_bwd(s["p"], s["rel"], s["qkv"], s["out"], s["lse"], s["peak"], s["d_out"], s["cu"], c["B"], s["idx"],
                                       s["o_dqkv"], s["o_dtable"], s["ws"], d_status=s["status"])
        return {"dqkv": s["o_dqkv"], "dtable": s["o_dtable"]}
    if c["direction"] == "forward":
        L.spa_sandwich_norm(s["p"], s["sw"], s["x"], s["z"], s["row"], s["o_y"], s["o_n"], s["o_stats"])
        return {"y": s["o_y"], "n": s["o_n"], "stats": s["o_stats"]}
    grads = ("dx", "dz", "dgate", "dscale", "dg_post", "db_post", "dg_pre", "db_pre")
    L.spa_sandwich_norm_bwd(s["p"], s["sw"], s["dn"], s["dy"], s["y"], s["z"], s["row"], s["stats"], workspace=s["ws"],
                            **{k: s["o_" + k] for k in grads})
    return {k: s["o_" + k] for k in grads if s["o_" + k] is not None}


# ---------------------------------------------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    """The definition, in 64 bits, on the inputs of this seed."""
    s = prepare(case, seed)
    f = {k: v.double() if isinstance(v, torch.Tensor) and v.is_floating_point() else v for k, v in s.items()}
    return (_exact_rel if case["op"] == "rel" else _exact_norm)(case, f)


def _exact_rel(c, f):
    C, H, R, K = c["C"], c["H"], c["rows"], c["cols"]
    d, Np, dev = C // H, f["qkv"].shape[0], f["qkv"].device
    pos = f["idx"].long() % (R * K)
    bias = f["table"][f["bucket"].long()].view(2 * R - 1, 2 * K - 1, H)
    dt = torch.float64
    if c["direction"] == "forward":
        out, lse, peak = torch.empty(Np, C, dtype=dt, device=dev), torch.empty(H, Np, dtype=dt, device=dev), torch.empty(H, Np, dtype=dt, device=dev)
    else:
        dqkv = torch.empty(Np, 3 * C, dtype=dt, device=dev)
        bins = torch.zeros(H, (2 * R - 1) * (2 * K - 1), dtype=dt, device=dev)
    r0 = 0
    for n in f["lens"]:
        sl = slice(r0, r0 + n)
        y, x = pos[sl] // K, pos[sl] % K
        dy, dx = y[:, None] - y[None] + R - 1, x[:, None] - x[None] + K - 1
        qkv = f["qkv"][sl].view(n, 3, H, d).permute(1, 2, 0, 3)
        S = torch.einsum("hie,hje->hij", qkv[0], qkv[1]) / math.sqrt(d) + bias[dy, dx].permute(2, 0, 1)
        if c["direction"] == "forward":
            z = torch.logsumexp(S, 2)
            lse[:, sl], peak[:, sl] = z, S.amax(2) - z
            out[sl] = torch.einsum("hij,hje->ihe", torch.exp(S - z[:, :, None]), qkv[2]).reshape(n, C)
        else:
            do, o = (f[k][sl].view(n, H, d).transpose(0, 1) for k in ("d_out", "out"))
            P = torch.exp(S - f["lse"][:, sl, None])
            dS = P * (torch.einsum("hie,hje->hij", do, qkv[2]) - (do * o).sum(2)[:, :, None])
            g = torch.stack((torch.einsum("hij,hje->hie", dS, qkv[1]) / math.sqrt(d),
                             torch.einsum("hij,hie->hje", dS, qkv[0]) / math.sqrt(d), torch.einsum("hij,hie->hje", P, do)))
            dqkv[sl] = g.permute(2, 0, 1, 3).reshape(n, 3 * C)
            at = (dy * (2 * K - 1) + dx).reshape(-1)
            for h in range(H):
                bins[h] += torch.bincount(at, weights=dS[h].reshape(-1), minlength=bins.shape[1])
        r0 += n
    if c["direction"] == "forward":
        return {"out": out, "lse": lse, "peak": peak}
    nb = f["table"].shape[0]
    return {"dqkv": dqkv, "dtable": torch.stack([torch.bincount(f["bucket"].long(), weights=b, minlength=nb) for b in bins], 1)}


def _exact_norm(c, f):
    B, N, C, layer = c["B"], c["N"], c["C"], c["kind"] == "layer"
    dt, dev = torch.float64, f["z"].device
    has = torch.ones(B * N, dtype=torch.bool, device=dev) if f["row"] is None else f["row"] >= 0
    t = has.nonzero()[:, 0]                   # the token of every row of z
    z = f["z"] if f["row"] is None else f["z"][f["row"][t].long()]
    zero = torch.zeros(C, dtype=dt, device=dev)
    b_post, b_pre = (f["b_post"], f["b_pre"]) if layer else (zero, zero)
    if c["gate"] == "none":
        gate = torch.ones(t.numel(), 1, dtype=dt, device=dev)
    elif c["gate"] == "score":
        gate = torch.sigmoid(f["gate"])[t, None]
    else:
        gate = f["gate"][t // N] if c["gate"] == "image" else f["gate"][t]

    def stats(v):
        m = v.mean(1) if layer else torch.zeros(v.shape[0], dtype=dt, device=dev)
        return m, 1.0 / torch.sqrt((v - m[:, None]).square().mean(1) + EPS)

    if c["direction"] == "forward":
        m1, r1 = stats(z)
        y = f["x"].clone()
        y[t] += ((z - m1[:, None]) * r1[:, None] * f["g_post"] + b_post) * f["scale"] * gate
        m2, r2 = stats(y)
        full = torch.zeros(4, B * N, dtype=dt, device=dev)
        full[0, t], full[1, t], full[2], full[3] = m1, r1, m2, r2
        return {"y": y, "n": (y - m2[:, None]) * r2[:, None] * f["g_pre"] + b_pre, "stats": full}
    m1, r1, m2, r2 = f["stats"]

    def through(g, vh, r):
        out = g - vh * (g * vh).sum(1, keepdim=True) / C
        return (out - g.sum(1, keepdim=True) / C if layer else out) * r[:, None]

    yh = (f["y"] - m2[:, None]) * r2[:, None]
    dx = f["dy"] + through(f["dn"] * f["g_pre"], yh, r2)
    d, zh = dx[t], (z - m1[t, None]) * r1[t, None]
    a = zh * f["g_post"] + b_post
    da = d * gate * f["scale"]
    dz = torch.empty_like(f["z"])
    dz[t if f["row"] is None else f["row"][t].long()] = through(da * f["g_post"], zh, r1[t])
    out = {"dx": dx, "dz": dz, "dscale": (d * gate * a).sum(0), "dg_post": (da * zh).sum(0), "dg_pre": (f["dn"] * yh).sum(0)}
    if layer:
        out.update(db_post=da.sum(0), db_pre=f["dn"].sum(0))
    dg = d * f["scale"] * a
    if c["gate"] == "score":
        out["dgate"] = torch.zeros(B * N, dtype=dt, device=dev)
        out["dgate"][t] = dg.sum(1) * gate[:, 0] * (1 - gate[:, 0])
    elif c["gate"] == "image":
        out["dgate"] = torch.zeros(B, C, dtype=dt, device=dev).index_add_(0, t // N, dg)
    elif c["gate"] == "token":
        out["dgate"] = torch.zeros(B * N, C, dtype=dt, device=dev)
        out["dgate"][t] = dg
    return out
