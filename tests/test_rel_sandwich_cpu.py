"""The oracle of the relative position bias and of the norms around a block, pinned by independent computations and by central
differences, and the refusals of the library's calls, which need no GPU."""
import ctypes

import numpy as np
import pytest

from oracle import rel_sandwich as R
from oracle import spa_oracle as O


@pytest.fixture(scope="module")
def lib():
    from paper_2410_23608_b200 import binding, build
    build.build()
    return binding


def rel_problem(seed=0, rows=3, cols=5, counts=(4, 0, 1, 9), H=2, d=4, nb=None):
    rng = np.random.default_rng(seed)
    N, C = rows * cols, H * d
    cu = np.concatenate(([0], np.cumsum(counts)))
    idx = np.concatenate([b * N + np.sort(rng.choice(N, n, replace=False)) for b, n in enumerate(counts)]).astype(np.int64)
    E = (2 * rows - 1) * (2 * cols - 1)
    bucket = np.arange(E) if nb is None else rng.integers(0, nb, E)
    table = rng.normal(size=(E if nb is None else nb, H))
    return dict(qkv=rng.normal(size=(cu[-1], 3 * C)), cu=cu, idx=idx, rows=rows, cols=cols, bucket=bucket, table=table, H=H)


def test_offsets_by_explicit_loops():
    rows, cols, idx = 3, 5, np.array([0, 4, 7, 14]) + 2 * 15
    off = R.offsets(idx, rows, cols)
    for a, i in enumerate(idx % 15):
        for b, j in enumerate(idx % 15):
            dy, dx = i // cols - j // cols, i % cols - j % cols
            assert off[a, b] == (dy + rows - 1) * (2 * cols - 1) + dx + cols - 1
    assert off.min() >= 0 and off.max() < 5 * 9


def test_zero_table_is_plain_attention():
    p = rel_problem()
    p["table"] = np.zeros_like(p["table"])
    f = R.rel_fwd(**p)
    ao, lse = O.attention_fwd(p["qkv"], p["cu"], p["H"])[:2]
    assert np.abs(f["out"] - ao).max() < 1e-13 and np.abs(f["lse"] - lse).max() < 1e-13


def test_masking_buckets_leave_the_other_keys_and_empty_rows():
    p = rel_problem()
    diag = R.offsets(p["idx"][:1], p["rows"], p["cols"])[0, 0]
    p["table"][:] = -np.inf
    p["table"][diag] = 0.3          # only the token itself: its own value comes back
    f = R.rel_fwd(**p)
    C = p["qkv"].shape[1] // 3
    assert np.allclose(f["out"], p["qkv"][:, 2 * C:]) and np.all(f["peak"] == 0)
    p["table"][:] = -np.inf
    f = R.rel_fwd(**p)
    assert np.all(f["out"] == 0) and np.all(f["lse"] == -np.inf)
    b = R.rel_bwd(p["qkv"], f["out"], f["lse"], np.ones_like(f["out"]), p["cu"], p["idx"], p["rows"], p["cols"], p["bucket"], p["table"], p["H"])
    assert np.all(b["dqkv"] == 0) and np.all(b["dtable"] == 0)


@pytest.mark.parametrize("nb", [None, 4])
def test_rel_gradients_against_differences(nb):
    p = rel_problem(seed=3, nb=nb)
    rng = np.random.default_rng(1)
    G = rng.normal(size=(p["cu"][-1], p["qkv"].shape[1] // 3))
    f = R.rel_fwd(**p)
    b = R.rel_bwd(p["qkv"], f["out"], f["lse"], G, p["cu"], p["idx"], p["rows"], p["cols"], p["bucket"], p["table"], p["H"])
    for name, grad in (("qkv", b["dqkv"]), ("table", b["dtable"])):
        for at in [tuple(rng.integers(0, s) for s in p[name].shape) for _ in range(12)]:
            v = []
            for h in (1e-6, -1e-6):
                q = dict(p, **{name: p[name].copy()})
                q[name][at] += h
                v.append((R.rel_fwd(**q)["out"] * G).sum())
            assert abs((v[0] - v[1]) / 2e-6 - grad[at]) < 1e-7 * max(1.0, abs(grad[at]))


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("gate_kind", ["none", "score", "image", "token"])
def test_sandwich_gradients_against_differences(kind, gate_kind):
    rng = np.random.default_rng(5)
    B, N, C, eps = 2, 3, 6, 1e-3
    row = np.array([0, -1, 2, 1, -1, 3])
    v = dict(x=rng.normal(size=(B * N, C)), z=rng.normal(size=(4, C)), scale=rng.normal(size=C), g_post=rng.normal(size=C),
             b_post=rng.normal(size=C), g_pre=rng.normal(size=C), b_pre=rng.normal(size=C),
             gate={"none": None, "score": rng.normal(size=B * N), "image": rng.normal(size=(B, C)), "token": rng.normal(size=(B * N, C))}[gate_kind])
    dn, dy = rng.normal(size=(B * N, C)), rng.normal(size=(B * N, C))

    def value(v):
        f = R.sandwich_fwd(v["x"], v["z"], row, v["gate"], gate_kind, v["scale"], v["g_post"], v["b_post"], v["g_pre"], v["b_pre"], kind, eps, B, N)
        return f, (f["n"] * dn).sum() + (f["y"] * dy).sum()

    f, _ = value(v)
    g = R.sandwich_bwd(dn, dy, f["y"], v["z"], row, f["stats"], v["gate"], gate_kind, v["scale"], v["g_post"], v["b_post"], v["g_pre"], kind, B, N)
    for name, grad in (("x", "dx"), ("z", "dz"), ("scale", "dscale"), ("g_post", "dg_post"), ("b_post", "db_post"), ("g_pre", "dg_pre"),
                       ("b_pre", "db_pre"), ("gate", "dgate")):
        if v[name] is None:
            continue
        for at in np.ndindex(v[name].shape):
            d = []
            for h in (1e-6, -1e-6):
                w = dict(v, **{name: v[name].copy()})
                w[name][at] += h
                d.append(value(w)[1])
            assert abs((d[0] - d[1]) / 2e-6 - g[grad][at]) < 1e-6 * max(1.0, abs(g[grad][at])), (name, at)
    assert np.array_equal(f["y"][row < 0], v["x"][row < 0])


def test_layer_norm_of_the_oracles_agree():
    rng = np.random.default_rng(2)
    x, g, b = rng.normal(size=(5, 8)), rng.normal(size=8), rng.normal(size=8)
    f = R.sandwich_fwd(x, np.zeros((1, 8)), np.full(5, -1), None, "none", g, g, b, g, b, "layer", 1e-5, 1, 5)
    assert np.abs(f["n"] - O.layer_norm(x[None], g, b)[0][0]).max() < 1e-13 and np.array_equal(f["y"], x)


# ------------------------------------------------------------------------------------ refusals
PTR = ctypes.c_void_p(4096)      # looked at on the host only for being there and aligned: every call below is refused
ODD = ctypes.c_void_p(4100)


def _rel(lib, rows=3, cols=5, nb=7, bucket=4096, table=4096):
    return lib.SpaRelBias(rows, cols, nb, bucket, table)


def _rel_call(lib, p, r, back, **kw):
    a = dict(qkv=PTR, out=PTR, lse=PTR, peak=PTR, d_out=PTR, seg=PTR, idx=PTR, dqkv=PTR, dtable=PTR, ws=PTR, n_seg=2)
    a.update(kw)
    pr = None if p is None else ctypes.byref(p)
    rr = None if r is None else ctypes.byref(r)
    if back:
        return lib.lib().spa_packed_attention_rel_bwd(pr, rr, a["qkv"], a["out"], a["lse"], a["peak"], a["d_out"], a["seg"], a["n_seg"], a["idx"],
                                                      a["dqkv"], a["dtable"], a["ws"], None, None)
    return lib.lib().spa_packed_attention_rel_fwd(pr, rr, a["qkv"], a["seg"], a["n_seg"], a["idx"], a["out"], a["lse"], a["peak"], a["ws"], None, None)


@pytest.mark.parametrize("back", [False, True])
def test_rel_calls_refuse(lib, back):
    p = lib.make_params(2, 15, 64, 2, "bf16")
    for bad in ("qkv", "out", "lse", "seg", "idx", "ws") + (("d_out", "dqkv", "dtable") if back else ("peak",)):
        for v in (None, ODD):
            assert _rel_call(lib, p, _rel(lib), back, **{bad: v}) == lib.SPA_ERR_INVALID_ARG, bad
    assert _rel_call(lib, p, _rel(lib), back, n_seg=-1) == lib.SPA_ERR_INVALID_ARG
    assert _rel_call(lib, None, _rel(lib), back) == lib.SPA_ERR_INVALID_ARG
    assert _rel_call(lib, p, None, back) == lib.SPA_ERR_INVALID_ARG
    for kw in (dict(rows=5), dict(rows=0), dict(rows=-3, cols=-5), dict(nb=0), dict(nb=-1), dict(bucket=None), dict(table=None), dict(table=4100)):
        assert _rel_call(lib, p, _rel(lib, **kw), back) == lib.SPA_ERR_INVALID_ARG, kw
    assert _rel_call(lib, p, _rel(lib, nb=1 << 26), back) == lib.SPA_ERR_UNSUPPORTED
    assert _rel_call(lib, lib.make_params(2, 15, 48, 2, "bf16"), _rel(lib), back) == lib.SPA_ERR_UNSUPPORTED      # heads of 24
    assert lib.spa_rel_workspace_bytes(p, _rel(lib, rows=5)) == 0 and lib.spa_rel_workspace_bytes(p, _rel(lib)) > 0


def _sandwich(lib, kind=0, gate_kind=0, eps=1e-5, gate=None, **kw):
    s = lib.SpaSandwich(kind, gate_kind, eps, gate)
    for k, v in kw.items():
        setattr(s, k, v)
    return s


def test_sandwich_calls_refuse(lib):
    L = lib.lib()
    p = lib.make_params(2, 15, 64, 1, "bf16")

    def fwd(s, p=p, x=PTR, z=PTR, row=None, y=PTR, n=PTR, stats=PTR):
        return L.spa_sandwich_norm(ctypes.byref(p), None if s is None else ctypes.byref(s), x, z, row, y, n, stats, None)

    def bwd(s, dn=PTR, dy=PTR, y=PTR, z=PTR, row=None, stats=PTR, dx=PTR, dz=PTR, dgate=None, dscale=None, ws=PTR):
        return L.spa_sandwich_norm_bwd(ctypes.byref(p), ctypes.byref(s), dn, dy, y, z, row, stats, dx, dz, dgate, dscale, None, None, None, None,
                                       ws, None)

    ok, bad = _sandwich(lib), lib.SPA_ERR_INVALID_ARG
    assert fwd(None) == bad
    for kw in (dict(x=None), dict(z=None), dict(y=None), dict(x=ODD), dict(row=ODD), dict(n=ODD), dict(stats=ODD)):
        assert fwd(ok, **kw) == bad, kw
    for kw in (dict(dn=None, dy=None), dict(y=None), dict(z=None), dict(stats=None), dict(dx=None), dict(dz=None), dict(ws=None), dict(dgate=PTR),
               dict(dscale=ODD)):
        assert bwd(ok, **kw) == bad, kw
    nan = float("nan")
    for s in (_sandwich(lib, kind=2), _sandwich(lib, kind=-1), _sandwich(lib, gate_kind=4), _sandwich(lib, gate_kind=1), _sandwich(lib, eps=-1.0),
              _sandwich(lib, eps=nan), _sandwich(lib, gate_kind=3, gate=4100), _sandwich(lib, scale=4100), _sandwich(lib, b_pre=4100)):
        assert fwd(s) == bad and bwd(s) == bad
    wide = lib.make_params(2, 15, 8192, 1, "f32")
    assert fwd(ok, p=wide) == lib.SPA_ERR_UNSUPPORTED and lib.spa_sandwich_workspace_bytes(wide, ok) == 0
    assert lib.spa_sandwich_workspace_bytes(lib.make_params(2, 15, 8192, 1, "bf16"), ok) > 0


def test_empty_batches_have_workspaces(lib):
    p = lib.make_params(0, 15, 64, 2, "bf16", capacity=1)
    for gate_kind in range(4):
        assert lib.spa_sandwich_workspace_bytes(p, _sandwich(lib, gate_kind=gate_kind, gate=4096)) > 0
    assert lib.spa_rel_workspace_bytes(p, _rel(lib)) > 0


def test_python_side_refusals(lib):
    import torch
    cpu = torch.zeros(45, dtype=torch.int32)
    with pytest.raises(ValueError):
        lib.rel_bias(3, 5, cpu, torch.zeros(4, 2))           # host tensors
    with pytest.raises(ValueError):
        lib.rel_bias(3, 4, cpu, torch.zeros(4, 2))           # a bucket for every offset
    with pytest.raises(ValueError):
        lib.rel_bias(3, 5, cpu.long(), torch.zeros(4, 2))
    with pytest.raises(ValueError):
        lib.sandwich("layer", "score", gate=torch.zeros(4, dtype=torch.bfloat16))  # scores are fp32
    with pytest.raises(ValueError):
        lib.sandwich("layer", "score")
    with pytest.raises(ValueError):
        lib.sandwich("rms", "image", gate=torch.zeros(4, 8))  # a host tensor


def test_struct_layouts(lib):
    assert ctypes.sizeof(lib.SpaRelBias) == 32 and ctypes.sizeof(lib.SpaSandwich) == 64
