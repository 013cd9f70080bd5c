"""What the binding refuses before an address reaches the library: tensors of another type or size than the problem's.  The library sees
addresses only; it would read such a tensor as what it is not, or past its end.  No GPU: the calls are refused before it matters."""
import pytest
import torch


@pytest.fixture
def lib(monkeypatch):
    from paper_2410_23608_b200 import binding, build
    build.build()
    monkeypatch.setattr(binding, "_ptr", lambda t: None if t is None else t.data_ptr())   # host tensors stand in for the device's
    monkeypatch.setattr(binding, "_stream", lambda stream: None)
    return binding


def _rel_calls(lib, p, rel):
    t, i = torch.zeros(64 * 192), torch.zeros(64, dtype=torch.int32)
    return (lambda: lib.spa_packed_attention_rel_fwd(p, rel, t, i, -1, i, t, t, t, t),
            lambda: lib.spa_packed_attention_rel_bwd(p, rel, t, t, t, t, t, i, -1, i, t, t, t))


@pytest.mark.parametrize("problem", ["f32", "bf16"])
@pytest.mark.parametrize("table,H", [(torch.float32, 2), (torch.bfloat16, 2), (torch.float32, 1), (torch.bfloat16, 3)])
def test_table_of_another_type_or_width(lib, problem, table, H):
    p = lib.make_params(2, 15, 64, 2, problem)
    rel = lib.rel_bias(3, 5, torch.zeros(45, dtype=torch.int32), torch.zeros(7, H, dtype=table))
    right = H == 2 and (table == torch.float32) == (problem == "f32")
    for call in _rel_calls(lib, p, rel):
        # n_seg = -1: what passes the binding is refused by the library, and launches nothing
        with pytest.raises(lib.SpaError if right else ValueError):
            call()


@pytest.mark.parametrize("dtype", [torch.float16, torch.float64, torch.int32])
def test_table_of_no_type_of_the_library(lib, dtype):
    with pytest.raises(ValueError):
        lib.rel_bias(3, 5, torch.zeros(45, dtype=torch.int32), torch.zeros(7, 2, dtype=dtype))


def _sandwich_calls(lib, p, s):
    t = torch.zeros(4096)
    return (lambda: lib.spa_sandwich_norm(p, s, None, t, None, t, t, t),                    # x = None: refused by the library, if not before
            lambda: lib.spa_sandwich_norm_bwd(p, s, t, t, None, t, None, t, t, t, workspace=t))


NAMES = ("scale", "g_post", "b_post", "g_pre", "b_pre")


@pytest.mark.parametrize("problem", ["f32", "bf16"])
@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("dtype,size", [(torch.float32, 64), (torch.bfloat16, 64), (torch.float32, 56), (torch.bfloat16, 72)])
def test_parameters_of_another_type_or_size(lib, problem, name, dtype, size):
    p = lib.make_params(2, 15, 64, 1, problem)
    s = lib.sandwich("layer", "none", **{name: torch.zeros(size, dtype=dtype)})
    right = size == 64 and (dtype == torch.float32) == (problem == "f32")
    for call in _sandwich_calls(lib, p, s):
        with pytest.raises(lib.SpaError if right else ValueError):
            call()


@pytest.mark.parametrize("problem", ["f32", "bf16"])
@pytest.mark.parametrize("kind,right", [("score", 30), ("image", 128), ("token", 1920)])
@pytest.mark.parametrize("size", [24, 32, 120, 128, 1912, 1920])   # a buffer for larger batches may be given
def test_gates_of_another_type_or_size(lib, problem, kind, right, size):
    p = lib.make_params(2, 15, 64, 1, problem)
    for dtype in (torch.float32, torch.bfloat16):
        if kind == "score" and dtype == torch.bfloat16:
            continue                                        # refused when it is made
        s = lib.sandwich("rms", kind, gate=torch.zeros(size, dtype=dtype))
        ok = size >= right and (kind == "score" or (dtype == torch.float32) == (problem == "f32"))
        for call in _sandwich_calls(lib, p, s):
            with pytest.raises(lib.SpaError if ok else ValueError):
                call()


def test_a_second_problem_is_looked_at_as_the_first(lib):
    s = lib.sandwich("rms", "image", gate=torch.zeros(4, 64), scale=torch.zeros(64))
    fit, wide, many = (lib.make_params(*a, 1, "f32") for a in ((4, 5, 64), (2, 5, 128), (5, 5, 64)))
    for p, right in ((fit, True), (fit, True), (wide, False), (many, False), (fit, True), (lib.make_params(4, 5, 64, 1, "bf16"), False)):
        for call in _sandwich_calls(lib, p, s):
            with pytest.raises(lib.SpaError if right else ValueError):
                call()


def test_parameters_that_differ_among_themselves(lib):
    f, b = torch.zeros(64), torch.zeros(64, dtype=torch.bfloat16)
    for kw in (dict(scale=f, g_pre=b), dict(scale=f, g_pre=f[:32]), dict(scale=b, gate=f, gate_kind="image"), dict(b_pre=f.half()),
               dict(gate=f.half(), gate_kind="token")):
        with pytest.raises(ValueError):
            lib.sandwich("layer", **kw)
    lib.sandwich("layer", "score", gate=f, scale=b)          # scores are fp32 beside parameters of any type
