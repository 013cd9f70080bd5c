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
