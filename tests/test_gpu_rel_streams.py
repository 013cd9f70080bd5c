"""The attention with a bias by relative position on a stream beside the default one: every element as on the default stream, and the rows behind
the last one as they were."""
import pytest
import torch

from tests.test_gpu_rel_attention import KINDS, Run, problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d,flags", KINDS)
@pytest.mark.parametrize("grid,counts,nb", [((14, 14), [(61 * i) % 180 + 10 for i in range(12)], 9), ((7, 7), [49, 30, 0, 17] * 6, None),
                                            ((33, 40), [700, 0, 320], None), ((24, 24), [576] * 9, 40)])
def test_on_another_stream(dtype, d, flags, grid, counts, nb):
    run = Run(problem(dtype, d, 4, *grid, counts, nb=nb, seed=2), flags)
    run.fwd(); run.bwd()
    torch.cuda.synchronize()
    first = {k: getattr(run, k).clone() for k in ("out", "lse", "peak", "dqkv", "dtable")}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for k in first:
            getattr(run, k).fill_(3.0)
        run.ws.fill_(0x55)
        run.fwd(); run.bwd()
    torch.cuda.synchronize()
    assert run.status.item() == 0
    for k, want in first.items():
        got = getattr(run, k)
        a, b = (got[:, :run.Np], want[:, :run.Np]) if k in ("lse", "peak") else (got[:run.Np], want[:run.Np]) if k != "dtable" else (got, want)
        assert torch.equal(a, b), k
        if k != "dtable":
            assert bool((got[:, run.Np:] if k in ("lse", "peak") else got[run.Np:]).eq(3.0).all()), k
