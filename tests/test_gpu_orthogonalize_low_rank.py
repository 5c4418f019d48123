"""orthogonalize of updates of low rank in 16 bits against the fp64 form (oracle/ops.py): the steps multiply what is
rounded off an update, outside of its few directions, by up to 3.4445^5. Bound: that of test_gpu_orthogonalize.py with
values held in two parts, and half a step of the result's type."""
import numpy as np
import pytest

from workloads import preset

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import ops    # noqa: E402
from scan_check import TYPES, rounding   # noqa: E402
from test_gpu_orthogonalize import NS, bound, fro   # noqa: E402


@pytest.fixture(scope="module")
def sim():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2607_05272_amd as bs
    with bs.Sim(preset("C1"), n_envs=1) as s:
        yield s


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("M,N,rank", [(96, 200, 1), (200, 96, 4), (130, 257, 1), (64, 64, 2)])
def test_low_rank(sim, M, N, rank, dtype):
    g = torch.Generator().manual_seed(M + rank)
    u = (torch.randn(M, rank, generator=g) @ torch.randn(rank, N, generator=g)).to(TYPES[dtype])
    got = sim.orthogonalize(u.cuda())
    sim.sync()
    want, way = ops.orthogonalize(u.double().numpy())
    e = bound(way, NS, True) + fro(rounding(want, u.dtype))
    assert e <= 0.06 * fro(want)   # 3 to 4% in bf16, whose rounding adds directions, 5% of a norm of 0.7 without them
    off = got.double().cpu().numpy() - want
    assert fro(off) <= e, (fro(off), e, fro(want))
    # and none of it is left outside of the rounding's reach: the rows' and the columns' errors
    for axis in (0, 1):
        assert (np.sqrt((off * off).sum(axis)) <= e).all()
