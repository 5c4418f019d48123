"""orthogonalize's three products, in every form (ortho_shapes.py), one step and one coefficient at a time, element by
element against torch in fp64 on the GPU.

With X = U / |U| and A = X X^T, one step gives a X, b A X and c A A X for one coefficient that is not 0. Bounds of an
element, from the magnitudes of its terms (u = 2^-24): a value held in two parts is off by 2^-22 of itself and 2^-35, X by
2 u more; a sum of K products takes three products of parts each, so at most (3 K + 4) u of the sum of their magnitudes
and 2^-22 of it for the product of parts that is left out; what its factors are off by goes through the product of
magnitudes. The results' rounding adds half a step of their type. The updates are one strong direction and noise,
so that an element of A A X or A X is a sum of about r terms of one sign: 64 columns of A, a tile, are 64 / r of it, and the
test asks that the bound is less than half of that."""
import pytest

from workloads import preset

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from ortho_shapes import FORMS   # noqa: E402
from scan_check import TYPES   # noqa: E402

U, HELD, TINY = 2.0 ** -24, 2.0 ** -22, 2.0 ** -35


@pytest.fixture(scope="module")
def sim():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2607_05272_amd as bs
    with bs.Sim(preset("C1"), n_envs=1) as s:
        yield s


def product(p, ep, q, eq):
    """p q and its bound, of factors off by ep and eq."""
    K = p.shape[1]
    lost = (3 * K + 4) * U + HELD
    return p @ q, lost * (p.abs() @ q.abs()) + ep @ q.abs() + p.abs() @ eq


def held(x, e):
    return e + HELD * (x.abs() + e) + TINY


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,M,N", sorted(FORMS))
def test_each_product(sim, n, M, N, dtype):
    g = torch.Generator(device="cuda").manual_seed(M)
    u = torch.randn(n, M, 1, generator=g, device="cuda") * torch.randn(n, 1, N, generator=g, device="cuda")
    u = (u + 0.1 * torch.randn(n, M, N, generator=g, device="cuda")).to(TYPES[dtype])
    got = [sim.orthogonalize(u, steps=1, coeffs=c, eps=0.0) for c in ((1.0, 0.0, 0.0), (0.0, 1.0, 0.0), (0.0, 0.0, 1.0))]
    sim.sync()
    for i in {0, n // 2, n - 1}:
        x = u[i].double()
        x = (x.t() if M > N else x).contiguous()
        r = x.shape[0]
        x = x / x.square().sum().sqrt()
        ex = held(x, 2 * U * x.abs())
        A, eA = product(x, ex, x.t().contiguous(), ex.t().contiguous())
        eA = held(A, eA)
        AA, eAA = product(A, eA, A, eA)
        eA2, eAA = held(A, eA + 2 * U * A.abs()), held(AA, eAA + U * AA.abs())
        for k, (w, e) in enumerate(((x, ex + 2 * U * x.abs()), product(A, eA2, x, ex), product(AA, eAA, x, ex))):
            assert k == 0 or r <= 64 or e.norm() <= 32 / r * w.norm()
            y = (got[k][i].t() if M > N else got[k][i]).double()
            f = torch.finfo(u.dtype)
            tol = e + 2 * U * w.abs() + f.eps / 2 * (w.abs() + e) + f.smallest_normal * f.eps
            off = ~((y - w).abs() <= tol)
            assert not off.any(), (k, int(off.sum()), off.nonzero()[0].tolist(), float((y - w).abs().max()))
