"""token_logprobs_grad where a token is none of the columns: of such a row the entropy's part is left, in every form of
either layout, against the fp64 form (oracle/ops.py) within the bounds of test_gpu_logprobs.py."""
import numpy as np
import pytest

from workloads import preset

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import ops    # noqa: E402
from scan_check import TYPES, near, rounding   # noqa: E402
from test_gpu_logprobs import U, errors, inputs, np_of   # noqa: E402


@pytest.fixture(scope="module")
def sim():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2607_05272_amd as bs
    with bs.Sim(preset("C1"), n_envs=1) as s:
        yield s


def entropy_gradient(z, dent, mask, live):
    """The entropies' part of the gradient alone, and its bound (check of test_gpu_logprobs.py at dlogp = 0)."""
    r = ops.token_logprobs(z, None, mask, live)
    want = ops.token_logprobs_grad(z, None, None, dent, mask, live)
    tol = np.zeros(z.shape)
    for n, (ls, p) in enumerate(zip(r["ls"], r["p"])):
        if p is not None:
            eL, eP, eH = errors(z.shape[1], np.where(p > 0, z[n], -np.inf), ls, p)
            H = r["entropy"][n]
            l0 = np.where(p > 0, np.abs(ls), 0.0)
            tol[n] = abs(dent[n]) * p * ((l0 + H) * (eP + 6 * U) + np.where(p > 0, eL, 0.0) + eH)
    return want, tol


@pytest.mark.parametrize("cols", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,A", [(9, 5), (300, 12), (70, 24), (9, 40), (131, 96), (20, 190), (20, 300), (7, 500)])
def test_a_token_that_is_no_column_leaves_the_entropys_part(sim, N, A, dtype, cols):
    """-1 is none; -2, A and, of 64 bits, those whose lower half is -1, -2 or a column are out of range, and told."""
    d = inputs(N, A, TYPES[dtype], N + A, masked=True, padded=True)
    lay = lambda t: t.cuda().t().contiguous().t() if cols else t.cuda()   # noqa: E731
    l, mk, live = lay(d["l"]), lay(d["mask"]), d["live"].cuda()
    want, tol = entropy_gradient(d["l"].double().numpy(), d["dent"].numpy(), np_of(d["mask"]), np_of(d["live"]))
    tol = tol + rounding(want, d["l"].dtype)
    for tok, kind in ((-1, torch.int64), (-1, torch.int32), (-2, torch.int32), (-2, torch.int64), (A, torch.int32), (A, torch.int64),
                      ((1 << 32) - 1, torch.int64), ((1 << 32) - 2, torch.int64), ((1 << 32) + 1, torch.int64), (-(1 << 32), torch.int64)):
        t = torch.full((N,), tok, dtype=kind, device="cuda")
        g = sim.token_logprobs_grad(l, t, d["dlogp"].cuda(), d["dent"].cuda(), mk, live)
        if tok == -1:
            sim.sync()
        else:
            with pytest.raises(Exception, match="action out of range"):
                sim.sync()
        near(g.double().cpu().numpy(), want, tol, f"token {tok}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_samples_of_no_column(sim, dtype):
    """193 to 384 columns of so many samples that they are held: as without tokens, bit by bit."""
    N, A = 33000, 200
    g = torch.Generator(device="cuda").manual_seed(1)
    l = (torch.randn(A, N, generator=g, device="cuda") * 2).to(TYPES[dtype]).t()
    dent = torch.randn(N, generator=g, device="cuda")
    want = sim.token_logprobs_grad(l, None, dentropy=dent)
    sim.sync()
    for tok in (-2, A, (1 << 32) - 2):
        got = sim.token_logprobs_grad(l, torch.full((N,), tok, device="cuda"), torch.ones(N, device="cuda"), dent)
        with pytest.raises(Exception, match="action out of range"):
            sim.sync()
        assert torch.equal(got, want)
