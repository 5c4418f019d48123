"""token_logprobs and its gradient where a row's numbers are not finite, in every form of either layout: a NaN, an
infinite logit, an infinite or NaN factor make what they are part of infinite or NaN, forbidden columns keep a gradient
of 0, and other rows are as without them."""
import pytest

from workloads import preset

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from scan_check import TYPES   # noqa: E402

ROWS = [(8, 3), (8, 40), (9, 500), (7, 2100), (8, 5001), (7, 50257), (200, 40000)]
COLS = [(8, 5), (9, 20), (130, 90), (7, 190), (8, 300), (9, 1500)]


@pytest.fixture(scope="module")
def sim():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2607_05272_amd as bs
    with bs.Sim(preset("C1"), n_envs=1) as s:
        yield s


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,A,cols", [(*s, False) for s in ROWS] + [(*s, True) for s in COLS])
def test_forbidden_columns_get_no_gradient(sim, N, A, cols, dtype):
    g = torch.Generator(device="cuda").manual_seed(A)
    lay = lambda t: t.t().contiguous().t() if cols else t   # noqa: E731
    l = torch.randn(N, A, generator=g, device="cuda").to(TYPES[dtype])
    mask = torch.rand(N, A, generator=g, device="cuda") > 0.4
    mask[:, 1] = True
    l[:, 2] = -float("inf")                     # forbidden by its logit
    tok = torch.ones(N, dtype=torch.int64, device="cuda")
    dl, dh = torch.randn(N, generator=g, device="cuda"), torch.randn(N, generator=g, device="cuda")
    clean = sim.token_logprobs(lay(l), tok, lay(mask))
    cg = sim.token_logprobs_grad(lay(l), tok, dl, dh, lay(mask))
    bad = l.clone()
    bad[1, 1], bad[2, 1] = float("nan"), float("inf")
    mask[3, 0] = False
    bad[3, 0] = float("nan")                    # a forbidden one: nothing
    cg3 = sim.token_logprobs_grad(lay(l), tok, dl, dh, lay(mask))[3]
    dl[4], dl[5], dh[6] = float("inf"), float("nan"), float("nan")
    r = sim.token_logprobs(lay(bad), tok, lay(mask))
    got = sim.token_logprobs_grad(lay(bad), tok, dl, dh, lay(mask))
    same = lay(bad).clone() if not cols else lay(bad.clone())
    sim.token_logprobs_grad(same, tok, dl, dh, lay(mask), grad=same)
    sim.sync()
    closed = ~mask | (l == -float("inf"))
    assert not got[closed].any() and not same[closed].any()
    assert not got[[1, 2, 4, 5, 6], 1].isfinite().any()
    for n in (1, 2):
        open_ = ~closed[n]
        assert not got[n][open_].isfinite().any()
        assert not r["logp"][n].isfinite() and r["entropy"][n].isnan()
    assert torch.equal(got[3], cg3)
    rest = [n for n in range(N) if n not in (1, 2, 3, 4, 5, 6)]
    assert torch.equal(got[rest], cg[rest]) and got[rest].isfinite().all()
    keep = [n for n in range(N) if n not in (1, 2, 3)]
    for k in ("logp", "entropy"):
        assert torch.equal(r[k][keep], clean[k][keep])
    assert torch.equal(got.isnan(), same.isnan())
    assert torch.equal(got.nan_to_num(), same.nan_to_num())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,A,cols", [(5, 50, False), (5, 900, False), (5, 2100, False), (3, 50257, False), (700, 5001, False),
                                      (5, 96, True), (5, 900, True), (5, 1500, True)])
def test_alternatives_of_what_is_not_finite(sim, N, A, cols, dtype):
    """NaN first, then +inf, then the finite ones, of equal ones the lowest column, however they are spread over a row;
    their log-probabilities are not finite, those of other rows what they are without."""
    top = 12
    g = torch.Generator(device="cuda").manual_seed(A)
    l = torch.randn(N, A, generator=g, device="cuda").to(TYPES[dtype])
    lay = lambda t: t.t().contiguous().t() if cols else t   # noqa: E731
    clean = sim.token_logprobs(lay(l), top=top)
    bad = l.clone()
    spread = torch.randperm(A, generator=g, device="cuda")[: top + 8]      # more NaNs than alternatives
    bad[0, spread] = float("nan")
    few = torch.randperm(A, generator=g, device="cuda")[:9]
    bad[1, few[:3]], bad[1, few[3:6]], bad[1, few[6:]] = float("nan"), float("inf"), -float("inf")
    bad[2, :] = -float("inf")
    bad[2, few[:2]] = float("inf")
    bad[2, few[2]] = 1.0
    r = sim.token_logprobs(lay(bad), top=top)
    sim.sync()
    assert torch.equal(r["top_index"][0], spread.sort().values[:top])
    assert r["top_logp"][0].isnan().all()
    want = torch.cat([few[:3].sort().values, few[3:6].sort().values])
    assert torch.equal(r["top_index"][1][:6], want)
    rest = l[1].float().clone()
    rest[few] = -float("inf")
    key = rest.double() * A - torch.arange(A, device="cuda") * 1e-9          # the lowest column of equal ones
    assert torch.equal(r["top_index"][1][6:], key.topk(top - 6).indices)
    assert r["top_logp"][1].isnan().all() and r["entropy"][1].isnan()
    assert torch.equal(r["top_index"][2][:3], torch.cat([few[:2].sort().values, few[2:3]]))
    assert (r["top_index"][2][3:] == -1).all() and (r["top_logp"][2][3:] == -float("inf")).all()
    assert not r["top_logp"][2][:3].isfinite().any()
    for k in ("top_index", "top_logp", "entropy"):
        assert torch.equal(r[k][3:], clean[k][3:])
