"""token_logprobs and its gradient against the fp64 form (oracle/ops.py): sizes, both layouts, types, masks, padding,
ties, infinities, refusals and graphs. Bounds: softmax_errors of loss_check.py; a log-probability is off by its
eL and its own rounding, an entropy by eH, and the gradient -p (g + h (log p + H)) by the usual rules (as
loss_check.check_policy has them), plus half a step of its type."""
import numpy as np
import pytest

from workloads import preset

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import loss_check as lc   # noqa: E402
from oracle import ops    # noqa: E402
from scan_check import TYPES, near, rounding   # noqa: E402

U = lc.U


@pytest.fixture(scope="module")
def sim():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2607_05272_amd as bs
    with bs.Sim(preset("C1"), n_envs=1) as s:
        yield s


def errors(A, z, ls, p):
    """eL of every log p_j, eP of p, eH of the entropy, of one row."""
    x = np.where(p > 0, z - z.max(), 0.0)
    l0 = np.where(p > 0, ls, 0.0)
    logS = -ls.max()
    eS, eP = lc.softmax_errors(A, x, p, logS)
    eL = eS + U * (np.abs(x) + np.abs(l0) + 3 * abs(logS) + 1)
    mx, mxx = (p * np.abs(x)).sum(), (p * x * x).sum()
    eH = eS * (1 + 2 * mx) + U * (3 * mxx + (16 + A / 64 + min(A, 96)) * mx + 4 * abs(logS) + 4)
    return eL, eP, eH


def inputs(N, A, dtype, seed, masked=False, padded=False, ties=False):
    g = torch.Generator().manual_seed(seed)
    l = torch.randn(N, A, generator=g) * 2
    if ties:
        l = (l * 2).round() / 2
    tok = torch.randint(0, A, (N,), generator=g)
    mask = live = None
    if masked:
        mask = torch.rand(N, A, generator=g) > 0.4
        if N > 2:
            mask[1] = False                      # nothing is open
            mask[2] = False
            mask[2, A // 2] = True               # one column is
    if padded:
        live = torch.rand(N, generator=g) > 0.3
    return dict(l=l.to(dtype), tok=tok, mask=mask, live=live, dlogp=torch.randn(N, generator=g),
                dent=torch.randn(N, generator=g) * 0.3)


def np_of(t):
    return None if t is None else t.numpy()


def check(sim, d, top=0, cols=False, mask_cols=None, grad=True):
    l, N, A = d["l"], *d["l"].shape
    z = l.double().numpy()
    lay = (lambda t, c: t.cuda().t().contiguous().t() if c else t.cuda())
    dl, mk = lay(l, cols), None if d["mask"] is None else lay(d["mask"], cols if mask_cols is None else mask_cols)
    tok, live = d["tok"].cuda(), None if d["live"] is None else d["live"].cuda()
    r = sim.token_logprobs(dl, tok, mk, live, top)
    g = sim.token_logprobs_grad(dl, tok, d["dlogp"].cuda(), d["dent"].cuda(), mk, live) if grad else None
    sim.sync()
    want = ops.token_logprobs(z, d["tok"].numpy(), np_of(d["mask"]), np_of(d["live"]), top)
    wg = ops.token_logprobs_grad(z, d["tok"].numpy(), d["dlogp"].numpy(), d["dent"].numpy(), np_of(d["mask"]), np_of(d["live"]))
    tl, te, tt, tg = np.zeros(N), np.zeros(N), np.zeros((N, top)), np.zeros((N, A))
    for n in range(N):
        ls, p = want["ls"][n], want["p"][n]
        if p is None:
            continue
        zz = np.where(p > 0, z[n], -np.inf)
        eL, eP, eH = errors(A, zz, ls, p)
        a = int(d["tok"][n])
        if 0 <= a < A and ls[a] > -np.inf:
            tl[n] = eL[a] + U * abs(ls[a])
        te[n] = eH
        for i, j in enumerate(want["top_index"][n]):
            if j >= 0:
                tt[n, i] = eL[j] + U * abs(ls[j])
        gl, h, hot = abs(float(d["dlogp"][n])), abs(float(d["dent"][n])), np.zeros(A)
        if 0 <= a < A:
            hot[a] = 1.0
        l0 = np.where(p > 0, np.abs(ls), 0.0)
        H = want["entropy"][n]
        tg[n] = gl * (p * eP + 3 * U * (hot + p)) + h * p * ((l0 + H) * (eP + 6 * U) + eL + eH)
    inf = np.isinf(want["logp"])
    got = r["logp"].double().cpu().numpy()
    assert np.array_equal(got[inf], want["logp"][inf])
    near(np.where(inf, 0, got), np.where(inf, 0, want["logp"]), tl, "logp")
    near(r["entropy"].double().cpu().numpy(), want["entropy"], te, "entropy")
    if top:
        assert np.array_equal(r["top_index"].cpu().numpy(), want["top_index"])
        got, none = r["top_logp"].double().cpu().numpy(), want["top_index"] < 0
        assert (got[none] == -np.inf).all()
        near(np.where(none, 0, got), np.where(none, 0, want["top_logp"]), tt, "top_logp")
    if grad:
        near(g.double().cpu().numpy(), wg, tg + rounding(wg, l.dtype), "grad")
    return r, g


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("N,A,top", [(1, 1, 1), (7, 6, 6), (33, 24, 5), (20, 96, 20), (5, 130, 64), (9, 515, 7), (6, 2100, 20),
                                     (3, 5001, 64), (2, 50257, 20)])
def test_rows(sim, N, A, top, dtype):
    check(sim, inputs(N, A, TYPES[dtype], N + A), top)
    check(sim, inputs(N, A, TYPES[dtype], N + A, masked=True, padded=True, ties=True), top)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,A,top", [(1, 6, 3), (64, 1, 1), (70, 6, 6), (130, 48, 5), (300, 96, 8), (65, 200, 64), (5, 700, 9)])
def test_columns(sim, N, A, top, dtype):
    """[A][N] logits, as sim.policy writes them, masks in either layout."""
    check(sim, inputs(N, A, TYPES[dtype], N + A, ties=True), top, cols=True)
    d = inputs(N, A, TYPES[dtype], N + A, masked=True, padded=True)
    check(sim, d, top, cols=True)
    check(sim, d, top, cols=True, mask_cols=False)
    check(sim, d, top, cols=False, mask_cols=True)


@pytest.mark.parametrize("N,A", [(1, 131072), (3, 70001), (2, 200001)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_long_rows(sim, N, A, dtype):
    check(sim, inputs(N, A, TYPES[dtype], A), 20)
    check(sim, inputs(N, A, TYPES[dtype], A, masked=True, padded=False), 3)


@pytest.mark.parametrize("cols", [False, True])
@pytest.mark.parametrize("A", [5, 64, 100, 384, 3001, 9000])
def test_alternatives_of_equal_and_ordered_rows(sim, A, cols):
    """All equal (the lowest columns), rising, falling, zeros of either sign, fewer than asked for."""
    l = torch.stack([torch.zeros(A), torch.arange(A).float() / A, -torch.arange(A).float() / A,
                     torch.where(torch.arange(A) % 2 == 0, -0.0, 0.0), torch.full((A,), -float("inf"))])
    l[4, A - 1] = 3.0
    d = dict(l=l, tok=torch.tensor([0, A - 1, 0, 1, A - 1]), mask=None, live=None, dlogp=torch.ones(5), dent=torch.ones(5))
    for top in (1, min(20, A), 64):
        check(sim, d, top, cols=cols)


def test_tokens_none_forbidden_and_out_of_range(sim):
    d = inputs(8, 40, torch.float32, 3, masked=True)
    d["tok"] = torch.tensor([-1, 3, 1, 4, 4, -1, 0, 39])
    d["mask"][3, 4] = False
    d["mask"][4, 4] = True
    d["l"][4, 4] = -float("inf")
    r, g = check(sim, d, 4)
    assert r["logp"][0] == 0 and r["logp"][3] == r["logp"][4] == -float("inf")
    for tok in (torch.tensor([40] + [0] * 7), torch.tensor([-2] + [0] * 7, dtype=torch.int32),
                torch.tensor([255] + [0] * 7, dtype=torch.uint8)):
        r = sim.token_logprobs(d["l"].cuda(), tok.cuda())
        with pytest.raises(Exception, match="action out of range"):
            sim.sync()
        assert r["logp"][0] == 0
        sim.token_logprobs_grad(d["l"].cuda(), tok.cuda(), dlogp=torch.ones(8, device="cuda"))
        with pytest.raises(Exception, match="action out of range"):
            sim.sync()
    for t in (torch.uint8, torch.int32):
        d["tok"] = torch.arange(8).to(t)
        check(sim, d, 0)
    r = sim.token_logprobs(d["l"].cuda(), None, top=2)
    assert r["logp"] is None
    sim.sync()


def test_nan_and_infinite_logits(sim):
    """A NaN (or +inf) makes its own row's numbers NaN and comes first; other rows are as before. Masked or in padding
    they do nothing."""
    d = inputs(6, 50, torch.float32, 5)
    clean, _ = check(sim, d, 4)
    l = d["l"].clone()
    l[1, 7] = float("nan")
    l[3, 9] = float("inf")
    r = sim.token_logprobs(l.cuda(), d["tok"].cuda(), top=4)
    sim.sync()
    for k in r:
        for n in (0, 2, 4, 5):
            assert torch.equal(r[k][n], clean[k][n])
    assert r["logp"][1].isnan() and r["entropy"][1].isnan() and r["entropy"][3].isnan()
    assert r["top_index"][1, 0] == 7 and r["top_index"][3, 0] == 9
    mask = torch.ones(6, 50, dtype=torch.bool)
    mask[1, 7] = mask[3, 9] = False
    if d["tok"][1] == 7 or d["tok"][3] == 9:
        d["tok"] = torch.zeros(6, dtype=torch.int64)
    d2 = dict(d, l=l, mask=mask)
    d2["l"] = torch.where(mask, l, torch.zeros(()))      # the oracle's copy
    want = ops.token_logprobs(d2["l"].double().numpy(), d["tok"].numpy(), mask.numpy(), None, 4)
    r = sim.token_logprobs(l.cuda(), d["tok"].cuda(), mask.cuda(), top=4)
    sim.sync()
    assert np.array_equal(r["top_index"].cpu().numpy(), want["top_index"])
    assert r["logp"].isfinite().all() and np.abs(r["logp"].cpu().numpy() - want["logp"]).max() < 1e-5
    live = torch.tensor([1, 0, 1, 0, 1, 1], dtype=torch.uint8)
    r = sim.token_logprobs(l.cuda(), d["tok"].cuda(), live=live.cuda(), top=4)
    g = sim.token_logprobs_grad(l.cuda(), d["tok"].cuda(), torch.ones(6, device="cuda"), torch.ones(6, device="cuda"), live=live.cuda())
    sim.sync()
    assert r["logp"][1] == r["entropy"][3] == 0 and (r["top_index"][[1, 3]] == -1).all()
    assert not g[[1, 3]].any() and g.isfinite().all()


@pytest.mark.parametrize("N,A,top", [(70000, 24, 4), (5000, 300, 8), (1500, 20000, 5)])
@pytest.mark.parametrize("cols", [False, True])
def test_many_rows(sim, N, A, top, cols):
    """More rows than workgroups take at once, against torch in fp64 (sums of A terms: bounds as above at |x| < 24)."""
    if cols and A > 384:
        N = 200
    g = torch.Generator(device="cuda").manual_seed(N)
    l = torch.randn((A, N) if cols else (N, A), generator=g, device="cuda") * 2
    l = (l.t() if cols else l)
    tok = torch.randint(0, A, (N,), generator=g, device="cuda")
    r = sim.token_logprobs(l, tok, top=top)
    dl = torch.randn(N, generator=g, device="cuda")
    grad = sim.token_logprobs_grad(l, tok, dl)
    sim.sync()
    ls = torch.log_softmax(l.double(), 1)
    p = ls.exp()
    eS = U * (3 * 24 + 4 + A / 64 + min(A, 96) + 16)
    eL = eS + U * (24 + 36 + 3 * 12 + 1 + 36)
    assert (r["logp"].double() - ls.gather(1, tok[:, None])[:, 0]).abs().max() <= eL
    v, i = l.double().topk(top, 1)          # fp32 normals: ties are next to none, and equal values as good
    assert torch.equal(l.double().gather(1, r["top_index"]), v)
    assert (r["top_logp"].double() - ls.gather(1, i)).abs().max() <= eL
    want = dl.double()[:, None] * (torch.zeros_like(p).scatter_(1, tok[:, None], 1.0) - p)
    tol = dl.double().abs()[:, None] * (p * (eS + U * (4 * 24 + 4 * 12 + 8 + 3)) + 3 * U) + U * want.abs()
    assert ((grad.double() - want).abs() <= tol).all()


def test_in_place_strides_repeats_and_graphs(sim):
    d = inputs(40, 700, torch.bfloat16, 6, masked=True, padded=True)
    wide = torch.full((40, 900), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, 13:713] = d["l"].cuda()
    l, tok, mk, live = wide[:, 13:713], d["tok"].cuda(), d["mask"].cuda(), d["live"].cuda()
    dl, dh = d["dlogp"].cuda(), d["dent"].cuda()
    a, g = check(sim, d, 6)
    b = sim.token_logprobs(l, tok, mk, live, 6)
    h = sim.token_logprobs_grad(l, tok, dl, dh, mk, live)
    same = l.clone()
    assert sim.token_logprobs_grad(same, tok, dl, dh, mk, live, grad=same) is same
    sim.sync()
    assert all(torch.equal(a[k], b[k]) for k in a) and torch.equal(g, h) and torch.equal(g, same)
    import paper_2607_05272_amd as bs
    st = torch.cuda.Stream()
    for l0 in (d["l"].cuda(), torch.randn(2, 131072, device="cuda")):
        with torch.cuda.stream(st), bs.Sim(preset("C1"), n_envs=1, stream=st) as own:
            st.wait_stream(torch.cuda.default_stream())
            cur = l0.clone()
            t = torch.zeros(len(cur), dtype=torch.int64, device="cuda")
            w = torch.ones(len(cur), device="cuda")
            own.token_logprobs(cur, t, top=5)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=st):
                out = own.token_logprobs(cur, t, top=5)
                og = own.token_logprobs_grad(cur, t, w, w)
            for f in (1.0, -1.0, 0.5):
                cur.copy_(l0 * f)
                graph.replay()
                want, wg = own.token_logprobs(cur, t, top=5), own.token_logprobs_grad(cur, t, w, w)
                st.synchronize()
                assert all(torch.equal(out[k], want[k]) for k in out) and torch.equal(og, wg)


def test_sizes_of_zero_and_refusals(sim):
    r = sim.token_logprobs(torch.zeros(0, 5, device="cuda"), torch.zeros(0, dtype=torch.int64, device="cuda"), top=2)
    assert r["logp"].shape == (0,) and r["top_index"].shape == (0, 2)
    assert sim.token_logprobs_grad(torch.zeros(0, 5, device="cuda")).shape == (0, 5)
    l, t = torch.randn(4, 6, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    import paper_2607_05272_amd as bs
    for a, kw in (((l.double(), t), {}), ((l, t[:3]), {}), ((l, t.float()), {}), ((l, t.cpu()), {}), ((l, t), dict(live=t)),
                  ((l, t), dict(mask=torch.ones(4, 5, dtype=torch.bool, device="cuda")))):
        with pytest.raises(ValueError):
            sim.token_logprobs(*a, **kw)
    with pytest.raises(bs.SimError, match="64"):
        sim.token_logprobs(l, t, top=65)
    with pytest.raises(bs.SimError, match="top must"):
        sim.token_logprobs(l, t, top=-1)
    with pytest.raises(bs.SimError, match="one stride"):
        sim.token_logprobs(torch.randn(8, 12, device="cuda")[::2, ::2], t)
    with pytest.raises(bs.SimError, match="needs tokens"):
        sim.token_logprobs_grad(l, None, torch.ones(4, device="cuda"))
    sim.sync()
