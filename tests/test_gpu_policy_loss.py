"""policy_loss against the fp64 form (oracle/ops.py) within the bounds of loss_check.py: sizes around
the kernels' row forms, both layouts, types, masks (rows left empty, infinities and NaN in masked
places, the type's lowest value), weights, the terms that may be absent, refusals, streams and graphs."""
import numpy as np
import pytest

from workloads import preset

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import loss_check as lc   # noqa: E402
from oracle import ops    # noqa: E402
from scan_check import TYPES   # noqa: E402


@pytest.fixture(scope="module")
def sim():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2607_05272_amd as bs
    with bs.Sim(preset("C1"), n_envs=1) as s:
        yield s


def inputs(N, A, dtype, seed, masked=False, padded=True):
    """Likely and unlikely actions, ratios inside and outside the clip range and none at its edge."""
    g = torch.Generator().manual_seed(seed)
    l = (torch.randn(N, A, generator=g) * 3).to(dtype)
    a = torch.randint(0, A, (N,), generator=g)
    mask = None
    if masked:
        mask = torch.rand(N, A, generator=g) > 0.4
        mask[torch.arange(N), a] = True
        mask[3::7] = False
    w = torch.rand(N, generator=g) / N
    if padded:
        w[2::5] = 0.0
    z = l.double()
    z = z if mask is None else z.masked_fill(~mask, -torch.inf)
    lp = torch.log_softmax(z, 1)[torch.arange(N), a].nan_to_num(0.0, 0.0, 0.0)
    rho = torch.exp(0.3 * torch.randn(N, generator=g).double())
    for edge in (1 - lc.CLIP, 1 + lc.CLIP):
        rho = torch.where((rho - edge).abs() < 1e-2, rho + 3e-2, rho)
    return dict(logits=l, actions=a, mask=mask, weight=w, old=(lp - rho.log()).float(),
                ref=(lp + 0.4 * torch.randn(N, generator=g)).float(), adv=torch.randn(N, generator=g))


def run(sim, s, c_kl=0.3, c_entropy=0.2, cols=False, grad=None, actions=torch.int64, **kw):
    d = {k: None if v is None else v.cuda() for k, v in s.items()}
    l = d["logits"]
    if cols:
        l = l.t().contiguous().t()
        d["mask"] = None if d["mask"] is None else d["mask"].t().contiguous().t()
    r = sim.policy_loss(l, d["actions"].to(actions), d["adv"], d["old"], d["ref"], d["weight"], d["mask"],
                        lc.CLIP, c_kl, c_entropy, grad=grad, **kw)
    sim.sync()
    return r


def check(sim, s, c_kl=0.3, c_entropy=0.2, **kw):
    r = run(sim, s, c_kl, c_entropy, **kw)
    h = {k: None if v is None else v.double().numpy() for k, v in s.items()}
    want = ops.policy_loss(h["logits"], h["actions"], h["adv"], h["old"], h["ref"], h["weight"], h["mask"],
                           lc.CLIP, c_kl, c_entropy)
    lc.check_policy(h, r, want, c_kl, c_entropy, s["logits"].dtype)
    return r


SIZES = [(1, 1), (5, 2), (64, 6), (65, 7), (130, 25), (33, 48), (20, 64), (21, 65), (40, 96), (17, 97), (9, 128),
         (9, 130), (12, 255), (6, 256), (6, 512), (7, 515), (5, 1000), (4, 1025), (4, 2048), (4, 2051), (3, 4096),
         (3, 4099), (3, 8192), (3, 8195), (2, 8200), (2, 16391), (2, 33000), (2, 50257), (2, 70001), (1, 131072), (1, 150001),
         (1, 300001), (40, 40000),
         (20, 70000)]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("N,A", SIZES)
def test_rows(sim, N, A, dtype):
    for masked in (False, True):
        check(sim, inputs(N, A, TYPES[dtype], N + A, masked))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("N,A", [(1, 6), (2, 1), (63, 6), (64, 7), (65, 24), (257, 48), (300, 97), (130, 255), (70, 600),
                                 (65, 2500)])
def test_columns(sim, N, A, dtype):
    """[A][N] logits, as sim_policy writes them."""
    for masked in (False, True):
        check(sim, inputs(N, A, TYPES[dtype], N + 3 * A, masked), cols=True)


@pytest.mark.parametrize("N,A", [(2000, 6), (3000, 48), (1500, 130), (600, 1100)])
@pytest.mark.parametrize("cols", [False, True])
def test_many_rows(sim, N, A, cols):
    check(sim, inputs(N, A, torch.float32, 5, True), cols=cols)


@pytest.mark.parametrize("N,A", [(33001, 255), (32767, 193), (40001, 384), (70001, 385)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_columns_held_and_read_twice(sim, N, A, dtype):
    check(sim, inputs(N, A, TYPES[dtype], 6, True), cols=True)


@pytest.mark.parametrize("A", [6, 300, 5000])
@pytest.mark.parametrize("without", ["old", "ref", "weight", "entropy", "kl"])
def test_absent_terms(sim, A, without):
    s = inputs(20, A, torch.float32, 1, padded=False)
    kw = {}
    if without in s:
        s[without] = None
    if without in ("ref", "kl"):
        kw["c_kl"] = 0.0
    if without == "entropy":
        kw["c_entropy"] = 0.0
    for cols in (False, True):
        check(sim, s, cols=cols, **kw)


@pytest.mark.parametrize("actions", [torch.uint8, torch.int32])
def test_types_of_actions_and_advantages(sim, actions):
    s = inputs(30, 96, torch.bfloat16, 2)
    a = check(sim, s, actions=actions)
    s["adv"] = s["adv"].double()
    b = check(sim, s, actions=actions)
    assert all(torch.equal(a[k], b[k]) for k in ("loss", "logp", "grad"))


@pytest.mark.parametrize("A", [7, 96, 700, 9000, 140001])
@pytest.mark.parametrize("cols", [False, True])
def test_masked_places_hold_anything(sim, A, cols):
    """Infinities and NaN where the mask forbids, -inf logits, the type's lowest value added as a mask."""
    if cols and A > 1000:
        A = 1000
    for dtype in (torch.float32, torch.bfloat16):
        s = inputs(11, A, dtype, 3, True)
        want = check(sim, s, cols=cols)
        dirty = dict(s, logits=s["logits"].clone())
        bad = ~s["mask"]
        places = torch.arange(bad.numel()).view(bad.shape)
        for i, v in enumerate((float("nan"), float("inf"), -float("inf"))):
            dirty["logits"][bad & (places % 3 == i)] = v
        got = run(sim, dirty, cols=cols)
        assert all(torch.equal(got[k], want[k]) for k in ("loss", "logp", "grad"))
        # -inf in place of the mask: the same
        inf = dict(s, mask=None, logits=s["logits"].masked_fill(bad, -float("inf")))
        got = run(sim, inf, cols=cols)
        assert all(torch.equal(got[k], want[k]) for k in ("loss", "logp", "grad"))
        # the lowest value in place of the mask: probability 0, but a row of nothing else is uniform
        low = dict(s, mask=None, logits=s["logits"].masked_fill(bad, torch.finfo(dtype).min))
        got = run(sim, low, cols=cols)
        live = s["mask"].any(1)
        assert torch.equal(got["logp"][live.cuda()], want["logp"][live.cuda()])
        assert torch.isfinite(got["grad"]).all() and torch.isfinite(got["loss"]).all()


@pytest.mark.parametrize("A", [5, 60, 3000, 140001])
def test_padding_and_empty_rows(sim, A):
    """Rows of weight 0 are not looked at (NaN logits, actions out of range); rows that the mask leaves
    empty give nothing."""
    s = inputs(12, A, torch.float32, 4, True)
    h = dict(s, logits=s["logits"].clone(), actions=s["actions"].clone())
    h["logits"][2::5] = float("nan")
    h["actions"][2::5] = -77
    want, got = check(sim, s), run(sim, h)
    assert all(torch.equal(got[k], want[k]) for k in ("loss", "logp", "grad"))
    assert (got["grad"][2::5] == 0).all() and (got["grad"][3::7] == 0).all() and (got["logp"][3::7] == 0).all()


@pytest.mark.parametrize("A", [6, 100, 4000])
def test_not_finite_rows_stay_apart(sim, A):
    s = inputs(9, A, torch.float32, 5, padded=False)
    want = run(sim, s)
    s["logits"][4, A // 2] = float("nan")
    s["logits"][6, 0] = float("inf")
    for cols in (False, True):
        got = run(sim, s, cols=cols)
        other = [0, 1, 2, 3, 5, 7, 8]
        assert torch.isnan(got["grad"][4]).all() and torch.isnan(got["logp"][[4, 6]]).all()
        assert torch.isnan(got["loss"][0])
        if not cols:
            assert torch.equal(got["grad"][other], want["grad"][other])
        assert torch.isfinite(got["grad"][other]).all()


@pytest.mark.parametrize("A", [6, 100, 4000])
@pytest.mark.parametrize("cols", [False, True])
def test_actions_that_are_not_open_are_latched(sim, A, cols):
    import paper_2607_05272_amd as bs
    s = inputs(20, A, torch.float32, 6, True, padded=False)
    s["actions"][5], s["actions"][9], s["actions"][11] = A, -1, 1
    s["mask"][11] = True
    s["mask"][11, 1] = False
    d = {k: v.cuda() for k, v in s.items()}
    lay = (lambda t: t.t().contiguous().t()) if cols else (lambda t: t)
    r = sim.policy_loss(lay(d["logits"]), d["actions"], d["adv"], d["old"], d["ref"], d["weight"], lay(d["mask"]),
                        lc.CLIP, 0.3, 0.2)
    with pytest.raises(bs.SimError, match="action out of range"):
        sim.sync()
    h = {k: v.double().numpy() for k, v in s.items()}
    want = ops.policy_loss(h["logits"], h["actions"], h["adv"], h["old"], h["ref"], h["weight"], h["mask"], lc.CLIP,
                           0.3, 0.2)
    assert want["bad"] == [5, 9, 11]
    lc.check_policy(h, r, want, 0.3, 0.2, torch.float32)
    sim.sync()


@pytest.mark.parametrize("N,A", [(40, 7), (50, 96), (20, 513), (3, 9001), (2, 140001)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides_and_gradient_in_place(sim, N, A, dtype):
    """Rows of an odd length and start, a gradient between guards, a mask of another layout, a mask
    row shared by all, the gradient over the logits."""
    dt = TYPES[dtype]
    s = inputs(N, A, dt, 7, True)
    want = check(sim, s)
    d = {k: v.cuda() for k, v in s.items()}
    room = torch.full((N, A + 5), 77.0, dtype=dt, device="cuda")
    l = room[:, 3:3 + A]
    l.copy_(d["logits"])
    out = torch.full((N, A + 3), 77.0, dtype=dt, device="cuda")
    args = (d["adv"], d["old"], d["ref"], d["weight"])
    m = d["mask"].t().contiguous().t()
    r = sim.policy_loss(l, d["actions"], *args, m, lc.CLIP, 0.3, 0.2, grad=out[:, 1:1 + A])
    sim.sync()
    assert all(torch.equal(r[k], want[k]) for k in ("loss", "logp", "grad"))
    assert (out[:, 0] == 77).all() and (out[:, 1 + A:] == 77).all() and (room[:, :3] == 77).all()
    r = sim.policy_loss(l, d["actions"], *args, d["mask"], lc.CLIP, 0.3, 0.2, grad=l)
    sim.sync()
    assert all(torch.equal(r[k], want[k]) for k in ("loss", "logp")) and torch.equal(l, want["grad"])
    assert (room[:, :3] == 77).all() and (room[:, 3 + A:] == 77).all()
    # in place over columns
    c = d["logits"].t().contiguous().t()
    w2 = sim.policy_loss(c, d["actions"], *args, m, lc.CLIP, 0.3, 0.2)
    r = sim.policy_loss(c, d["actions"], *args, m, lc.CLIP, 0.3, 0.2, grad=c)
    sim.sync()
    assert torch.equal(c, w2["grad"]) and torch.equal(r["loss"], w2["loss"])
    # one mask row for all
    s["mask"] = (torch.rand(A, generator=torch.Generator().manual_seed(1)) > 0.3)[None].expand(N, A).clone()
    s["mask"][:, s["actions"]] = True
    want = check(sim, s)
    r = sim.policy_loss(d["logits"], d["actions"], *args, s["mask"][0].cuda()[None].expand(N, A), lc.CLIP, 0.3, 0.2)
    sim.sync()
    assert all(torch.equal(r[k], want[k]) for k in ("loss", "logp", "grad"))


def test_without_gradient_and_without_samples(sim):
    s = inputs(30, 48, torch.float32, 8)
    want = check(sim, s)
    r = run(sim, s, want_grad=False)
    assert r["grad"] is None and torch.equal(r["loss"], want["loss"]) and torch.equal(r["logp"], want["logp"])
    e = torch.empty(0, 48, device="cuda")
    r = sim.policy_loss(e, torch.empty(0, dtype=torch.int64, device="cuda"), torch.empty(0, device="cuda"))
    sim.sync()
    assert (r["loss"] == 0).all() and r["grad"].shape == (0, 48)
    for A in (1, 700, 5000, 200000):
        for e in (torch.empty(0, A, device="cuda"), torch.empty(A, 0, device="cuda").t()):
            r = sim.policy_loss(e, torch.empty(0, dtype=torch.int64, device="cuda"), torch.empty(0, device="cuda"))
            sim.sync()
            assert (r["loss"] == 0).all()


def test_far_rows(sim):
    """Rows more than 2^31 elements apart, in the logits, the gradient and the mask."""
    N, A, far = 3, 5000, (1 << 30) + 8
    s = inputs(N, A, torch.bfloat16, 9, True, padded=False)
    want = check(sim, s)
    d = {k: v.cuda() for k, v in s.items()}
    room = torch.empty(2 * far + 2 * A, dtype=torch.bfloat16, device="cuda")
    l, g = (room[i * A:].as_strided((N, A), (far, 1)) for i in (0, 1))
    m = torch.empty(2 * far + A, dtype=torch.uint8, device="cuda").as_strided((N, A), (far, 1))
    l.copy_(d["logits"])
    m.copy_(d["mask"])
    r = sim.policy_loss(l, d["actions"], d["adv"], d["old"], d["ref"], d["weight"], m, lc.CLIP, 0.3, 0.2, grad=g)
    sim.sync()
    assert all(torch.equal(r[k], want[k]) for k in ("loss", "logp", "grad"))


def test_refusals(sim):
    import paper_2607_05272_amd as bs
    N, A = 4, 6
    l, a, adv = torch.zeros(N, A, device="cuda"), torch.zeros(N, dtype=torch.int64, device="cuda"), torch.zeros(N, device="cuda")
    for bad in (lambda: sim.policy_loss(l.double(), a, adv), lambda: sim.policy_loss(l, a.short(), adv),
                lambda: sim.policy_loss(l, a[:3], adv), lambda: sim.policy_loss(l, a, adv.half()),
                lambda: sim.policy_loss(l.cpu(), a, adv), lambda: sim.policy_loss(l, a, adv, mask=l),
                lambda: sim.policy_loss(l, a, adv, weight=adv.double()),
                lambda: sim.policy_loss(l, a, adv, grad=l.half())):
        with pytest.raises(ValueError):
            bad()
    for bad, what in ((dict(clip=0.0), "clip"), (dict(clip=1.0), "clip"), (dict(c_kl=0.1), "reference"),
                      (dict(c_kl=-0.1), ">= 0"), (dict(c_entropy=float("nan")), ">= 0"),
                      (dict(grad=torch.zeros(1, A, device="cuda").expand(N, A)), "share memory"),
                      (dict(grad=l.view(-1).as_strided((N, A), (1, N))), "other strides")):
        with pytest.raises(bs.SimError, match=what):
            sim.policy_loss(l, a, adv, **bad)
    with pytest.raises(bs.SimError, match="stride"):
        sim.policy_loss(torch.zeros(N, A, 2, device="cuda")[..., 0], a, adv)
    sim.sync()


def test_graphs(sim):
    """Two captured calls on one context, replayed on streams of their own with eager work between."""
    import paper_2607_05272_amd as bs
    sets = [{k: v.cuda() for k, v in inputs(N, A, torch.float32, A, True).items()} for N, A in ((3000, 48), (3, 9000))]
    def call(s, d):   # noqa: E306
        return s.policy_loss(d["logits"], d["actions"], d["adv"], d["old"], d["ref"], d["weight"], d["mask"],
                             lc.CLIP, 0.3, 0.2)
    want = [call(sim, d) for d in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    with bs.Sim(preset("C1"), n_envs=1, stream=streams[0]) as s0:
        torch.cuda.synchronize()
        graphs, got = [], []
        for d in sets:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=streams[0]):
                got.append(call(s0, d))
            graphs.append(g)
        for _ in range(4):
            for o in got:
                for t in o.values():
                    t.fill_(-1.0)
            torch.cuda.synchronize()
            for g, st in zip(graphs, streams):
                with torch.cuda.stream(st):
                    g.replay()
            call(sim, sets[0])
            torch.cuda.synchronize()
            for w, o in zip(want, got):
                assert all(torch.equal(w[k], o[k]) for k in w)


@pytest.mark.parametrize("N,A,cols", [(20, 6, False), (20, 6, True), (15, 48, True), (9, 300, False), (70, 600, True),
                                      (6, 5000, False), (3, 9000, False), (2, 140001, False), (2, 300001, False)])
@pytest.mark.parametrize("ref", [-float("inf"), 120.0, 1000.0, float("nan")])
def test_a_reference_without_its_coefficient_tells_the_kl_term_alone(sim, N, A, cols, ref):
    """c_kl = 0 with a reference that forbids the action, lies far above its probability or is NaN: the
    KL term is infinite, huge or NaN, all else that of a call without a reference."""
    s = inputs(N, A, torch.float32, 10, True, padded=False)
    want = run(sim, dict(s, ref=None), c_kl=0.0, cols=cols)
    s["ref"][0] = ref
    got = run(sim, s, c_kl=0.0, cols=cols)
    assert torch.isfinite(want["loss"]).all() and torch.isfinite(want["grad"]).all()
    assert all(torch.equal(got[k], want[k]) for k in ("logp", "grad"))
    assert torch.equal(got["loss"][[0, 1, 3]], want["loss"][[0, 1, 3]])
    kl = got["loss"][2].item()
    assert kl > 1e40 or kl == float("inf") or kl != kl


@pytest.mark.parametrize("A,cols", [(10007, True), (50000, True), (10007, False), (50000, False), (300000, False)])
def test_many_small_probabilities(sim, A, cols):
    """Sixteen logits of 0, then thousands whose exponential is 0.9 half steps of fp32 at 1: a sum that takes
    them one after another loses them all (50000 columns: 1.7e-4 of the sum, the bound is 5e-5)."""
    l = torch.full((3, A), 24 * -np.log(2.0) + np.log(0.9))
    l[:, :16] = 0.0
    s = dict(logits=l, actions=torch.tensor([0, 5, A - 1]), mask=None, weight=None, old=None, ref=None,
             adv=torch.tensor([1.0, -2.0, 0.5]))
    check(sim, s, 0.0, 0.2, cols=cols)
