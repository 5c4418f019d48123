"""balance_loss against the fp64 form (oracle/ops.py) within the bounds of loss_check.py: sizes, both
layouts, types, groups, padding, choices that are none or out of range, refusals and graphs."""
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


def inputs(N, A, k, dtype, seed, index=torch.int64):
    g = torch.Generator().manual_seed(seed)
    l = (torch.randn(N, A, generator=g) * 2 + torch.randn(1, A, generator=g)).to(dtype)
    idx = l.float().topk(k, dim=1).indices
    return l, idx.to(index), torch.rand(N, generator=g) > 0.2


def check(sim, l, idx, live, group=1, coef=0.7, cols=False, **kw):
    d = l.cuda()
    d = d.t().contiguous().t() if cols else d
    r = sim.balance_loss(d, idx.cuda(), None if live is None else live.cuda(), group, coef, **kw)
    sim.sync()
    want = ops.balance_loss(l.double().numpy(), idx.numpy(), None if live is None else live.numpy(), group, coef)
    on = np.ones(len(l), bool) if live is None else live.numpy()
    lc.check_balance(r, want, l.double().numpy(), on, group, coef, l.dtype)
    return r


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("N,A,k", [(1, 1, 1), (7, 4, 2), (64, 8, 2), (100, 60, 4), (65, 64, 1), (50, 65, 8), (40, 128, 8),
                                   (33, 130, 3), (20, 256, 8), (15, 384, 2), (9, 515, 4), (5, 1100, 6), (4, 4096, 3)])
def test_rows(sim, N, A, k, dtype):
    l, idx, live = inputs(N, A, k, TYPES[dtype], N + A)
    check(sim, l, idx, live)
    check(sim, l, idx, None, coef=-3.0)


@pytest.mark.parametrize("index", [torch.uint8, torch.int32])
@pytest.mark.parametrize("N,K", [(1, 1), (63, 1), (200, 4), (130, 8), (300, 16)])
def test_servers_of_the_simulator(sim, N, K, index):
    """The simulator's actions in groups of 6, logits in either layout."""
    l, idx, live = inputs(N, 6 * K, 1, torch.float32, K, index)
    for cols in (False, True):
        check(sim, l, idx, live, group=6, cols=cols)


@pytest.mark.parametrize("N,A,k,group", [(3000, 16, 2, 1), (5000, 48, 1, 6), (2500, 200, 8, 1), (20000, 6, 1, 2)])
def test_many_rows(sim, N, A, k, group):
    l, idx, live = inputs(N, A, k, torch.float32, 3)
    for cols in (False, True):
        check(sim, l, idx, live, group, cols=cols)


@pytest.mark.parametrize("N,A,group", [(70001, 200, 1), (400, 200, 8), (400, 720, 6), (300000, 7, 1)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_columns_held_and_read_twice(sim, N, A, group, dtype):
    l, idx, live = inputs(N, A, 2, TYPES[dtype], 5)
    check(sim, l, idx, live, group, cols=True)


def test_wide_groups(sim):
    l, idx, live = inputs(6, 9000, 3, torch.bfloat16, 4)
    check(sim, l, idx, live, group=3)
    check(sim, l, idx, live, group=9000)


def test_padding_and_forbidden_columns(sim):
    """Rows that are not live may hold anything; columns at -inf have probability 0; rows of nothing
    but -inf add nothing to P."""
    l, idx, live = inputs(40, 30, 2, torch.float32, 5)
    l[:, 7] = -float("inf")
    l[4] = -float("inf")
    idx[idx == 7] = 8
    live[4] = True
    want = check(sim, l, idx, live)
    l2, i2 = l.clone(), idx.clone()
    l2[~live] = float("nan")
    i2[~live] = 1000
    r = sim.balance_loss(l2.cuda(), i2.cuda(), live.cuda(), 1, 0.7)
    sim.sync()
    assert all(torch.equal(r[k], want[k]) for k in r)
    assert (r["grad"][4] == 0).all() and (r["grad"][~live] == 0).all() and (r["grad"][:, 7] == 0).all()


def test_no_live_rows(sim):
    l, idx, live = inputs(9, 12, 2, torch.float32, 6)
    r = sim.balance_loss(l.cuda(), idx.cuda(), torch.zeros(9, dtype=torch.bool, device="cuda"))
    e = sim.balance_loss(torch.empty(0, 12, device="cuda"), torch.empty(0, 2, dtype=torch.int32, device="cuda"))
    sim.sync()
    for x in (r, e):
        assert x["loss"] == 0 and (x["counts"] == 0).all() and (x["grad"] == 0).all()


def test_choices_that_are_none_or_out_of_range(sim):
    import paper_2607_05272_amd as bs
    l, idx, live = inputs(50, 20, 3, torch.float32, 7)
    idx[::4, 1] = -1
    check(sim, l, idx, live)
    check(sim, l, idx.to(torch.int32), live)
    idx[live.nonzero()[0], 0] = 20
    r = sim.balance_loss(l.cuda(), idx.cuda(), live.cuda(), 1, 0.7)
    with pytest.raises(bs.SimError, match="out of range"):
        sim.sync()
    want = ops.balance_loss(l.double().numpy(), idx.numpy(), live.numpy(), 1, 0.7)
    assert want["bad"] == 1
    lc.check_balance(r, want, l.double().numpy(), live.numpy(), 1, 0.7, torch.float32)
    sim.sync()


@pytest.mark.parametrize("A", [30, 700])
def test_strides_and_gradient_in_place(sim, A):
    l, idx, live = inputs(30, A, 2, torch.bfloat16, 8)
    want = check(sim, l, idx, live)
    room = torch.full((30, A + 5), 77.0, dtype=torch.bfloat16, device="cuda")
    v = room[:, 3:3 + A]
    v.copy_(l)
    r = sim.balance_loss(v, idx.cuda(), live.cuda(), 1, 0.7, grad=v)
    sim.sync()
    assert torch.equal(v, want["grad"]) and torch.equal(r["loss"], want["loss"])
    assert (room[:, :3] == 77).all() and (room[:, 3 + A:] == 77).all()
    none = sim.balance_loss(l.cuda(), idx.cuda(), live.cuda(), 1, 0.7, want_grad=False)
    sim.sync()
    assert none["grad"] is None and torch.equal(none["loss"], want["loss"]) and torch.equal(none["counts"], want["counts"])


def test_far_rows(sim):
    l, idx, live = inputs(3, 200, 2, torch.bfloat16, 9)
    want = check(sim, l, idx, live)
    far = (1 << 30) + 8
    room = torch.empty(2 * far + 400, dtype=torch.bfloat16, device="cuda")
    a, b = (room[i * 200:].as_strided((3, 200), (far, 1)) for i in (0, 1))
    a.copy_(l)
    r = sim.balance_loss(a, idx.cuda(), live.cuda(), 1, 0.7, grad=b)
    sim.sync()
    assert all(torch.equal(r[k], want[k]) for k in r)


def test_refusals(sim):
    import paper_2607_05272_amd as bs
    l, i = torch.zeros(4, 6, device="cuda"), torch.zeros(4, 1, dtype=torch.int64, device="cuda")
    for bad in (lambda: sim.balance_loss(l.double(), i), lambda: sim.balance_loss(l, i[:3]),
                lambda: sim.balance_loss(l, i[:, 0]), lambda: sim.balance_loss(l, i.float()),
                lambda: sim.balance_loss(l, i, live=l[:, 0])):
        with pytest.raises(ValueError):
            bad()
    for kw, what in ((dict(group=4), "divide"), (dict(group=0), "divide"),
                     (dict(grad=torch.zeros(4, 1, device="cuda").expand(4, 6)), "share memory")):
        with pytest.raises(bs.SimError, match=what):
            sim.balance_loss(l, i, **kw)
    with pytest.raises(bs.SimError, match="4096"):
        sim.balance_loss(torch.zeros(2, 5000, device="cuda"), i[:2])
    sim.sync()


def test_graphs(sim):
    import paper_2607_05272_amd as bs
    sets = [[t.cuda() for t in inputs(N, A, 2, torch.float32, A)] for N, A in ((3000, 48), (40, 8))]
    want = [sim.balance_loss(l, i, v) for l, i, v in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    with bs.Sim(preset("C1"), n_envs=1, stream=streams[0]) as s0:
        torch.cuda.synchronize()
        graphs, got = [], []
        for l, i, v in sets:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=streams[0]):
                got.append(s0.balance_loss(l, i, v))
            graphs.append(g)
        for _ in range(4):
            for o in got:
                for t in o.values():
                    t.fill_(-1)
            torch.cuda.synchronize()
            for g, st in zip(graphs, streams):
                with torch.cuda.stream(st):
                    g.replay()
            sim.balance_loss(*sets[0])
            torch.cuda.synchronize()
            for w, o in zip(want, got):
                assert all(torch.equal(w[k], o[k]) for k in w)


@pytest.mark.parametrize("A,cols", [(10000, True), (48000, True), (48000, False)])
def test_many_small_probabilities(sim, A, cols):
    """Sixteen logits of 0, then thousands whose exponential is 0.9 half steps of fp32 at 1: a sum that takes
    them one after another loses them all (48000 columns: 1.6e-4 of the sum)."""
    l = torch.full((3, A), 24 * -np.log(2.0) + np.log(0.9))
    l[:, :16] = 0.0
    check(sim, l, torch.tensor([[0], [17], [3]]), None, group=16, cols=cols)
