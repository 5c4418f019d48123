"""linear_attn and its gradient against the fp64 form (oracle/ops.py) within the bounds of attn_check.py: sizes
from one step to several runs of steps, odd channels, types, shared heads, lengths, strides, decays at their
bounds, states in place, refusals and graphs."""
import numpy as np
import pytest

from workloads import preset

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import attn_check as ac   # noqa: E402
from oracle import ops    # noqa: E402
from scan_check import TYPES   # noqa: E402


@pytest.fixture(scope="module")
def sim():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2607_05272_amd as bs
    with bs.Sim(preset("C1"), n_envs=1) as s:
        yield s


def cuda(d):
    return {k: v.cuda() if torch.is_tensor(v) else v for k, v in d.items()}


def both(sim, d, grad=True):
    c = cuda(d)
    y, state = sim.linear_attn(c["q"], c["k"], c["v"], c["decay"], c["s0"], c["lengths"], c["scale"])
    g = None
    if grad:
        g = sim.linear_attn_grad(c["q"], c["k"], c["v"], c["decay"], c["dy"], c["s0"], c["dstate"], c["lengths"], c["scale"])
    sim.sync()
    ac.check_forward(d, y, state)
    if grad:
        ac.check_grad(d, *g)
    return y, state, g


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("B,T,H,Hk,Dk,Dv", [
    (1, 1, 1, 1, 1, 1), (3, 1, 4, 2, 64, 64), (2, 1, 2, 1, 128, 256), (2, 2, 3, 3, 33, 130), (1, 16, 2, 2, 16, 20),
    (1, 17, 2, 2, 16, 20), (2, 63, 2, 1, 64, 64), (1, 64, 1, 1, 64, 128), (2, 65, 4, 2, 72, 80), (1, 100, 2, 2, 7, 3),
    (1, 130, 2, 1, 128, 128), (1, 200, 1, 1, 256, 64), (1, 161, 1, 1, 40, 256), (1, 96, 1, 1, 130, 250)])
def test_sizes(sim, B, T, H, Hk, Dk, Dv, dtype):
    both(sim, ac.inputs(B, T, H, Hk, Dk, Dv, TYPES[dtype], 100 * T + Dk))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("B,T,H,Hk,Dk,Dv", [(6, 1, 2, 2, 8, 8), (7, 40, 4, 1, 24, 32), (5, 129, 3, 3, 64, 48), (6, 200, 2, 1, 96, 72)])
def test_lengths(sim, B, T, H, Hk, Dk, Dv, dtype):
    """Whole, empty and ragged sequences; padding may hold anything."""
    d = ac.inputs(B, T, H, Hk, Dk, Dv, TYPES[dtype], T, lengths=True)
    y, state, g = both(sim, d)
    e = cuda(d)
    for n in ("q", "k", "v", "dy"):
        x = e[n].clone()
        x[torch.arange(T, device="cuda")[None] >= e["lengths"][:, None]] = float("nan")
        e[n] = x
    y2, s2 = sim.linear_attn(e["q"], e["k"], e["v"], e["decay"], e["s0"], e["lengths"], e["scale"])
    g2 = sim.linear_attn_grad(e["q"], e["k"], e["v"], e["decay"], e["dy"], e["s0"], e["dstate"], e["lengths"], e["scale"])
    sim.sync()
    for a, b in zip((y, state, *g), (y2, s2, *g2)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("T", [1, 9, 150])
def test_decays_at_their_bounds(sim, T):
    """0 forgets everything but the step itself, 1 nothing; tiny ones underflow over a run."""
    both(sim, ac.inputs(2, T, 5, 1, 32, 16, torch.float32, 3, decays=[0.0, 1.0, 1e-30, 0.5, 1 - 2.0 ** -20]))
    both(sim, ac.inputs(2, T, 5, 5, 32, 16, torch.bfloat16, 4, decays=[0.0, 1.0, 1e-30, 0.5, 1 - 2.0 ** -20]))


@pytest.mark.parametrize("T", [3, 70])
def test_decays_and_lengths_out_of_range_are_told(sim, T):
    d = ac.inputs(3, T, 3, 3, 16, 16, torch.float32, 5, lengths=True)
    bad = cuda(d)
    bad["decay"] = torch.tensor([1.5, -0.25, float("nan")], device="cuda")
    y, s = sim.linear_attn(bad["q"], bad["k"], bad["v"], bad["decay"], bad["s0"], bad["lengths"], bad["scale"])
    with pytest.raises(Exception, match="decay out of range"):
        sim.sync()
    d["decay"] = torch.tensor([1.0, 0.0, 0.0])
    ac.check_forward(d, y, s)
    bad = cuda(d)
    bad["lengths"] = torch.tensor([T + 1, -1, 1], dtype=torch.int32, device="cuda")
    y, s = sim.linear_attn(bad["q"], bad["k"], bad["v"], bad["decay"], bad["s0"], bad["lengths"], bad["scale"])
    with pytest.raises(Exception, match="sequence length out of range"):
        sim.sync()
    d["lengths"] = torch.tensor([T, 0, 1], dtype=torch.int32)
    ac.check_forward(d, y, s)
    for want in ((0,), (1,), (2,)):      # the gradient tells whichever of its outputs are wanted
        sizes = dict(dq=None, dk=None, dv=None)
        sim.linear_attn_grad(bad["q"], bad["k"], bad["v"], bad["decay"], bad["dy"], bad["s0"], bad["dstate"],
                             bad["lengths"], bad["scale"], **sizes)
        with pytest.raises(Exception, match="sequence length out of range"):
            sim.sync()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 5, 90])
def test_strides(sim, T, dtype):
    """Time-major, channels cut out of wider rows at odd places, sequences and steps broadcast, heads outermost."""
    d = ac.inputs(3, T, 4, 2, 40, 24, TYPES[dtype], 6)
    c = cuda(d)
    a = sim.linear_attn(c["q"], c["k"], c["v"], c["decay"], c["s0"], None, c["scale"])
    ga = sim.linear_attn_grad(c["q"], c["k"], c["v"], c["decay"], c["dy"], c["s0"], c["dstate"], None, c["scale"])

    def lay(x, how):
        if how == 0:
            return x.transpose(0, 1).contiguous().transpose(0, 1)
        if how == 1:
            w = torch.full((*x.shape[:3], x.shape[3] + 7), float("nan"), device="cuda", dtype=x.dtype)
            w[..., 3:3 + x.shape[3]] = x
            return w[..., 3:3 + x.shape[3]]
        return x.permute(2, 0, 1, 3).contiguous().permute(1, 2, 0, 3)
    for how in range(3):
        q, k, v, dy = (lay(c[n], (how + i) % 3) for i, n in enumerate(("q", "k", "v", "dy")))
        out = lay(torch.zeros_like(a[0]), how)
        b = sim.linear_attn(q, k, v, c["decay"], c["s0"], None, c["scale"], y=out)
        outs = [lay(torch.zeros_like(x), how) for x in ga[:3]]
        gb = sim.linear_attn_grad(q, k, v, c["decay"], dy, c["s0"], c["dstate"], None, c["scale"], *outs)
        sim.sync()
        for x, z in zip((*a, *ga), (*b, *gb)):
            assert torch.equal(x, z), how
    # one sequence's keys and one step's values for all
    k, v = c["k"][:1].expand(3, T, 2, 40), c["v"][:, :1].expand(3, T, 2, 24)
    x = sim.linear_attn(c["q"], k, v, c["decay"], c["s0"], None, c["scale"])
    z = sim.linear_attn(c["q"], k.contiguous(), v.contiguous(), c["decay"], c["s0"], None, c["scale"])
    sim.sync()
    assert all(torch.equal(p, r) for p, r in zip(x, z))


@pytest.mark.parametrize("T", [1, 4, 80, 300])
def test_state_in_place_and_runs_that_follow_each_other(sim, T):
    """A sequence in two calls, the state carried in place, is the sequence in one; ds0 over dstate; y or gradients
    left out change nothing else."""
    d = ac.inputs(2, 2 * T, 2, 1, 64, 64, torch.float32, 7)
    c = cuda(d)
    state = c["s0"].clone()
    y1, st = sim.linear_attn(c["q"][:, :T], c["k"][:, :T], c["v"][:, :T], c["decay"], state, None, c["scale"], state=state)
    y2, _ = sim.linear_attn(c["q"][:, T:], c["k"][:, T:], c["v"][:, T:], c["decay"], state, None, c["scale"], state=state)
    assert st is state
    ds = c["dstate"].clone()
    g = sim.linear_attn_grad(c["q"], c["k"], c["v"], c["decay"], c["dy"], c["s0"], ds, None, c["scale"], ds0=ds)
    h = sim.linear_attn_grad(c["q"], c["k"], c["v"], c["decay"], c["dy"], c["s0"], c["dstate"], None, c["scale"])
    none, only = sim.linear_attn(c["q"], c["k"], c["v"], c["decay"], c["s0"], None, c["scale"], want_y=False)
    sim.sync()
    ac.check_forward(d, torch.cat([y1, y2], 1), state)
    ac.check_grad(d, *g)
    assert g[3] is ds and all(torch.equal(a, b) for a, b in zip(g, h))
    assert none is None
    ac.check_forward(d, None, only)


def test_sizes_of_zero(sim):
    for B, T in ((0, 5), (2, 0), (0, 0)):
        z = lambda h, c: torch.zeros(B, T, h, c, device="cuda")   # noqa: E731
        s0 = torch.randn(B, 2, 8, 8, device="cuda")
        l = torch.full((2,), 0.5, device="cuda")
        y, s = sim.linear_attn(z(2, 8), z(1, 8), z(1, 8), l, s0)
        dq, dk, dv, ds0 = sim.linear_attn_grad(z(2, 8), z(1, 8), z(1, 8), l, z(2, 8), s0, s0)
        sim.sync()
        assert y.shape == (B, T, 2, 8) and torch.equal(s, s0) and torch.equal(ds0, s0)


def test_a_length_of_zero_keeps_the_state(sim):
    d = cuda(ac.inputs(2, 40, 2, 2, 16, 16, torch.bfloat16, 8))
    n = torch.zeros(2, dtype=torch.int32, device="cuda")
    y, s = sim.linear_attn(d["q"], d["k"], d["v"], d["decay"], d["s0"], n, d["scale"])
    g = sim.linear_attn_grad(d["q"], d["k"], d["v"], d["decay"], d["dy"], d["s0"], d["dstate"], n, d["scale"])
    sim.sync()
    assert torch.equal(s, d["s0"]) and torch.equal(g[3], d["dstate"])
    assert not y.any() and not any(x.any() for x in g[:3])


@pytest.mark.parametrize("T", [1, 33, 200])
def test_an_infinity_stays_in_its_sequence(sim, T):
    d = cuda(ac.inputs(3, T, 2, 2, 16, 16, torch.bfloat16, 9))
    d["v"][1, 0, 0, 0] = float("inf")
    y, s = sim.linear_attn(d["q"], d["k"], d["v"], d["decay"], d["s0"], None, d["scale"])
    sim.sync()
    assert y[[0, 2]].isfinite().all() and s[[0, 2]].isfinite().all() and y[1, :, 1].isfinite().all()
    assert not y[1, 0, 0, 0].isfinite()


@pytest.mark.parametrize("dtype,T", [("bf16", 1), ("bf16", 300), ("f32", 70), ("f16", 130)])
def test_repeated_calls_and_graphs(sim, dtype, T):
    """The same bits each time; captured, replayed on new inputs between eager calls."""
    a = cuda(ac.inputs(2, T, 4, 2, 64, 64, TYPES[dtype], 10, lengths=T > 1))
    b = cuda(ac.inputs(2, T, 4, 2, 64, 64, TYPES[dtype], 11, lengths=T > 1))

    def call(d):
        return (*sim.linear_attn(d["q"], d["k"], d["v"], d["decay"], d["s0"], d["lengths"], 0.2),
                *sim.linear_attn_grad(d["q"], d["k"], d["v"], d["decay"], d["dy"], d["s0"], d["dstate"], d["lengths"], 0.2))
    ra, rb = call(a), call(b)
    assert all(torch.equal(x, y) for x, y in zip(ra, call(a)))
    import paper_2607_05272_amd as bs
    st = torch.cuda.Stream()
    with torch.cuda.stream(st), bs.Sim(preset("C1"), n_envs=1, stream=st) as own:
        cur = {k: v.clone() if torch.is_tensor(v) else v for k, v in a.items()}
        st.wait_stream(torch.cuda.default_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            out = (*own.linear_attn(cur["q"], cur["k"], cur["v"], cur["decay"], cur["s0"], cur["lengths"], 0.2),
                   *own.linear_attn_grad(cur["q"], cur["k"], cur["v"], cur["decay"], cur["dy"], cur["s0"], cur["dstate"],
                                         cur["lengths"], 0.2))
        for d, want in ((a, ra), (b, rb), (a, ra)):
            for k, v in d.items():
                if torch.is_tensor(v):
                    cur[k].copy_(v)
            graph.replay()
            st.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(out, want))
            own.linear_attn(b["q"], b["k"], b["v"], b["decay"])
            st.synchronize()


def test_gradient_against_differences(sim):
    """The directional derivative of sum(y dy) + sum(state dstate) along a random direction: both linear in each input
    on its own, so a difference of two calls gives it exactly but for rounding (fp32: 1e-4 of the terms' size)."""
    d = cuda(ac.inputs(1, 50, 2, 1, 24, 20, torch.float32, 12))
    g = sim.linear_attn_grad(d["q"], d["k"], d["v"], d["decay"], d["dy"], d["s0"], d["dstate"], None, d["scale"])
    gen = torch.Generator(device="cuda").manual_seed(1)

    def total(c):
        y, s = sim.linear_attn(c["q"], c["k"], c["v"], c["decay"], c["s0"], None, c["scale"])
        return (y.double() * d["dy"].double()).sum() + (s.double() * d["dstate"].double()).sum()
    for i, n in enumerate(("q", "k", "v", "s0")):
        e = torch.randn(d[n].shape, generator=gen, device="cuda")
        num = (total({**d, n: d[n] + e}) - total({**d, n: d[n] - e})) / 2
        ref = (g[i].double() * e.double()).sum()
        size = (g[i].double().abs() * e.double().abs()).sum() + 1
        assert abs(num - ref) <= 1e-4 * size, n


def test_refusals(sim):
    d = cuda(ac.inputs(2, 8, 4, 2, 16, 16, torch.float32, 13))
    q, k, v, l = d["q"], d["k"], d["v"], d["decay"]
    bad = [((q.double(), k, v, l), {}), ((q, k.bfloat16(), v, l), {}), ((q, k[:, :7], v, l), {}), ((q, k, v, l[:3]), {}),
           ((q, k, v, l.double()), {}), ((q.cpu(), k, v, l), {}), ((q[0], k, v, l), {}), ((q, k, v[:, :, :1], l), {}),
           ((q, k, v, l), dict(s0=d["s0"].bfloat16())), ((q, k, v, l), dict(s0=d["s0"].transpose(2, 3))),
           ((q, k, v, l), dict(lengths=torch.zeros(3, dtype=torch.int32, device="cuda"))),
           ((q, k, v, l), dict(state=d["s0"][:1])), ((q[..., ::2], k[..., ::2], v, l), {})]
    for a, kw in bad:
        with pytest.raises(ValueError):
            sim.linear_attn(*a, **kw)
    import paper_2607_05272_amd as bs
    with pytest.raises(bs.SimError, match="divide"):
        sim.linear_attn(q[:, :, :3], k, v, l[:3].contiguous())
    with pytest.raises(bs.SimError, match="scale"):
        sim.linear_attn(q, k, v, l, scale=float("nan"))
    with pytest.raises(bs.SimError, match="256"):
        w = torch.zeros(1, 2, 1, 257, device="cuda")
        sim.linear_attn(w, w, w, l[:1].contiguous())
    with pytest.raises(bs.SimError, match="share memory"):
        sim.linear_attn(q, k, v, l, y=torch.empty(1, 8, 4, 16, device="cuda").expand(2, 8, 4, 16))
