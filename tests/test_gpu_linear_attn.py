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


def reference(d, grad=True):
    """The steps taken by torch in fp64 on the GPU: y, state and (dq, dk, dv, ds0), with the sums of their terms'
    magnitudes."""
    def run(q, k, v, l, dy, s0, ds, n, scale):
        B, T, H, Dk = q.shape
        g = H // k.shape[2]
        S, G = s0.clone(), ds.clone()
        l = l[:, None, None]
        y, dq = torch.zeros_like(dy), torch.zeros_like(q)
        dk, dv = torch.zeros_like(q), torch.zeros_like(dy)
        for t in range(T):
            on = (t < n)[:, None, None, None]
            kt, vt = k[:, t].repeat_interleave(g, 1), v[:, t].repeat_interleave(g, 1)
            S = torch.where(on, l * S + kt[..., None] * vt[..., None, :], S)
            y[:, t] = torch.where(on[..., 0], scale * (q[:, t][..., None] * S).sum(2), 0.0)
            dq[:, t] = torch.where(on[..., 0], scale * (S * dy[:, t][..., None, :]).sum(3), 0.0)
        for t in reversed(range(T) if grad else range(0)):
            on = (t < n)[:, None, None, None]
            kt, vt = k[:, t].repeat_interleave(g, 1), v[:, t].repeat_interleave(g, 1)
            Gt = G + scale * q[:, t][..., None] * dy[:, t][..., None, :]
            dk[:, t] = torch.where(on[..., 0], (Gt * vt[..., None, :]).sum(3), 0.0)
            dv[:, t] = torch.where(on[..., 0], (Gt * kt[..., None]).sum(2), 0.0)
            G = torch.where(on, l * Gt, G)
        share = lambda x: x.unflatten(2, (H // g, g)).sum(3)   # noqa: E731
        return y, S, dq, share(dk), share(dv), G
    a = [d[x].double() for x in ("q", "k", "v", "decay", "dy", "s0", "dstate")]
    n = d["lengths"] if d["lengths"] is not None else torch.full((d["q"].shape[0],), d["q"].shape[1], device="cuda")
    return run(*a, n, d["scale"]), run(*(x.abs() for x in a), n, abs(d["scale"]))


@pytest.mark.parametrize("dtype", ["bf16", "f32", "f16"])
@pytest.mark.parametrize("B,T,H,Hk,Dk,Dv,lengths", [
    (2, 2500, 2, 1, 64, 64, True), (1, 3000, 1, 1, 128, 128, False), (1, 1111, 3, 1, 200, 96, False), (3, 700, 2, 2, 48, 130, True),
    (40, 70, 4, 2, 64, 64, True), (100, 40, 4, 4, 128, 128, False), (70, 100, 4, 1, 100, 120, True), (130, 33, 3, 3, 64, 40, True),
    (5, 600, 1, 1, 256, 256, True), (7000, 20, 2, 1, 8, 8, True), (30000, 3, 1, 1, 16, 16, True)])
def test_segments_and_many_sequences(sim, B, T, H, Hk, Dk, Dv, lengths, dtype):
    """Every form of a run: time in segments, 64 and 128 columns, halves, more sequences than the chip holds."""
    if B * T * H * max(Dk, Dv) > 1 << 22 and dtype == "f16":
        pytest.skip("the types share their forms")
    d = cuda(ac.inputs(B, T, H, Hk, Dk, Dv, TYPES[dtype], T, lengths=lengths))
    y, state = sim.linear_attn(d["q"], d["k"], d["v"], d["decay"], d["s0"], d["lengths"], d["scale"])
    g = sim.linear_attn_grad(d["q"], d["k"], d["v"], d["decay"], d["dy"], d["s0"], d["dstate"], d["lengths"], d["scale"])
    sim.sync()
    want, size = reference(d)
    D = max(Dk, Dv) + H // Hk
    for name, got, w, m in zip(("y", "state", "dq", "dk", "dv", "ds0"), (y, state, *g), want, size):
        e = ac._loss(got.dtype, T, D)
        tol = e * m + torch.finfo(got.dtype).eps / 2 * w.abs() + torch.finfo(got.dtype).smallest_normal * torch.finfo(got.dtype).eps
        off = ~((got.double() - w).abs() <= tol)
        assert not off.any(), (name, int(off.sum()), off.nonzero()[0].tolist())


def test_single_outputs_of_the_entry_points(sim):
    """Through the C entry points: each gradient alone is what it is with the others; nothing else is read or written."""
    import ctypes as C
    from paper_2607_05272_amd import _lib as L
    from paper_2607_05272_amd.sim import _heads
    for T in (5, 100, 700):
        d = cuda(ac.inputs(2, T, 4, 2, 32, 48, torch.bfloat16, 15))
        all_of = sim.linear_attn_grad(d["q"], d["k"], d["v"], d["decay"], d["dy"], d["s0"], d["dstate"], None, d["scale"])
        sizes = L.SimLinearAttn(2, T, 4, 2, 32, 48, 2, d["scale"])
        for i in range(4):
            out = [torch.empty_like(x) if j == i else None for j, x in enumerate(all_of)]
            ptr = lambda x: None if x is None else x.data_ptr()   # noqa: E731
            q = d["q"] if i else None                  # q is not needed for dq, k not for dk, v not for dv and ds0
            k = d["k"] if i in (0, 2) else None
            v = d["v"] if i in (0, 1) else None
            sim._call("linear_attn_grad", sizes, _heads(q), _heads(k), _heads(v), ptr(d["decay"]), _heads(d["dy"]), None, ptr(d["s0"]),
                      ptr(d["dstate"]), _heads(out[0]), _heads(out[1]), _heads(out[2]), ptr(out[3]))
            sim.sync()
            assert torch.equal(out[i], all_of[i]), (T, i)
    assert C.sizeof(L.SimHeads) == 32


def test_from_another_stream(sim):
    """Called while another stream is current: ordered after its work, and its later work after the call."""
    d = ac.inputs(2, 300, 2, 2, 64, 64, torch.float32, 16)
    c = cuda(d)
    want = sim.linear_attn(c["q"], c["k"], c["v"], c["decay"], c["s0"], None, c["scale"])
    sim.sync()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        st.wait_stream(torch.cuda.default_stream())
        for _ in range(3):
            big = torch.randn(4096, 4096, device="cuda")
            for _ in range(8):
                big = big @ big * 1e-3             # keeps the stream busy before the inputs are there
            q = c["q"] + 0.0 * big[0, 0].nan_to_num(0.0, 0.0, 0.0)
            y, s = sim.linear_attn(q, c["k"], c["v"], c["decay"], c["s0"], None, c["scale"])
            copy = y.clone()
            st.synchronize()
            assert torch.equal(copy, want[0]) and torch.equal(s, want[1])


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


@pytest.mark.parametrize("dtype", ["bf16", "f32", "f16"])
@pytest.mark.parametrize("T,Dk,Dv", [(9, 16, 24), (150, 16, 24), (150, 96, 40), (90, 128, 128), (70, 200, 40)])
def test_what_is_not_finite_reaches_only_what_it_is_part_of(sim, T, Dk, Dv, dtype):
    """An infinity or NaN in a live step: results that the formulas make without it are what they are without
    it (the steps before it above all), the others are not finite."""
    d = ac.inputs(2, T, 2, 2, Dk, Dv, TYPES[dtype], 17)

    def call(d):
        c = cuda(d)
        y, s = sim.linear_attn(c["q"], c["k"], c["v"], c["decay"], c["s0"], None, c["scale"])
        g = sim.linear_attn_grad(c["q"], c["k"], c["v"], c["decay"], c["dy"], c["s0"], c["dstate"], None, c["scale"])
        sim.sync()
        return [x.cpu() for x in (y, s, *g)]
    clean = call(d)
    for i, name in enumerate(("q", "k", "v", "dy")):
        e = dict(d)
        e[name] = d[name].clone()
        e[name][1, (2 * T) // 3, 1, 3] = float("nan") if i % 2 else float("inf")
        a = [e[n].double().numpy() for n in ("q", "k", "v", "decay", "dy", "s0", "dstate")]
        with np.errstate(invalid="ignore"):
            want = (*ops.linear_attn(*a[:4], a[5], None, d["scale"]), *ops.linear_attn_grad(*a, None, d["scale"]))
        got = call(e)
        mixed = []
        for x, w, c in zip(got, want, clean):
            free = torch.from_numpy(np.isfinite(w))
            assert not x[~free].isfinite().any(), name
            mixed.append(torch.where(free, x, c))
        ac.check_forward(d, *mixed[:2])
        ac.check_grad(d, *mixed[2:])


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
