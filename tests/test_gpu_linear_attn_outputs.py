"""linear_attn_grad with some of its outputs alone, through the C entry point: what is out of range is told whichever of
them are wanted, and time in segments whose number differs between dk's and dv's passes gives what the formulas do."""
import pytest

from workloads import preset

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import attn_check as ac   # noqa: E402
from scan_check import TYPES   # noqa: E402
from test_gpu_linear_attn import cuda, reference   # noqa: E402

NAMES = ("dq", "dk", "dv", "ds0")


@pytest.fixture(scope="module")
def sim():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2607_05272_amd as bs
    with bs.Sim(preset("C1"), n_envs=1) as s:
        yield s


def grad_of(sim, d, want, ds0=None):
    """{name: gradient} of the wanted ones; the inputs that none of them needs are absent."""
    from paper_2607_05272_amd import _lib as L
    from paper_2607_05272_amd.sim import _FLOAT, _heads
    q, k, v = d["q"], d["k"], d["v"]
    B, T, H, Dk = q.shape
    out = {n: torch.full_like(x, float("nan")) for n, x in zip(NAMES, (q, k, v, d["s0"])) if n in want}
    if ds0 is not None:
        out["ds0"] = ds0
    sizes = L.SimLinearAttn(B, T, H, k.shape[2], Dk, v.shape[3], _FLOAT[q.dtype], d["scale"])
    ptr = lambda x: None if x is None else x.data_ptr()   # noqa: E731
    some = lambda x, *names: _heads(x if any(n in want for n in names) else None)   # noqa: E731
    sim._call("linear_attn_grad", sizes, some(q, "dk", "dv", "ds0"), some(k, "dq", "dv"), some(v, "dq", "dk"), ptr(d["decay"]),
              _heads(d["dy"]), ptr(d["lengths"]), ptr(d["s0"]), ptr(d["dstate"]), *(_heads(out.get(n)) for n in NAMES[:3]),
              ptr(out.get("ds0")))
    return out


@pytest.mark.parametrize("T", [3, 70, 700])
@pytest.mark.parametrize("want", [("dq",), ("dk",), ("dv",), ("ds0",), ("dk", "dv"), ("dv", "ds0"), NAMES])
def test_what_is_out_of_range_is_told_with_any_outputs(sim, T, want):
    good = cuda(ac.inputs(3, T, 3, 3, 32, 48, torch.float32, 5, lengths=True))
    first = grad_of(sim, good, want)
    sim.sync()
    for name, bad, as_if, what in (
            ("lengths", [T + 1, -1, 1], [T, 0, 1], "sequence length out of range"),
            ("decay", [1.5, -0.25, float("nan")], [1.0, 0.0, 0.0], "decay out of range")):
        d = dict(good)
        d[name] = torch.tensor(bad, dtype=good[name].dtype, device="cuda")
        got = grad_of(sim, d, want)
        with pytest.raises(Exception, match=what):
            sim.sync()
        d[name] = torch.tensor(as_if, dtype=good[name].dtype, device="cuda")
        same = grad_of(sim, d, want)
        sim.sync()
        assert all(torch.equal(got[n], same[n]) for n in want)
    again = grad_of(sim, good, want)
    sim.sync()
    assert all(torch.equal(first[n], again[n]) for n in want)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("B,T,H,Hk,Dk,Dv", [(16, 600, 4, 2, 64, 256), (16, 600, 4, 1, 256, 64), (5, 900, 6, 3, 200, 40)])
def test_passes_of_differing_segments(sim, B, T, H, Hk, Dk, Dv, dtype):
    """Wide keys and narrow values, and the other way round; each output alone is what it is with the others."""
    d = cuda(ac.inputs(B, T, H, Hk, Dk, Dv, TYPES[dtype], T, lengths=True))
    ds = d["dstate"].clone()
    g = sim.linear_attn_grad(d["q"], d["k"], d["v"], d["decay"], d["dy"], d["s0"], ds, d["lengths"], d["scale"], ds0=ds)
    assert g[3] is ds
    alone = [grad_of(sim, d, (n,))[n] for n in NAMES]
    over = d["dstate"].clone()
    grad_of(sim, dict(d, dstate=over), ("ds0",), ds0=over)
    y, state = sim.linear_attn(d["q"], d["k"], d["v"], d["decay"], d["s0"], d["lengths"], d["scale"])
    sim.sync()
    for n, a, b in zip(NAMES, g, alone):
        assert torch.equal(a, b), n
    assert torch.equal(over, ds)
    want, size = reference(d)
    D = max(Dk, Dv) + H // Hk
    for name, got, w, m in zip(("y", "state", *NAMES), (y, state, *g), want, size):
        f = torch.finfo(got.dtype)
        tol = ac._loss(got.dtype, T, D) * m + f.eps / 2 * w.abs() + f.smallest_normal * f.eps
        off = ~((got.double() - w).abs() <= tol)
        assert not off.any(), (name, int(off.sum()), off.nonzero()[0].tolist())
