"""orthogonalize against the fp64 form (oracle/ops.py).

Bound: with e_i the error that step i adds to X (Frobenius norm) and L_i how far the steps after it stretch a small
change of X_i, the result is off by at most sum e_i L_i, to first order (10% more for the rest). L_i is exact: in the
singular vectors of X_i a change's symmetric part is multiplied by (f(s) - f(t)) / (s - t) (f'(s) on the diagonal),
its other part by (f(s) + f(t)) / (s + t), f the remaining steps' map of singular values. e_i: a value held in
parts is off by r (2^-11 in one fp16 part, 2^-22 in two) of itself and 2^-35 (half the smallest fp16 number times 2^-10)
at most, a sum of K products by (K + 4) 2^-24 of the sum of their magnitudes (one part), plus for two parts 2^-22 of it
(the product of two second parts that is left out)."""
import numpy as np
import pytest

from workloads import preset

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import ops    # noqa: E402
from scan_check import TYPES, rounding   # noqa: E402

U, NS = 2.0 ** -24, (3.4445, -4.7750, 2.0315)


@pytest.fixture(scope="module")
def sim():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2607_05272_amd as bs
    with bs.Sim(preset("C1"), n_envs=1) as s:
        yield s


def fro(x):
    return np.sqrt((x * x).sum())


def stretch(s, coeffs, steps):
    """The largest factor on a change of X with singular values s, over `steps` steps."""
    a, b, c = coeffs
    f, d = s.copy(), np.ones_like(s)
    for _ in range(steps):
        d = d * (a + 3 * b * f ** 2 + 5 * c * f ** 4)
        f = a * f + b * f ** 3 + c * f ** 5
    gap = s[:, None] - s[None]
    close = np.abs(gap) < 1e-7
    sym = np.where(close, np.abs(d[:, None]), np.abs(f[:, None] - f[None]) / np.where(close, 1.0, np.abs(gap)))
    tot = s[:, None] + s[None]
    low = tot < 1e-7
    skew = np.where(low, abs(a) ** steps, np.abs(f[:, None] + f[None]) / np.where(low, 1.0, tot))
    return max(1.0, sym.max(), skew.max(), abs(a) ** steps)


def bound(way, coeffs, two):
    a, b, c = (abs(x) for x in coeffs)
    r = 2.0 ** -22 if two else 2.0 ** -11
    tiny = 2.0 ** -35
    left = 2.0 ** -22 if two else 0.0
    total = 0.0
    steps = len(way) - 1
    for i in range(steps):
        x, ax = way[i], np.abs(way[i])
        R, C = x.shape
        A = x @ x.T
        nA, nX = np.linalg.norm(A, 2), np.linalg.norm(x, 2)
        B = coeffs[1] * A + coeffs[2] * A @ A
        root = np.sqrt(R * R)
        eA = ((C + 4) * U + left) * fro(ax @ ax.T) + r * fro(A) + tiny * root
        eB = (b + 2 * c * nA) * eA + c * ((R + 4) * U + left) * fro(np.abs(A) @ np.abs(A)) + 4 * U * (b * fro(A) + c * fro(A @ A)) \
            + r * fro(B) + tiny * root
        e = eB * nX + ((R + 4) * U + left) * fro(np.abs(B) @ ax) + 4 * U * (a * fro(x) + fro(B @ x))
        s = np.linalg.svd(way[i + 1], compute_uv=False)
        e += r * fro(way[i + 1]) + tiny * np.sqrt(x.size)
        total += e * stretch(s, coeffs, steps - 1 - i)
    s = np.linalg.svd(way[0], compute_uv=False)
    total += (r * fro(way[0]) + 4 * U * fro(way[0]) + tiny * np.sqrt(way[0].size)) * stretch(s, coeffs, steps)
    return 1.1 * total


def check(sim, u, **kw):
    d = u.cuda()
    got = sim.orthogonalize(d, **kw)
    sim.sync()
    assert got.dtype == u.dtype and got.shape == u.shape
    many = u if u.dim() == 3 else u[None]
    for x, y in zip(many, got.double().cpu().numpy().reshape(many.shape)):
        want, way = ops.orthogonalize(x.double().numpy(), **{k: v for k, v in kw.items() if k != "out"})
        e = bound(way, kw.get("coeffs", NS), u.dtype != torch.bfloat16) * abs(kw.get("scale", 1.0))
        e += fro(rounding(want, u.dtype))
        assert fro(y - want) <= e, (fro(y - want), e, fro(want))
    return got


def update(n, M, N, dtype, seed, scale=1e-3):
    g = torch.Generator().manual_seed(seed)
    r = max(1, min(M, N) // 8)
    u = torch.randn(n, M, r, generator=g) @ torch.randn(n, r, N, generator=g) * r ** -0.5 + 0.5 * torch.randn(n, M, N, generator=g)
    return (u * scale).to(dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,M,N", [(1, 1, 1), (2, 1, 9), (3, 7, 5), (1, 16, 16), (2, 33, 65), (1, 64, 200), (2, 130, 96), (1, 128, 128),
                                   (1, 96, 257), (1, 300, 129), (1, 256, 256)])
def test_sizes(sim, n, M, N, dtype):
    check(sim, update(n, M, N, TYPES[dtype], M + N))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_larger(sim, dtype):
    got = check(sim, update(1, 520, 700, TYPES[dtype], 5))
    s = np.linalg.svd(got[0].double().cpu().numpy(), compute_uv=False)
    assert 0.5 < s.min() and s.max() < 1.3


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,M,N", [(94, 256, 256), (43, 512, 600), (1, 64, 4000), (2, 2100, 130), (1, 200, 1100)])
def test_tiles_and_shares(sim, n, M, N, dtype):
    """Batches that are given the larger tiles, and few rows of many columns, whose sums are shared by workgroups: one
    matrix n times, so every result is the first one's."""
    u = update(1, M, N, TYPES[dtype], M)
    d = u.cuda().expand(n, M, N)
    got = sim.orthogonalize(d)
    sim.sync()
    assert all(torch.equal(got[i], got[0]) for i in range(1, n))
    want, way = ops.orthogonalize(u[0].double().numpy())
    e = bound(way, NS, dtype != "bf16") + fro(rounding(want, u.dtype))
    assert fro(got[0].double().cpu().numpy() - want) <= e


@pytest.mark.parametrize("steps", [0, 1, 2, 7])
def test_steps_coefficients_and_scale(sim, steps):
    check(sim, update(2, 40, 70, torch.float32, 7), steps=steps, scale=0.25)
    check(sim, update(1, 70, 40, torch.float32, 8), steps=steps, coeffs=(1.5, -0.5, 0.0), eps=0.0)
    check(sim, update(1, 48, 48, torch.bfloat16, 9), steps=steps, coeffs=(1.875, -1.25, 0.375), scale=-2.0)


def test_strides_in_place_and_repeats(sim):
    u = update(3, 40, 72, torch.float32, 10).cuda()
    a = sim.orthogonalize(u)
    t = u.transpose(1, 2).contiguous().transpose(1, 2)
    b = sim.orthogonalize(t)
    wide = torch.full((3, 50, 90), float("nan"), device="cuda")
    wide[:, 5:45, 11:83] = u
    out = torch.full((3, 50, 90), 7.0, device="cuda")
    c = sim.orthogonalize(wide[:, 5:45, 11:83], out=out[:, 5:45, 11:83])
    d = torch.empty(40, 3, 72, device="cuda").transpose(0, 1)
    sim.orthogonalize(u, out=d)
    one = sim.orthogonalize(u[1])
    e = u[:1].expand(3, 40, 72)
    same = u.clone()
    f = sim.orthogonalize(same, out=same)
    rows = sim.orthogonalize(e)
    sim.sync()
    assert f is same and all(torch.equal(a, x) for x in (b, c, d, f)) and torch.equal(one, a[1])
    assert all(torch.equal(rows[i], a[0]) for i in range(3))
    out[:, 5:45, 11:83] = 7.0
    assert (out == 7.0).all()
    # tall: the transposed wide one, bit for bit
    assert torch.equal(sim.orthogonalize(u.transpose(1, 2).contiguous()), a.transpose(1, 2))


def test_zeros_tiny_huge_and_not_finite(sim):
    u = torch.zeros(5, 24, 40)
    u[1] = update(1, 24, 40, torch.float32, 11)[0] * 1e-30
    u[2] = update(1, 24, 40, torch.float32, 12)[0] * 1e30
    u[3] = update(1, 24, 40, torch.float32, 13)[0]
    u[3, 2, 5] = float("nan")
    u[4] = update(1, 24, 40, torch.float32, 14)[0]
    u[4, 0, 0] = float("inf")
    r = sim.orthogonalize(u.cuda())
    sim.sync()
    assert not r[0].any() and r[3].isnan().all() and r[4].isnan().all()
    check(sim, u[2])
    # below eps the norm counts for little: X = U / eps
    want, _ = ops.orthogonalize(u[1].double().numpy())
    assert np.abs(r[1].double().cpu().numpy() - want).max() <= 1e-3 * np.abs(want).max() + 3.4445 ** 5 * 2.0 ** -35
    check(sim, u[1], eps=0.0)
    assert not sim.orthogonalize(torch.zeros(4, 6, device="cuda"), eps=0.0).any()


def test_graphs(sim):
    import paper_2607_05272_amd as bs
    a, b = (update(2, 100, 150, torch.bfloat16, s).cuda() for s in (15, 16))
    ra, rb = sim.orthogonalize(a), sim.orthogonalize(b)
    st = torch.cuda.Stream()
    with torch.cuda.stream(st), bs.Sim(preset("C1"), n_envs=1, stream=st) as own:
        st.wait_stream(torch.cuda.default_stream())
        cur = a.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            out = own.orthogonalize(cur)
        for x, want in ((a, ra), (b, rb), (a, ra)):
            cur.copy_(x)
            graph.replay()
            st.synchronize()
            assert torch.equal(out, want)
            own.orthogonalize(b)
            st.synchronize()


def test_sizes_of_zero_and_refusals(sim):
    import paper_2607_05272_amd as bs
    for s in ((0, 4, 5), (2, 0, 5), (2, 4, 0), (0, 0)):
        assert sim.orthogonalize(torch.zeros(s, device="cuda")).shape == s
    u = torch.randn(4, 6, device="cuda")
    for bad, kw in ((u.double(), {}), (u.cpu(), {}), (u[0], {}), (u, dict(out=u.t())), (u, dict(out=u.bfloat16()))):
        with pytest.raises(ValueError):
            sim.orthogonalize(bad, **kw)
    for kw, what in ((dict(steps=-1), "steps"), (dict(steps=33), "steps"), (dict(eps=-1.0), "eps"), (dict(scale=float("inf")), "finite"),
                     (dict(coeffs=(1.0, float("nan"), 0.0)), "finite"), (dict(out=torch.empty(1, 6, device="cuda").expand(4, 6)), "share memory")):
        with pytest.raises(bs.SimError, match=what):
            sim.orthogonalize(u, **kw)
    sim.sync()
