"""Linear attention, log-probabilities and orthogonalised updates over arrays whose elements lie more than 2^32 elements
apart: the same bits as over adjacent ones."""
import pytest

from workloads import preset

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

FAR = (1 << 32) + 24


@pytest.fixture(scope="module")
def sim():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    if torch.cuda.mem_get_info()[0] < 48 << 30:
        pytest.skip("needs 48 GB of free memory")
    import paper_2607_05272_amd as bs
    with bs.Sim(preset("C1"), n_envs=1) as s:
        yield s


@pytest.fixture(scope="module")
def room():
    """Twice 2^32 elements of 16 bits; what a test leaves outside of its own elements is not looked at."""
    m = torch.empty(2 * FAR + (1 << 26), dtype=torch.bfloat16, device="cuda")
    yield m
    del m


def far(room, x, strides, at):
    """x laid out in room by these strides, from element `at` on"""
    t = room.as_strided(x.shape, strides, at)
    t.copy_(x)
    return t


@pytest.mark.parametrize("T", [1, 3, 40])
def test_linear_attn(sim, room, T):
    B, H, Hk, Dk, Dv = 2, 2, 1, 32, 40
    g = torch.Generator(device="cuda").manual_seed(T)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()   # noqa: E731
    q, k, v, dy = r(B, T, H, Dk), r(B, T, Hk, Dk), r(B, T, Hk, Dv), r(B, T, H, Dv)
    l = torch.tensor([0.9, 0.99], device="cuda")
    n = torch.tensor([T, max(0, T - 2)], dtype=torch.int32, device="cuda")
    want = (*sim.linear_attn(q, k, v, l, lengths=n), *sim.linear_attn_grad(q, k, v, l, dy, lengths=n))
    place = iter(range(0, 1 << 26, 1 << 20))

    def apart(x):    # sequences far apart, or heads
        h, d = x.shape[2:]
        return far(room, x, (FAR, h * d, d, 1) if h == 1 else (T * d, d, FAR, 1), next(place))
    Q, K, V, DY = map(apart, (q, k, v, dy))
    y, dq, dk, dv = map(apart, (dy, q, k, v))
    _, state = sim.linear_attn(Q, K, V, l, lengths=n, y=y)
    _, _, _, ds0 = sim.linear_attn_grad(Q, K, V, l, DY, lengths=n, dq=dq, dk=dk, dv=dv)
    sim.sync()
    for a, b in zip(want, (y, state, dq, dk, dv, ds0)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("A", [3, 40, 500, 2100, 40000])
def test_log_probabilities_of_rows(sim, room, A):
    g = torch.Generator(device="cuda").manual_seed(A)
    l = torch.randn(3, A, generator=g, device="cuda").bfloat16()
    t, w = torch.arange(3, device="cuda"), torch.randn(3, generator=g, device="cuda")
    far_l = far(room, l, (FAR, 1), 5)
    a, ga = sim.token_logprobs(l, t, top=3), sim.token_logprobs_grad(l, t, w, w)
    b, gb = sim.token_logprobs(far_l, t, top=3), sim.token_logprobs_grad(far_l, t, w, w, grad=far_l)
    sim.sync()
    assert all(torch.equal(a[k], b[k]) for k in a) and torch.equal(ga, gb)


@pytest.mark.parametrize("A", [6, 40, 300, 500])
def test_log_probabilities_of_columns(sim, room, A):
    """A column's samples are adjacent, the last columns' beyond 2^32 elements."""
    N, step = 200, (2 * FAR) // A
    g = torch.Generator(device="cuda").manual_seed(A)
    l = torch.randn(A, N, generator=g, device="cuda").bfloat16().t()
    t, w = torch.arange(N, device="cuda") % A, torch.randn(N, generator=g, device="cuda")
    far_l = far(room, l, (1, step), 7)
    a, ga = sim.token_logprobs(l, t, top=3), sim.token_logprobs_grad(l, t, w, w)
    b, gb = sim.token_logprobs(far_l, t, top=3), sim.token_logprobs_grad(far_l, t, w, w, grad=far_l)
    sim.sync()
    assert all(torch.equal(a[k], b[k]) for k in a) and torch.equal(ga, gb)


def test_orthogonalize(sim, room):
    g = torch.Generator(device="cuda").manual_seed(1)
    u = torch.randn(2, 3, 70, generator=g, device="cuda").bfloat16()
    want = sim.orthogonalize(u)
    rows = far(room, u, (100, FAR, 1), 1)
    b = sim.orthogonalize(rows)
    sim.orthogonalize(u, out=rows)
    apart = far(room, u, (FAR, 70, 1), 1 << 20)
    c = sim.orthogonalize(apart, out=apart)
    sim.sync()
    assert torch.equal(b, want) and torch.equal(rows, want) and c is apart and torch.equal(c, want)
