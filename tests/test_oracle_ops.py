"""The plain forms of the operators (oracle/ops.py): gradients against central differences of the
losses they belong to, and against torch autograd in fp64."""
import numpy as np
import pytest
import torch

from oracle import ops


def differences(f, x, h=1e-6):
    g = np.zeros_like(x)
    it = np.nditer(x, flags=["multi_index"])
    for _ in it:
        i = it.multi_index
        x0 = x[i]
        x[i] = x0 + h
        up = f()
        x[i] = x0 - h
        down = f()
        x[i] = x0
        g[i] = (up - down) / (2 * h)
    return g


@pytest.mark.parametrize("kind", ["linear", "sigmoid"])
@pytest.mark.parametrize("reverse", [False, True])
def test_scan_gradient(kind, reverse):
    r = np.random.default_rng(1)
    B, T, D = 3, 5, 2
    gate, x, dy = (r.normal(size=(B, T, D)) for _ in range(3))
    h0, ds = r.normal(size=(B, D)), r.normal(size=(B, D))
    n = np.array([5, 3, 0])

    def loss():
        y, h = ops.gated_scan(gate, x, h0, n, kind, reverse)
        return (y * dy).sum() + (h * ds).sum()
    y, h = ops.gated_scan(gate, x, h0, n, kind, reverse)
    assert (y[1, 3:] == 0).all() and (y[2] == 0).all() and (h[2] == h0[2]).all()
    dg, dx, dh0 = ops.gated_scan_grad(gate, x, y, dy, h0, ds, n, kind, reverse)
    for a, g in ((gate, dg), (x, dx), (h0, dh0)):
        np.testing.assert_allclose(g, differences(loss, a), rtol=1e-6, atol=1e-8)


def test_scan_is_the_returns_recurrence():
    import oracle
    r = np.random.default_rng(2)
    T, E = 40, 3
    rew, v = r.normal(size=(T, E)), r.normal(size=(T + 1, E)).astype(np.float32)
    adv, _ = oracle.gae(rew, v, 0.99, 0.95)
    v = v.astype(np.float64)
    delta = rew + 0.99 * v[1:] - v[:-1]
    y, _ = ops.gated_scan(np.full((1, T, E), 0.99 * 0.95), delta[None], reverse=True)
    np.testing.assert_allclose(y[0], adv, rtol=1e-12, atol=1e-12)


@pytest.mark.parametrize("masked", [False, True])
def test_policy_loss_gradient(masked):
    r = np.random.default_rng(3)
    N, A = 6, 5
    z, adv = r.normal(size=(N, A)) * 2, r.normal(size=N)
    act = r.integers(0, A, N)
    mask = r.random((N, A)) < 0.6
    mask[np.arange(N), act] = True
    mask[4] = False
    w = r.random(N)
    w[1] = 0.0
    kw = dict(mask=mask if masked else None, weight=w, c_kl=0.3, c_entropy=0.2)
    lp = np.array([p["ls"][a] if p else 0.0 for p, a in
                   zip(ops.policy_loss(z, act, adv, **kw)["parts"], act)])
    rho = np.array([0.9, 1.5, 0.6, 1.1, 1.0, 1.4])     # inside and outside the clip range
    old, ref = lp - np.log(rho), lp + r.normal(size=N) * 0.5
    got = ops.policy_loss(z, act, adv, old, ref, **kw)
    want = differences(lambda: ops.policy_loss(z, act, adv, old, ref, **kw)["loss"][0], z)
    np.testing.assert_allclose(got["grad"], want, rtol=1e-6, atol=1e-9)
    t = torch.tensor(z, requires_grad=True)
    tm = torch.tensor(mask) if masked else torch.ones(N, A, dtype=torch.bool)
    keep = torch.tensor(w != 0) & tm.any(1)
    ls = torch.log_softmax(t.masked_fill(~tm, -torch.inf)[keep], 1)
    a = torch.tensor(act)[keep, None]
    l = ls.gather(1, a)[:, 0]
    rt = torch.exp(l - torch.tensor(old)[keep])
    ad, d = torch.tensor(adv)[keep], torch.tensor(ref)[keep] - l
    lsf = ls.masked_fill(~tm[keep], 0.0)
    loss = (torch.tensor(w)[keep] * (-torch.minimum(rt * ad, rt.clamp(0.8, 1.2) * ad)
                                     + 0.3 * (torch.exp(d) - d - 1)
                                     + 0.2 * (torch.exp(ls) * lsf).sum(1))).sum()
    loss.backward()
    np.testing.assert_allclose(got["loss"][0], loss.item(), rtol=1e-12)
    np.testing.assert_allclose(got["grad"], t.grad.numpy(), rtol=1e-9, atol=1e-12)


@pytest.mark.parametrize("group,k", [(1, 2), (3, 1)])
def test_balance_gradient(group, k):
    r = np.random.default_rng(4)
    N, A = 7, 6
    z = r.normal(size=(N, A))
    idx = r.integers(0, A, (N, k))
    live = np.array([1, 1, 0, 1, 1, 0, 1])
    got = ops.balance_loss(z, idx, live, group, 0.7)
    assert got["counts"].sum() == k * 5
    want = differences(lambda: ops.balance_loss(z, idx, live, group, 0.7)["loss"], z)
    np.testing.assert_allclose(got["grad"], want, rtol=1e-6, atol=1e-9)
    # every target equally often and equally likely: the loss's value is coef
    even = np.tile(np.arange(A), (A, 1)).T[:, :1]
    np.testing.assert_allclose(ops.balance_loss(np.zeros((A, A)), even, coef=0.7)["loss"], 0.7)


def test_a_reference_without_its_coefficient_tells_the_kl_term_alone():
    """c_kl = 0 with a reference that forbids an action (-inf) or is far above it: the KL term is infinite or
    huge, loss, policy term and gradient are those of a call without a reference."""
    r = np.random.default_rng(5)
    z, adv, act = r.normal(size=(4, 5)), r.normal(size=4), np.array([0, 1, 2, 3])
    for ref in (np.array([-np.inf, -1.0, 0.0, -2.0]), np.array([1000.0, -1.0, 0.0, -2.0])):
        with np.errstate(over="ignore"):
            got = ops.policy_loss(z, act, adv, logp_ref=ref, c_entropy=0.1)
        want = ops.policy_loss(z, act, adv, c_entropy=0.1)
        assert got["loss"][2] == np.inf
        np.testing.assert_array_equal(got["loss"][[0, 1, 3]], want["loss"][[0, 1, 3]])
        np.testing.assert_array_equal(got["grad"], want["grad"])
