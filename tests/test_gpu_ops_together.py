"""The operators as a training program uses them together, and at sizes where their kernels' workgroups go
round their loops: the policy's own logits through the losses against the built-in minibatch
gradient, advantages by the recurrence, many rows and many sequences."""
import numpy as np
import pytest

from workloads import preset

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import loss_check as lc   # noqa: E402
import scan_check as sc   # noqa: E402
from oracle import ops    # noqa: E402


@pytest.fixture(scope="module")
def bs():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2607_05272_amd as m
    m.load()
    return m


def test_policy_update_from_its_logits(bs):
    """A rollout's advantages by gated_scan, then the policy's logits on a PPO minibatch through
    policy_loss: the sum of its gradient over the samples is the minibatch gradient of the output
    layer's bias, and its terms are the minibatch's. Both are fp32 forwards of the same network whose
    sums run in other orders (a logit off by some 1e-6), so 1e-5 of the sum of magnitudes."""
    w = preset("C1", value_head=1)
    E, T, M, A, ch = 256, 16, 1024, 6, 0.01
    with bs.Sim(w, n_envs=E) as sim, bs.Sim(w, n_envs=M) as net:
        wts = sim.init_weights(7)
        sim.reset(11)
        tr = sim.rollout(wts, T, store_obs=True)
        v = tr.value.double()
        delta = (tr.reward + 0.99 * v[1:]) - v[:-1]
        gate = torch.full((T, E), 0.99 * 0.95, dtype=torch.float64, device="cuda")
        adv, _ = sim.gated_scan(gate, delta, reverse=True)
        ref, ret = sim.returns_gae(tr.reward, tr.value, 0.99, 0.95)
        sim.sync()
        np.testing.assert_allclose(adv.cpu().numpy(), ref.cpu().numpy(), rtol=1e-11, atol=1e-9)
        # old log-probabilities of another policy, so that ratios spread over the clip range
        old = tr.logp + 0.2 * torch.randn(T, E, generator=torch.Generator().manual_seed(1)).cuda()
        adv = (adv - adv.mean()) / adv.std()
        g, loss, idx = sim.ppo_minibatch_grad(wts, tr.obs, tr.actions, old, adv, ret, M, 5, c_entropy=ch,
                                              want_index=True)
        t, e = idx // E, idx % E
        net.reset(1)
        logits = net.policy(wts, tr.obs[t, :, e].t().contiguous(), 0, want_logits=True)["logits"][:A].t()
        r = sim.policy_loss(logits, tr.actions[t, e], adv[t, e], logp_old=old[t, e], c_entropy=ch)
        b = sim.balance_loss(logits, tr.actions[t, e][:, None], group=6, coef=0.1)
        sim.sync()
        net.sync()
        b3 = sim.unflatten_grads(g.cpu().numpy())["b3"][:A]
        size = r["grad"].abs().double().sum(0).cpu().numpy()
        assert (np.abs(b3 - r["grad"].double().sum(0).cpu().numpy()) <= 1e-5 * size).all()
        got, want = r["loss"].double().cpu().numpy(), loss.cpu().numpy()
        np.testing.assert_allclose(got[1], want[1], rtol=1e-4, atol=1e-5)
        np.testing.assert_allclose(-ch * got[3], want[3], rtol=1e-4)
        # one server: every choice falls on it, and there is nothing to balance
        assert b["counts"].tolist() == [M] and abs(b["loss"].item() - 0.1) < 1e-6
        assert b["grad"].abs().max().item() < 1e-9


def test_recurrent_policy_step(bs):
    """A recurrent policy over padded episodes in bf16: states by gated_scan, logits of them, both losses on
    the same logits (the second written over a copy in place), the gradient back through the recurrence."""
    g = torch.Generator().manual_seed(2)
    B, T, D, A = 6, 90, 40, 24
    n = torch.tensor([90, 0, 1, 50, 89, 30], dtype=torch.int32)
    gate, x = (torch.randn(B, T, D, generator=g).bfloat16() for _ in range(2))
    head = torch.randn(D, A, generator=g) * 0.3
    act = torch.randint(0, A, (B * T,), generator=g)
    adv = torch.randn(B * T, generator=g)
    live = (torch.arange(T)[None] < n[:, None]).reshape(-1)
    weight = live.float() / live.sum()
    with bs.Sim(preset("C1"), n_envs=1) as sim:
        y, h = sim.gated_scan(gate.cuda(), x.cuda(), lengths=n.cuda(), kind="sigmoid")
        logits = y.float().reshape(B * T, D) @ head.cuda()
        pol = sim.policy_loss(logits, act.cuda(), adv.cuda(), weight=weight.cuda(), c_entropy=0.02)
        both = logits.clone()
        bal = sim.balance_loss(both, act.cuda()[:, None], live=live.cuda(), group=6, coef=0.5, grad=both)
        dl = pol["grad"] + bal["grad"]
        dy = (dl @ head.cuda().t()).reshape(B, T, D).bfloat16()
        dg, dx, dh0 = sim.gated_scan_grad(gate.cuda(), x.cuda(), y, dy, lengths=n.cuda(), kind="sigmoid")
        sim.sync()
    d = dict(gate=gate, x=x, dy=dy.cpu(), h0=None, dstate=None, lengths=n)
    sc.check_forward(d, y, h, "sigmoid", False)
    sc.check_grad(d, y, dg, dx, dh0, "sigmoid", False)
    z = logits.double().cpu().numpy()
    want = ops.policy_loss(z, act.numpy(), adv.numpy(), weight=weight.numpy(), c_entropy=0.02)
    s = dict(actions=act.numpy(), weight=weight.numpy(), adv=adv.numpy(), old=None, ref=None)
    lc.check_policy(s, pol, want, 0.0, 0.02, torch.float32)
    wb = ops.balance_loss(z, act.numpy()[:, None], live.numpy(), 6, 0.5)
    lc.check_balance(bal, wb, z, live.numpy(), 6, 0.5, torch.float32)
    assert (dl[~live.cuda()] == 0).all() and (dg[:, 50:][3] == 0).all()


def sample_of(N):
    """Rows from all over, the first and the last ones among them."""
    r = np.unique(np.concatenate([np.arange(3), np.linspace(0, N - 1, 40).astype(int), np.arange(N - 3, N)]))
    return r[(r >= 0) & (r < N)]


@pytest.mark.parametrize("N,A,dtype,cols,masked", [
    (300000, 6, "f32", False, False), (20000, 1000, "bf16", False, False), (20000, 1000, "f32", False, True),
    (5000, 2100, "bf16", False, True), (1300, 20000, "bf16", False, False), (1200, 20000, "bf16", False, True),
    (700, 50257, "bf16", False, False), (700, 40001, "f16", False, True), (300, 131072, "bf16", False, False),
    (600, 70001, "f32", False, False), (1300000, 3, "f32", True, True), (600000, 13, "bf16", True, False),
    (600001, 40, "f16", True, False), (530000, 90, "bf16", True, True), (270000, 200, "bf16", True, False),
    (270000, 400, "bf16", True, False)])
def test_many_rows(bs, N, A, dtype, cols, masked):
    """More rows than workgroups take at once: rows from all over against the fp64 form, the loss
    against its terms summed from the rows' own log-probabilities in fp64. A tenth of the rows is
    padding."""
    dt = sc.TYPES[dtype]
    g = torch.Generator(device="cuda").manual_seed(N + A)
    l = (torch.randn((A, N) if cols else (N, A), generator=g, device="cuda", dtype=dt) * 2)
    l = l.t() if cols else l
    act = torch.randint(0, A, (N,), generator=g, device="cuda")
    mask = None
    if masked:
        mask = torch.rand((A, N) if cols else (N, A), generator=g, device="cuda") > 0.3
        mask = mask.t() if cols else mask
        mask.scatter_(1, act[:, None], True)
    w = (torch.rand(N, generator=g, device="cuda") > 0.1).float() * torch.rand(N, generator=g, device="cuda") / N
    adv = torch.randn(N, generator=g, device="cuda")
    scale = 65536.0 if dtype == "f16" else 1.0
    w = w * scale
    with bs.Sim(preset("C1"), n_envs=1) as sim:
        r = sim.policy_loss(l, act, adv, weight=w, mask=mask, c_entropy=0.1)
        again = sim.policy_loss(l, act, adv, weight=w, mask=mask, c_entropy=0.1)
        sim.sync()
        assert all(torch.equal(r[k], again[k]) for k in r)
        at = torch.from_numpy(sample_of(N)).cuda()
        s = {k: v[at].double().cpu().numpy() for k, v in (("logits", l), ("actions", act), ("weight", w), ("adv", adv))}
        m = None if mask is None else mask[at].cpu().numpy()
        want = ops.policy_loss(s["logits"], s["actions"].astype(int), s["adv"], weight=s["weight"], mask=m, c_entropy=0.1)
        got = dict(logp=r["logp"][at], grad=r["grad"][at], loss=torch.from_numpy(want["loss"]))
        lc.check_policy(dict(s, old=None, ref=None), got, want, 0.0, 0.1, dt)
        # rho = 1: the policy term is -sum w adv whatever the logits; entropies by the rows' softmax
        pol = -(w.double() * adv.double()).sum().item()
        size = (w.double() * adv.double().abs()).sum().item()
        assert abs(r["loss"][1].item() - pol) <= 4 * lc.U * size + 2 * lc.U * abs(pol)
        H = 0.0
        for i in range(0, N, max(1, (1 << 26) // A)):
            z = l[i:i + max(1, (1 << 26) // A)].double()
            if mask is not None:
                z = z.masked_fill(~mask[i:i + len(z)], -torch.inf)
            ls = torch.log_softmax(z, 1)
            H += (w[i:i + len(z)].double() * -(ls.exp() * ls.clamp(min=-1e300)).sum(1)).sum().item()
        # loss_check's bound of a row's entropy, with mean |x| below 20 and mean x^2 below 400
        eS = lc.U * (3 * 20 + 4 + A / 64 + min(A, 96) + 16)
        eH = eS * 41 + lc.U * (1200 + (16 + A / 64 + min(A, 96)) * 20 + 4 * 20 + 4)
        assert abs(r["loss"][3].item() - H) <= eH * w.double().sum().item() + 2 * lc.U * abs(H)


@pytest.mark.parametrize("N,A,k,group,dtype,cols", [
    (300000, 24, 1, 6, "f32", False), (300000, 12, 1, 6, "f32", True), (100000, 16, 8, 1, "bf16", False),
    (20000, 1000, 2, 1, "bf16", False), (3000, 4096, 4, 1, "f32", False), (600000, 5, 2, 1, "bf16", True)])
def test_many_routed_rows(bs, N, A, k, group, dtype, cols):
    dt = sc.TYPES[dtype]
    g = torch.Generator(device="cuda").manual_seed(N + A)
    l = torch.randn((A, N) if cols else (N, A), generator=g, device="cuda", dtype=dt)
    l = l.t() if cols else l
    idx = torch.randint(0, A, (N, k), generator=g, device="cuda")
    live = torch.rand(N, generator=g, device="cuda") > 0.1
    with bs.Sim(preset("C1"), n_envs=1) as sim:
        r = sim.balance_loss(l, idx, live, group, 0.5)
        again = sim.balance_loss(l, idx, live, group, 0.5)
        sim.sync()
    assert all(torch.equal(r[x], again[x]) for x in r)
    G, W = A // group, int(live.sum())
    counts = torch.bincount((idx[live] // group).reshape(-1), minlength=G)
    assert torch.equal(r["counts"], counts)
    f = (counts.double() / (k * W)).repeat_interleave(group)
    p = torch.softmax(l.double(), 1)
    s = (p * f).sum(1)
    loss = 0.5 * G / W * (s * live).sum().item()
    eP = lc.U * (3 * 10 + 4 + A / 64 + min(A, 96) + 16 + 4 * 10 + 4 * 20 + 8)   # |x| below 10 where p counts
    assert abs(r["loss"].item() - loss) <= 2 * eP * loss + 4 * lc.U * loss
    want = 0.5 * G / W * p * (f - s[:, None]) * live[:, None]
    tol = 0.5 * G / W * p * (f + s[:, None]) * 2 * (eP + 8 * lc.U) + torch.finfo(dt).eps / 2 * want.abs() + 1e-40
    x = (l.double() - l.double().amax(1, keepdim=True)).abs()
    tol += 0.5 * G / W * p * (f + s[:, None]) * lc.U * 7 * x
    assert ((r["grad"].double() - want).abs() <= tol).all()


@pytest.mark.parametrize("B,T,D", [(4_300_000, 5, 2), (3000, 20, 1), (70000, 6, 1), (40000, 9, 7)])
def test_many_sequences(bs, B, T, D):
    """More sequences than workgroups of a launch, against the steps taken by torch in fp64; |gate| < 1, so a
    state is off by at most 3 T + 64 roundings of the sum of its terms' magnitudes."""
    g = torch.Generator(device="cuda").manual_seed(B)
    gate = torch.rand(B, T, D, generator=g, device="cuda") * 2 - 1
    x, dy = (torch.randn(B, T, D, generator=g, device="cuda") for _ in range(2))
    n = torch.randint(0, T + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    with bs.Sim(preset("C1"), n_envs=1) as sim:
        y, h = sim.gated_scan(gate, x, lengths=n)
        dg, dx, dh0 = sim.gated_scan_grad(gate, x, y, dy, lengths=n)
        sim.sync()
    s = torch.zeros(B, D, dtype=torch.float64, device="cuda")
    m, prev = s.clone(), [None] * T
    for t in range(T):
        on = (t < n)[:, None]
        prev[t] = y[:, t - 1].double() if t else torch.zeros_like(s)
        s = torch.where(on, gate[:, t].double() * s + x[:, t].double(), s)
        m = torch.where(on, gate[:, t].double().abs() * m + x[:, t].double().abs(), m)
        off = (y[:, t].double() - torch.where(on, s, 0.0)).abs()
        assert (off <= sc.unit(torch.float32) * (3 * T + 65) * m).all(), t
    assert ((h.double() - s).abs() <= sc.unit(torch.float32) * (3 * T + 65) * m).all()
    C, m = torch.zeros_like(s), torch.zeros_like(s)
    for t in reversed(range(T)):
        on = (t < n)[:, None]
        G, M = dy[:, t].double() + C, dy[:, t].double().abs() + m
        u = sc.unit(torch.float32) * (3 * T + 66) * M
        assert ((dx[:, t].double() - torch.where(on, G, 0.0)).abs() <= u).all()
        assert ((dg[:, t].double() - torch.where(on, G * prev[t], 0.0)).abs() <= (u + sc.unit(torch.float32) * 2 * M) * prev[t].abs()).all()
        C, m = torch.where(on, gate[:, t].double() * G, C), torch.where(on, gate[:, t].double().abs() * M, m)
    assert ((dh0.double() - C).abs() <= sc.unit(torch.float32) * (3 * T + 66) * m + 1e-45).all()


def policy_rows(l, act, adv, w, mask, c):
    """Rows [n][A] at rho = 1 and without a KL term, in fp64: grad, logp and loss_check's bounds of both."""
    A, U = l.shape[1], lc.U
    z = l.double() if mask is None else l.double().masked_fill(~mask, -torch.inf)
    x = z - z.amax(1, keepdim=True)
    logS = x.exp().sum(1, keepdim=True).log()
    ls = x - logS
    p = ls.exp()
    x, ls = (v.masked_fill(p == 0, 0.0) for v in (x, ls))
    H = -(p * ls).sum(1, keepdim=True)
    hot = torch.zeros_like(p).scatter_(1, act[:, None], 1.0)
    w, q = w.double()[:, None], -adv.double()[:, None]
    grad = w * (q * (hot - p) + c * p * (ls + H))
    logp = ls.gather(1, act[:, None]) * (w != 0)
    adds = A / 64 + min(A, 96) + 16
    eS = U * (p * (3 * x.abs() + 4)).sum(1, keepdim=True) + U * adds
    eP = eS + U * (4 * x.abs() + 4 * logS.abs() + 8)
    eL = eS + U * (x.abs() + ls.abs() + 3 * logS.abs() + 1)
    mx, mxx = (p * x.abs()).sum(1, keepdim=True), (p * x * x).sum(1, keepdim=True)
    eH = eS * (1 + 2 * mx) + U * (3 * mxx + adds * mx + 4 * logS.abs() + 4)
    dq = q.abs() * 6 * U   # rho = 1 as it stands, clipped bounds and products: 4, and 2 as there
    tol = w * (dq * (hot + p) + q.abs() * p * eP + q.abs() * 3 * U * (hot + p)
               + c * p * ((ls.abs() + H) * (eP + 6 * U) + eL + eH))
    tol = tol + torch.finfo(l.dtype).eps / 2 * grad.abs() + torch.finfo(l.dtype).smallest_normal * torch.finfo(l.dtype).eps
    return grad, logp[:, 0], tol, (eL.gather(1, act[:, None])[:, 0] + U * logp[:, 0].abs())


@pytest.mark.parametrize("N,A,dtype,cols,masked", [
    (300000, 6, "f32", False, False), (20000, 1000, "bf16", False, False), (20000, 1000, "f32", False, True),
    (5000, 2100, "bf16", False, True), (1300, 20000, "bf16", False, False), (1200, 20000, "bf16", False, True),
    (700, 50257, "bf16", False, False), (300, 131072, "bf16", False, False), (600, 70001, "f32", False, False),
    (20, 90001, "bf16", False, True), (2200000, 6, "f32", True, True), (1060000, 13, "f32", True, False), (530000, 40, "f32", True, True),
    (530000, 90, "f32", True, False), (600001, 40, "f16", True, False), (530000, 90, "bf16", True, True),
    (530000, 190, "f32", True, False), (270000, 400, "bf16", True, True)])
def test_every_row(bs, N, A, dtype, cols, masked):
    """More rows than workgroups take at once: every row's gradient and log-probability against the closed
    form in fp64. A tenth of the rows is padding."""
    dt = sc.TYPES[dtype]
    g = torch.Generator(device="cuda").manual_seed(N + A)
    l = (torch.randn((A, N) if cols else (N, A), generator=g, device="cuda", dtype=dt) * 2)
    l = l.t() if cols else l
    act = torch.randint(0, A, (N,), generator=g, device="cuda")
    mask = None
    if masked:
        mask = torch.rand((A, N) if cols else (N, A), generator=g, device="cuda") > 0.3
        mask = mask.t() if cols else mask
        mask.scatter_(1, act[:, None], True)
    w = (torch.rand(N, generator=g, device="cuda") > 0.1).float() * torch.rand(N, generator=g, device="cuda") / N
    w = w * (65536.0 if dtype == "f16" else 1.0)
    adv = torch.randn(N, generator=g, device="cuda")
    with bs.Sim(preset("C1"), n_envs=1) as sim:
        r = sim.policy_loss(l, act, adv, weight=w, mask=mask, c_entropy=0.1)
        sim.sync()
    rows = max(1, (1 << 24) // A)
    for i in range(0, N, rows):
        at = slice(i, min(N, i + rows))
        grad, logp, tol, tl = policy_rows(l[at], act[at], adv[at], w[at], None if mask is None else mask[at], 0.1)
        off = ~((r["grad"][at].double() - grad).abs() <= tol)
        assert not off.any(), (i + off.any(1).nonzero()[0].item(), int(off.sum()))
        off = ~((r["logp"][at].double() - logp).abs() <= tl)
        assert not off.any(), (i + off.nonzero()[0].item(), int(off.sum()))
