"""Linear attention, log-probabilities, the policy loss and orthogonalised updates as a training program uses them
together, and as a serving one does."""
import numpy as np
import pytest

from workloads import preset

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import attn_check as ac   # noqa: E402
from oracle import ops    # noqa: E402


@pytest.fixture(scope="module")
def sim():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2607_05272_amd as bs
    with bs.Sim(preset("C1"), n_envs=1) as s:
        yield s


def test_training_step(sim):
    """A sequence policy over padded episodes in fp32: y by linear_attn, logits by a head, log-probabilities of the taken
    actions under it (the next update's logp_old, and policy_loss's own at rho = 1), a loss over log-probabilities and
    entropies back through the head and the layer, an orthogonalised update of the head. Against torch's autograd of the
    whole in fp64: fp32 sums of some hundred terms, so 1e-4 of each gradient's norm."""
    g = torch.Generator().manual_seed(0)
    B, T, F, H, D, A = 5, 90, 24, 2, 16, 12
    n = torch.tensor([90, 0, 1, 50, 89], dtype=torch.int32)
    x = torch.randn(B, T, F, generator=g)
    wq, wk, wv = (torch.randn(F, H * D, generator=g) * F ** -0.5 for _ in range(3))
    head = torch.randn(H * D, A, generator=g) * 0.3
    act = torch.randint(0, A, (B * T,), generator=g)
    adv = torch.randn(B * T, generator=g)
    decay = torch.tensor([0.9, 0.99])
    live = (torch.arange(T)[None] < n[:, None]).reshape(-1)
    w = live.float() / live.sum()
    c = 0.02
    dev = [t.cuda() for t in (x, wq, wk, wv, head, act, adv, decay, n, live, w)]
    X, Wq, Wk, Wv, Hd, Act, Adv, Dec, N, Live, W = dev
    q, k, v = ((X @ m).view(B, T, H, D) for m in (Wq, Wk, Wv))
    y, _ = sim.linear_attn(q, k, v, Dec, lengths=N, scale=D ** -0.5)
    flat = y.reshape(B * T, H * D)
    logits = flat @ Hd
    lp = sim.token_logprobs(logits, Act, live=Live, top=3)
    pol = sim.policy_loss(logits, Act, Adv, logp_old=lp["logp"], weight=W, c_entropy=c)
    dl = sim.token_logprobs_grad(logits, Act, dlogp=-W * Adv, dentropy=-c * W, live=Live)
    dy = (dl @ Hd.t()).reshape(B, T, H, D)
    dhead = flat.t() @ dl
    dq, dk, dv, _ = sim.linear_attn_grad(q, k, v, Dec, dy, lengths=N, scale=D ** -0.5)
    grads = [X.reshape(-1, F).t() @ t.reshape(-1, H * D) for t in (dq, dk, dv)] + [dhead]
    step = sim.orthogonalize(dhead, scale=0.2)
    sim.sync()
    # in fp64
    p = [t.double().requires_grad_() for t in (wq, wk, wv, head)]
    Q, K, V = ((x.double() @ m).view(B, T, H, D) for m in p[:3])
    gap = torch.arange(T)[:, None] - torch.arange(T)
    wt = torch.where(gap >= 0, decay.double()[:, None, None] ** gap.clamp(min=0), 0.0)
    Y = torch.einsum("bths,bshd->bthd", torch.einsum("bthd,bshd->bths", Q, K) * wt.permute(1, 0, 2), V) * D ** -0.5
    Y = torch.where(live.view(B, T, 1, 1), Y, 0.0)
    ls = torch.log_softmax(Y.reshape(B * T, H * D) @ p[3], 1)
    logp = ls.gather(1, act[:, None])[:, 0]
    ent = -(ls.exp() * ls).sum(1)
    loss = (w.double() * (-adv.double() * logp - c * ent)).sum()
    loss.backward()
    for got, t in zip(grads, p):
        assert (got.double().cpu() - t.grad).norm() <= 1e-4 * t.grad.norm()
    assert (lp["logp"].double().cpu() - torch.where(live, logp, 0.0).detach()).abs().max() < 1e-4
    assert (lp["entropy"].double().cpu() - torch.where(live, ent, 0.0).detach()).abs().max() < 1e-4
    # at rho = 1 the policy loss is the same loss but for its value: -adv for -adv logp
    assert (pol["grad"] - dl).norm() <= 1e-5 * dl.norm()
    # two sums of the same row in other orders: each log-probability is off by at most eL + u |log p| of loss_check.py, with
    # |x| at most the row's spread s, |log p| at most s + log 12 and log S at most log 12:
    # (3 s + 4) + (12/64 + 12 + 16) + (s + s + 2.5 + 3 2.5 + 1) + s + 2.5 <= 6 s + 46 u
    spread = (logits.amax(1) - logits.amin(1)).max()
    assert (pol["logp"] - lp["logp"])[Live].abs().max() <= 2 * (6 * spread + 46) * 2.0 ** -24
    top = ls.detach().sort(1, descending=True).values[:, :3]
    assert (lp["top_logp"].double().cpu()[live] - top[live]).abs().max() < 1e-4
    assert (lp["top_index"][~Live] == -1).all() and not dl[~Live].any()
    want, _ = ops.orthogonalize(dhead.double().cpu().numpy(), scale=0.2)
    assert np.abs(step.double().cpu().numpy() - want).max() < 1e-4 * np.abs(want).max() + 1e-5


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_serving(sim, dtype):
    """Prompts of unequal lengths at once, then token after token on the state in place, each told with its log-probability
    and alternatives: as the whole sequences in one call."""
    B, P, M, H, Hk, D = 3, 70, 12, 4, 2, 32
    d = ac.inputs(B, P + M, H, Hk, D, D, dtype, 3, s0=False)
    n = torch.tensor([70, 1, 33], dtype=torch.int32)
    c = {k: v.cuda() if torch.is_tensor(v) else v for k, v in d.items()}
    y, state = sim.linear_attn(c["q"][:, :P], c["k"][:, :P], c["v"][:, :P], c["decay"], lengths=n.cuda(), scale=0.2)
    rows = []
    for t in range(M):
        at = slice(P + t, P + t + 1)
        z, same = sim.linear_attn(c["q"][:, at], c["k"][:, at], c["v"][:, at], c["decay"], s0=state, scale=0.2, state=state)
        assert same is state
        logits = z.reshape(B, H * D)
        r = sim.token_logprobs(logits, logits.argmax(1), top=2)
        rows.append((z, r, logits))
    sim.sync()
    for b in range(B):
        keep = list(range(int(n[b]))) + list(range(P, P + M))
        one = {k: (v[b:b + 1, keep] if k in ("q", "k", "v") else v) for k, v in d.items()}
        one.update(s0=None, lengths=None, scale=0.2)
        ac.check_forward(one, torch.cat([y[b:b + 1, :int(n[b])]] + [z[b:b + 1] for z, _, _ in rows], 1), state[b:b + 1])
    for z, r, logits in rows:
        assert torch.equal(r["top_index"][:, 0], logits.double().max(1).indices) or \
            torch.equal(logits.gather(1, r["top_index"][:, :1])[:, 0], logits.max(1).values)
        assert torch.equal(r["top_logp"][:, 0], r["logp"])
