"""The fp64 forms of linear attention, log-probabilities and orthogonalised updates (oracle/ops.py) against
closed forms, torch's autograd and differences."""
import numpy as np
import torch

from oracle import ops


def attn_inputs(seed=0, B=2, T=7, H=4, Hk=2, Dk=3, Dv=5):
    r = np.random.default_rng(seed)
    return (r.normal(size=(B, T, H, Dk)), r.normal(size=(B, T, Hk, Dk)), r.normal(size=(B, T, Hk, Dv)),
            np.array([0.0, 0.5, 0.9, 1.0])[:H], r.normal(size=(B, H, Dk, Dv)), r)


def test_linear_attn_is_the_sum_over_earlier_steps():
    q, k, v, l, s0, _ = attn_inputs()
    n = np.array([7, 4])
    y, S = ops.linear_attn(q, k, v, l, s0, n, 0.3)
    for b in range(2):
        for h in range(4):
            K, V = k[b, :, h // 2], v[b, :, h // 2]
            for t in range(n[b]):
                w = sum(l[h] ** (t - s) * (q[b, t, h] @ K[s]) * V[s] for s in range(t + 1))
                np.testing.assert_allclose(y[b, t, h], 0.3 * (w + l[h] ** (t + 1) * q[b, t, h] @ s0[b, h]), rtol=1e-12, atol=1e-12)
            end = sum(l[h] ** (n[b] - 1 - s) * np.outer(K[s], V[s]) for s in range(n[b])) + l[h] ** n[b] * s0[b, h]
            np.testing.assert_allclose(S[b, h], end, rtol=1e-12, atol=1e-12)
    assert not y[1, 4:].any()


def test_linear_attn_grad_against_autograd():
    q, k, v, l, s0, r = attn_inputs(1)
    n, scale = np.array([7, 4]), 0.3
    dy, ds = r.normal(size=(2, 7, 4, 5)), r.normal(size=s0.shape)
    ts = [torch.tensor(x, requires_grad=True) for x in (q, k, v, s0)]
    Q, K, V, S = ts
    K, V = K.repeat_interleave(2, 2), V.repeat_interleave(2, 2)
    total = 0.0
    for b in range(2):
        s = S[b]
        for t in range(n[b]):
            s = torch.tensor(l)[:, None, None] * s + K[b, t, :, :, None] * V[b, t, :, None, :]
            total = total + (scale * (Q[b, t, :, None, :] @ s)[:, 0] * torch.tensor(dy[b, t])).sum()
        total = total + (s * torch.tensor(ds[b])).sum()
    total.backward()
    got = ops.linear_attn_grad(q, k, v, l, dy, s0, ds, n, scale)
    for a, b in zip(got, ts):
        np.testing.assert_allclose(a, b.grad.numpy(), rtol=1e-11, atol=1e-12)


def test_token_logprobs_and_their_gradient():
    r = np.random.default_rng(2)
    z = r.normal(size=(6, 9)) * 2
    z[0, 3] = z[0, 5]                       # a tie
    z[1, 2] = -np.inf
    tok = np.array([4, 2, -1, 0, 8, 8])
    mask = r.random((6, 9)) > 0.2
    mask[np.arange(6), tok] = True
    mask[5] = False
    live = np.array([1, 1, 1, 0, 1, 1], bool)
    got = ops.token_logprobs(z, tok, mask, live, top=9)
    t = torch.tensor(z, requires_grad=True)
    ls = torch.log_softmax(t.masked_fill(torch.tensor(~mask), -torch.inf), 1)
    p = ls.exp()
    H = -(p * ls.masked_fill(p == 0, 0.0)).sum(1)
    for n in (0, 2, 4):
        np.testing.assert_allclose(got["entropy"][n], H[n].item(), rtol=1e-12)
    np.testing.assert_allclose(got["logp"][[0, 4]], ls[[0, 4], [4, 8]].detach().numpy(), rtol=1e-12)
    assert got["logp"][1] == -np.inf and got["logp"][2] == got["logp"][3] == got["logp"][5] == 0
    assert (got["top_index"][[3, 5]] == -1).all()
    for n in (0, 1, 2, 4):
        idx = got["top_index"][n][got["top_index"][n] >= 0]
        assert len(idx) == (mask[n] & (z[n] > -np.inf)).sum() and mask[n][idx].all()
        assert (np.diff(z[n][idx]) <= 0).all()
    if mask[0, 3] and mask[0, 5]:
        order = list(got["top_index"][0])
        assert order.index(3) + 1 == order.index(5)
    dl, dh = r.normal(size=6), r.normal(size=6)
    rows = [0, 4]
    (sum(dl[n] * ls[n, tok[n]] + dh[n] * H[n] for n in rows)).backward()
    want = ops.token_logprobs_grad(z, tok, dl, dh, mask, live)
    np.testing.assert_allclose(want[rows], t.grad.numpy()[rows], rtol=1e-10, atol=1e-12)
    assert not want[[3, 5]].any()
    # the entropy's part by differences, of a row without a token
    e = 1e-6
    for j in range(9):
        d = np.zeros_like(z)
        d[2, j] = e
        num = (ops.token_logprobs(z + d, tok, mask, live)["entropy"][2] - ops.token_logprobs(z - d, tok, mask, live)["entropy"][2]) / (2 * e)
        assert abs(num * dh[2] - want[2, j]) < 1e-8


def test_orthogonalize_maps_singular_values():
    r = np.random.default_rng(3)
    for M, N in ((4, 9), (9, 4), (5, 5), (1, 6)):
        u = r.normal(size=(M, N))
        x, way = ops.orthogonalize(u, scale=2.0)
        U, s, Vt = np.linalg.svd(u, full_matrices=False)
        f = s / (np.sqrt((u * u).sum()) + 1e-7)
        for _ in range(5):
            f = 3.4445 * f - 4.7750 * f ** 3 + 2.0315 * f ** 5
        np.testing.assert_allclose(x, 2 * U @ np.diag(f) @ Vt, rtol=1e-9, atol=1e-10)
        assert len(way) == 6
    assert not ops.orthogonalize(np.zeros((3, 4)))[0].any()
