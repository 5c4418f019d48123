"""Plain fp64 forms of the operators for the caller's own networks, one step or one sample at
a time, with what the tests' error bounds are made of. Shares nothing with the HIP path.

gated_scan        h = g_t h + x_t, or h = f h + (1 - f) x_t with f = 1/(1 + exp(-g_t))
gated_scan_grad   its gradient, from the stored y
policy_loss       the clipped policy loss with a KL term over logits, and its gradient
balance_loss      a router's balance loss, its counts and its gradient
linear_attn       S = decay S + k v^T, y = scale S^T q, and linear_attn_grad
token_logprobs    log-probabilities, entropies, alternatives, and token_logprobs_grad
orthogonalize     Newton-Schulz products of an update
"""
import numpy as np


def _sigmoid(g):
    """f and 1 - f, each to its own relative accuracy."""
    e = np.exp(-np.abs(g))
    big, small = 1.0 / (1.0 + e), e / (1.0 + e)
    return np.where(g < 0, small, big), np.where(g < 0, big, small)


def _order(T, reverse):
    return range(T - 1, -1, -1) if reverse else range(T)


def gated_scan(gate, x, h0=None, lengths=None, kind="linear", reverse=False):
    """y [B][T][D], last state [B][D]."""
    B, T, D = gate.shape
    n = np.full(B, T) if lengths is None else np.asarray(lengths)
    h = np.zeros((B, D)) if h0 is None else np.array(h0, np.float64)
    y = np.zeros((B, T, D))
    for t in _order(T, reverse):
        on = t < n
        g, u = gate[on, t].astype(np.float64), x[on, t].astype(np.float64)
        f, r = _sigmoid(g) if kind == "sigmoid" else (g, 1.0)
        h[on] = f * h[on] + r * u
        y[on, t] = h[on]
    return y, h


def gated_scan_grad(gate, x, y, dy, h0=None, dstate=None, lengths=None, kind="linear",
                    reverse=False):
    """dgate, dx [B][T][D], dh0 [B][D]."""
    B, T, D = gate.shape
    n = np.full(B, T) if lengths is None else np.asarray(lengths)
    first = np.zeros((B, D)) if h0 is None else np.asarray(h0, np.float64)
    C = np.zeros((B, D)) if dstate is None else np.array(dstate, np.float64)
    dg, dx = np.zeros((B, T, D)), np.zeros((B, T, D))
    for t in reversed(list(_order(T, reverse))):
        for b in np.nonzero(t < n)[0]:
            tp = t + 1 if reverse else t - 1
            hp = np.asarray(y[b, tp], np.float64) if 0 <= tp < n[b] else first[b]
            g = gate[b, t].astype(np.float64)
            G = dy[b, t].astype(np.float64) + C[b]
            if kind == "sigmoid":
                f, r = _sigmoid(g)
                dg[b, t] = G * (hp - x[b, t].astype(np.float64)) * f * r
                dx[b, t] = r * G
                C[b] = f * G
            else:
                dg[b, t], dx[b, t], C[b] = G * hp, G, g * G
    return dg, dx, C


def scan_majorants(gate, b, h0, lengths, kind, reverse):
    """M_t = |a_t| M + |b_t| and E_t = |a_t| E + M_t in the order of a scan with inputs b: the sum
    of the magnitudes of a state's terms, and the same with each term counted once for every step
    that it has passed. Also the last ones [B][D]."""
    B, T, D = gate.shape
    n = np.full(B, T) if lengths is None else np.asarray(lengths)
    m = np.zeros((B, D)) if h0 is None else np.abs(np.asarray(h0, np.float64))
    e = m.copy()
    M, E = np.zeros((B, T, D)), np.zeros((B, T, D))
    for t in _order(T, reverse):
        on = t < n
        g = gate[on, t].astype(np.float64)
        a = _sigmoid(g)[0] if kind == "sigmoid" else np.abs(g)
        m[on] = a * m[on] + np.abs(b[on, t])
        e[on] = a * e[on] + m[on]
        M[on, t], E[on, t] = m[on], e[on]
    return M, E, m, e


def policy_loss(logits, actions, adv, logp_old=None, logp_ref=None, weight=None, mask=None, clip=0.2,
                c_kl=0.0, c_entropy=0.0):
    """dict(loss [4], logp [N], grad [N][A], parts) with `parts` what error bounds are made of."""
    z = np.array(logits, np.float64)
    N, A = z.shape
    w = np.full(N, 1.0 / max(N, 1)) if weight is None else np.asarray(weight, np.float64)
    z[np.isnan(z) & (w == 0)[:, None]] = 0.0
    allowed = np.ones((N, A), bool) if mask is None else np.asarray(mask) != 0
    allowed = allowed & ~(z == -np.inf)
    loss, logp, grad = np.zeros(3), np.zeros(N), np.zeros((N, A))
    parts = [None] * N
    bad = []
    for n in range(N):
        if w[n] == 0 or not allowed[n].any():
            continue
        a, ok = int(actions[n]), allowed[n]
        if not 0 <= a < A or not ok[a]:
            bad.append(n)
            continue
        v = z[n, ok]
        m = v.max()
        ls = np.full(A, -np.inf)
        ls[ok] = v - m - np.log(np.exp(v - m).sum())
        p = np.exp(ls)
        lsf = np.where(ok, ls, 0.0)
        H = -(p * lsf).sum()
        lp = ls[a]
        rho = 1.0 if logp_old is None else np.exp(lp - float(logp_old[n]))
        ad = float(adv[n])
        clipped = (rho > 1 + clip and ad > 0) or (rho < 1 - clip and ad < 0)
        term = -ad * min(max(rho, 1 - clip), 1 + clip) if clipped else -ad * rho
        q = 0.0 if clipped else -ad * rho
        kl = 0.0
        if logp_ref is not None:
            d = float(logp_ref[n]) - lp
            kl = np.expm1(d) - d
            q -= c_kl * np.expm1(d) if c_kl else 0.0
        g = -q * p
        g[a] += q
        g += c_entropy * p * (lsf + H)
        grad[n], logp[n] = w[n] * g, lp
        loss += w[n] * np.array([term, kl, H])
        parts[n] = dict(p=p, ls=lsf, H=H, q=q, rho=rho, x=np.where(ok, z[n] - m, 0.0), term=term)
    total = loss[0] + (c_kl * loss[1] if c_kl else 0.0) - (c_entropy * loss[2] if c_entropy else 0.0)
    return dict(loss=np.concatenate([[total], loss]), logp=logp, grad=grad, parts=parts, bad=bad)


def balance_loss(logits, index, live=None, group=1, coef=1.0):
    """dict(loss, counts [G], grad [N][A])."""
    z = np.array(logits, np.float64)
    N, A = z.shape
    G, k = A // group, index.shape[1]
    on = np.ones(N, bool) if live is None else np.asarray(live) != 0
    counts = np.zeros(G, np.int64)
    bad = 0
    for n in np.nonzero(on)[0]:
        for a in index[n]:
            if 0 <= a < A:
                counts[int(a) // group] += 1
            elif a != -1:
                bad += 1
    W = int(on.sum())
    f = np.repeat(counts / (k * max(W, 1)), group)
    grad, P = np.zeros((N, A)), np.zeros((N, A))
    for n in np.nonzero(on)[0]:
        if (z[n] == -np.inf).all():
            continue
        e = np.exp(z[n] - z[n].max())
        P[n] = e / e.sum()
        grad[n] = coef * G / W * P[n] * (f - (f * P[n]).sum())
    return dict(loss=coef * G / max(W, 1) * (P * f).sum(), counts=counts, grad=grad, p=P, f=f, bad=bad)


def grad_majorants(gate, dy, dstate, lengths, kind, reverse):
    """As scan_majorants for G_t = dy_t + C, C = a_t G_t: of G at every step and of dh0."""
    B, T, D = gate.shape
    n = np.full(B, T) if lengths is None else np.asarray(lengths)
    m = np.zeros((B, D)) if dstate is None else np.abs(np.asarray(dstate, np.float64))
    e = m.copy()
    M, E = np.zeros((B, T, D)), np.zeros((B, T, D))
    for t in reversed(list(_order(T, reverse))):
        on = t < n
        g = gate[on, t].astype(np.float64)
        a = _sigmoid(g)[0] if kind == "sigmoid" else np.abs(g)
        M[on, t] = np.abs(dy[on, t].astype(np.float64)) + m[on]
        E[on, t] = M[on, t] + e[on]
        m[on], e[on] = a * M[on, t], a * E[on, t] + a * M[on, t]
    return M, E, m, e


def linear_attn(q, k, v, decay, s0=None, lengths=None, scale=1.0):
    """y [B][T][H][Dv] and the last state [B][H][Dk][Dv]: S = decay S + k_t v_t^T, y_t = scale S^T q_t."""
    B, T, H, Dk = q.shape
    g, Dv = H // k.shape[2], v.shape[3]
    n = np.full(B, T) if lengths is None else np.asarray(lengths)
    S = np.zeros((B, H, Dk, Dv)) if s0 is None else np.array(s0, np.float64)
    y = np.zeros((B, T, H, Dv))
    for t in range(T):
        on = t < n
        kt, vt = (np.repeat(x[on, t].astype(np.float64), g, axis=1) for x in (k, v))
        S[on] = decay[:, None, None] * S[on] + kt[..., :, None] * vt[..., None, :]
        y[on, t] = scale * (q[on, t].astype(np.float64)[..., None, :] @ S[on])[..., 0, :]
    return y, S


def linear_attn_grad(q, k, v, decay, dy, s0=None, dstate=None, lengths=None, scale=1.0):
    """dq, dk, dv, ds0 of linear_attn, from the states of every step."""
    B, T, H, Dk = q.shape
    Hk, Dv = v.shape[2:]
    g = H // Hk
    n = np.full(B, T) if lengths is None else np.asarray(lengths)
    S = np.zeros((B, H, Dk, Dv)) if s0 is None else np.array(s0, np.float64)
    G = np.zeros((B, H, Dk, Dv)) if dstate is None else np.array(dstate, np.float64)
    dq, dk, dv = (np.zeros(x.shape) for x in (q, k, v))
    l = decay[:, None, None]
    for t in range(T):
        on = t < n
        kt, vt = (np.repeat(x[on, t].astype(np.float64), g, axis=1) for x in (k, v))
        S[on] = l * S[on] + kt[..., :, None] * vt[..., None, :]
        dq[on, t] = scale * (S[on] @ dy[on, t].astype(np.float64)[..., None])[..., 0]
    for t in range(T - 1, -1, -1):
        on = t < n
        kt, vt = (np.repeat(x[on, t].astype(np.float64), g, axis=1) for x in (k, v))
        qt, dt = q[on, t].astype(np.float64), dy[on, t].astype(np.float64)
        Gt = G[on] + scale * qt[..., :, None] * dt[..., None, :]
        dk[on, t] = (Gt @ vt[..., None])[..., 0].reshape(-1, Hk, g, Dk).sum(2)
        dv[on, t] = (kt[..., None, :] @ Gt)[..., 0, :].reshape(-1, Hk, g, Dv).sum(2)
        G[on] = l * Gt
    return dq, dk, dv, G


def token_logprobs(logits, tokens=None, mask=None, live=None, top=0):
    """Dict: logp, entropy [N], top_index, top_logp [N][top], and ls, p [N][A] of the rows that give anything."""
    N, A = logits.shape
    r = dict(logp=np.zeros(N), entropy=np.zeros(N), top_index=np.full((N, top), -1), top_logp=np.full((N, top), -np.inf),
             ls=[None] * N, p=[None] * N)
    for n in range(N):
        z = logits[n].astype(np.float64)
        if mask is not None:
            z = np.where(mask[n], z, -np.inf)
        if (live is not None and not live[n]) or not (z > -np.inf).any():
            continue
        x = z - z.max()
        ls = x - np.log(np.exp(x).sum())
        p = np.exp(ls)
        r["ls"][n], r["p"][n] = ls, p
        r["entropy"][n] = -(p[p > 0] * ls[p > 0]).sum()
        if tokens is not None and 0 <= tokens[n] < A:
            r["logp"][n] = ls[tokens[n]]
        order = [j for j in sorted(range(A), key=lambda j: (-z[j], j)) if z[j] > -np.inf][:top]
        r["top_index"][n, :len(order)] = order
        r["top_logp"][n, :len(order)] = ls[order]
    return r


def token_logprobs_grad(logits, tokens, dlogp, dentropy, mask=None, live=None):
    """The gradient of sum(dlogp logp + dentropy H); rows whose token is none or forbidden keep H's part."""
    r = token_logprobs(logits, tokens, mask, live)
    d = np.zeros(logits.shape)
    for n in range(len(logits)):
        ls, p = r["ls"][n], r["p"][n]
        if p is None:
            continue
        a = -1 if tokens is None else int(tokens[n])
        g = float(dlogp[n]) if dlogp is not None and 0 <= a < len(p) and ls[a] > -np.inf else 0.0
        h = 0.0 if dentropy is None else float(dentropy[n])
        d[n] = -p * (g + h * (np.where(p > 0, ls, 0.0) + r["entropy"][n]))
        if g:
            d[n, a] += g
    return d


def orthogonalize(u, steps=5, coeffs=(3.4445, -4.7750, 2.0315), eps=1e-7, scale=1.0):
    """One matrix [M][N]; and every X on the way, with the shorter side as rows."""
    a, b, c = coeffs
    x = np.asarray(u, np.float64)
    x = x.T if x.shape[0] > x.shape[1] else x
    x = x / (np.sqrt((x * x).sum()) + eps)
    way = [x]
    for _ in range(steps):
        A = x @ x.T
        x = a * x + (b * A + c * A @ A) @ x
        way.append(x)
    return scale * (x.T if u.shape[0] > u.shape[1] else x), way
