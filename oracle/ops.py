"""Plain fp64 forms of the operators for the caller's own networks, one step or one sample at
a time, with what the tests' error bounds are made of. Shares nothing with the HIP path.

gated_scan        h = g_t h + x_t, or h = f h + (1 - f) x_t with f = 1/(1 + exp(-g_t))
gated_scan_grad   its gradient, from the stored y
policy_loss       the clipped policy loss with a KL term over logits, and its gradient
balance_loss      a router's balance loss, its counts and its gradient
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
