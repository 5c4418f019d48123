"""Inputs and error bounds of the policy loss's and the balance loss's tests (u = 2^-24).

With x = l - m: exp(x) is off by (3 |x| + 4) u of itself (x, the exponent's argument and exp2, each
rounded), S = sum exp(x) by the mean of that and one u per addition on a term's way (at most
A/64 + min(A, 96) + 16), log S by eS plus its own rounding; logp = x_a - log S, p = exp(x)/S or
exp(x - log S), H = log S - sum(exp(x) x)/S and the loss's terms follow by the usual rules. The
gradient's bound adds half a step of its type."""
import numpy as np
import torch

from scan_check import near, rounding

U = 2.0 ** -24
CLIP = 0.2


def softmax_errors(A, x, p, logS):
    eS = U * (p * (3 * np.abs(x) + 4)).sum() + U * (A / 64 + min(A, 96) + 16)
    eP = eS + U * (4 * np.abs(x) + 4 * abs(logS) + 8)
    return eS, eP


def check_policy(s, got, want, c_kl, c_entropy, dtype):
    """got: dict of tensors; want: oracle.ops.policy_loss of the same inputs s (numpy)."""
    N, A = want["grad"].shape
    tg, tl, terms = np.zeros((N, A)), np.zeros(N), np.zeros(3)
    for n, r in enumerate(want["parts"]):
        if r is None:
            continue
        a, p, ls, x, H, q, rho = int(s["actions"][n]), r["p"], r["ls"], r["x"], r["H"], r["q"], r["rho"]
        w = 1.0 / N if s["weight"] is None else abs(float(s["weight"][n]))
        ad, lp = abs(float(s["adv"][n])), want["logp"][n]
        logS = x[a] - lp
        eS, eP = softmax_errors(A, x, p, logS)
        eL = eS + U * (np.abs(x) + np.abs(ls) + 3 * abs(logS) + 1)          # of log p
        mx, mxx = (p * np.abs(x)).sum(), (p * x * x).sum()
        eH = eS * (1 + 2 * mx) + U * (3 * mxx + (16 + A / 64 + min(A, 96)) * mx + 4 * abs(logS) + 4)
        eR = eL[a] + U * (abs(lp - float(s["old"][n])) + 6) if s["old"] is not None else U
        dq, dt = (rho * ad * (eR + 3 * U), rho * ad * (eR + 3 * U)) if q != 0 or r["term"] == 0 \
            else (0.0, 2 * ad * 3 * U)
        dk = 0.0
        if s["ref"] is not None:
            d = float(s["ref"][n]) - lp
            e = abs(np.expm1(d))
            eD = eL[a] + U * abs(d)
            dq += c_kl * (np.exp(d) * eD + 4 * U * e) + U * abs(q)
            dk = e * eD + U * (8 * e + 4 * abs(d))
        dq += abs(q) * 2 * U
        hot = np.zeros(A)
        hot[a] = 1.0
        tg[n] = w * (dq * (hot + p) + abs(q) * p * eP + abs(q) * 3 * U * (hot + p)
                     + c_entropy * p * ((np.abs(ls) + H) * (eP + 6 * U) + eL + eH))
        tl[n] = eL[a] + U * abs(lp)
        terms += w * (np.array([dt, dk, eH]) + 2 * U * np.abs([r["term"], dk, H]))
    near(got["logp"].double().cpu().numpy(), want["logp"], tl, "logp")
    if got["grad"] is not None:
        near(got["grad"].double().cpu().numpy(), want["grad"], tg + rounding(want["grad"], dtype), "grad")
    tot = terms[0] + c_kl * terms[1] + c_entropy * terms[2]
    tol = np.concatenate([[tot], terms])
    near(got["loss"].double().cpu().numpy(), want["loss"], tol + rounding(want["loss"], torch.float32), "loss")


def check_balance(got, want, z, live, group, coef, dtype):
    N, A = want["grad"].shape
    G, W = A // group, max(1, int(live.sum()))
    f, P = want["f"], want["p"]
    tg, tl = np.zeros((N, A)), 0.0
    for n in range(N):
        if not P[n].any():
            continue
        ok = P[n] > 0
        x = np.where(ok, z[n] - z[n].max(), 0.0)
        logS = -np.log(P[n].max())
        eS, eP = softmax_errors(A, x, P[n], logS)
        si = (f * P[n]).sum()
        # the kernel works on f' = f - 1/G, rounded once, and si' = sum p f': |f'| takes f's place in every
        # rounding, and si - 1/G that of si
        fc = np.abs(f - 1.0 / G)
        sc = (fc * P[n]).sum()
        dsi = (P[n] * fc * eP).sum() + sc * (eS + (20 + A / 64 + min(A, 96)) * U)
        # the oracle's own fp64: f - si from a sum of A products, each step off by at most 2^-53 of f or si;
        # where f is even their difference is nothing but that
        o64 = (A + 8) * 2.0 ** -53 * (f + si)
        tg[n] = abs(coef) * G / W * P[n] * (np.abs(f - si) * (eP + 8 * U) + 2 * U * fc + 2 * U * sc + dsi + o64)
        tl += abs(coef) * G / W * dsi
    near(got["grad"].double().cpu().numpy(), want["grad"], tg + rounding(want["grad"], dtype), "grad")
    assert np.array_equal(got["counts"].cpu().numpy(), want["counts"]), "counts"
    l = np.array(want["loss"])
    near(got["loss"].double().cpu().numpy(), l, np.array(tl) + 4 * U * abs(l) + rounding(l, torch.float32), "loss")
