"""Inputs and error bounds of linear attention's tests (u = 2^-24).

With M the sum of the magnitudes of a result's terms (the same call on the inputs' magnitudes), a result is off
by at most what its terms lose on their way:
  - products are held in fp32 and summed in fp32: a term passes at most Dk (or Dv, in the gradient) additions
    over the channels, 64 within a run of steps, 4 per run of at least 32 steps or per join of runs behind it
    (two products and two sums), and where steps are taken one after another (T <= 16) 3 a step; 24 more for its
    weights (powers of the decay, the scale) and the join of heads that share: u each;
  - for T > 16, values are split into parts of 8 bits: 16-bit types keep 16 bits of the four values that are
    split or multiplied on a term's way (the product q k, its weighted sum, the weighted k or v, the state), each
    off by at most 2^-17 (half a step of the second part), and leave out the product of two second parts, at most
    2^-18, in up to two products: 4 2^-17 + 2 2^-18 <= 2^-14.6; fp32, and states of any type, keep three parts, 24
    bits: 4 u and four products of a second and a third part, 2^-26 each, and of two third ones: 6 u in all.
The output's rounding adds half a step of its type."""
import numpy as np
import torch

from oracle import ops
from scan_check import host, near, rounding

U = 2.0 ** -24


def inputs(B, T, H, Hk, Dk, Dv, dtype, seed, s0=True, lengths=False, decays=None):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)   # noqa: E731
    d = dict(q=r(B, T, H, Dk).to(dtype), k=r(B, T, Hk, Dk).to(dtype), v=r(B, T, Hk, Dv).to(dtype),
             dy=r(B, T, H, Dv).to(dtype), dstate=r(B, H, Dk, Dv).float(), s0=r(B, H, Dk, Dv).float() if s0 else None,
             decay=(1.0 - torch.exp2(-1.0 - 7.0 * torch.rand(H, generator=g))).float(), lengths=None,
             scale=Dk ** -0.5)
    if decays is not None:
        d["decay"] = torch.tensor([decays[i % len(decays)] for i in range(H)], dtype=torch.float32)
    if lengths:
        n = torch.randint(0, T + 1, (B,), generator=g)
        n[: min(B, 4)] = torch.tensor([T, 0, min(1, T), max(0, T - 1)])[: min(B, 4)]
        d["lengths"] = n.to(torch.int32)
    return d


def _args(d, names):
    return [host(d[n]) for n in names]


def _loss(dtype, T, D):
    parts = 0.0 if T <= 16 else (6 * U if dtype == torch.float32 else 2.0 ** -14.6)
    return parts + U * (D + 64 + 24 + T / 8 + 3 * min(T, 16))


def check_forward(d, y, state):
    q, k, v, l, s0 = _args(d, ("q", "k", "v", "decay", "s0"))
    n = None if d["lengths"] is None else d["lengths"].cpu().numpy()
    want, last = ops.linear_attn(q, k, v, l, s0, n, d["scale"])
    m, ms = ops.linear_attn(*map(np.abs, (q, k, v, l)), None if s0 is None else np.abs(s0), n, abs(d["scale"]))
    e, es = (_loss(t, q.shape[1], q.shape[3]) for t in (d["q"].dtype, torch.float32))
    if y is not None:
        near(host(y), want, e * m + rounding(want, d["q"].dtype), "y")
    if state is not None:
        near(host(state), last, es * ms + rounding(last, torch.float32), "state")


def check_grad(d, dq, dk, dv, ds0):
    q, k, v, l, dy, s0, ds = _args(d, ("q", "k", "v", "decay", "dy", "s0", "dstate"))
    n = None if d["lengths"] is None else d["lengths"].cpu().numpy()
    want = ops.linear_attn_grad(q, k, v, l, dy, s0, ds, n, d["scale"])
    a = [None if x is None else np.abs(x) for x in (q, k, v, l, dy, s0, ds)]
    m = ops.linear_attn_grad(*a, n, abs(d["scale"]))
    D = max(q.shape[3], v.shape[3]) + q.shape[2] // k.shape[2]
    for name, got, w, b, dt in zip(("dq", "dk", "dv", "ds0"), (dq, dk, dv, ds0), want, m,
                                   [d["q"].dtype] * 3 + [torch.float32]):
        if got is not None:
            near(host(got), w, _loss(dt, q.shape[1], D) * b + rounding(w, dt), name)
