"""Inputs and error bounds of the gated recurrence's tests.

A computed state differs from the exact one by the roundings on each term's way to it: two per step
(a product and a sum; three where a run's gates are multiplied up first and then applied) and a
few per join of runs, at most 64 in all, each at most u = 2^-24 (fp64: 2^-53) of the term. With
M the sum of the terms' magnitudes and E the same with each term counted once for every step that
it has passed (oracle.ops.scan_majorants), |error| <= u (3 E + 64 M). A sigmoid gate (and 1 minus
it) is itself off by at most (1.5 |g| + 6) u: the exponent's argument |g| log2(e), rounded twice,
then exp2, a sum, a reciprocal and a product of one ulp each; that is added to the 3. The output's rounding
adds half a step of its type."""
import numpy as np
import torch

from oracle import ops

TYPES = {"f64": torch.float64, "f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def wide(dtype):
    return torch.float64 if dtype == torch.float64 else torch.float32


def unit(dtype):
    return 2.0 ** -53 if dtype == torch.float64 else 2.0 ** -24


def rounding(v, dtype):
    """Half a step of `dtype` at the values v (and of its smallest numbers)."""
    f = torch.finfo(dtype)
    return f.eps / 2 * np.abs(v) + f.smallest_normal * f.eps


def host(t):
    """The values of a tensor, in numpy fp64 (None stays None)."""
    return None if t is None else t.detach().double().cpu().numpy()


def inputs(B, T, D, dtype, kind, seed, h0=True, lengths=False, device="cpu"):
    """Gates near one (and zero ones among them), inputs, upstream gradients: dict of tensors."""
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)   # noqa: E731
    gate = r(B, T, D) * 2.0 + 2.0
    if kind == "linear":
        gate = torch.sigmoid(gate) * torch.where(r(B, T, D) > 2.0, -1.0, 1.0)
        gate = torch.where(r(B, T, D) > 2.3, torch.zeros(()).double(), gate)
    d = dict(gate=gate.to(dtype), x=r(B, T, D).to(dtype), dy=r(B, T, D).to(dtype), h0=None,
             dstate=r(B, D).to(wide(dtype)), lengths=None)
    if h0:
        d["h0"] = r(B, D).to(wide(dtype))
    if lengths:
        n = torch.randint(0, T + 1, (B,), generator=g)
        n[: min(B, 3)] = torch.tensor([T, 0, min(1, T)])[: min(B, 3)]
        d["lengths"] = n.to(torch.int32)
    return {k: None if v is None else v.to(device) for k, v in d.items()}


def _gate_error(gate, kind):
    return 3.0 + (1.5 * np.abs(gate).max(initial=0.0) + 6.0 if kind == "sigmoid" else 0.0)


def check_forward(d, y, state, kind, reverse):
    dt = d["gate"].dtype
    gate, x, h0 = host(d["gate"]), host(d["x"]), host(d["h0"])
    n = None if d["lengths"] is None else d["lengths"].cpu().numpy()
    want, last = ops.gated_scan(gate, x, h0, n, kind, reverse)
    b = (ops._sigmoid(gate)[1] if kind == "sigmoid" else 1.0) * x
    M, E, m, e = ops.scan_majorants(gate, b, h0, n, kind, reverse)
    k, u = _gate_error(gate, kind), unit(dt)
    if y is not None:
        near(host(y), want, u * (k * E + 64 * M) + rounding(want, dt), "y")
    near(host(state), last, u * (k * e + 64 * m) + rounding(last, wide(dt)), "state")
    return want, last


def check_grad(d, y, dgate, dx, dh0, kind, reverse):
    dt = d["gate"].dtype
    gate, x, dy, ys = host(d["gate"]), host(d["x"]), host(d["dy"]), host(y)
    h0, ds = host(d["h0"]), host(d["dstate"])
    n = None if d["lengths"] is None else d["lengths"].cpu().numpy()
    want = ops.gated_scan_grad(gate, x, np.zeros_like(x) if ys is None else ys, dy, h0, ds, n, kind,
                               reverse)
    M, E, m, e = ops.grad_majorants(gate, dy, ds, n, kind, reverse)
    k, u = _gate_error(gate, kind), unit(dt)
    eG = u * (k * E + 64 * M)
    f, r = ops._sigmoid(gate) if kind == "sigmoid" else (1.0, 1.0)
    near(host(dx), want[1], r * eG + 2 * k * u * r * M + rounding(want[1], dt), "dx")
    if dgate is not None:
        B, T, D = gate.shape
        hp = np.zeros_like(x)
        z = np.zeros((B, 1, D)) if h0 is None else h0[:, None]
        if reverse:
            hp = np.concatenate([ys[:, 1:], z], 1)
            for b in range(B):
                if n is not None and 0 < n[b] <= T:
                    hp[b, n[b] - 1] = z[b, 0]
        else:
            hp = np.concatenate([z, ys[:, :-1]], 1)
        c = np.abs(hp - x) * f * r if kind == "sigmoid" else np.abs(hp)
        c = np.where(M > 0, c, 0.0)
        near(host(dgate), want[0], c * eG + (2 * k + 6) * u * c * M + rounding(want[0], dt), "dgate")
    near(host(dh0), want[2], u * (k * e + 64 * m) + rounding(want[2], wide(dt)), "dh0")


def near(got, want, tol, what):
    assert got.shape == want.shape, f"{what}: {got.shape}, expected {want.shape}"
    off = ~(np.abs(got - want) <= tol)
    if off.any():
        i = np.unravel_index(np.argmax(np.where(off, np.abs(got - want) / np.maximum(tol, 1e-300), 0)), off.shape)
        raise AssertionError(f"{what}: {off.sum()} of {off.size} outside; at {i} got {got[i]!r}, "
                             f"expected {want[i]!r} +- {tol[i]!r}")
