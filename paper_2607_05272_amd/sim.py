"""Python face of the C ABI in include/batchsim.h (argument marshalling only).

Tensors passed in or returned are CUDA (HIP) tensors owned by torch; the library writes
into them on the context's stream. Layouts follow the ABI: [T][E] time-major arrays and
[F][E] observations.
"""
import ctypes as C
import threading

import numpy as np
import torch

from . import _lib as L


def _p(t):
    return None if t is None else C.c_void_p(t.data_ptr())


_FLOAT = {torch.float64: 0, torch.float32: 1, torch.bfloat16: 2, torch.float16: 3}
_INT = {torch.uint8: 0, torch.int32: 1, torch.int64: 2}


def _a(t):
    """A tensor's address (None: absent)."""
    return None if t is None else t.data_ptr()


def _seq(t):
    """sim_seq of a [B][T][D] tensor (None: absent)."""
    if t is None:
        return None
    sb, st, sd = t.stride()
    if sd != 1 and t.shape[2] > 1:
        raise ValueError("channels (the last dimension) must be adjacent in memory")
    return C.byref(L.SimSeq(t.data_ptr(), sb, st))


def _mat(t):
    return None if t is None else C.byref(L.SimMat(t.data_ptr(), *t.stride()))


def weights_layout(w):
    """Byte offsets of the policy weight buffer for workload `w` (sim_weights_layout)."""
    lib = L.load()
    cfg = L.make_cfg(w, n_envs=max(1, w.get("n_envs", 1)))
    lay = L.SimWLayout()
    L.check(lib.sim_weights_layout(C.byref(cfg), C.byref(lay)), "sim_weights_layout")
    return dict(w1=lay.w1, b1=lay.b1, w2=lay.w2, b2=lay.b2, w3=lay.w3, b3=lay.b3,
                bytes=lay.bytes, n_out=lay.n_out, elem_bytes=lay.elem_bytes)


def attn_layout(w):
    """Byte offsets of the attention policy's weights (sim_attn_weights_layout) and their
    shapes ([in][out] matrices, vectors)."""
    lib = L.load()
    cfg = L.make_cfg(w, n_envs=max(1, w.get("n_envs", 1)))
    lay = L.SimAttnLayout()
    L.check(lib.sim_attn_weights_layout(C.byref(cfg), C.byref(lay)), "sim_attn_weights_layout")
    F, D, A = w["obs_dim"], w["attn_embed"], 6 * w["n_servers"]
    Hp, Hv = w["mlp_h1"], w["mlp_h2"]
    shapes = dict(w_in=(F, D), b_in=(D,), w_qkv=(D, 3 * D), b_qkv=(3 * D,), w_o=(D, D),
                  b_o=(D,), wp1=(D, Hp), bp1=(Hp,), wp2=(Hp, A), bp2=(A,), wv1=(D, Hv),
                  bv1=(Hv,), wv2=(Hv, 1), bv2=(1,))
    return {k: getattr(lay, k) for k in L.ATTN_KEYS}, shapes, lay.bytes


def _is_attn(w):
    return w.get("policy_kind", L.POLICY_MLP) == L.POLICY_ATTN


def _dims(w, n_out):
    return [w["obs_dim"], w["mlp_h1"], w["mlp_h2"], n_out]


def pack_weights(w, arrays):
    """Host bytes of the ABI weight buffer from arrays w1,b1,w2,b2,w3,b3 ([in][out]).
    Matrices must hold fp32 values (bf16-representable ones in bf16 mode). For the attention
    policy: the fp32 arrays named by sim_attn_weights_layout."""
    if _is_attn(w):
        off, shapes, nbytes = attn_layout(w)
        buf = np.zeros(nbytes, np.uint8)
        for k in L.ATTN_KEYS:
            a = np.ascontiguousarray(arrays[k], dtype=np.float64).reshape(shapes[k])
            f32 = a.astype(np.float32)
            if not np.array_equal(f32.astype(np.float64), a):
                raise ValueError(f"{k} is not fp32-representable")
            raw = f32.tobytes()
            buf[off[k]:off[k] + len(raw)] = np.frombuffer(raw, np.uint8)
        return buf
    lay = weights_layout(w)
    buf = np.zeros(lay["bytes"], np.uint8)
    dims = _dims(w, lay["n_out"])
    for l in range(3):
        W = np.ascontiguousarray(arrays[f"w{l + 1}"], dtype=np.float64).reshape(dims[l], dims[l + 1])
        f32 = W.astype(np.float32)
        if not np.array_equal(f32.astype(np.float64), W):
            raise ValueError(f"w{l + 1} is not fp32-representable")
        if lay["elem_bytes"] == 2:
            bits = f32.view(np.uint32)
            if np.any(bits & 0xFFFF):
                raise ValueError(f"w{l + 1} is not bf16-representable")
            raw = (bits >> 16).astype(np.uint16).tobytes()
        else:
            raw = f32.tobytes()
        o = lay[f"w{l + 1}"]
        buf[o:o + len(raw)] = np.frombuffer(raw, np.uint8)
        b = np.ascontiguousarray(arrays[f"b{l + 1}"], dtype=np.float32).reshape(dims[l + 1])
        o = lay[f"b{l + 1}"]
        buf[o:o + b.nbytes] = np.frombuffer(b.tobytes(), np.uint8)
    return buf


def unpack_weights(w, buf):
    """fp64 arrays of the values held in an ABI weight buffer (host bytes)."""
    if _is_attn(w):
        off, shapes, _ = attn_layout(w)
        buf = np.asarray(buf, dtype=np.uint8)
        out = {}
        for k in L.ATTN_KEYS:
            n = int(np.prod(shapes[k]))
            out[k] = np.frombuffer(buf[off[k]:off[k] + 4 * n].tobytes(),
                                   np.float32).astype(np.float64).reshape(shapes[k])
        return out
    lay = weights_layout(w)
    buf = np.asarray(buf, dtype=np.uint8)
    dims = _dims(w, lay["n_out"])
    out = {}
    for l in range(3):
        n = dims[l] * dims[l + 1]
        o = lay[f"w{l + 1}"]
        if lay["elem_bytes"] == 2:
            bits = np.frombuffer(buf[o:o + 2 * n].tobytes(), np.uint16).astype(np.uint32) << 16
            W = bits.view(np.float32)
        else:
            W = np.frombuffer(buf[o:o + 4 * n].tobytes(), np.float32)
        out[f"w{l + 1}"] = W.astype(np.float64).reshape(dims[l], dims[l + 1])
        o = lay[f"b{l + 1}"]
        out[f"b{l + 1}"] = np.frombuffer(buf[o:o + 4 * dims[l + 1]].tobytes(),
                                         np.float32).astype(np.float64)
    return out


class Trajectory:
    """Caller-owned device buffers of one rollout (sim_traj)."""

    def __init__(self, T, E, F, device, value=False, shadow=False, obs=False, rchk=False,
                 logp=True, reward=True):
        self.T, self.E = T, E
        self.actions = torch.empty((T, E), dtype=torch.uint8, device=device)
        self.logp = torch.empty((T, E), dtype=torch.float32, device=device) if logp else None
        self.reward = torch.empty((T, E), dtype=torch.float64, device=device) if reward else None
        self.reward_shadow = (torch.empty((T, E), dtype=torch.float64, device=device)
                              if shadow else None)
        self.value = torch.empty((T + 1, E), dtype=torch.float32, device=device) if value else None
        self.obs = torch.empty((T + 1, F, E), dtype=torch.float32, device=device) if obs else None
        self.rchk = torch.empty((T, E), dtype=torch.int64, device=device) if rchk else None

    def struct(self):
        return L.SimTraj(*(None if t is None else t.data_ptr() for t in
                           (self.actions, self.logp, self.reward, self.reward_shadow,
                            self.value, self.obs, self.rchk)))


class Sim:
    """One simulator context (sim_create ... sim_destroy) on the current HIP device."""

    def __init__(self, w, n_envs=None, device="cuda", stream=None):
        self.lib = L.load()
        self.w = w
        self.cfg = L.make_cfg(w, n_envs)
        self.E = self.cfg.n_envs
        self.F = w["obs_dim"]
        self.K = w["n_servers"]
        self.A = 6 * self.K
        self.Ap = self.A + (1 if w["value_head"] else 0)
        self.device = torch.device(device)
        self._index = (self.device.index if self.device.index is not None
                       else torch.cuda.current_device())
        self._device = torch.device("cuda", self._index)
        self._work = threading.local()
        self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
        self._raw_stream = self.stream.cuda_stream
        self._ctx = C.c_void_p()
        self._keep = []
        with torch.cuda.device(self._device):
            L.check(self.lib.sim_create(C.byref(self.cfg), C.c_void_p(self.stream.cuda_stream),
                                        C.byref(self._ctx)), "sim_create")

    def close(self):
        if self._ctx:
            L.check(self.lib.sim_destroy(self._ctx), "sim_destroy")
            self._ctx = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *a):
        self.close()

    # -- environment ------------------------------------------------------------------
    def set_trace(self, times, classes, counts):
        """Device tensors times [E][L] f64, classes [E][L] u8, counts [E] i32."""
        self._keep = [times, classes, counts]
        L.check(self.lib.sim_set_trace(self._ctx, _p(times), _p(classes), _p(counts)),
                "sim_set_trace")

    def reset(self, seed):
        L.check(self.lib.sim_reset(self._ctx, C.c_uint64(seed)), "sim_reset")

    def obs(self):
        o = torch.empty((self.F, self.E), dtype=torch.float32, device=self.device)
        L.check(self.lib.sim_obs(self._ctx, _p(o)), "sim_obs")
        return o

    def step(self, actions, want_obs=True, want_reward=True):
        obs = (torch.empty((self.F, self.E), dtype=torch.float32, device=self.device)
               if want_obs else None)
        r = torch.empty(self.E, dtype=torch.float64, device=self.device) if want_reward else None
        rs = (torch.empty(self.E, dtype=torch.float64, device=self.device)
              if want_reward and self.w["shadow"] else None)
        L.check(self.lib.sim_step(self._ctx, _p(actions), _p(obs), _p(r), _p(rs)), "sim_step")
        return obs, r, rs

    def tick(self):
        t = C.c_int32()
        L.check(self.lib.sim_tick(self._ctx, C.byref(t)), "sim_tick")
        return t.value

    # -- policy -----------------------------------------------------------------------
    def init_weights(self, seed):
        lay = weights_layout(self.w)
        buf = torch.zeros(lay["bytes"], dtype=torch.uint8, device=self.device)
        L.check(self.lib.sim_init_weights(self._ctx, C.c_uint64(seed), _p(buf)), "sim_init_weights")
        return buf

    def upload_weights(self, arrays):
        return torch.from_numpy(pack_weights(self.w, arrays)).to(self.device)

    def policy(self, weights, obs, step, want_logits=False):
        E = obs.shape[1]
        assert E == self.E and obs.shape[0] == self.F
        act = torch.empty(E, dtype=torch.uint8, device=self.device)
        logp = torch.empty(E, dtype=torch.float32, device=self.device)
        val = torch.empty(E, dtype=torch.float32, device=self.device) if self.w["value_head"] else None
        lg = torch.empty((self.Ap, E), dtype=torch.float32, device=self.device) if want_logits else None
        L.check(self.lib.sim_policy(self._ctx, _p(weights), _p(obs), C.c_uint32(step), _p(act),
                                    _p(logp), _p(val), _p(lg)), "sim_policy")
        return dict(actions=act, logp=logp, value=val, logits=lg)

    def policy_hidden(self, weights, obs, step):
        """sim_policy_hidden: the policy's outputs plus the hidden activations h1 [H1][E] and
        h2 [H2][E] that the kernel passes between layers."""
        E = obs.shape[1]
        assert E == self.E and obs.shape[0] == self.F
        H1, H2 = self.w["mlp_h1"], self.w["mlp_h2"]
        act = torch.empty(E, dtype=torch.uint8, device=self.device)
        logp = torch.empty(E, dtype=torch.float32, device=self.device)
        val = torch.empty(E, dtype=torch.float32, device=self.device) if self.w["value_head"] else None
        lg = torch.empty((self.Ap, E), dtype=torch.float32, device=self.device)
        hid = torch.empty((H1 + H2, E), dtype=torch.float32, device=self.device)
        L.check(self.lib.sim_policy_hidden(self._ctx, _p(weights), _p(obs), C.c_uint32(step),
                                           _p(act), _p(logp), _p(val), _p(lg), _p(hid)),
                "sim_policy_hidden")
        return dict(actions=act, logp=logp, value=val, logits=lg, h1=hid[:H1], h2=hid[H1:])

    def rollout(self, weights, T, store_obs=False, rchk=False, traj=None):
        if traj is None:
            traj = Trajectory(T, self.E, self.F, self.device, value=bool(self.w["value_head"]),
                              shadow=bool(self.w["shadow"]), obs=store_obs, rchk=rchk)
        st = traj.struct()
        L.check(self.lib.sim_rollout(self._ctx, _p(weights), T, C.byref(st)), "sim_rollout")
        return traj

    def returns_gae(self, r, v, gamma, lam, adv=None, ret=None):
        T = r.shape[0]
        adv = torch.empty_like(r) if adv is None else adv
        ret = torch.empty_like(r) if ret is None else ret
        L.check(self.lib.returns_gae(self._ctx, T, _p(r), _p(v), C.c_double(gamma),
                                     C.c_double(lam), _p(adv), _p(ret)), "returns_gae")
        return adv, ret

    def ppo_grad_count(self):
        n = C.c_int64()
        L.check(self.lib.sim_ppo_grad_count(C.byref(self.cfg), C.byref(n)), "sim_ppo_grad_count")
        return n.value

    def ppo_minibatch_grad(self, weights, obs, actions, logp_old, adv, ret, M, seed, clip=0.2,
                           c_value=0.5, c_entropy=0.01, want_index=False, grads=None, loss=None,
                           noalloc=False):
        """One PPO minibatch: obs [T(+1)][F][E] (rows 0..T-1 used), actions/logp_old/adv/ret
        [T][E]. Returns (grads fp32 flat W1,b1,W2,b2,W3,b3; loss [4] fp64; index or None).
        noalloc=True calls ppo_minibatch_grad_noalloc (the library's fixed scratch)."""
        T = actions.shape[0]
        assert actions.shape[1] == self.E and obs.shape[1] == self.F and obs.shape[0] >= T
        grads = (torch.empty(self.ppo_grad_count(), dtype=torch.float32, device=self.device)
                 if grads is None else grads)
        loss = torch.empty(4, dtype=torch.float64, device=self.device) if loss is None else loss
        idx = torch.empty(M, dtype=torch.int64, device=self.device) if want_index else None
        name = "ppo_minibatch_grad_noalloc" if noalloc else "ppo_minibatch_grad"
        L.check(getattr(self.lib, name)(self._ctx, _p(weights), T, _p(obs), _p(actions),
                                        _p(logp_old), _p(adv), _p(ret), M, C.c_uint64(seed),
                                        clip, c_value, c_entropy, _p(grads), _p(loss), _p(idx)),
                name)
        return grads, loss, idx

    def reinforce_minibatch_grad(self, weights, obs, actions, adv, ret, M, seed, c_value=0.5,
                                 c_entropy=0.01, want_index=False, grads=None, loss=None):
        """REINFORCE with baseline on one minibatch (adv = G - V, ret = G)."""
        T = actions.shape[0]
        assert actions.shape[1] == self.E and obs.shape[1] == self.F and obs.shape[0] >= T
        grads = (torch.empty(self.ppo_grad_count(), dtype=torch.float32, device=self.device)
                 if grads is None else grads)
        loss = torch.empty(4, dtype=torch.float64, device=self.device) if loss is None else loss
        idx = torch.empty(M, dtype=torch.int64, device=self.device) if want_index else None
        L.check(self.lib.reinforce_minibatch_grad(self._ctx, _p(weights), T, _p(obs), _p(actions),
                                                  _p(adv), _p(ret), M, C.c_uint64(seed), c_value,
                                                  c_entropy, _p(grads), _p(loss), _p(idx)),
                "reinforce_minibatch_grad")
        return grads, loss, idx

    # -- operators for the caller's own networks -------------------------------------------
    # They work on the tensors' memory and are no part of torch's autograd: results do not require
    # gradients, and a gradient is computed where its function is called.
    def _check(self, name, t, shape, dtypes):
        """`t` is a tensor on the context's device, of this shape and one of these types."""
        if t.dtype in dtypes and t.shape == shape and t.device == self._device:
            return
        if t.device != self._device:
            raise ValueError(f"{name} is on {t.device}, the context on {self._device}")
        if t.shape != shape:
            raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
        raise ValueError(f"{name} is {t.dtype}, expected {' or '.join(map(str, dtypes))}")

    def _flat(self, name, t, shape, dtypes):
        """As _check, of a tensor (or None) that is read as one contiguous array."""
        if t is None:
            return
        self._check(name, t, shape, dtypes)
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")

    def _call(self, name, sizes, *args):
        """An operator's entry point with work memory, ordered after the work of the current
        stream, and that stream after it, where the context has another one. The memory is kept
        from call to call, per thread, where calls follow one another on the context's stream;
        a captured call, whose replays do not, gets its own, and so does one from another
        stream, whose allocations torch orders by that stream, or made while another device is the
        current one, whose capture alone torch tells of."""
        sizes_p, need = C.byref(sizes), C.c_size_t()
        L.check(getattr(self.lib, name + "_work")(sizes_p, C.byref(need)), name)
        work, need = None, need.value
        same = torch._C._cuda_getCurrentRawStream(self._index) == self._raw_stream
        if need:
            work = getattr(self._work, "memory", None)
            if (not same or torch.cuda.current_device() != self._index
                    or torch.cuda.is_current_stream_capturing()):
                work = torch.empty(need, dtype=torch.uint8, device=self._device)
            elif work is None or work.numel() < need:
                work = self._work.memory = torch.empty(need, dtype=torch.uint8, device=self._device)
        if not same:
            now = torch.cuda.current_stream(self._device)
            self.stream.wait_stream(now)
        rc = getattr(self.lib, name)(self._ctx, sizes_p, *args, _a(work), need)
        if not same:   # `work` is held until here: what it is given to next comes after the call
            now.wait_stream(self.stream)
        if rc:
            L.check(rc, name)

    def gated_scan(self, gate, x, h0=None, lengths=None, kind="linear", reverse=False, y=None,
                   state=None, want_y=True):
        """The recurrence h = gate_t h + x_t (kind "linear") or, with f = sigmoid(gate_t),
        h = f h + (1 - f) x_t ("sigmoid") over gate, x [B][T][D], or [T][D] for one sequence, from
        h0 [B][D] (fp64 for fp64 inputs, otherwise fp32; default 0), backwards in t with
        `reverse`. lengths [B] int32: later steps are padding. Returns (y, state): the state
        after each step, in the inputs' type (None unless want_y), and the last state, which
        may be written over h0 (state=h0). With more than 4 steps the gates of runs of steps are
        multiplied up: linear gates beyond 1 need products over any run that stay finite in the
        state's type (gated_scan in batchsim.h)."""
        one = gate.dim() == 2
        if one:
            gate, x, y = gate[None], x[None], None if y is None else y[None]
            h0, state = (None if s is None else s.view(1, -1) for s in (h0, state))
        B, T, D = gate.shape
        wide = torch.float64 if gate.dtype == torch.float64 else torch.float32
        self._check("gate", gate, (B, T, D), _FLOAT)
        self._check("x", x, (B, T, D), (gate.dtype,))
        self._flat("h0", h0, (B, D), (wide,))
        self._flat("lengths", lengths, (B,), (torch.int32,))
        if y is not None:
            self._check("y", y, (B, T, D), (gate.dtype,))
        elif want_y:
            y = gate.new_empty((B, T, D))
        if state is None:
            state = gate.new_empty((B, D), dtype=wide)
        else:
            self._flat("state", state, (B, D), (wide,))
        sizes = L.SimScan(_FLOAT[gate.dtype], L.GATE_KINDS[kind], int(reverse), B, T, D)
        self._call("gated_scan", sizes, _seq(gate), _seq(x), _a(lengths), _a(h0), _seq(y), _a(state))
        return (None if y is None else y[0], state[0]) if one else (y, state)

    def gated_scan_grad(self, gate, x, y, dy, h0=None, dstate=None, lengths=None, kind="linear",
                        reverse=False, dgate=None, dx=None, dh0=None, want_gate=True):
        """Gradient of gated_scan: gate, x, y (its output), dy [B][T][D] or [T][D], dstate [B][D]
        the gradient of its last state. Returns (dgate, dx, dh0) of the inputs' full shapes (sum
        over the dimensions that an input was broadcast along); with want_gate=False dgate is
        None and y (and x) may be. Products of gates must be finite as for gated_scan, with any
        number of steps."""
        one = gate.dim() == 2
        if one:
            gate, x, y, dy, dgate, dx = (None if t is None else t[None]
                                         for t in (gate, x, y, dy, dgate, dx))
            h0, dstate, dh0 = (None if s is None else s.view(1, -1) for s in (h0, dstate, dh0))
        B, T, D = gate.shape
        wide = torch.float64 if gate.dtype == torch.float64 else torch.float32
        self._check("gate", gate, (B, T, D), _FLOAT)
        for name, t in (("x", x), ("y", y), ("dy", dy), ("dgate", dgate), ("dx", dx)):
            if t is not None:
                self._check(name, t, (B, T, D), (gate.dtype,))
        self._flat("h0", h0, (B, D), (wide,))
        self._flat("dstate", dstate, (B, D), (wide,))
        self._flat("lengths", lengths, (B,), (torch.int32,))
        if dgate is None and want_gate:
            dgate = gate.new_empty((B, T, D))
        if dx is None:
            dx = gate.new_empty((B, T, D))
        if dh0 is None:
            dh0 = gate.new_empty((B, D), dtype=wide)
        else:
            self._flat("dh0", dh0, (B, D), (wide,))
        sizes = L.SimScan(_FLOAT[gate.dtype], L.GATE_KINDS[kind], int(reverse), B, T, D)
        self._call("gated_scan_grad", sizes, _seq(gate), _seq(x), _seq(y), _seq(dy), _a(lengths),
                   _a(h0), _a(dstate), _seq(dgate), _seq(dx), _a(dh0))
        if one:
            return None if dgate is None else dgate[0], dx[0], dh0[0]
        return dgate, dx, dh0

    def _grad_like(self, logits, grad, want):
        if grad is not None:
            self._check("grad", grad, logits.shape, (logits.dtype,))
            return grad
        if not want:
            return None
        N, A = logits.shape
        if logits.stride(1) == 1 or A == 1:
            return logits.new_empty((N, A))
        return logits.new_empty((A, N)).t()

    def policy_loss(self, logits, actions, adv, logp_old=None, logp_ref=None, weight=None,
                    mask=None, clip=0.2, c_kl=0.0, c_entropy=0.0, grad=None, want_grad=True):
        """Clipped policy loss with a KL term over logits [N][A] of any network (rows of actions,
        or sim.policy's [A][E] logits transposed) and its gradient: actions [N] uint8, int32 or
        int64, adv [N] fp32 or fp64, logp_old, logp_ref, weight [N] fp32 (0: padding; default
        1/N), mask [N][A] bool or uint8 (0 forbids). Returns dict(loss [4] fp32: total, policy, KL and
        entropy terms; logp [N]; grad [N][A] in the logits' type, which may be the logits
        themselves: grad=logits). Few samples of more than 384 actions are much faster as rows."""
        N, A = logits.shape
        self._check("logits", logits, (N, A), (torch.float32, torch.bfloat16, torch.float16))
        self._flat("actions", actions, (N,), _INT)
        self._flat("adv", adv, (N,), (torch.float32, torch.float64))
        for name, t in (("logp_old", logp_old), ("logp_ref", logp_ref), ("weight", weight)):
            self._flat(name, t, (N,), (torch.float32,))
        if mask is not None:
            self._check("mask", mask, (N, A), (torch.bool, torch.uint8))
        grad = self._grad_like(logits, grad, want_grad)
        loss = logits.new_empty(4, dtype=torch.float32)
        logp = logits.new_empty(N, dtype=torch.float32)
        sizes = L.SimPolicyLoss(N, A, _FLOAT[logits.dtype], _INT[actions.dtype], _FLOAT[adv.dtype],
                                clip, c_kl, c_entropy)
        self._call("policy_loss", sizes, _mat(logits), _mat(mask), _a(actions), _a(weight),
                   _a(logp_old), _a(logp_ref), _a(adv), _mat(grad), _a(logp), _a(loss))
        return dict(loss=loss, logp=logp, grad=grad)

    def balance_loss(self, logits, index, live=None, group=1, coef=1.0, grad=None, want_grad=True):
        """Balance loss of a router's logits [N][A] whose rows chose the columns index [N][k]
        (uint8, int32 or int64; -1: none), its counts and its gradient; `group` consecutive
        columns count as one target (6 for the simulator's actions). live [N] bool or uint8: the
        other rows are padding. Returns dict(loss (fp32 scalar), counts [A/group] int64, grad
        [N][A])."""
        N, A = logits.shape
        self._check("logits", logits, (N, A), (torch.float32, torch.bfloat16, torch.float16))
        if index.dim() != 2:
            raise ValueError("index has shape [N][k]")
        k = index.shape[1]
        self._flat("index", index, (N, k), _INT)
        self._flat("live", live, (N,), (torch.bool, torch.uint8))
        grad = self._grad_like(logits, grad, want_grad)
        counts = logits.new_empty(max(1, A // max(1, group)), dtype=torch.int64)
        loss = logits.new_empty((), dtype=torch.float32)
        sizes = L.SimBalance(N, A, k, group, _FLOAT[logits.dtype], _INT[index.dtype], coef)
        self._call("balance_loss", sizes, _mat(logits), _a(index), _a(live), _mat(grad), _a(counts),
                   _a(loss))
        return dict(loss=loss, counts=counts, grad=grad)

    def params_from_weights(self, weights):
        p = torch.empty(self.ppo_grad_count(), dtype=torch.float32, device=self.device)
        L.check(self.lib.sim_params_from_weights(self._ctx, _p(weights), _p(p)),
                "sim_params_from_weights")
        return p

    def adam_update(self, params, grads, m, v, step, lr, beta1=0.9, beta2=0.999, eps=1e-8,
                    weights=None):
        L.check(self.lib.adam_update(self._ctx, _p(params), _p(grads), _p(m), _p(v), step, lr,
                                     beta1, beta2, eps, _p(weights)), "adam_update")

    def update(self, weights, params, m, v, step, obs, actions, logp_old, adv, ret, algo,
               epochs, minibatches, M, seed, lr, clip=0.2, c_value=0.5, c_entropy=0.01,
               beta1=0.9, beta2=0.999, eps=1e-8, want_losses=True):
        """sim_update: epochs x minibatches of gradient + Adam; returns (new step, losses)."""
        T = actions.shape[0]
        cfg = L.SimUpdateCfg(algo, epochs, minibatches, M, seed, clip, c_value, c_entropy, lr,
                             beta1, beta2, eps)
        st = C.c_int32(step)
        losses = (torch.empty((epochs * minibatches, 4), dtype=torch.float64, device=self.device)
                  if want_losses else None)
        L.check(self.lib.sim_update(self._ctx, C.byref(cfg), _p(weights), _p(params), _p(m),
                                    _p(v), C.byref(st), T, _p(obs), _p(actions), _p(logp_old),
                                    _p(adv), _p(ret), _p(losses)), "sim_update")
        return st.value, losses

    def unflatten_grads(self, g):
        """Split a flat gradient vector (host numpy) into the policy's arrays (W1,b1,W2,b2,W3,b3,
        or the attention policy's fourteen in sim_attn_layout order)."""
        if _is_attn(self.w):
            _, sh, _ = attn_layout(self.w)
            shapes = [(k, sh[k]) for k in L.ATTN_KEYS]
        else:
            F, H1, H2, Ap = self.F, self.w["mlp_h1"], self.w["mlp_h2"], self.Ap
            shapes = [("w1", (F, H1)), ("b1", (H1,)), ("w2", (H1, H2)), ("b2", (H2,)),
                      ("w3", (H2, Ap)), ("b3", (Ap,))]
        out, o = {}, 0
        for k, sh in shapes:
            n = int(np.prod(sh))
            out[k] = np.asarray(g[o:o + n]).reshape(sh)
            o += n
        return out

    # -- checkpoint / resume ------------------------------------------------------------
    def get_state(self, device=True):
        """Snapshot of every environment's state, the tick counter and the seed, as a uint8
        tensor on the device (or in host memory)."""
        n = C.c_size_t()
        L.check(self.lib.sim_get_state(self._ctx, None, C.byref(n)), "sim_get_state")
        buf = torch.empty(n.value, dtype=torch.uint8, device=self.device if device else "cpu")
        L.check(self.lib.sim_get_state(self._ctx, _p(buf), C.byref(n)), "sim_get_state")
        return buf

    def set_state(self, buf):
        L.check(self.lib.sim_set_state(self._ctx, _p(buf), buf.numel()), "sim_set_state")

    # -- statistics -------------------------------------------------------------------
    def counters(self):
        cnt = torch.empty((2, L.NCNT, self.E), dtype=torch.int64, device=self.device)
        sums = torch.empty((2, L.NSUM, self.E), dtype=torch.float64, device=self.device)
        L.check(self.lib.sim_counters(self._ctx, _p(cnt), _p(sums)), "sim_counters")
        return cnt, sums

    def checksums(self):
        chk = torch.empty((2, self.E), dtype=torch.int64, device=self.device)
        L.check(self.lib.sim_checksums(self._ctx, _p(chk)), "sim_checksums")
        return chk

    def stats(self):
        t = L.SimTotals()
        L.check(self.lib.sim_stats(self._ctx, C.byref(t)), "sim_stats")
        return dict(cnt=np.array([[t.cnt[s][i] for i in range(L.NCNT)] for s in range(2)]),
                    sum=np.array([[t.sum[s][i] for i in range(L.NSUM)] for s in range(2)]))

    def sync(self):
        L.check(self.lib.sim_sync(self._ctx), "sim_sync")

    # -- tracing ----------------------------------------------------------------------
    def set_timing(self, on):
        L.check(self.lib.sim_set_timing(self._ctx, 1 if on else 0), "sim_set_timing")

    def set_graphs(self, on):
        """Rollout graphs on (default) or off (every rollout launched eagerly)."""
        L.check(self.lib.sim_set_graphs(self._ctx, 1 if on else 0), "sim_set_graphs")

    def set_fused_rollout(self, mode):
        """Fused small-batch rollouts: FUSE_AUTO (default), FUSE_ON or FUSE_OFF (per-tick
        launches); see sim_set_fused_rollout."""
        L.check(self.lib.sim_set_fused_rollout(self._ctx, int(mode)), "sim_set_fused_rollout")

    def graph_stats(self):
        """(graphs captured, rollouts replayed from a graph)."""
        c, r = C.c_int64(0), C.c_int64(0)
        L.check(self.lib.sim_graph_stats(self._ctx, C.byref(c), C.byref(r)), "sim_graph_stats")
        return c.value, r.value

    def get_timing(self, clear=True):
        """Per kernel class: (total ms, launches) from HIP events on the context's stream."""
        ms = (C.c_double * len(L.KERNEL_CLASSES))()
        n = (C.c_int64 * len(L.KERNEL_CLASSES))()
        L.check(self.lib.sim_get_timing(self._ctx, ms, n, 1 if clear else 0), "sim_get_timing")
        return {k: (ms[i], n[i]) for i, k in enumerate(L.KERNEL_CLASSES)}
