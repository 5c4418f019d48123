"""The entry points of linear attention, log-probabilities and orthogonalised updates without a GPU (as
test_ops_host.py, over ops_stub.cpp's recording HIP runtime): what they refuse, that a refused call launches nothing,
that a call is launched on the context's device and allocates nothing, and the launches' limits over the sizes."""
import ctypes as C
import itertools

import pytest

import ops_stub
from paper_2607_05272_amd import _lib as L
from seq_ops_stub import run

P = 1 << 40


@pytest.fixture(scope="module")
def stub(tmp_path_factory):
    return ops_stub.build(str(tmp_path_factory.mktemp("stub") / "libopsstub.so"))


def attn(**kw):
    return dict(dict(B=3, T=40, H=4, Hk=2, Dk=16, Dv=24, dtype=2, scale=0.25), **kw)


def logp(**kw):
    return dict(dict(N=100, A=48, top=4, dtype=1, token_type=2), **kw)


def orth(**kw):
    return dict(dict(n=2, M=40, N=50, steps=5, dtype=1, a=3.4445, b=-4.775, c=2.0315, eps=1e-7, scale=1.0), **kw)


def heads(i, H, D, T=40):
    return [P + (i << 32), T * H * D, H * D, D]


def mat(i, sn=48, sa=1):
    return [P + (i << 32), sn, sa]


def mats(i, M=40, N=50):
    return [P + (i << 32), M * N, N, 1]


ARGS = {"linear_attn": [heads(1, 4, 16), heads(2, 2, 16), heads(3, 2, 24), P, P, P, heads(4, 4, 24), P],
        "linear_attn_grad": [heads(1, 4, 16), heads(2, 2, 16), heads(3, 2, 24), P, heads(4, 4, 24), P, P, P,
                             heads(5, 4, 16), heads(6, 2, 16), heads(7, 2, 24), P],
        "token_logprobs": [mat(1), None, P, None, P, P, P, P],
        "token_logprobs_grad": [mat(1), None, P, None, P, P, mat(2)],
        "orthogonalize": [mats(1), mats(2)]}
SIZES = {"linear_attn": attn, "linear_attn_grad": attn, "token_logprobs": logp, "token_logprobs_grad": logp,
         "orthogonalize": orth}


def call(name, sizes=(), **kw):
    """A good call of `name` with some sizes and some arguments (by place: a0, a1, ...) replaced."""
    a, extra = list(ARGS[name]), {}
    for k, v in kw.items():
        if k[0] == "a" and k[1:].isdigit():
            a[int(k[1:])] = v
        else:
            extra[k] = v
    return dict(call=name, sizes=SIZES[name](**dict(sizes)), args=a, **extra)


def launches(log):
    return [l for l in log if l[0] != "need"]


def test_good_calls_launch_on_the_contexts_device_and_allocate_nothing(stub):
    calls = [call(n) for n in ARGS]
    out = run(stub, calls + [dict(device=1)] + calls)
    n = len(calls)
    for (rc, msg, log), (rc1, _, log1) in zip(out[:n], out[n + 1:]):
        log, log1 = launches(log), launches(log1)
        assert rc == rc1 == 0, msg
        assert log and all(l[0] == "launch" for l in log)
        assert log1[0] == ["device", "0"] and log1[-1] == ["device", "1"]
        assert log1[1:-1] == log


@pytest.mark.parametrize("name", sorted(ARGS))
def test_common_refusals(stub, name):
    bad = [dict(call(name), sizes=None), dict(call(name), no_ctx=True), call(name, dict(dtype=9)), call(name, dict(dtype=-1)),
           call(name, dict(dtype=0))]
    need = int(run(stub, [call(name)])[0][2][-1][1])
    if need:
        bad += [call(name, less=-1), call(name, work=0), call(name, at=ops_stub.WORK + 8)]
    for c, (rc, msg, log) in zip(bad, run(stub, bad)):
        assert rc == -1 and msg and not launches(log), (c, rc, msg, log)


def refused(stub, bad):
    for (what, c), (rc, msg, log) in zip(bad, run(stub, [c for _, c in bad])):
        assert rc in (-1, -5) and what in msg and not launches(log), (what, msg, log)


def accepted(stub, good):
    for c, (rc, msg, _) in zip(good, run(stub, good)):
        assert rc == 0, (c, msg)


def test_linear_attn_refusals(stub):
    f, g = "linear_attn", "linear_attn_grad"
    refused(stub, [
        (">= 0", call(f, dict(B=-1))), (">= 0", call(f, dict(T=-1))), ("2^30", call(f, dict(T=1 << 30))), ("2^21", call(f, dict(B=1 << 19))),
        ("divide", call(f, dict(H=3))), ("divide", call(f, dict(Hk=0))), ("divide", call(f, dict(H=0))), (">= 1", call(f, dict(Dk=0))),
        ("256", call(f, dict(Dk=257))), ("256", call(f, dict(Dv=257))), ("scale", call(f, dict(scale=float("nan")))),
        ("scale", call(f, dict(scale=float("inf")))), ("q is NULL", call(f, a0=None)), ("k is NULL", call(f, a1=None)),
        ("v is NULL", call(f, a2=None)), ("decay is NULL", call(f, a3=None)), ("negative", call(f, a0=[P, -1, 64, 16])),
        ("2^62", call(f, a0=[P, 1 << 61, 64, 16])), ("share memory", call(f, a6=[P, 3840, 95, 24])),
        ("share memory", call(f, a6=[P, 3840, 96, 23])), ("share memory", call(f, a6=[P, 0, 96, 24])),
        ("aligned", call(f, a0=[P + 1, 2560, 64, 16])), ("aligned", call(f, a3=P + 2)), ("aligned", call(f, a4=P + 2)),
        ("aligned", call(f, a5=P + 2)), ("aligned", call(f, a7=P + 2)),
        ("q is NULL", call(g, a0=None)), ("k is NULL", call(g, a1=None)), ("v is NULL", call(g, a2=None)), ("dy is NULL", call(g, a4=None)),
        ("share memory", call(g, a9=[P, 1280, 32, 15])), ("aligned", call(g, a11=P + 2)), ("aligned", call(g, a7=P + 1))])
    accepted(stub, [
        call(f, a6=None), call(f, a0=None, a6=None), call(f, a7=None), call(f, a4=None, a5=None), call(f, dict(B=0), a0=None, a3=None),
        call(f, dict(T=0), a0=None, a1=None, a2=None), call(f, a0=[P, 0, 0, 0]), call(f, a6=[P, 24, 288, 72]),
        call(f, dict(B=1), a6=[P, 0, 96, 24]), call(g, a2=None, a8=None, a9=None), call(g, a1=None, a8=None, a10=None),
        call(g, a1=None, a2=None, a8=None, a9=None, a10=None), call(g, a8=None, a9=None, a10=None, a11=None), call(g, a5=None, a6=None, a7=None)])


def test_logprob_refusals(stub):
    f, g = "token_logprobs", "token_logprobs_grad"
    refused(stub, [
        ("N must", call(f, dict(N=-1))), ("N must", call(f, dict(N=1 << 31))), ("A must", call(f, dict(A=0))), ("2^30", call(f, dict(A=1 << 30))),
        ("top must", call(f, dict(top=-1))), ("64", call(f, dict(top=65))), ("token type", call(f, dict(token_type=3))),
        ("logits is NULL", call(f, a0=None)), ("needs tokens", call(f, a2=None)), ("one stride", call(f, a0=mat(1, 96, 2))),
        ("negative", call(f, a1=mat(3, -1, 1))), ("aligned", call(f, a2=P + 4)), ("aligned", call(f, a4=P + 2)), ("aligned", call(f, a6=P + 4)),
        ("aligned", call(f, a7=P + 2)), ("grad is NULL", call(g, a6=None)), ("needs tokens", call(g, a2=None)),
        ("share memory", call(g, a6=mat(2, 47))), ("other strides", call(g, a6=mat(1, 49))), ("aligned", call(g, a5=P + 2)),
        ("one stride", call(g, a6=mat(2, 96, 2)))])
    accepted(stub, [
        call(f, dict(N=0), a0=None, a2=None), call(f, a2=None, a4=None), call(f, a4=None, a5=None, a6=None, a7=None), call(f, a1=mat(3, 0, 1)),
        call(f, a3=P), call(f, dict(top=0), a6=None, a7=None), call(f, a6=None), call(f, a7=None), call(f, a0=mat(1, 1, 100)),
        call(g, a6=mat(1)), call(g, a4=None, a5=None), call(g, a2=None, a4=None), call(g, dict(N=0), a0=None, a6=None)])


def test_orthogonalize_refusals(stub):
    f = "orthogonalize"
    refused(stub, [
        (">= 0", call(f, dict(M=-1))), (">= 0", call(f, dict(n=-1))), ("65536", call(f, dict(N=65537))), ("65536", call(f, dict(n=65536))),
        ("steps", call(f, dict(steps=-1))), ("steps", call(f, dict(steps=33))), ("finite", call(f, dict(a=float("nan")))),
        ("finite", call(f, dict(scale=float("inf")))), ("eps", call(f, dict(eps=-1.0))), ("update is NULL", call(f, a0=None)),
        ("out is NULL", call(f, a1=None)), ("negative", call(f, a0=[P, 2000, -50, 1])), ("share memory", call(f, a1=[P, 2000, 49, 1])),
        ("share memory", call(f, a1=[P, 0, 50, 1])), ("aligned", call(f, a0=[P + 2, 2000, 50, 1])), ("2^62", call(f, a0=[P, 1 << 62, 50, 1]))])
    accepted(stub, [call(f, a0=[P, 0, 0, 0]), call(f, a1=mats(1)), call(f, a1=[P, 1, 100, 2]), call(f, dict(n=0), a0=None, a1=None),
                    call(f, dict(M=0), a0=None, a1=None), call(f, dict(steps=0)), call(f, dict(n=1), a1=[P, 0, 50, 1])])


def test_every_size_launches_within_limits(stub):
    """Grids, blocks and LDS of the launches over the range of sizes, types and layouts."""
    calls = []
    for name, (B, T, H, Hk), (Dk, Dv), dt in itertools.product(
            ("linear_attn", "linear_attn_grad"),
            [(1, 1, 1, 1), (64, 1, 16, 4), (8, 2048, 16, 4), (1, 32768, 8, 8), ((1 << 21) - 1, 1, 1, 1), ((1 << 21) - 1, 17, 1, 1), (3, 17, 1 << 19, 1 << 10), (1, (1 << 30) - 1, 2, 1),
             (1, 1 << 20, 64, 64), (2, 5, 1, 1), (2, 0, 3, 1), (40000, 20, 2, 2)],
            [(1, 1), (64, 64), (128, 128), (256, 256), (256, 1), (33, 200)], (1, 2, 3)):
        h = lambda i, n, d: [P + (i << 42), T * n * d, n * d, d]   # noqa: E731
        s = dict(B=B, T=T, H=H, Hk=Hk, Dk=Dk, Dv=Dv, dtype=dt)
        if name == "linear_attn":
            calls.append(call(name, s, a0=h(1, H, Dk), a1=h(2, Hk, Dk), a2=h(3, Hk, Dv), a6=h(4, H, Dv)))
        else:
            calls.append(call(name, s, a0=h(1, H, Dk), a1=h(2, Hk, Dk), a2=h(3, Hk, Dv), a4=h(4, H, Dv), a8=h(5, H, Dk), a9=h(6, Hk, Dk), a10=h(7, Hk, Dv)))
    for (N, A), top, dt, lay, name in itertools.product(
            [(1, 1), (256, 6), (131072, 96), (32, 131072), (2048, 50257), ((1 << 31) - 1, 3), (1, (1 << 30) - 1), (5, 700), (100000, 2000)],
            (0, 1, 20, 64), (1, 2, 3), (lambda i, n, a: mat(i, a, 1), lambda i, n, a: mat(i, 1, n)), ("token_logprobs", "token_logprobs_grad")):
        extra = {"a0": lay(1, N, A)}
        if name == "token_logprobs_grad":
            extra["a6"] = lay(2, N, A)
        calls.append(call(name, dict(N=N, A=A, top=top, dtype=dt), **extra))
    for (n, M, N), dt, steps in itertools.product(
            [(1, 1, 1), (4, 256, 256), (12, 1365, 512), (1, 4096, 8192), (65535, 8, 8), (1, 65536, 65536), (3, 65536, 1), (2, 130, 4000), (100, 512, 512)],
            (1, 2, 3), (0, 5)):
        calls.append(call("orthogonalize", dict(n=n, M=M, N=N, dtype=dt, steps=steps), a0=mats(1, M, N), a1=mats(2, M, N)))
    for c, (rc, msg, log) in zip(calls, run(stub, calls)):
        assert rc == 0, (c, msg)
        for l in launches(log):
            assert l[0] == "launch", (c, l)
            gx, gy, gz, bx, by, bz, lds, limit = map(int, l[-8:])
            assert 1 <= gx < 1 << 31 and 1 <= gy < 65536 and 1 <= gz < 65536, (c, l)
            assert gx * bx < 1 << 32 and 64 <= bx * by * bz <= 1024 and lds <= limit, (c, l)


def test_struct_sizes():
    assert C.sizeof(L.SimHeads) == C.sizeof(L.SimMats) == 32
    assert C.sizeof(L.SimLinearAttn) == 16 + 6 * 4
    assert C.sizeof(L.SimLogprobs) == 8 + 4 * 4
    assert C.sizeof(L.SimOrtho) == 24 + 2 * 4 + 5 * 4 + 4
