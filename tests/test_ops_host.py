"""The operators' entry points without a GPU: what they refuse, that a refused call launches
nothing, that a call is launched on the context's device, and that none allocates."""
import ctypes as C
import itertools

import pytest

import ops_stub
from paper_2607_05272_amd import _lib as L

P = 1 << 40


@pytest.fixture(scope="module")
def stub(tmp_path_factory):
    return ops_stub.build(str(tmp_path_factory.mktemp("stub") / "libopsstub.so"))


def scan(**kw):
    return dict(dict(dtype=1, kind=1, reverse=0, B=3, T=40, D=16), **kw)


def pol(**kw):
    return dict(dict(N=100, A=48, dtype=1, action_type=2, adv_type=1, clip=0.2, c_kl=0.1, c_entropy=0.01), **kw)


def bal(**kw):
    return dict(dict(N=100, A=48, k=2, group=6, dtype=1, index_type=2, coef=0.1), **kw)


def seq(n, st=16, sb=640):
    return [P + (n << 32), sb, st]


def mat(n, sn=48, sa=1):
    return [P + (n << 32), sn, sa]


ARGS = {"gated_scan": [seq(1), seq(2), None, P, seq(3), P],
        "gated_scan_grad": [seq(1), seq(2), seq(3), seq(4), None, P, P, seq(5), seq(6), P],
        "policy_loss": [mat(1), None, P, P, P, P, P, mat(2), P, P],
        "balance_loss": [mat(1), P, P, mat(2), P, P]}
SIZES = {"gated_scan": scan, "gated_scan_grad": scan, "policy_loss": pol, "balance_loss": bal}


def call(name, sizes=(), **args):
    """A good call of `name` with some sizes and some arguments (by place: a0, a1, ...) replaced."""
    a = list(ARGS[name])
    extra = {}
    for k, v in args.items():
        if k[0] == "a" and k[1:].isdigit():
            a[int(k[1:])] = v
        else:
            extra[k] = v
    return dict(call=name, sizes=SIZES[name](**dict(sizes)), args=a, **extra)


def test_good_calls_launch_on_the_contexts_device_and_allocate_nothing(stub):
    calls = [call(n) for n in ARGS]
    out = ops_stub.run(stub, calls + [dict(device=1)] + calls)
    n = len(calls)
    for (rc, msg, log), (rc1, _, log1) in zip(out[:n], out[n + 1:]):
        assert rc == rc1 == 0, msg
        assert log and all(l[0] == "launch" for l in log)
        # device 0 while launching, then device 1 again
        assert log1[0] == ["device", "0"] and log1[-1] == ["device", "1"]
        assert log1[1:-1] == log


@pytest.mark.parametrize("name", sorted(ARGS))
def test_common_refusals(stub, name):
    work = int(ops_stub.run(stub, [dict(work_of=name, sizes=SIZES[name]())])[0][1])
    bad = [dict(call(name), sizes=None), dict(call(name), no_ctx=True), call(name, dict(dtype=9)),
           call(name, dict(dtype=-1))]
    if work:
        bad += [call(name, work=work - 1), call(name, work=0), call(name, at=ops_stub.WORK + 8)]
    for c, (rc, msg, log) in zip(bad, ops_stub.run(stub, bad)):
        assert rc == -1 and msg and not log, (c, rc, msg, log)


def test_scan_refusals(stub):
    bad = [("kind", call("gated_scan", dict(kind=2))), ("reverse", call("gated_scan", dict(reverse=2))),
           (">= 0", call("gated_scan", dict(T=-1))), ("2^30", call("gated_scan", dict(T=1 << 30))),
           ("2^31", call("gated_scan", dict(B=1 << 20, D=1 << 20))), ("gate is NULL", call("gated_scan", a0=None)),
           ("x is NULL", call("gated_scan", a1=None)), ("negative", call("gated_scan", a1=[P, -1, 16])),
           ("2^62", call("gated_scan", a1=[P, 1 << 61, 16])), ("share memory", call("gated_scan", a4=seq(3, st=15))),
           ("share memory", call("gated_scan", a4=seq(3, sb=0))),
           ("share memory", call("gated_scan", a4=[P, 20, 16])),
           ("not aligned", call("gated_scan", a0=[P + 2, 640, 16])), ("aligned", call("gated_scan", a3=P + 2)),
           ("aligned", call("gated_scan", a2=P + 2)),
           ("y is NULL", call("gated_scan_grad", a2=None)), ("x is NULL", call("gated_scan_grad", a1=None)),
           ("dy is NULL", call("gated_scan_grad", a3=None)), ("share memory", call("gated_scan_grad", a8=[P, 640, 0])),
           ("aligned", call("gated_scan_grad", dict(dtype=0), a5=P + 4))]
    for (what, c), (rc, msg, log) in zip(bad, ops_stub.run(stub, [c for _, c in bad])):
        assert rc in (-1, -5) and what in msg and not log, (what, msg, log)
    good = [call("gated_scan", a4=[P, 16, 48]), call("gated_scan", a0=[P, 0, 0]), call("gated_scan", a4=None),
            call("gated_scan", a3=None, a5=None), call("gated_scan", dict(B=0)), call("gated_scan", dict(T=0), a0=None, a1=None),
            call("gated_scan", dict(B=1), a4=[P, 0, 16]),
            call("gated_scan_grad", dict(kind=0), a1=None), call("gated_scan_grad", a1=None, a2=None, a7=None),
            call("gated_scan_grad", a4=P, a5=None, a6=None, a9=None)]
    for c, (rc, msg, _) in zip(good, ops_stub.run(stub, good)):
        assert rc == 0, (c, msg)


def test_policy_refusals(stub):
    bad = [("N must", call("policy_loss", dict(N=-1))), ("N must", call("policy_loss", dict(N=1 << 31))),
           ("A must", call("policy_loss", dict(A=0))), ("A must", call("policy_loss", dict(A=1 << 30))), ("type 0", call("policy_loss", dict(dtype=0))),
           ("action type", call("policy_loss", dict(action_type=3))), ("advantages", call("policy_loss", dict(adv_type=2))),
           ("clip", call("policy_loss", dict(clip=0.0))), ("clip", call("policy_loss", dict(clip=float("nan")))),
           (">= 0", call("policy_loss", dict(c_kl=-1.0))), ("reference", call("policy_loss", a5=None)),
           ("logits is NULL", call("policy_loss", a0=None)), ("one stride", call("policy_loss", a0=mat(1, 96, 2))),
           ("one stride", call("policy_loss", a7=mat(1, 96, 2))), ("negative", call("policy_loss", a1=mat(3, -1, 1))),
           ("share memory", call("policy_loss", a7=mat(2, 0, 1))), ("share memory", call("policy_loss", a7=mat(2, 47, 1))),
           ("share memory", call("policy_loss", a7=mat(2, 1, 99))), ("other strides", call("policy_loss", a7=mat(1, 49, 1))),
           ("NULL", call("policy_loss", a2=None)), ("NULL", call("policy_loss", a6=None)), ("NULL", call("policy_loss", a9=None)),
           ("aligned", call("policy_loss", a2=P + 4)), ("aligned", call("policy_loss", a0=[P + 2, 48, 1])),
           ("aligned", call("policy_loss", dict(adv_type=0), a6=P + 4)), ("2^62", call("policy_loss", a0=mat(1, 1 << 60, 1)))]
    for (what, c), (rc, msg, log) in zip(bad, ops_stub.run(stub, [c for _, c in bad])):
        assert rc in (-1, -5) and what in msg and not log, (what, msg, log)
    good = [call("policy_loss", a0=mat(1, 1, 100), a7=mat(1, 1, 100)), call("policy_loss", a7=None, a8=None),
            call("policy_loss", dict(c_kl=0.0), a3=None, a4=None, a5=None), call("policy_loss", a1=mat(3, 0, 1)),
            call("policy_loss", dict(N=0), a0=None, a2=None, a6=None), call("policy_loss", dict(N=1), a0=mat(1, 7, 1)),
            call("policy_loss", dict(A=1), a0=mat(1, 7, 3), a7=mat(2, 7, 3))]
    for c, (rc, msg, _) in zip(good, ops_stub.run(stub, good)):
        assert rc == 0, (c, msg)


def test_balance_refusals(stub):
    bad = [("N must", call("balance_loss", dict(N=-1))), (">= 1", call("balance_loss", dict(k=0))),
           (">= 1", call("balance_loss", dict(A=0))), ("2^30", call("balance_loss", dict(A=1 << 30, group=1 << 20))), ("N*k", call("balance_loss", dict(N=1 << 30, k=2))),
           ("divide", call("balance_loss", dict(group=5))), ("divide", call("balance_loss", dict(group=-6))),
           ("4096", call("balance_loss", dict(A=4097, group=1), a0=mat(1, 4097), a3=mat(2, 4097))),
           ("index type", call("balance_loss", dict(index_type=-1))), ("type 0", call("balance_loss", dict(dtype=0))),
           ("NULL", call("balance_loss", a1=None)), ("NULL", call("balance_loss", a4=None)),
           ("NULL", call("balance_loss", a5=None)), ("logits is NULL", call("balance_loss", a0=None)),
           ("aligned", call("balance_loss", a1=P + 4)), ("share memory", call("balance_loss", a3=mat(2, 47, 1)))]
    for (what, c), (rc, msg, log) in zip(bad, ops_stub.run(stub, [c for _, c in bad])):
        assert rc in (-1, -5) and what in msg and not log, (what, msg, log)
    good = [call("balance_loss", a2=None), call("balance_loss", a3=None), call("balance_loss", a3=mat(1)),
            call("balance_loss", dict(N=0), a0=None, a1=None), call("balance_loss", a0=mat(1, 1, 100))]
    for c, (rc, msg, _) in zip(good, ops_stub.run(stub, good)):
        assert rc == 0, (c, msg)


def test_every_size_launches_within_limits(stub):
    """Grids, blocks and LDS of the launches over the range of sizes, types and layouts."""
    calls = [call("gated_scan" if g == 0 else "gated_scan_grad", dict(B=b, T=t, D=d, dtype=dt, kind=k),
                  **{f"a{i}": [P + (i << 33), t * d, d] for i in ((0, 1, 4) if g == 0 else (0, 1, 2, 3, 7, 8))})
             for g, (b, t, d), dt, k in itertools.product(
                 (0, 1), [(1, 1, 1), (64, 1, 2048), (1, 1000, 256), (512, 2047, 1), (8, 2048, 2048), (1, 65536, 512),
                          (1, 1, 1 << 30), (1 << 20, 3, 7), (1, (1 << 30) - 1, 1), (16, 1025, 1536), (1, 300000, 5)], range(4), (0, 1))]
    calls += [call("policy_loss", dict(N=n, A=a, dtype=dt, action_type=t), a0=m(1, n, a), a7=m(2, n, a))
              for (n, a), dt, t, m in itertools.product(
                  [(1, 1), (256, 6), (131072, 96), (2048, 50257), (4096, 131072), ((1 << 31) - 1, 3), (1, (1 << 30) - 1), (0, 6), (0, 700), (0, 5000),
                   (0, 200000)],
                  (1, 2, 3), (0, 2), (lambda i, n, a: mat(i, a, 1), lambda i, n, a: mat(i, 1, n)))]
    calls += [call("balance_loss", dict(N=n, A=a, k=k, group=g, dtype=dt), a0=m(1, n, a), a3=m(2, n, a))
              for (n, a, k, g), dt, m in itertools.product(
                  [(1, 1, 1, 1), (65536, 48, 1, 6), (131072, 128, 8, 1), ((1 << 30), 4096, 1, 1), (10, 1023 << 20, 1, 1 << 20), (0, 8, 1, 1)],
                  (1, 2, 3), (lambda i, n, a: mat(i, a, 1), lambda i, n, a: mat(i, 1, n)))]
    for c, (rc, msg, log) in zip(calls, ops_stub.run(stub, calls)):
        assert rc == 0, (c, msg)
        for l in log:
            assert l[0] == "launch", (c, l)
            gx, gy, gz, bx, by, bz, lds, limit = map(int, l[-8:])
            assert 1 <= gx < 1 << 31 and 1 <= gy < 65536 and 1 <= gz < 65536, (c, l)
            assert gx * bx < 1 << 32 and 64 <= bx * by * bz <= 1024 and lds <= limit, (c, l)


def test_struct_sizes():
    assert C.sizeof(L.SimSeq) == C.sizeof(L.SimMat) == 24
    assert C.sizeof(L.SimScan) == 16 + 24
    assert C.sizeof(L.SimPolicyLoss) == 8 + 7 * 4 + 4
    assert C.sizeof(L.SimBalance) == 8 + 6 * 4
