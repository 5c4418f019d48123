"""The forms that orthogonalize takes for the shapes of test_gpu_orthogonalize_forms.py, over ops_stub.cpp's recording
HIP runtime: the tiles of the three products and the shares of the first one's sum, so that a change of the rule that
picks them leaves no form untested."""
import re

import pytest

import ops_stub
from ortho_shapes import FORMS
from seq_ops_stub import run

P = 1 << 40


@pytest.fixture(scope="module")
def stub(tmp_path_factory):
    return ops_stub.build(str(tmp_path_factory.mktemp("stub") / "libopsstub.so"))


def test_the_shapes_reach_every_form(stub):
    calls = []
    for n, M, N in FORMS:
        for dt in (1, 2, 3):
            calls.append(dict(call="orthogonalize", sizes=dict(n=n, M=M, N=N, steps=1, dtype=dt, a=1.0, b=1.0, c=1.0, eps=0.0, scale=1.0),
                              args=[[P, M * N, N, 1], [P + (1 << 38), M * N, N, 1]]))
    out = run(stub, calls)
    seen = set()
    for c, (rc, msg, log) in zip(calls, out):
        assert rc == 0, msg
        muls = [(re.search(r"ortho_mul_kILi(\d+)ELi(\d+)E", l[1]), int(l[4])) for l in log if l[0] == "launch"]
        muls = [(int(m[1]), int(m[2]), z) for m, z in muls if m]
        assert [k for _, k, _ in muls] == [0, 1, 2]
        got = (muls[0][0], muls[2][0], muls[0][2])
        s = c["sizes"]
        assert got == FORMS[s["n"], s["M"], s["N"]] and muls[1][0] == got[0], (s, got)
        assert any("ortho_sum_k" in l[1] for l in log if l[0] == "launch") == (got[2] > 1)
        seen |= {(t, k) for t, k, _ in muls}
    assert seen == {(t, k) for t in (64, 128, 256) for k in (0, 1, 2)}
    assert {h for h, _, z in FORMS.values() if z > 1} == {64, 128, 256} == {h for h, _, z in FORMS.values() if z == 1} | {256}
