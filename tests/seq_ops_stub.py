"""The entry points of linear attention, log-probabilities and orthogonalised updates of the built library over
ops_stub.cpp's recording HIP runtime, on a machine without a GPU. Run as a program (a process of its own): reads a list
of calls as JSON from stdin and prints for each its status, its message and what it launched.

    {"call": name, "sizes": {field: value}, "args": [...]}
        an entry point; an argument is null, a pointer (nothing is read) or [pointer, strides...]; "work" the bytes of
        work memory, or "less" what it has less than the *_work call asks for; "at" its address
    {"device": d}                        the current device from here on (the context is on 0)
"""
import ctypes as C
import importlib.util
import json
import os
import subprocess
import sys

import ops_stub

KINDS = {"linear_attn": "SimLinearAttn", "linear_attn_grad": "SimLinearAttn", "token_logprobs": "SimLogprobs",
         "token_logprobs_grad": "SimLogprobs", "orthogonalize": "SimOrtho"}


def run(stub, calls):
    """[(status, message, log lines split into words)], in a process where no other HIP runtime is loaded"""
    sys.path.insert(0, os.path.dirname(ops_stub.HERE))
    from workloads import preset
    r = subprocess.run([sys.executable, os.path.abspath(__file__), stub], input=json.dumps([preset("C1"), calls]),
                       capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
    return [(rc, msg, [l.split() for l in log]) for rc, msg, log in json.loads(r.stdout.splitlines()[-1])]


def main(path):
    lib = C.CDLL(path, mode=C.RTLD_GLOBAL)
    lib.stub_log.restype = C.c_char_p
    spec = importlib.util.spec_from_file_location("_lib", os.path.join(ops_stub.PKG, "_lib.py"))
    M = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(M)
    dll, ctx, out = M.load(), C.c_void_p(), []
    w, calls = json.load(sys.stdin)
    cfg = M.make_cfg(w, 1)
    assert dll.sim_create(C.byref(cfg), C.c_void_p(8), C.byref(ctx)) == 0
    for c in calls:
        lib.stub_clear()
        if "device" in c:
            lib.stub_device(c["device"])
            out.append((0, "", []))
            continue
        name = c["call"]
        sizes = None if c["sizes"] is None else C.byref(getattr(M, KINDS[name])(**c["sizes"]))
        need = C.c_size_t()
        getattr(dll, name + "_work")(sizes, C.byref(need))
        args = [C.byref({3: M.SimMat, 4: M.SimHeads}[len(a)](*a)) if isinstance(a, list) else a for a in c["args"]]
        have = c["work"] if "work" in c else max(0, need.value + c.get("less", 0))
        rc = getattr(dll, name)(None if c.get("no_ctx") else ctx, sizes, *args, c.get("at", ops_stub.WORK) if have else None, have)
        out.append((rc, dll.sim_last_error().decode() if rc else "", lib.stub_log().decode().splitlines() + [f"need {need.value}"]))
    print(json.dumps(out))


if __name__ == "__main__":
    main(sys.argv[1])
