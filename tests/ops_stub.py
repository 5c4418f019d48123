"""The operators' entry points of the built library over ops_stub.cpp's recording HIP runtime, on a
machine without a GPU. Run as a program (a process of its own): reads a list of calls as JSON from
stdin and prints for each its status, its message and what it launched.

    {"call": name, "sizes": {field: value}, "args": [...], "work": bytes}
        an entry point; an argument is null, a pointer (nothing is read) or [pointer, stride,
        stride]; "work" the bytes of work memory (absent: what the *_work call asks for)
    {"work_of": name, "sizes": {..}}     the bytes that name_work gives, as the message
    {"device": d}                        the current device from here on (the context is on 0)
"""
import ctypes as C
import importlib.util
import json
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
PKG = os.path.join(os.path.dirname(HERE), "paper_2607_05272_amd")
WORK = 1 << 44


def build(out):
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-D__HIP_PLATFORM_AMD__", "-w",
                    "-I", "/opt/rocm/include", os.path.join(HERE, "ops_stub.cpp"), "-o", out],
                   check=True)
    return out


def run(stub, calls):
    """[(status, message, log lines split into words)]"""
    sys.path.insert(0, os.path.dirname(HERE))
    from workloads import preset
    r = subprocess.run([sys.executable, os.path.abspath(__file__), stub],
                       input=json.dumps([preset("C1"), calls]), capture_output=True, text=True,
                       timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
    return [(rc, msg, [l.split() for l in log]) for rc, msg, log in json.loads(r.stdout.splitlines()[-1])]


def main(path):
    stub = C.CDLL(path, mode=C.RTLD_GLOBAL)
    stub.stub_log.restype = C.c_char_p
    spec = importlib.util.spec_from_file_location("_lib", os.path.join(PKG, "_lib.py"))
    L = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(L)
    lib, ctx, out = L.load(), C.c_void_p(), []
    w, calls = json.load(sys.stdin)
    cfg = L.make_cfg(w, 1)
    assert lib.sim_create(C.byref(cfg), C.c_void_p(8), C.byref(ctx)) == 0
    kinds = {"gated_scan": L.SimScan, "gated_scan_grad": L.SimScan, "policy_loss": L.SimPolicyLoss,
             "balance_loss": L.SimBalance}
    for c in calls:
        stub.stub_clear()
        if "device" in c:
            stub.stub_device(c["device"])
            out.append((0, "", []))
            continue
        name = c.get("call") or c["work_of"]
        sizes = None if c["sizes"] is None else C.byref(kinds[name](**c["sizes"]))
        need = C.c_size_t()
        rc = getattr(lib, name + "_work")(sizes, C.byref(need))
        if "work_of" in c:
            out.append((rc, str(need.value) if rc == 0 else lib.sim_last_error().decode(), []))
            continue
        args = [C.byref(L.SimSeq(*a)) if isinstance(a, list) else a for a in c["args"]]
        have = c.get("work", need.value)
        rc = getattr(lib, name)(None if c.get("no_ctx") else ctx, sizes, *args, c.get("at", WORK) if have else None, have)
        out.append((rc, lib.sim_last_error().decode() if rc else "", stub.stub_log().decode().splitlines()))
    print(json.dumps(out))


if __name__ == "__main__":
    main(sys.argv[1])
