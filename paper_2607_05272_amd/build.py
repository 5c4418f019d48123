"""Compile the HIP library libbatchsim.so for gfx950 (in-tree).

Every translation unit is built with -ffp-contract=off (no implicit fma: the fp64
simulator must round exactly where its source says) and with packed fp32 instructions
disabled. Translation units compile in parallel, then link into one shared library.
"""
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
ROOT = os.path.dirname(HERE)
LIB = os.path.join(HERE, "libbatchsim.so")
BUILD = os.path.join(HERE, "_build")
SOURCES = ["runtime.cpp", "sim_kernels.hip", "mlp_kernels.hip", "gae_kernels.hip",
           "ppo_kernels.hip", "ppo_fused.hip", "train_kernels.hip", "attn_kernels.hip",
           "prim_kernels.hip", "rollout_kernels.hip", "rollout_wide.hip", "ops.cpp", "scan_kernels.hip",
           "logit_kernels.hip"]
HEADERS = ["devmath.hpp", "params.hpp", "policy_dev.hpp", "sim_dev.hpp", "ppo_dev.hpp", "train_dev.hpp",
           "rollout_dev.hpp", "ops.hpp", "ops_dev.hpp"]
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-ffp-contract=off",
         "-fno-fast-math", "-Wall", "-Wno-unused-function",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-I", os.path.join(ROOT, "include")]
# kernels whose loop over the ticks holds the whole simulator and policy: hoisting constants and
# parameters out of it costs more registers than there are (140 spilled vector registers
# against 50; rollouts of 16384 environments of the 8-server system 37.7 -> 30.4 us per tick)
EXTRA = {"rollout_wide.hip": ["-mllvm", "-disable-machine-licm"]}
LINK = []


def _hipcc():
    for p in ("/opt/rocm/bin/hipcc", "hipcc"):
        if os.path.sep not in p or os.path.exists(p):
            return p
    return "hipcc"


def build(force=True, verbose=False):
    """Compile all sources and link libbatchsim.so. Always recompiles when force=True."""
    os.makedirs(BUILD, exist_ok=True)
    deps = [os.path.join(CSRC, f) for f in SOURCES + HEADERS] + [
        os.path.join(ROOT, "include", "batchsim.h")]
    if not force and os.path.exists(LIB) and os.path.getmtime(LIB) >= max(map(os.path.getmtime, deps)):
        return LIB
    hipcc = _hipcc()
    procs = []
    objs = []
    for src in SOURCES:
        obj = os.path.join(BUILD, src.rsplit(".", 1)[0] + ".o")
        objs.append(obj)
        extra = EXTRA.get(src, [])
        cmd = [hipcc, *FLAGS, *extra, "-c", os.path.join(CSRC, src), "-o", obj]
        if src.endswith(".cpp"):
            cmd = [hipcc, *FLAGS, "-x", "hip", "-c", os.path.join(CSRC, src), "-o", obj]
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT,
                                            text=True)))
    failed = []
    for src, p in procs:
        out, _ = p.communicate()
        lines = [l for l in out.splitlines() if "packed-fp32-ops" not in l]
        if p.returncode != 0:
            failed.append((src, "\n".join(lines)))
        elif verbose and lines:
            print("\n".join(lines), file=sys.stderr)
    if failed:
        raise RuntimeError("HIP build failed:\n" + "\n\n".join(f"[{s}]\n{o}" for s, o in failed))
    tmp = LIB + ".tmp"
    subprocess.run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", *objs, *LINK, "-o", tmp],
                   check=True)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose=True))
