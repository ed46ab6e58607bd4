"""Builds liblc.so (the HIP library behind include/lc.h) in-tree with hipcc for gfx950."""
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "liblc.so")
SOURCES = ["lc_encode.hip", "lc_decode.hip", "lc_decode_one.hip", "lc_api.hip", "lc_w4.hip", "lc_i8.hip", "lc_kv.hip", "lc_prompt.hip", "lc_pages.hip",
           "lc_draft.hip"]
FLAGS = ["-O3", "--offload-arch=gfx950", "-std=c++17", "-shared", "-fPIC", "-ffp-contract=off",
         # packed fp32 instructions stay off: some of their forms have given wrong results on this hardware
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]
# the attention's sums live in vector registers from end to end; left to itself the compiler moves them to the accumulation
# registers and back for every tile
MORE_FLAGS = {"lc_kv.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1"], "lc_prompt.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1"]}


def _run(cmd, verbose):
    res = subprocess.run(cmd, capture_output=True, text=True)
    if verbose or res.returncode != 0:
        print(res.stdout + res.stderr)
    if res.returncode != 0:
        raise RuntimeError("hipcc failed building liblc.so")


def build_library(verbose=False):
    """One hipcc per source file, side by side, then the link."""
    from concurrent.futures import ThreadPoolExecutor
    objdir = os.path.join(HERE, "_build")
    os.makedirs(objdir, exist_ok=True)
    compile_flags = [f for f in FLAGS if f != "-shared"]
    objs = [os.path.join(objdir, s.replace(".hip", ".o")) for s in SOURCES]
    cmds = [["hipcc"] + compile_flags + MORE_FLAGS.get(s, []) + ["-c", "-o", o, os.path.join(CSRC, s)] for s, o in zip(SOURCES, objs)]
    with ThreadPoolExecutor(len(cmds)) as pool:
        list(pool.map(lambda c: _run(c, verbose), cmds))
    _run(["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB] + objs, verbose)
    return LIB


if __name__ == "__main__":
    print(build_library(verbose=True))
