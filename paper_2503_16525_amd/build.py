"""Builds libkvshare_hip.so (gfx950) in-tree with hipcc.  `python -m paper_2503_16525_amd.build`."""
from __future__ import annotations

import concurrent.futures
import glob
import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
OBJ_DIR = os.path.join(PKG, "_build")
LIB_PATH = os.path.join(PKG, "libkvshare_hip.so")
# the same library with the large-launch attention kernel pinned at compile time, and with a switch that sends paged attention
# to its kernel of many rows: only the test suite loads it, to run those kernels at sizes the oracle can follow
# (the shipped library has no run-time switch)
LIB_BIGATTN_PATH = os.path.join(PKG, "libkvshare_hip_bigattn.so")

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-fvisibility=hidden",
    "-Wall", "-Wextra", "-Wno-unused-parameter",
    # keep the compiler from forming packed-fp32 VALU ops
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I", INCLUDE, "-I", CSRC,
]


# per-file additions: the 256-row attention kernel wants its score tiles in vector registers (the
# softmax reads them there); by default the compiler puts every MFMA result into accumulation
# registers and copies the scores out one by one
EXTRA_FLAGS = {
    "attention_mfma2.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"],
    "attention_paged_large.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"],
    "impact.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"],
}


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.hip")))


def _compile(src: str, force: bool, defines=(), tag: str = "") -> str:
    obj = os.path.join(OBJ_DIR, os.path.basename(src) + tag + ".o")
    deps = [src] + glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(INCLUDE, "*.h"))
    if not force and os.path.exists(obj) and all(os.path.getmtime(obj) >= os.path.getmtime(d) for d in deps):
        return obj
    cmd = [HIPCC] + FLAGS + EXTRA_FLAGS.get(os.path.basename(src), []) + list(defines) + ["-c", src, "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    msgs = "\n".join(l for l in (r.stdout + r.stderr).splitlines()
                     if "is not a recognized feature for this target" not in l)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed on {src}:\n{msgs}")
    if msgs.strip():
        sys.stderr.write(msgs + "\n")
    return obj


def _link(objs, lib: str, force: bool) -> None:
    if force or not os.path.exists(lib) or any(os.path.getmtime(o) > os.path.getmtime(lib) for o in objs):
        tmp = lib + f".tmp{os.getpid()}"
        r = subprocess.run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp] + list(objs),
                           capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError("link failed:\n" + r.stdout + r.stderr)
        os.replace(tmp, lib)


def build(force: bool = False, jobs: int = 8) -> str:
    os.makedirs(OBJ_DIR, exist_ok=True)
    srcs = sources()
    # the files that hold the choices between the attention kernels
    pinned = {"attention_mfma.hip": "-DKVS_ATTN_FORCE=2", "attention_paged.hip": "-DKVS_PAGED_TEST", "attention_paged_large.hip": "-DKVS_PAGED_TEST"}
    with concurrent.futures.ThreadPoolExecutor(max_workers=jobs) as ex:
        big = {name: ex.submit(_compile, os.path.join(CSRC, name), force, (define,), ".bigattn") for name, define in pinned.items()}
        objs = list(ex.map(lambda s: _compile(s, force), srcs))
        big_objs = {os.path.join(OBJ_DIR, name + ".o"): obj.result() for name, obj in big.items()}
    _link(objs, LIB_PATH, force)
    _link([big_objs.get(o, o) for o in objs], LIB_BIGATTN_PATH, force)
    return LIB_PATH


if __name__ == "__main__":
    print(build(force="--force" in sys.argv))
