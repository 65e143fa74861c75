"""Build libtrimul.so (the C-ABI library, HIP for gfx950) in-tree with hipcc.

    python -m paper_2603_14806_amd.build
"""
import concurrent.futures
import os
import shutil
import subprocess
import sys
import tempfile

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libtrimul.so")
SOURCES = ["api.hip", "project.hip", "contract.hip", "epilogue.hip", "backward.hip", "opm.hip", "triattn.hip",
           "crossattn.hip", "crossattn_backward.hip", "dropout.hip"]
ARCH = "gfx950"


def hipcc():
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found (set HIPCC or install ROCm under /opt/rocm)")


FLAGS = [f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC",
         # no packed-fp32 instructions in device code
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wall", "-Wno-unused-function", "-Wno-unused-variable",
         "-I", os.path.join(ROOT, "include")]


def _run(cmd):
    """(exit code, messages) of one compiler call."""
    r = subprocess.run(cmd, capture_output=True, text=True)
    return r.returncode, [ln for ln in (r.stdout + r.stderr).splitlines() if "packed-fp32-ops" not in ln]


def build(verbose=False):
    """Compiles the sources side by side and links the library."""
    with tempfile.TemporaryDirectory() as tmp:
        objects = [os.path.join(tmp, s.replace(".hip", ".o")) for s in SOURCES]
        cmds = [[hipcc()] + FLAGS + ["-c", os.path.join(CSRC, s), "-o", o] for s, o in zip(SOURCES, objects)]
        link = [hipcc(), f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", LIB + ".tmp"] + objects
        if verbose:
            print("\n".join(" ".join(c) for c in cmds + [link]), flush=True)
        with concurrent.futures.ThreadPoolExecutor(min(8, os.cpu_count() or 1)) as pool:
            done = list(pool.map(_run, cmds))
        msgs = [ln for _, m in done for ln in m]
        if all(rc == 0 for rc, _ in done):
            done.append(_run(link))
            msgs += done[-1][1]
        if any(rc != 0 for rc, _ in done):
            raise RuntimeError("hipcc failed:\n" + "\n".join(msgs))
    if verbose and msgs:
        print("\n".join(msgs))
    os.replace(LIB + ".tmp", LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-q" not in sys.argv))
