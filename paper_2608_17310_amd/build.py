"""Build libesopt.so for gfx950 with hipcc (in-tree, next to this file)."""
import os
import shutil
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
SOURCES = [os.path.join(HERE, "csrc", f) for f in ("esopt.hip", "eskv.hip", "eshead.hip")]
OUT = os.path.join(HERE, "libesopt.so")

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # rounding is spelled out in the source: no implicit contraction
    "-ffp-contract=off",
    # no packed-fp32 VALU forms (v_pk_fma_f32 and friends)
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Werror=return-type",
]


def hipcc():
    for cand in (shutil.which("hipcc"), "/opt/rocm/bin/hipcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found")


def _run(cmd):
    res = subprocess.run(cmd, capture_output=True, text=True)
    noise = "packed-fp32-ops"        # the host pass does not know the feature
    msgs = [l for l in (res.stdout + res.stderr).splitlines() if noise not in l]
    if res.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + "\n".join(msgs))
    return msgs


def build(verbose=False):
    """Compile every source each time it is called (the sources at the same
    time); write the library atomically."""
    tmp = OUT + ".tmp"
    with tempfile.TemporaryDirectory() as work:
        objects = [os.path.join(work, os.path.basename(s) + ".o") for s in SOURCES]
        with ThreadPoolExecutor(len(SOURCES)) as pool:
            msgs = [m for out in pool.map(
                lambda so: _run([hipcc(), *HIPCC_FLAGS, "-c", so[0], "-o", so[1]]),
                zip(SOURCES, objects)) for m in out]
        msgs += _run([hipcc(), "--offload-arch=gfx950", "-shared", "-o", tmp, *objects])
    if verbose and msgs:
        print("\n".join(msgs), file=sys.stderr)
    os.replace(tmp, OUT)
    return OUT


if __name__ == "__main__":
    print(build(verbose=True))
