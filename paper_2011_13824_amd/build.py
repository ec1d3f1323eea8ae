"""Build the gfx950 HIP library ``liblirpa.so`` in-tree with hipcc."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
LIB = os.path.join(PKG, "liblirpa.so")

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # packed fp32 VALU ops stay off: only scalar fp32 and MFMA arithmetic is emitted
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I", os.path.join(ROOT, "include"),
]

# translation units, and the flags that only they take
UNITS = {
    # MFMA results in ordinary VGPRs (no accumulator-register copies before the VALU reads them)
    "lirpa.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=true"],
    "blocks.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=true"],
}


def _run(cmds, verbose):
    """Runs the commands side by side; raises with their output if one fails."""
    procs = []
    for cmd in cmds:
        if verbose:
            print(" ".join(cmd), flush=True)
        procs.append(subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT,
                                      text=True))
    outs = [p.communicate()[0] for p in procs]
    for p, cmd, out in zip(procs, cmds, outs):
        if p.returncode != 0:
            sys.stderr.write(out)
            raise RuntimeError("hipcc failed for " + cmd[-1])


def build(verbose: bool = False) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    tmp = LIB + ".tmp%d" % os.getpid()
    with tempfile.TemporaryDirectory() as work:
        objs = {u: os.path.join(work, u + ".o") for u in UNITS}
        _run([[hipcc] + HIPCC_FLAGS + extra + ["-c", os.path.join(PKG, "csrc", u), "-o", objs[u]]
              for u, extra in UNITS.items()], verbose)
        _run([[hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", *objs.values(), "-o", tmp]],
             verbose)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
