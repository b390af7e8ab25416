"""Compiles the HIP sources of this package for gfx950 into libcondensa.so (in-tree)."""
from __future__ import annotations

import os
import subprocess
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
SOURCES = [os.path.join(HERE, "csrc", name) for name in ("api.hip", "adamw.hip", "adapter.hip")]
LIB = os.path.join(HERE, "libcondensa.so")

FLAGS = [
    "-O3", "--offload-arch=gfx950", "-std=c++17", "-fPIC",
    "-ffp-contract=off",                                   # one rounding per operation, as specified
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
]


def build(verbose: bool = False) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    flags = list(FLAGS)
    if os.environ.get("CONDENSA_PLAIN_STREAM_STORES") == "1":
        # the compiler's own non-temporal stores instead of the buffer stores with system-scope bits: a build to
        # cross-check a parity failure against (csrc/common.h)
        flags.append("-DCONDENSA_PLAIN_STREAM_STORES")
    if os.environ.get("CONDENSA_INTEGER_F16") == "1":
        # binary16 rounding and widening in integer arithmetic throughout, instead of the conversion instructions
        flags.append("-DCONDENSA_INTEGER_F16")
    # the sources compile side by side, each into a code object of its own
    with tempfile.TemporaryDirectory() as tmp:
        objects = [os.path.join(tmp, os.path.basename(src) + ".o") for src in SOURCES]
        commands = [[hipcc] + flags + ["-c", "-o", obj, src] for obj, src in zip(objects, SOURCES)]
        running = [subprocess.Popen(cmd, stdout=subprocess.DEVNULL, stderr=subprocess.PIPE, text=True) for cmd in commands]
        results = [(p.communicate()[1], p.returncode) for p in running]
        if all(rc == 0 for _, rc in results):
            link = subprocess.run([hipcc, "--offload-arch=gfx950", "-shared", "-o", LIB] + objects, capture_output=True, text=True)
            results.append((link.stderr, link.returncode))
    noise = "packed-fp32-ops"
    err = "\n".join(l for text, _ in results for l in text.splitlines() if noise not in l)
    if verbose and err.strip():
        print(err)
    if any(rc != 0 for _, rc in results):
        raise RuntimeError("hipcc failed:\n" + err)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
