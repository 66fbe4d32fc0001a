"""Build the HIP library (libsaber.so) for gfx950 with hipcc, in-tree."""
from __future__ import annotations

import glob
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libsaber.so")
OPS_CSRC = os.path.join(HERE, "ops", "csrc")
SOURCES = [os.path.join(CSRC, "saber.hip"), os.path.join(OPS_CSRC, "saber_ops.hip")]
# every header the sources include: an edit to any of them marks the library stale
DEPS = SOURCES + sorted(glob.glob(os.path.join(CSRC, "*.hpp"))) + sorted(glob.glob(os.path.join(OPS_CSRC, "*.hpp"))) + sorted(glob.glob(os.path.join(os.path.dirname(HERE), "include", "*.h")))

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    "-ffp-contract=off",                               # products and sums round separately, as documented
    "-fhip-fp32-correctly-rounded-divide-sqrt",        # Eq. 2's division must be IEEE-rounded
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-command-line-argument",
]


def stale() -> bool:
    return not os.path.exists(LIB) or any(os.path.getmtime(LIB) < os.path.getmtime(d) for d in DEPS)


def build(force: bool = True) -> str:
    """Compile libsaber.so.  ``force=False`` rebuilds only when a source is newer than the library."""
    if not force and not stale():
        return LIB
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    tmp = LIB + ".tmp%d" % os.getpid()
    objects = ["%s.%d.o" % (tmp, i) for i in range(len(SOURCES))]
    flags = [f for f in HIPCC_FLAGS if f != "-shared"]
    try:
        _run([[hipcc] + flags + ["-c", "-o", o, src] for o, src in zip(objects, SOURCES)])
        _run([[hipcc] + HIPCC_FLAGS + ["-o", tmp] + objects])
        os.replace(tmp, LIB)
    finally:
        for path in objects + [tmp]:
            if os.path.exists(path):
                os.remove(path)
    return LIB


def _run(commands):
    """Runs the commands side by side; raises with the output of the first that fails."""
    running = [subprocess.Popen(c, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True) for c in commands]
    done = [(p.communicate()[0], p.returncode) for p in running]
    for out, code in done:
        if code != 0:
            raise RuntimeError("hipcc failed:\n" + "\n".join(ln for ln in out.splitlines() if "is not a recognized feature" not in ln))


if __name__ == "__main__":
    print(build())
