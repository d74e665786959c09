"""Build libnetkv.so for gfx950 with hipcc (in-tree)."""
import os
import subprocess
import sys
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
SRC = os.path.join(HERE, "csrc", "netkv.hip")
# the selection path and the handle; the flow-level transfer simulation; the
# decode instance's block cache, rotary positions and the eviction
SOURCES = [SRC] + [os.path.join(HERE, "csrc", f) for f in ("flowsim.hip", "blockcache.hip", "diffattend.hip", "append.hip",
                                                           "evict.hip")]
LIB = os.path.join(HERE, "libnetkv.so")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-result",
]


def build(verbose: bool = False) -> str:
    """The sources are compiled side by side and linked."""
    with tempfile.TemporaryDirectory() as tmp:
        objs = [os.path.join(tmp, os.path.basename(s) + ".o") for s in SOURCES]
        cmds = [[HIPCC, *FLAGS, "-c", "-I", os.path.join(ROOT, "include"), "-o", o, s] for s, o in zip(SOURCES, objs)]
        if verbose:
            for cmd in cmds:
                print(" ".join(cmd), flush=True)
        running = [subprocess.Popen(cmd) for cmd in cmds]
        failed = [cmd for p, cmd in zip(running, cmds) if p.wait()]
        if failed:
            raise subprocess.CalledProcessError(1, failed[0])
        out = LIB + ".tmp%d" % os.getpid()
        subprocess.check_call([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", out, *objs])
        os.replace(out, LIB)
    return LIB


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
