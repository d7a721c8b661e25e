"""Builds libmori.so in-tree with hipcc for gfx950."""
from __future__ import annotations

import concurrent.futures
import glob
import os
import subprocess
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libmori.so")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # idleness decides the ranking: IEEE binary32 with no contraction, correctly
    # rounded division and no flushing of denormals, exactly like the oracle
    "-ffp-contract=off", "-fno-fast-math", "-fhip-fp32-correctly-rounded-divide-sqrt",
    "-fno-gpu-flush-denormals-to-zero",
    # packed fp32 instructions stay off (see the design notes)
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # host loops begin on a fetch line wherever the code before them ends (replica
    # admission is otherwise up to 7% slower after a change to another file)
    "-Xarch_host", "-falign-loops=32",
    "-Wall", "-Wno-unused-result",
]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.hip")))


def _run(cmd) -> str:
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + res.stdout + res.stderr)
    return res.stderr


def build(verbose: bool = False) -> str:
    """Compile every HIP source into paper_2606_00866_amd/libmori.so (always rebuilds), a
    process a source: the attention kernels have many forms and take a minute in all."""
    tmp = LIB + ".tmp%d" % os.getpid()
    with tempfile.TemporaryDirectory() as to, concurrent.futures.ThreadPoolExecutor(os.cpu_count() or 4) as pool:
        objects = {s: os.path.join(to, os.path.basename(s) + ".o") for s in sources()}
        said = list(pool.map(lambda s: _run([HIPCC, *FLAGS, "-I", os.path.join(HERE, "..", "include"), "-c", s, "-o",
                                             objects[s]]), objects))
        said.append(_run([HIPCC, "--offload-arch=gfx950", "-shared", "-o", tmp, *objects.values()]))
    if verbose and any(s.strip() for s in said):
        print("".join(said))
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
