"""Builds libflce.so (the gfx950 HIP kernels and their C ABI) in-tree with hipcc."""
from __future__ import annotations

import glob
import os
import subprocess
import tempfile
from concurrent.futures import ThreadPoolExecutor

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG_DIR, "csrc")
LIB_PATH = os.path.join(PKG_DIR, "libflce.so")

LINK_FLAGS = ["--offload-arch=gfx950", "-fPIC", "-shared", "-fvisibility=hidden"]
HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-fvisibility=hidden",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wextra", "-Wno-unused-parameter",
]


def _hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if cand and (os.path.sep not in cand or os.path.exists(cand)):
            return cand
    raise RuntimeError("hipcc not found")


def sources() -> list[str]:
    return sorted(glob.glob(os.path.join(CSRC, "*.hip")))


def is_stale() -> bool:
    if not os.path.exists(LIB_PATH):
        return True
    t = os.path.getmtime(LIB_PATH)
    deps = glob.glob(os.path.join(CSRC, "*")) + glob.glob(os.path.join(PKG_DIR, "..", "include", "*.h"))
    return any(os.path.getmtime(d) > t for d in deps)


def build(verbose: bool = False) -> str:
    """Compile every HIP source for gfx950 into libflce.so (always recompiles; the sources side by side)."""
    def run(cmd):
        res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
        out = "\n".join(l for l in res.stdout.splitlines() if "packed-fp32-ops" not in l)
        if res.returncode != 0:
            raise RuntimeError("hipcc failed:\n" + out)
        return out

    with tempfile.TemporaryDirectory() as tmp:
        objects = {src: os.path.join(tmp, os.path.basename(src) + ".o") for src in sources()}
        with ThreadPoolExecutor(len(objects)) as pool:
            outs = list(pool.map(lambda so: run([_hipcc(), *HIPCC_FLAGS, "-c", so[0], "-o", so[1]]), objects.items()))
        outs.append(run([_hipcc(), *LINK_FLAGS, *objects.values(), "-o", LIB_PATH]))
    if verbose:
        for out in filter(str.strip, outs):
            print(out)
    # A shared library links even when a kernel's host-side launch stub was not
    # emitted; it would only fail when loaded.  Catch that here.
    nm = subprocess.run(["nm", "-D", "--undefined-only", LIB_PATH], stdout=subprocess.PIPE, text=True)
    missing = [l.split()[-1] for l in nm.stdout.splitlines() if "__device_stub__" in l]
    if missing:
        raise RuntimeError("libflce.so has undefined kernel launch stubs: " + ", ".join(missing))
    return LIB_PATH


if __name__ == "__main__":
    print(build(verbose=True))
