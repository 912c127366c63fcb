"""Build the native library libcs.so in-tree for gfx950.

    python -m paper_2112_13896_amd.build

Compiles the HIP kernels and C ABI (csrc/cs_api.hip, the sparse layers;
csrc/q8_api.hip, the 8-bit attention-layer operators; csrc/mx4_api.hip, the
4-bit cache and attention; csrc/step_api.hip, rotary positions and step plans)
and the host pack routine (csrc/cs_pack.cpp) with hipcc and links them, once as the product
library and once with the product counter compiled in (libcs_count.so, used by
tests).  Packed-fp32 instruction generation is switched off for all device
code.
"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(HERE, "libcs.so")
COUNT_LIB = os.path.join(HERE, "libcs_count.so")
STAMP_LIB = os.path.join(HERE, "libcs_stamps.so")
ARCH = "gfx950"

DEVICE_FLAGS = ["-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found")


def sources() -> list:
    """Translation units; only the first knows the instrumented builds' defines."""
    return [os.path.join(CSRC, f) for f in ("cs_api.hip", "q8_api.hip", "mx4_api.hip",
                                          "step_api.hip", "cs_pack.cpp")]


def source_digest() -> str:
    """SHA-256 over every source and header the layer kernels (csrc/cs_api.hip, csrc/cs_pack.cpp)
    are built from: the native sources but those of the attention-layer operators."""
    import hashlib
    h = hashlib.sha256()
    files = sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC)
                   if f.endswith((".hip", ".cpp", ".h"))
                   and not f.startswith(("q8_", "mx4_", "step_")))
    files.append(os.path.join(INCLUDE, "cs.h"))
    for f in files:
        h.update(os.path.basename(f).encode())
        h.update(open(f, "rb").read())
    return h.hexdigest()


def _compile(src: str, out: str, extra: list) -> list:
    return [hipcc(), f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC", "-c", "-Wall",
            "-Wno-unused-command-line-argument", *DEVICE_FLAGS, "-I", INCLUDE, "-I", CSRC, *extra,
            "-o", out, src]


def _link(out: str, objects: list) -> list:
    return [hipcc(), f"--offload-arch={ARCH}", "-fPIC", "-shared", "-o", out, *objects]


def _run(cmds: list, verbose: bool) -> None:
    """The commands side by side; raises when one fails, after all have ended."""
    procs = []
    for cmd in cmds:
        if verbose:
            print(" ".join(cmd), flush=True)
        procs.append((cmd, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT,
                                            text=True)))
    failed = None
    noise = "is not a recognized feature for this target"
    for cmd, p in procs:
        text = p.communicate()[0]
        if p.returncode != 0:
            sys.stderr.write(text)
            failed = failed or (f"hipcc failed with exit code {p.returncode} "
                                f"({os.path.basename(cmd[cmd.index('-o') + 1])})")
            continue
        msgs = [ln for ln in text.splitlines() if noise not in ln and ln.strip()]
        if msgs and verbose:
            print("\n".join(msgs))
    if failed:
        raise RuntimeError(failed)


def build(verbose: bool = False, extra: list | None = None, counting: bool = True) -> str:
    """Compile libcs.so (always recompiles) and, with `counting`, the two
    instrumented builds: libcs_count.so (every multiply-route-sum kernel counts
    the products it forms; tests only) and libcs_stamps.so (phase stamps; the
    benchmark's phase report), the compilations side by side.  The other
    sources know neither define: the three libraries share their objects.
    Returns the path of libcs.so."""
    extra = list(extra or [])
    libs = [(LIB, [])]
    if counting:
        libs += [(COUNT_LIB, ["-DCS_COUNT_PRODUCTS"]), (STAMP_LIB, ["-DCS_PHASE_STAMPS"])]
    api, *shared = sources()
    with tempfile.TemporaryDirectory(prefix="cs_build_") as tmp:
        cmds, links = [], []
        common = [os.path.join(tmp, os.path.basename(s) + ".o") for s in shared]
        for i, (lib, define) in enumerate(libs):
            obj = os.path.join(tmp, f"{i}.o")
            cmds.append(_compile(api, obj, extra + define))
            links.append(_link(lib + ".tmp", [obj, *common]))
        cmds += [_compile(s, o, extra) for s, o in zip(shared, common)]
        _run(cmds, verbose)
        _run(links, verbose)
    for lib, _ in libs:
        os.replace(lib + ".tmp", lib)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
