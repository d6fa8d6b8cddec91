"""Build the gfx950 HIP library in place (hipcc, no CUDA, no JIT).

Three builds of the same sources:

* ``libtopk.so``       -- the library;
* ``libtopk_check.so`` -- with ``TOPK_CHECK_INDICES``: forward calls wait for their
  stream and report asynchronous kernel errors, and the finalize counts selected
  indices outside the value matrix (``topk_debug_bad_indices``);
* ``libtopk_san.so``   -- the host code built with AddressSanitizer and
  UndefinedBehaviorSanitizer (device code unchanged), for the CPU tests of the
  C ABI's argument checks and planning; it needs the sanitizer runtime preloaded.

``libtopk.so`` and ``libtopk_check.so`` are refused where the compiler spills vector registers of one of the
kernels of ``NO_SPILLS``.

Run as ``python -m paper_2106_06899_amd.build`` or call ``build()``.
"""
from __future__ import annotations

import glob
import os
import re
import subprocess
import sys
import tempfile

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
SOURCES = ["csrc/topk_kernels.hip", "csrc/topk_rows.hip", "csrc/topk_cells.hip", "csrc/topk_few.hip", "csrc/topk_keep.hip",
           "csrc/topk_dense.hip", "csrc/topk_rope.hip", "csrc/topk_prefix.hip",
           "csrc/topk_packed.hip", "csrc/topk_packed_bwd.hip", "csrc/topk_pages.hip", "csrc/topk_tree.hip", "csrc/topk_api.hip"]
LIB = os.path.join(PKG, "libtopk.so")
LIB_CHECK = os.path.join(PKG, "libtopk_check.so")
LIB_SAN = os.path.join(PKG, "libtopk_san.so")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-mllvm", "-amdgpu-mfma-vgpr-form=1",      # MFMA accumulators in VGPRs: no accvgpr copies
    "-Wall", "-Wno-unused-function",
]
# Kernels that hold operands of matrix instructions in all the registers there are while rows come to LDS directly. A
# build of the gradients' kernel with spilled vector registers has given NaN, with sources that give right results
# without; what the compiler made of the spills was not found out, so a build that has any does not count as one.
NO_SPILLS = ("k_packed", "k_packed_dq", "k_packed_dkv", "k_tree")
VARIANTS = {
    "main": (LIB, []),
    "check": (LIB_CHECK, ["-DTOPK_CHECK_INDICES"]),
    # host code only: each -fsanitize= applies to the host compilation
    "san": (LIB_SAN, ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
                      "-Xarch_host", "-fno-omit-frame-pointer", "-shared-libsan", "-O1"]),
}


def sanitizer_runtime() -> str | None:
    """The ASan runtime a process must preload to load libtopk_san.so."""
    pats = ["/opt/rocm/llvm/lib/clang/*/lib/linux/libclang_rt.asan-x86_64.so",
            "/opt/rocm/lib/llvm/lib/clang/*/lib/linux/libclang_rt.asan-x86_64.so"]
    for p in pats:
        hits = sorted(glob.glob(p))
        if hits:
            return hits[-1]
    return None


def _command(out: str, extra: list[str]) -> list[str]:
    return [HIPCC, *FLAGS, *extra, "-I", os.path.join(ROOT, "include"), "-I", os.path.join(PKG, "csrc"),
            *[os.path.join(PKG, s) for s in SOURCES], "-o", out + ".tmp"]


def spills(log: str) -> list[str]:
    """The kernels of NO_SPILLS of which the compiler's remarks (-Rpass-analysis=kernel-resource-usage) name spilled
    vector registers, and those that the remarks lack altogether."""
    left, found, name = set(NO_SPILLS), [], None
    for line in log.splitlines():
        if m := re.search(r"remark: .*Function Name: (\S+)", line):
            mangled = m.group(1)
            name = next((k for k in NO_SPILLS if f"{len(k)}{k}I" in mangled), None)  # (I: its template arguments)
        elif name and (m := re.search(r"remark: .*VGPRs Spill: (\d+)", line)):
            left.discard(name)
            if int(m.group(1)):
                found.append(f"{mangled}: {m.group(1)} vector registers spilled")
    return found + [f"{k}: not in the compiler's remarks" for k in sorted(left)]


def build(verbose: bool = False, variants=("main", "check", "san")) -> str:
    """Compile every HIP source for gfx950 into each requested library (always
    recompiles; the builds run in parallel). Returns the path of libtopk.so."""
    procs = []
    for name in variants:
        out, extra = VARIANTS[name]
        cmd = _command(out, extra + ([] if name == "san" else ["-Rpass-analysis=kernel-resource-usage"]))
        if verbose:
            print(" ".join(cmd), flush=True)
        said = tempfile.TemporaryFile("w+")  # (the remarks are more than a pipe holds, and the builds are waited for in turn)
        procs.append((name, out, said, subprocess.Popen(cmd, stdout=said, stderr=subprocess.STDOUT)))
    failed = []
    for name, out, said, p in procs:
        p.wait()
        said.seek(0)
        log = said.read()
        spilled = [] if p.returncode or name == "san" else spills(log)
        if p.returncode != 0:
            sys.stderr.write(log)
            failed.append(os.path.basename(out))
        elif spilled:
            sys.stderr.write("\n".join(spilled) + "\n")
            os.remove(out + ".tmp")
            failed.append(os.path.basename(out))
        else:
            os.replace(out + ".tmp", out)
    if failed:
        raise RuntimeError("hipcc failed building " + ", ".join(failed))
    return LIB


if __name__ == "__main__":
    which = tuple(sys.argv[1:]) or ("main", "check", "san")
    print(build(verbose=True, variants=which))
