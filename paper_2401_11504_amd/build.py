"""Build libtemplora.so (gfx950 only) in-tree with hipcc.

    python -m paper_2401_11504_amd.build

Objects go to paper_2401_11504_amd/_build/ (git-ignored); the shared library is
written next to this file so that it travels with the source tree.
"""
from __future__ import annotations

import os
import re
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OUT = os.path.join(HERE, "libtemplora.so")
SOURCES = ["templora.hip", "gemm_bf16.hip", "gemm_f32.hip", "attention.hip", "elementwise.hip", "decode.hip",
           "cache8.hip", "choose.hip", "sample.hip", "paged.hip", "attn_weights.hip"]
# packed-fp32 VALU forms are switched off for device code on purpose: the compiler otherwise emits v_pk_*_f32
# forms that have been seen to give wrong results on these machines
FLAGS = ["-O3", "-std=c++17", "-fPIC", "--offload-arch=gfx950", "-Xclang", "-target-feature", "-Xclang",
         "-packed-fp32-ops", "-Wall", "-Wno-unused-function", "-Wno-unknown-warning-option"]


def _hipcc() -> str:
    for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if c and (os.path.isabs(c) and os.path.exists(c) or not os.path.isabs(c)):
            return c
    raise RuntimeError("hipcc not found")


# What the compiler reports of every kernel.  None may reserve scratch memory: a choice between two addresses in it turns loads into
# flat ones that are waited for one by one (dropout_low_rank_add_kernel over 2048 x 4096, 192 contraction elements: 28 us, 25 without),
# and a spilled accumulator of the GEMM tiles would be stored ahead of the wait for its matrix instruction, which the compiler does not see.
USAGE = ["-Rpass-analysis=kernel-resource-usage"]
_REMARK = re.compile(r"^.*remark: .*\[-Rpass-analysis=kernel-resource-usage\]\n(?: *\d* \|.*\n)*", re.M)


def scratch_users(remarks: str) -> dict:
    """{kernel: bytes per lane} of the kernels that reserve scratch memory."""
    out, name = {}, None
    for m in re.finditer(r"remark: +(Function Name|ScratchSize \[bytes/lane\]): (\S+)", remarks):
        if m[1] == "Function Name":
            name = m[2]
        elif int(m[2]):
            out[name] = int(m[2])
    return out


def build(verbose: bool = False, jobs: int = 8) -> str:
    bdir = os.path.join(HERE, "_build")
    os.makedirs(bdir, exist_ok=True)
    hipcc = _hipcc()

    def compile_one(src):
        obj = os.path.join(bdir, src.replace(".hip", ".o"))
        cmd = [hipcc, *FLAGS, *USAGE, "-c", os.path.join(CSRC, src), "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError("hipcc failed for %s:\n%s\n%s" % (src, " ".join(cmd), _REMARK.sub("", r.stderr)[-8000:]))
        scratch = scratch_users(r.stderr)
        if scratch:
            raise RuntimeError("%s: kernels that reserve scratch memory (bytes per lane): %s" % (src, scratch))
        rest = _REMARK.sub("", r.stderr)
        if verbose and rest.strip():
            print(rest, file=sys.stderr)
        return obj

    with ThreadPoolExecutor(max_workers=max(1, min(jobs, len(SOURCES)))) as ex:
        objs = list(ex.map(compile_one, SOURCES))
    cmd = [hipcc, "-shared", "-fPIC", "--offload-arch=gfx950", *objs, "-o", OUT]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n%s" % r.stderr[-8000:])
    return OUT


if __name__ == "__main__":
    print(build(verbose=True))
