"""Build libmoe355.so (HIP kernels + C ABI) for gfx950, in-tree, with hipcc."""
from __future__ import annotations

import os
import re
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
OBJDIR = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libmoe355.so")

SOURCES = ["moe_api.hip", "route.hip", "permute.hip", "gemm_bf16.hip", "gemm_stream.hip", "gemm_ring.hip", "gemm_f32.hip", "static_baseline.hip",
           "expert_cache.hip", "placement.hip", "quant.hip", "gate_topk.hip", "attn_api.hip", "kv_append.hip", "attn_decode.hip", "attn_prefill.hip", "sample.hip",
           "b128_api.hip", "select_experts.hip", "quant_b128.hip", "gemm_b128_stream.hip", "gemm_b128_tile.hip", "gemm_b128_small.hip"]

# packed fp32 instructions are switched off for all device code
HIPCC_FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall", "-Wno-unused-function",
               "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
               "-I", INCLUDE, "-I", CSRC]


def _hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if cand and (os.path.sep not in cand or os.path.exists(cand)):
            return cand
    raise RuntimeError("hipcc not found")


# The MFMA GEMM kernels sit at the register limit (256 accumulators + staging registers): a harmless
# looking edit can tip one of them into scratch spills and cost 10-20 % with no other symptom, so the
# compiler's per-kernel resource report is read and a spill there fails the build.  In gemm_b128_tile.hip it would
# cost more than time: a spilled accumulator is read without the wait that its inline MFMA needs.
NO_SPILL_SOURCES = {"gemm_bf16.hip", "gemm_stream.hip", "gemm_ring.hip", "gemm_b128_tile.hip"}


def spilled_kernels(report: str):
    """(kernel name, spilled VGPRs) for every kernel of a -Rpass-analysis=kernel-resource-usage
    report that spills."""
    out = []
    for block in report.split("Function Name: ")[1:]:
        name = block.split("\n", 1)[0].strip()
        m = re.search(r"VGPRs Spill: (\d+)", block)
        if m and int(m.group(1)) > 0:
            out.append((name, int(m.group(1))))
    return out


def _compile(src: str, verbose: bool) -> str:
    obj = os.path.join(OBJDIR, src.replace(".hip", ".o"))
    cmd = [_hipcc(), *HIPCC_FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
    check = src in NO_SPILL_SOURCES
    if check:
        cmd.insert(-4, "-Rpass-analysis=kernel-resource-usage")
    r = subprocess.run(cmd, capture_output=True, text=True)
    if check:
        bad = spilled_kernels(r.stderr)
        if r.returncode == 0 and bad:
            raise RuntimeError("register spills in %s: %s" % (src, ", ".join("%s (%d VGPRs)" % b for b in bad)))
        r.stderr = "\n".join(l for l in r.stderr.splitlines()
                              if "remark:" not in l and not re.match(r"^\s*\d*\s*\|", l))
    err = "\n".join(l for l in r.stderr.splitlines() if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError("hipcc failed for %s:\n%s" % (src, err))
    if verbose and err.strip():
        print(err, file=sys.stderr)
    return obj


def build(verbose: bool = False) -> str:
    """Compile every HIP source and link the shared library.  Always recompiles."""
    os.makedirs(OBJDIR, exist_ok=True)
    with ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as ex:
        objs = list(ex.map(lambda s: _compile(s, verbose), SOURCES))
    cmd = [_hipcc(), "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objs]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n" + r.stderr)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
