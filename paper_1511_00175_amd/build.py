"""Build libfc.so (aggregation and update) and libfc_lm.so (the operators of
fc_lm.h), HIP kernels + C ABI each, for gfx950, in place, with hipcc.

Flags that matter for results:
  -ffp-contract=off   no fused multiply-add: every operation is rounded once
  no -ffast-math, no -fgpu-flush-denormals-to-zero: subnormals are kept
  -Xclang -target-feature -Xclang -packed-fp32-ops: no packed fp32 ALU ops
"""
import os
import re
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(PKG, "libfc.so")
SOURCES = ["fc_reduce_f32.hip", "fc_reduce_f16.hip", "fc_update.hip", "fc_api.cpp"]
SOURCES_LM = ["fc_embed.hip", "fc_xent.hip", "fc_muon.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
ARCH = "gfx950"
FLAGS = ["-O3", "-std=c++17", "-fPIC", f"--offload-arch={ARCH}", "-ffp-contract=off",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wall", "-Wno-unused-function", f"-I{INCLUDE}", f"-I{CSRC}"]


RESOURCES = os.path.join(PKG, "_build", "kernel_resources.txt")
_REMARK = re.compile(r"remark:\s+(Function Name|VGPRs|AGPRs|ScratchSize \[bytes/lane\]|Occupancy \[waves/SIMD\]|"
                     r"LDS Size \[bytes/block\]):\s+(\S+)")


def _resources(stderr):
    """Per-kernel resource usage from the compiler's kernel-resource-usage
    remarks: {kernel: {field: value}}."""
    out, cur = {}, None
    for ln in stderr.splitlines():
        m = _REMARK.search(ln)
        if not m:
            continue
        key, val = m.group(1).split(" ")[0], m.group(2)
        if key == "Function":
            cur = out.setdefault(val, {})
        elif cur is not None:
            cur[key] = int(val)
    return out


def _compile(src, obj, extra):
    lang = ["-x", "hip"] if src.endswith(".hip") else []
    remarks = ["-Rpass-analysis=kernel-resource-usage"] if src.endswith(".hip") else []
    cmd = [HIPCC, *FLAGS, *remarks, *extra, *lang, "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    # the host pass does not know the packed-fp32 feature and says so; that is harmless
    noise = [ln for ln in r.stderr.splitlines() if ln.strip() and "packed-fp32-ops" not in ln
             and "ignoring feature" not in ln and "remark:" not in ln and "kernel-resource-usage" not in ln]
    if r.returncode:
        raise RuntimeError(f"hipcc failed for {src}:\n" + "\n".join(noise))
    return _resources(r.stderr)


def build(out=LIB, extra=()):
    """Compile every source and link the shared libraries, libfc.so as `out` and
    libfc_lm.so beside it; returns the first's path."""
    objdir = os.path.join(PKG, "_build")
    os.makedirs(objdir, exist_ok=True)
    sources = SOURCES + SOURCES_LM
    objs = [os.path.join(objdir, s + ".o") for s in sources]
    with ThreadPoolExecutor(len(sources)) as ex:
        usage = {}
        for u in ex.map(lambda a: _compile(*a, list(extra)), zip(sources, objs)):
            usage.update(u)
    # every kernel keeps its sums and tiles in registers and LDS: no scratch memory
    with open(RESOURCES, "w") as f:
        for name in sorted(usage):
            f.write(name + " " + " ".join(f"{k}={v}" for k, v in sorted(usage[name].items())) + "\n")
    spill = [n for n, u in usage.items() if u.get("ScratchSize", 0)]
    if spill:
        raise RuntimeError("kernels using scratch memory: " + ", ".join(spill))
    for lib, part in ((out, objs[:len(SOURCES)]), (os.path.join(os.path.dirname(out), "libfc_lm.so"), objs[len(SOURCES):])):
        tmp = lib + ".tmp"
        subprocess.run([HIPCC, "-shared", "-fPIC", f"--offload-arch={ARCH}", *part, "-o", tmp], check=True)
        os.replace(tmp, lib)
    return out


if __name__ == "__main__":
    print(build(extra=sys.argv[1:]))
