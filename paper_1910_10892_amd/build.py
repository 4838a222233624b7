"""Build step of libmrfmp: nineteen hipcc compilations side by side and a link, in-tree output next to
the sources."""
from __future__ import annotations

import os
import re
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.abspath(__file__)), "csrc")
LIB_PATH = os.path.join(CSRC, "libmrfmp.so")
SOURCES = ["mrfmp.hip"]
LEARN_SOURCES = ["mrfmp_norm.hip", "mrfmp_bucket.hip", "mrfmp_policy.hip",
                 "mrfmp_attention.hip", "mrfmp_attention_bwd.hip", "mrfmp_rotate.hip", "mrfmp_scan.hip"]
HEADERS = ["mrfmp_attention.h", "mrfmp_learn.h", "mrfmp_rows.h", "mrfmp_device.h", "mrfmp_fwd.h", "mrfmp_bwd.h", "mrfmp_bwd_sum.h", "mrfmp_head.h", "../../include/mrfmp.h"]

# -ffp-contract=off: the only fused multiply-add is the explicit one of the message update,
#   so that floating point decisions (argmins) match a plain C evaluation order.
# packed-fp32 instructions are switched off: some of their forms have given wrong results now and then.
HIPCC_FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared", "-ffp-contract=off", "-munsafe-fp-atomics",
               "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wall"]


# The attention's sums stay where the other instructions reach them: left to itself the compiler keeps them in the accumulation registers and moves hundreds of
# values a tile to and fro.  (Kernels that have no room for that are units of their own, without this flag.)  None of these kernels may need scratch memory beside
# accumulation registers: this compiler has made wrong code of such ones, so the build fails if there is one.
UNIT_FLAGS = {"mrfmp_attention.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"], "mrfmp_attention_bwd.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"]}


REPORT_FLAG = "-Rpass-analysis=kernel-resource-usage"


def kernels_with_scratch_and_accumulation(report: str) -> list[str]:
    """Names of the kernels that the compiler's resource report has with both."""
    found, name, used = [], None, {}
    for line in report.splitlines():
        m = re.search(r"remark: .*?(Function Name|AGPRs|ScratchSize \[bytes/lane\]): (\S+)", line)
        if not m:
            continue
        if m.group(1) == "Function Name":
            name, used = m.group(2), {}
            continue
        used[m.group(1)[:5]] = int(m.group(2))
        if len(used) == 2 and all(used.values()):
            found.append(name)
    return found


def is_stale() -> bool:
    if not os.path.exists(LIB_PATH):
        return True
    t = os.path.getmtime(LIB_PATH)
    return any(os.path.getmtime(os.path.join(CSRC, f)) > t for f in SOURCES + LEARN_SOURCES + HEADERS)


def build(verbose: bool = False) -> str:
    """Compile libmrfmp.so for gfx950 (cross-compiles without a GPU): the sweeps' source as nine
    translation units (the schedules, the entry points, a family of sweeps each) and a source or two per
    learning and sequence operator side by side, then link."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    objdir = os.path.join(CSRC, "_build")
    os.makedirs(objdir, exist_ok=True)
    flags = [f for f in HIPCC_FLAGS if f != "-shared"]
    jobs = []
    units = [("mrfmp_part%d.o" % part, ["-DMRF_PART=%d" % part], SOURCES) for part in range(1, 10)]
    units += [(f.replace(".hip", ".o"), UNIT_FLAGS.get(f, []), [f]) for f in LEARN_SOURCES]
    units += [(f.replace(".hip", "_f32.o"), ["-DMRF_ATTENTION_F32"], [f]) for f in UNIT_FLAGS]
    units.append(("mrfmp_attention_bwd_128.o", ["-DMRF_ATTENTION_128"], ["mrfmp_attention_bwd.hip"]))
    for name, defines, sources in units:
        obj = os.path.join(objdir, name)
        cmd = [hipcc, *flags, *defines, "-c", "-o", obj, *sources]
        if sources[0] in UNIT_FLAGS:
            cmd.insert(1, REPORT_FLAG)
        jobs.append((obj, subprocess.Popen(cmd, cwd=CSRC, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    failed, both, reported = False, [], 0
    for obj, proc in jobs:
        out, _ = proc.communicate()
        if REPORT_FLAG in proc.args:
            both += kernels_with_scratch_and_accumulation(out)
            reported += out.count("Function Name")
        if verbose or proc.returncode != 0:
            print(out)
        failed = failed or proc.returncode != 0
    if failed:
        raise RuntimeError("hipcc failed compiling libmrfmp")
    if both or not reported:
        raise RuntimeError("kernels with scratch memory beside accumulation registers: %s" % (both or "no report of the compiler's to tell by"))
    cmd = [hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB_PATH, *[obj for obj, _ in jobs]]
    res = subprocess.run(cmd, cwd=CSRC, capture_output=True, text=True)
    if verbose or res.returncode != 0:
        print(res.stdout)
        print(res.stderr)
    if res.returncode != 0:
        raise RuntimeError("hipcc failed linking libmrfmp.so")
    return LIB_PATH


if __name__ == "__main__":
    print(build(verbose=True))
