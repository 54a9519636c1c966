"""Compile the HIP library for gfx950 into paper_2508_06041_amd/libdpllm.so and the binding's native part into _calls.so (in-tree)."""
import os
import re
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libdpllm.so")
SOURCES = ["dpllm_api.hip", "token_api.hip", "attention_api.hip", "token_host.hip"]
CALLS = os.path.join(HERE, "_calls.so")
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall", "-Wno-unused-result",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         # the first kernel arguments arrive in scalar registers with the launch instead of being loaded from memory
         "-mllvm", "-amdgpu-kernarg-preload-count=14"]


def spilled(report: str) -> list:
    """The kernels that keep vector registers in scratch memory, from what the compiler says about the resources of each: their code is
    written for the registers there are, and one that does not fit makes every launch of it slower without any other sign."""
    kernels = []
    for part in report.split("Function Name: ")[1:]:
        used = {k: int(v) for k, v in re.findall(r"(ScratchSize|VGPRs Spill)[^:\n]*: (\d+)", part)}
        if any(used.values()):
            kernels.append(part.split()[0])
    return kernels


def build(verbose: bool = False, extra=()) -> str:
    """Every source becomes an object of its own, all at once, so that the code of one does not move when another changes."""
    objects = os.path.join(HERE, "_build")
    os.makedirs(objects, exist_ok=True)
    hipcc = "/opt/rocm/bin/hipcc"
    made = [os.path.join(objects, s.replace(".hip", ".o")) for s in SOURCES]
    cmds = [["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", "-Wextra", "-I" + sysconfig.get_paths()["include"], "-o", CALLS,
             os.path.join(CSRC, "py_calls.cpp")]]
    cmds += [[hipcc, *FLAGS, *extra, "-Rpass-analysis=kernel-resource-usage", "-fno-caret-diagnostics", "-c", os.path.join(CSRC, s), "-o", o]
             for s, o in zip(SOURCES, made)]
    link = [hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *made]
    if verbose:
        print("\n".join(" ".join(c) for c in [*cmds, link]))
    running = [subprocess.Popen(c, stderr=subprocess.PIPE, text=True) for c in cmds]
    reports = [p.communicate()[1] for p in running]
    for report in reports:
        sys.stderr.write("".join(line for line in report.splitlines(True) if "[-Rpass-analysis" not in line and not line.startswith("In file included")))
    for p, c in zip(running, cmds):
        if p.returncode:
            raise subprocess.CalledProcessError(p.returncode, c)
    bad = [k for report in reports for k in spilled(report)]
    if bad:
        raise RuntimeError("vector registers spilled: " + ", ".join(bad))
    subprocess.run(link, check=True)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
