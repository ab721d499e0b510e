"""Kernels whose lanes hand values to each other through LDS without a barrier of the workgroup: the order is said to the compiler, on what it makes of them."""
import os
import re
import subprocess

from paper_2509_23410_amd import build


def test_lanes_of_a_wavefront_meet_around_what_they_hand_on(tmp_path):
    """weigh_wide_kernel: 32 lanes write the rows' lse and limits, all 64 read them, step after step.  A lane is a thread to the compiler, which may move a lane's loads over
    other lanes' stores, and the other way round, where no fence is in between."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    out = str(tmp_path / "w.ll")
    subprocess.run([hipcc, *[f for f in build.HIPCC_FLAGS if f not in ("-shared", "-fPIC")], "-S", "-emit-llvm", "--cuda-device-only", "-I", os.path.join(build.ROOT, "include"),
                    "-I", build.CSRC, "-o", out, os.path.join(build.CSRC, "attention_weights.hip")], check=True, capture_output=True)
    bodies = re.findall(r"^define [^\n]*weigh_wide_kernel[^\n]*\{\n(.*?)^\}", open(out).read(), re.S | re.M)
    assert len(bodies) == 9
    for body in bodies:
        events = ""
        for line in body[:body.index('fence syncscope("workgroup")')].splitlines():
            if re.match(r"\s*fence ", line):
                events += "F"
            elif "ptr addrspace(3)" in line and re.search(r"(= load|^\s*store) ", line):
                events += "L" if "= load" in line else "S"
        assert re.fullmatch("F+S+F+L+S", events), events          # the last: a wavefront's sums, which the workgroup's barrier is behind
