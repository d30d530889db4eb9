"""Registers that the attention's kernels spill, from the compiler's report (no GPU)."""
import os
import re
import subprocess

from paper_2509_24859_amd import build

# kernel, type, channels, wavefronts: the most that is known and stands at the kernels; all others spill none
KNOWN = {("forward", "bf16", 128, 4): 11, ("forward", "f16", 128, 4): 11,
         ("grad_queries", "bf16", 128, 8): 3, ("grad_queries", "f16", 128, 8): 7, ("grad_queries", "bf16", 128, 4): 16, ("grad_queries", "f16", 128, 4): 23,
         ("grad_keys", "bf16", 128, 4): 9, ("grad_keys", "f16", 128, 4): 10}


def test_no_more_registers_are_spilled_than_is_said(tmp_path):
    flags = [f for f in build.HIPCC_FLAGS if f not in ("-shared", "-Wall")]
    report = subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), *flags, "--cuda-device-only", "-c", "-w", "-Rpass-analysis=kernel-resource-usage",
                             "-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC, os.path.join(build.CSRC, "op_attention.hip"),
                             "-o", str(tmp_path / "device.o")], capture_output=True, text=True, check=True).stderr
    kernel, spilled = None, {}
    for line in report.splitlines():
        name = re.search(r"Function Name: \S*?(forward|grad_queries|grad_keys)IDF16(b|_)Li(\d+)ELi(\d)E", line)
        if "Function Name:" in line:
            kernel = name and (name.group(1), "bf16" if name.group(2) == "b" else "f16", int(name.group(3)), int(name.group(4)))
        count = re.search(r"VGPRs Spill: (\d+)", line)
        if count and kernel:
            spilled[kernel] = int(count.group(1))
    assert len(spilled) == 3 * 2 * 3 * 2
    more = {k: n for k, n in spilled.items() if n > KNOWN.get(k, 0)}
    assert not more, more
