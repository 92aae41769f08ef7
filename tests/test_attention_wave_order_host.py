"""The attention kernels for short sequences hand rows from lane to lane of a wave through the LDS before their first barrier.  In their intermediate code,
compiled as the library is, every change from writing the LDS to reading it and back has a barrier of the wave in between, so that the order is what the
program says and not what the compiler happens to leave."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = os.path.join(ROOT, "paper_2304_08480_amd", "csrc", "attention_kernels.hip")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    if shutil.which(HIPCC) is None:
        pytest.skip("no hipcc")
    from paper_2304_08480_amd.build import FLAGS
    out = tmp_path_factory.mktemp("ir") / "attention.ll"
    subprocess.run([HIPCC, *FLAGS, "--offload-device-only", "-emit-llvm", "-S", SOURCE, "-o", str(out)], check=True, capture_output=True, timeout=600)
    found = re.finditer(r"^define [^\n]*amdgpu_kernel[^\n]*@\S*(k_attention_(fwd|bwd)_shortILi\d+ELi(\d+))\S*\(.*?^}", out.read_text(), re.S | re.M)
    return {m.group(1): (m.group(2), int(m.group(3)), m.group(0)) for m in found}


def _events(body):
    """Of what happens before the first barrier of the workgroup: W writes of the LDS, R reads, w barriers of the wave with fences; runs of one as one."""
    text = ""
    for line in body.splitlines():
        if "@llvm.amdgcn.s.barrier" in line:
            break
        if re.search(r"= load .*addrspace\(3\)", line):
            text += "R"
        elif re.match(r"\s*store .*addrspace\(3\)", line):
            text += "W"
        elif "@llvm.amdgcn.wave.barrier" in line:
            text += "w"
        elif re.search(r'fence syncscope\("wavefront"\) (release|acquire)', line):
            text += "f"
    return re.sub(r"(.)\1*", r"\1", text.replace("fwf", "w"))


def test_rows_change_lanes_in_the_order_of_the_program(kernels):
    assert len(kernels) == 32                     # forward and backward, head widths of 32 and 64 in five numbers of tiles, of 96 and 128 in three
    for name, (way, tiles, body) in kernels.items():
        events = _events(body)
        assert "R" in events and "WR" not in events and "RW" not in events and "f" not in events, (name, events)
