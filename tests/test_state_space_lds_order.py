"""Exchanges between the lanes of one wave through LDS, in what the compiler is given to order: its own intermediate code of the kernels."""
import os
import re
import subprocess

import pytest

from paper_1907_03329_amd import build


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{kernel: its lines} of the reverse scan, compiled for the device alone."""
    out = tmp_path_factory.mktemp("code") / "backward.ll"
    subprocess.run([build.HIPCC] + build.FLAGS + ["--cuda-device-only", "-S", "-emit-llvm", "-o", str(out), os.path.join(build.CSRC, "selective_backward_kernels.hip")],
                   check=True, capture_output=True)
    text = out.read_text()
    return {m.group(1): m.group(2).splitlines() for m in re.finditer(r"^define [^\n]*@(\w*selective_backward_kernel\w*)\([^\n]*\{\n(.*?)^\}", text, re.M | re.S)}


def unordered(lines):
    """Accesses that follow, with nothing between that keeps the order, one of the other kind: a read of what other lanes have written, a write over what they read."""
    seen, found, fences = set(), [], set()
    for line in lines:
        if "s_barrier" in line and "~{memory}" in line:
            seen.clear()
        if m := re.search(r'fence syncscope\("wavefront"\) (\w+)', line):
            fences.add(m.group(1))
            if fences == {"release", "acquire"} or "acq_rel" in fences:
                seen.clear()
                fences.clear()
        kind = "read" if re.search(r"= load .*ptr addrspace\(3\)", line) else "write" if re.search(r"^\s*store .*ptr addrspace\(3\)", line) else None
        if kind:
            fences.clear()
            if seen - {kind}:
                found.append(line.strip())
            seen.add(kind)
    return found


def test_the_check_finds_what_it_is_for():
    write, read = "  store <4 x float> %1, ptr addrspace(3) %2, align 16", "  %3 = load <4 x float>, ptr addrspace(3) %4, align 16"
    order = ['  fence syncscope("wavefront") release', "  tail call void @llvm.amdgcn.wave.barrier()", '  fence syncscope("wavefront") acquire']
    barrier = ['  tail call void asm sideeffect "s_waitcnt lgkmcnt(0)\\0A\\09s_barrier", "~{memory}"()']
    assert unordered([write, read]) == [read.strip()] and unordered([read, write]) == [write.strip()] and unordered([write, order[0], read])
    assert not unordered([write, write, *order, read, read, *order, write, *barrier, read])


def test_sums_over_the_lanes_of_a_wave_are_ordered(kernels):
    """The reverse scan's lanes leave values in LDS, read other lanes', and leave the next ones in the same places."""
    assert len(kernels) == 20
    for name, lines in kernels.items():
        accesses = [line for line in lines if re.search(r"(= load|^\s*store) .*ptr addrspace\(3\)", line)]
        assert len(accesses) >= 32, name
        assert not unordered(lines), name
