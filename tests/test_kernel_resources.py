"""Registers and scratch memory of the kernels as built, from the notes the compiler leaves in the library for the runtime that loads them.

A wave may have 512 vector registers of a SIMD's divided by the waves that stand on it, in steps of eight: 84 or fewer leave room for six."""
import os
import re
import struct
import subprocess

import pytest

import paper_2402_14118_amd as mm

READELF = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "llvm-readelf")


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """Mangled name -> the figures of every kernel in the library."""
    data, found, at = open(mm.LIB_PATH, "rb").read(), {}, 0
    path = tmp_path_factory.mktemp("notes") / "object"
    while (at := data.find(b"\x7fELF\x02\x01\x01\x40", at)) >= 0:       # (64 bits, little-endian, the ABI of device code)
        sections, = struct.unpack_from("<Q", data, at + 0x28)
        entry, count = struct.unpack_from("<HH", data, at + 0x3A)
        path.write_bytes(data[at:at + sections + entry * count])
        text = subprocess.run([READELF, "--notes", str(path)], check=True, capture_output=True, text=True).stdout
        for kernel in re.split(r"\n  - (?=\.agpr_count)", text)[1:]:
            figures = {k: int(v) for k, v in re.findall(r"\n    \.(vgpr_count|vgpr_spill_count|private_segment_fixed_size): +(\d+)", kernel)}
            found[re.search(r"\n    \.name: +(\S+)", kernel).group(1)] = figures
        at += sections
    assert len(found) > 300
    return found


def pairs(kernels, fused, ks):
    """Instances of the pair kernel by (mangled element type, block width, waves along the columns, words)."""
    out = {}
    for name, figures in kernels.items():
        m = re.search(r"mmm_pairs_kernelI(\w+?)Li(\d+)ELi(\d+)ELi(\d+)ELi(\d+)ELb([01])E", name)
        if m and (m.group(6) == "1") == fused and int(m.group(4)) == ks:
            out.setdefault((m.group(1), int(m.group(2)), int(m.group(3)), int(m.group(5))), []).append(figures)
    return out


def test_pairs_keep_their_sums_in_registers(kernels):
    for fused, ks in ((False, 1), (False, 4), (True, 1), (True, 2), (True, 4), (True, 8)):
        instances = pairs(kernels, fused, ks)
        assert instances
        for which, both in instances.items():
            assert all(f["private_segment_fixed_size"] == 0 for f in both), (fused, ks, which)


def test_many_rows_leave_room_for_other_waves(kernels):
    """The mask evaluated inside, 512 columns to a workgroup: its loads wait, and other waves have to work meanwhile."""
    instances = pairs(kernels, True, 1)
    for which in (("f", 16, 8, 32), ("f", 32, 8, 32), ("f", 32, 8, 64), ("t", 32, 8, 32)):
        for figures in instances[which]:
            assert figures["vgpr_count"] <= 84, (which, figures)


def test_no_other_kernel_uses_scratch(kernels):
    """But norms of more than one piece for each lane, and two instances that put one or two registers by."""
    for name, figures in kernels.items():
        if figures["private_segment_fixed_size"] == 0:
            continue
        wide = re.search(r"mmm_block_norm(_grad)?_kernelI\w+Li[24]ELi(8|16)E", name)
        few = re.search(r"mmm_build_kernel|mmm_matmul_kernel", name) and figures["vgpr_spill_count"] <= 2
        assert wide or few, (name, figures)
