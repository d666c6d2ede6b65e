"""What the compiler made of the kernels of the calls around a verification, read from the metadata of the library that was built."""

import os
import re
import struct
import subprocess

import pytest
import yaml

import paper_2602_16994_amd as mpv

LLVM = "/opt/rocm/llvm/bin"


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """Every kernel of every code object in the library (one for each translation unit)."""
    if not os.path.exists(f"{LLVM}/llvm-objcopy"):
        pytest.skip("no LLVM tools of ROCm")
    tmp = tmp_path_factory.mktemp("code")
    subprocess.run([f"{LLVM}/llvm-objcopy", f"--dump-section=.hip_fatbin={tmp}/bundles", mpv.lib_path(), f"{tmp}/copy.so"], check=True)
    data = (tmp / "bundles").read_bytes()
    found = {}
    for start in (m.start() for m in re.finditer(b"__CLANG_OFFLOAD_BUNDLE__", data)):
        entries, = struct.unpack_from("<Q", data, start + 24)
        at = start + 32
        for _ in range(entries):
            offset, size, length = struct.unpack_from("<QQQ", data, at)
            target = data[at + 24:at + 24 + length].decode()
            at += 24 + length
            if "gfx950" not in target or not size:
                continue
            (tmp / "object").write_bytes(data[start + offset:start + offset + size])
            notes = subprocess.run([f"{LLVM}/llvm-readelf", "--notes", f"{tmp}/object"], check=True, capture_output=True, text=True).stdout
            found.update({k[".name"]: k for k in yaml.safe_load(notes[notes.index("---"):notes.index("\n...")])["amdhsa.kernels"]})
    return found


def test_tree_attention(kernels):
    """Two waves a SIMD: 256 registers a lane.  Nothing lies in private memory, but for the 16-row kernel of the longest float32 rows, whose
    query and sums take 192 registers: 7 of them."""
    attention = {n: k for n, k in kernels.items() if "attention_kernel" in n}
    assert len(attention) == 13 + 14 + 14
    for name, k in attention.items():
        widest = "AttentionILi0ELi256ELi1ELi1E" in name
        assert k[".vgpr_count"] <= 256, name
        assert k[".vgpr_spill_count"] <= (7 if widest else 0) and k[".private_segment_fixed_size"] <= (32 if widest else 0), name
        assert k[".sgpr_spill_count"] <= 181, name              # (to lanes of vector registers)


@pytest.mark.parametrize("kernel,count", [("14combine_kernel", 41), ("11part_kernel", 3), ("11draw_kernel", 3), ("12chain_kernel", 3), ("18plan_tables_kernel", 1),
                                          ("16fill_rows_kernel", 1), ("18fill_packed_kernel", 1), ("13append_kernel", 1)])
def test_the_others_keep_all_in_registers(kernels, kernel, count):
    found = {n: k for n, k in kernels.items() if kernel in n}
    assert len(found) == count
    for name, k in found.items():
        assert k[".vgpr_spill_count"] == 0 and k[".sgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0, name
        assert k[".vgpr_count"] <= 128, name                    # (1024 threads a workgroup: 128 registers a lane)
