"""Registers and LDS of the chunk kernels, as the compiler's metadata in the library's gfx950 code objects gives them: what decides how many
workgroups a compute unit holds.  No GPU needed."""
import re
import struct
import subprocess

import pytest

READELF = "/opt/rocm/llvm/bin/llvm-readelf"


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{mangled name: {"vgpr_count": n, "vgpr_spill_count": n, "group_segment_fixed_size": bytes}} of all code objects."""
    from paper_2601_18383_amd import build
    data = open(build.build(force=False), "rb").read()
    out, at, n = {}, data.find(b"__CLANG_OFFLOAD_BUNDLE__"), 0
    while at >= 0:
        count, pos = struct.unpack_from("<Q", data, at + 24)[0], at + 32
        for _ in range(count):
            offset, size, length = struct.unpack_from("<QQQ", data, pos)
            if b"gfx950" in data[pos + 24:pos + 24 + length]:
                path = tmp_path_factory.mktemp("code") / ("gfx950_%d.co" % n)
                path.write_bytes(data[at + offset:at + offset + size])
                notes = subprocess.run([READELF, "--notes", str(path)], capture_output=True, text=True, check=True).stdout
                for block in notes.split("\n  - .a")[1:]:
                    field = lambda k: re.search(r"\.%s:\s*(\S+)" % k, block)
                    if field("symbol"):
                        out[field("name").group(1)] = {k: int(field(k).group(1)) for k in
                                                       ("vgpr_count", "vgpr_spill_count", "group_segment_fixed_size")}
            pos += 24 + length
        n += 1
        at = data.find(b"__CLANG_OFFLOAD_BUNDLE__", at + 24)
    return out


def _named(kernels, pattern, count):
    found = {n: k for n, k in kernels.items() if re.search(pattern, n)}
    assert len(found) == count, sorted(found)
    return found


def test_many_rows_keep_three_workgroups_a_compute_unit(kernels):
    for name, k in _named(kernels, r"chunk_attend_kernelILi128E", 4).items():
        assert k["vgpr_count"] <= 168 and 3 * k["group_segment_fixed_size"] <= 160 * 1024, name
    for name, k in _named(kernels, r"chunk_attend_kernelILi64E", 4).items():
        assert k["vgpr_count"] <= 128 and k["vgpr_spill_count"] == 0, name
    plain, = _named(kernels, r"chunk_attend_kernelILi128ELb0ELb0ELb0EE", 1).values()
    assert plain["vgpr_spill_count"] == 0


def test_few_rows_do_not_spill(kernels):
    for name, k in _named(kernels, r"chunk_attend_few_kernelILi(64|128)E", 4).items():
        assert k["vgpr_count"] <= 256 and k["vgpr_spill_count"] == 0 and k["group_segment_fixed_size"] <= 160 * 1024, name


def test_scores_keep_three_workgroups_a_compute_unit(kernels):
    for name, k in _named(kernels, r"chunk_scores_kernelILi(64|128)E", 6).items():
        assert k["vgpr_count"] <= 168 and 3 * k["group_segment_fixed_size"] <= 160 * 1024, name
    for name, k in _named(kernels, r"chunk_scores_kernelILi(64|128)ELb0ELb0EE", 2).items():
        assert k["vgpr_spill_count"] == 0, name


def test_scores_of_few_slots_do_not_spill(kernels):
    for name, k in _named(kernels, r"chunk_scores_few_kernelILi(64|128)E", 6).items():
        assert k["vgpr_count"] <= 256 and k["vgpr_spill_count"] == 0, name
