"""Kernels that are bound by memory keep what they hold in registers: what the compiler says of them."""
import os
import re
import subprocess

from paper_2608_26004_gb300 import build


def test_no_write_into_the_4_bit_cache_spills(tmp_path):
    done = subprocess.run([build.nvcc_path(), "-gencode", build.GENCODE, "-O3", "-std=c++17", "-I" + build.INCLUDE,
                           "-Xptxas=-v", "-c", os.path.join(build.CSRC, "cache4.cu"), "-o", str(tmp_path / "cache4.o")],
                          capture_output=True, text=True, check=True)
    found = re.findall(r"Function properties for \S*cache4_(write|read)_kernel\S*\n.*?(\d+) bytes spill stores, (\d+) bytes spill",
                       done.stderr)
    assert sorted(name for name, _, _ in found) == ["read"] * 4 + ["write"] * 4
    assert all((stores, loads) == ("0", "0") for _, stores, loads in found), found
