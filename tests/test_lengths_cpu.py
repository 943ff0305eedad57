"""Lengths have 31 bits: the pages of the longest are counted without an overflow (no GPU needed: the helper is plain C++), and the kernel that makes
block tables counts pages with nothing else."""
import os
import re
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_23815_b200", "csrc")
MAIN = """
#include <cstdio>
#include <initializer_list>
#include "lengths.h"
int main() {
  for (unsigned n : {0u, 1u, 15u, 16u, 17u, 1u << 30, 0x7fffffefu, 0x7ffffff0u, 0x7ffffff1u, 0x7ffffffeu, 0x7fffffffu}) std::printf("%u %d\\n", n, kvattn::pages_of((int)n));
}
"""


def test_pages_of_the_longest_lengths(tmp_path):
    src, exe = tmp_path / "m.cpp", tmp_path / "m"
    src.write_text(MAIN)
    r = subprocess.run(["g++", "-std=c++17", "-fsanitize=undefined", "-fno-sanitize-recover=all", f"-I{CSRC}", str(src), "-o", str(exe)], capture_output=True, text=True)
    if r.returncode:
        pytest.fail(r.stderr)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0, out.stderr
    rows = [tuple(map(int, x.split())) for x in out.stdout.splitlines()]
    assert len(rows) == 11 and all(pages == -(-n // 16) for n, pages in rows)


@pytest.mark.parametrize("name", ["step_tables.cu"])
def test_no_sum_of_a_length_and_a_page_in_signed_32_bits(name):
    code = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
    sums = [m.group(0) for m in re.finditer(r"\(([^()]|\([^()]*\))*\+ kPageSize - 1\) / kPageSize", code)]
    assert [s for s in sums if "(int64_t)" not in s] == []
