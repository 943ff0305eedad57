"""How few blocks of a kernel that is launched early are laid over the SMs (no GPU needed): the rule is plain C++."""
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_23815_b200", "csrc")
MAIN = """
#include <cstdio>
#include <initializer_list>
#include "spread.h"
int main() {
  for (int sms : {1, 2, 7, 132, 148})
    for (long blocks = 1; blocks <= 5L * sms; ++blocks) {
      const int smem = kvattn::few_blocks_smem(blocks, sms), share = (int)((blocks + sms - 1) / sms);
      std::printf("%d %ld %d %d\\n", sms, blocks, share, smem);
    }
}
"""


def test_few_blocks_do_not_pile_up_on_an_sm(tmp_path):
    src, exe = tmp_path / "m.cpp", tmp_path / "m"
    src.write_text(MAIN)
    r = subprocess.run(["g++", "-std=c++17", f"-I{CSRC}", str(src), "-o", str(exe)], capture_output=True, text=True)
    if r.returncode:
        pytest.fail(r.stderr)
    rows = [tuple(map(int, x.split())) for x in subprocess.run([str(exe)], capture_output=True, text=True).stdout.splitlines()]
    assert len(rows) == 5 * sum((1, 2, 7, 132, 148))
    for sms, blocks, share, smem in rows:
        if share > 3:
            assert smem == 0
            continue
        per_sm = 228 * 1024 // (smem + 1024)                       # (every block takes 1 KB more)
        want = 2 if share == 1 and 2 * blocks > sms else share     # a second stream's blocks find room beside
        assert per_sm == want and smem <= 227 * 1024
