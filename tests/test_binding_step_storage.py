"""Tensors without storage are an error of the calls around attention as well, and not a crash: here, where the current device cannot be had either, and on a GPU."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

_SCRIPT = """
import faulthandler; faulthandler.enable()
import torch
from torch._subclasses.fake_tensor import FakeTensorMode
from paper_2607_23815_b200 import kvattn
class NoPool:
    ptr, n_kv_heads, head_dim = None, 2, 64
if torch.cuda.is_available():
    torch.zeros(1, device="cuda")
with FakeTensorMode():
    e = lambda t, *s: torch.empty(3, *s, dtype=t, device="cuda")
    args = [e(torch.bfloat16, 2, 4, 64), e(torch.bfloat16, 2, 2, 64), e(torch.int32, 2, 8), e(torch.int32, 2, 2, 5), e(torch.int32, 2), e(torch.int32, 2, 2),
            e(torch.float32, 32), e(torch.float32, 2, 4), e(torch.int32, 3)]
calls = {
    "tables": lambda q, k, bt, lists, two, counts, inv, lse, three: kvattn.kv_step_tables(NoPool, two, two, two, bt, three, two, two, two, None, None, 0),
    "rotary": lambda q, k, bt, lists, two, counts, inv, lse, three: kvattn.kv_append_rotary(NoPool, q, k, k, two, two, inv, None, q, False, 0),
    "rotary of keys": lambda q, k, bt, lists, two, counts, inv, lse, three: kvattn.kv_append_rotary(NoPool, None, k, k, two, two, inv, None, None, False, 0),
    "bounds": lambda q, k, bt, lists, two, counts, inv, lse, three: kvattn.kv_page_bounds(NoPool, two, q, 0),
    "choice": lambda q, k, bt, lists, two, counts, inv, lse, three: kvattn.attn_select_pages(NoPool, q, k, bt, two, 64, 0, 0, lists, counts, 0),
    "selected": lambda q, k, bt, lists, two, counts, inv, lse, three: kvattn.attn_decode_selected(NoPool, q, bt, two, 64, lists, counts, 1.0, q, lse, 0),
}
def refused(*tensors):
    for name, call in calls.items():
        for _ in range(3):
            try:
                call(*tensors)
            except RuntimeError as e:
                assert not isinstance(e, kvattn.KvError), name
            else:
                raise SystemExit(name + ": no error")
    return tensors[0]
torch.vmap(refused)(*args)
print("all refused")
"""


def _check():
    r = subprocess.run([sys.executable, "-c", _SCRIPT], capture_output=True, text=True, cwd=ROOT, timeout=300)
    assert r.returncode == 0 and "all refused" in r.stdout, (r.returncode, r.stdout, r.stderr[-2000:])


def test_tensors_without_storage_here():
    _check()


@pytest.mark.gpu
def test_tensors_without_storage_on_a_gpu():
    _check()
