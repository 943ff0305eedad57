"""kv_page_bounds against the definition (a choice among stored values: equal)."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import paged_attention as orc
from oracle import paged_step as step
from paper_2607_23815_b200 import kvattn
from step_harness import Pages, from_gpu, guarded, i32, randn_bits

pytestmark = pytest.mark.gpu


def _run(pages, slots):
    b, check = guarded((pages.n, pages.heads, 2, pages.d), torch.bfloat16, 9.0)
    kvattn.kv_page_bounds(pages.pool, i32(slots), b)
    torch.cuda.synchronize()
    assert check()
    want = step.page_bounds(pages.host, slots, np.full(b.shape, 9.0))
    return orc.widen(from_gpu(b)), want


CASES = [(8, 128, [(1483, 1)], 0), (2, 64, [(0, 1)], 0), (8, 128, [(i, 1) for i in range(40)], 6), (1, 128, [(15, 1), (15, 2), (0, 16), (0, 17), (3, 13)], 0),
         (3, 64, [(5, 300), (0, 15)], 33), (8, 64, [(0, 4000), (1, 31)], 0), (8, 128, [(0, 2100)] * 3, 1)]


@pytest.mark.parametrize("heads,d,seqs,pad", CASES)
def test_bounds_of_the_pages_that_were_written(heads, d, seqs, pad):
    rng = np.random.default_rng(heads * d + len(seqs))
    count = sum(-(-(a % 16 + b) // 16) for a, b in seqs) + 2
    pages, ids, slots, at = Pages(count, heads, d), rng.permutation(count), [], 0
    for a, b in seqs:
        t = np.arange(a % 16 + b)
        rows = ids[at + t // 16] * 16 + t % 16
        pages.host.k[rows // 16, :, rows % 16] = randn_bits(rng, len(rows), heads, d)   # (slots behind stay what they are: no numbers)
        slots += rows[a % 16:].tolist()
        at += -(-(a % 16 + b) // 16)
    pages.upload()
    got, want = _run(pages, np.array(slots + [-1] * pad))
    assert np.array_equal(got, want) and pages.status() == 0


def test_keys_that_are_infinite_or_not_numbers():
    rng = np.random.default_rng(2)
    pages = Pages(3, 2, 64)
    pages.host.k[:] = randn_bits(rng, 3, 2, 16, 64)
    pages.host.k[1, 0, 4, 7], pages.host.k[1, 1, 15, 63], pages.host.k[0, 0, 0, :2], pages.host.k[2, 1, 9, 33] = 0x7FC0, 0xFFFF, [0x7F80, 0xFF80], 0xFF80
    pages.upload()
    got, want = _run(pages, np.arange(48))
    assert np.array_equal(got, want, equal_nan=True) and np.isnan(got).sum() == 4


def test_slots_outside_are_recorded_and_nothing_to_do():
    pages = Pages(2, 1, 64)
    pages.host.k[:] = 0x3F80
    pages.upload()
    got, want = _run(pages, np.array([-1, -1, -5]))
    assert np.array_equal(got, want) and pages.status() == 0
    b = torch.full((2, 1, 2, 64), 9.0, dtype=torch.bfloat16, device="cuda")
    kvattn.kv_page_bounds(pages.pool, i32([3, 32, 0x7fffffff, 17]), b)
    assert pages.status() == kvattn.KV_ERR_BOUNDS and float(b.sum()) == 256.0
    n0 = kvattn.kvattn_launch_count()
    kvattn.kv_page_bounds(pages.pool, i32([]), b)
    p = lambda off=0: C.c_void_p(b.data_ptr() + off)
    call = kvattn.lib().kv_page_bounds
    h, inv = pages.pool.handle, kvattn.KV_ERR_INVALID
    assert call(None, p(), 1, p(), None) == call(h, None, 1, p(), None) == call(h, p(), 1, None, None) == call(h, p(), -1, p(), None) == inv
    assert call(h, p(), 1, p(8), None) == inv and call(h, p(), (1 << 30) + 1, p(), None) == kvattn.KV_ERR_UNSUPPORTED
    assert kvattn.kvattn_launch_count() == n0
    assert kvattn.kv_page_bounds_bytes(pages.pool) == 2 * 2 * 64 * 2 and kvattn.lib().kv_page_bounds_bytes(None) == 0
    with pytest.raises(ValueError):
        kvattn.kv_page_bounds(pages.pool, i32([1]), b[:1])
    with pytest.raises(TypeError):
        kvattn.kv_page_bounds(pages.pool, i32([1]), b.float())
