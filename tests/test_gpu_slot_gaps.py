"""Slot maps that leave slots out inside a page: the rows are stored, the slots between them stay, what lies behind a page's last row is cleared, and its
bounds are those of the page up to that row, however the rows fall on warps and blocks."""
import numpy as np
import pytest
import torch

from oracle import paged_attention as orc
from oracle import paged_step as step
from paper_2607_23815_b200 import kvattn
from step_harness import Pages, from_gpu, i32, randn_bits, to_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,d", [(8, 128), (2, 64), (33, 64)])
@pytest.mark.parametrize("n", [1, 3, 700])
def test_rows_with_slots_left_out_between_them(heads, d, n):
    rng = np.random.default_rng(heads + n)
    pages = Pages(n + 2, heads, d)
    pages.host.k[:], pages.host.v[:] = randn_bits(rng, 2, n + 2, heads, 16, d)
    pages.upload()
    slots = []
    for page in rng.permutation(n + 2)[:n]:
        some = [[3, 5], [0, 15], [0, 2, 4, 6, 8], [14], list(range(1, 16, 2)), [0, 1, 2, 9, 10, 12]][rng.integers(6)]
        slots += [int(page) * 16 + s for s in some]
    slots = np.array(slots + [-1] * 5)
    real, T = slots >= 0, len(slots)
    k, v = randn_bits(rng, 2, T, heads, d)
    kvattn.kv_append_rotary(pages.pool, None, to_gpu(k), to_gpu(v), i32(slots), i32(np.zeros(T)), torch.ones(d // 2, device="cuda"), None, None)   # (turned by nothing)
    bounds = torch.full((n + 2, heads, 2, d), 9.0, dtype=torch.bfloat16, device="cuda")
    kvattn.kv_page_bounds(pages.pool, i32(slots), bounds)
    page, at = slots[real] // 16, slots[real] % 16
    for image, rows in ((pages.host.k, k), (pages.host.v, v)):
        image[page, :, at] = rows[real]
        for p in np.unique(page):
            image[p, :, at[page == p].max() + 1:] = 0
    for got, want in zip(pages.image(), (pages.host.k, pages.host.v)):
        assert np.array_equal(got, want)
    want = step.page_bounds(pages.host, slots, np.full(bounds.shape, 9.0))
    assert np.array_equal(orc.widen(from_gpu(bounds)), want) and pages.status() == 0


def test_page_0_and_padding_behind_it():
    pages = Pages(2, 1, 64)
    one = torch.ones(3, 1, 64, dtype=torch.bfloat16, device="cuda")
    slots = i32([4, -1, -16])                                                  # (no slot of page 0, though a sixteenth of it is)
    kvattn.kv_append_rotary(pages.pool, None, one, one, slots, slots * 0, torch.ones(32, device="cuda"), None, None)
    for image in pages.image():
        assert np.all(image[0, 0, 4] == 0x3F80) and np.all(image[0, 0, 5:] == 0) and np.all(image[0, 0, :4] == 0x7FC1) and np.all(image[1] == 0x7FC1)
    pages.k.zero_()
    bounds = torch.full((2, 1, 2, 64), 9.0, dtype=torch.bfloat16, device="cuda")
    kvattn.kv_page_bounds(pages.pool, slots, bounds)
    assert bool((bounds[0] == 0).all()) and bool((bounds[1] == 9).all()) and pages.status() == 0
