"""The bounds and the rotary append where one launch's blocks go round several times and a warp of the bounds looks at sixteen and at thirty-two rows (sizes for a
device of 148 SMs)."""
import numpy as np
import pytest
import torch

from oracle import paged_attention as orc
from oracle import paged_step as step
from paper_2607_23815_b200 import kvattn
from step_harness import Pages, from_gpu, i32, randn_bits, to_gpu
from test_gpu_append_rotary import _close, _slots

pytestmark = pytest.mark.gpu


def _seqs(rng, total):
    out, left = [], total
    while left:
        new = min(left, int(rng.integers(1, 3000)))
        out.append((int(rng.integers(0, 40)), new))
        left -= new
    return out


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads,total", [(8, 12001), (8, 100003), (3, 250001)])
def test_bounds_of_many_rows(heads, total, d):
    rng = np.random.default_rng(total + d)
    seqs = _seqs(rng, total)
    count = sum(-(-(a % 16 + b) // 16) for a, b in seqs) + 2
    slots = _slots(rng, count, *zip(*seqs), 37)
    few = randn_bits(rng, 97, heads, 16, d)                                    # (pages of other numbers, drawn from a few)
    pages = Pages(count, heads, d)
    pages.host.k[:] = few[rng.integers(0, 97, count)]
    pages.host.k[:, :, 15] = 0x7FC0                                            # what lies behind a page's last row is no number, unless it has sixteen
    full = slots[(slots >= 0) & (slots % 16 == 15)] // 16
    pages.host.k[full, :, 15] = few[0, :, 15]
    pages.upload()
    bounds = torch.full((count, heads, 2, d), 9.0, dtype=torch.bfloat16, device="cuda")
    kvattn.kv_page_bounds(pages.pool, i32(slots), bounds)
    want = step.page_bounds(pages.host, slots, np.full(bounds.shape, 9.0))
    assert np.array_equal(orc.widen(from_gpu(bounds)), want) and pages.status() == 0


@pytest.mark.parametrize("hq,hkv,d,total,neighbours", [(32, 8, 128, 2501, False), (64, 8, 128, 1403, True), (1, 1, 128, 6007, False), (16, 4, 64, 5003, True)])
def test_rotation_of_many_rows(hq, hkv, d, total, neighbours):
    rng = np.random.default_rng(total)
    seqs = _seqs(rng, total)
    count = sum(-(-(a % 16 + b) // 16) for a, b in seqs) + 2
    pages, slots = Pages(count, hkv, d), _slots(rng, count, *zip(*seqs), 11)
    T = len(slots)
    q, k, v = (randn_bits(rng, T, h, d) for h in (hq, hkv, hkv))
    pos, inv = rng.integers(0, 200000, (1, T)), (10000.0 ** (-np.arange(d // 2) * 2 / d)).astype(np.float32)
    row = to_gpu(np.concatenate([x.reshape(T, -1) for x in (q, k, v)], 1))
    tq, tk, tv = (x.unflatten(1, (-1, d)) for x in row.split([hq * d, hkv * d, hkv * d], 1))
    out = torch.full((T, hq, d), -3.0, dtype=torch.bfloat16, device="cuda")
    kvattn.kv_append_rotary(pages.pool, tq, tk, tv, i32(slots), i32(pos[0]), torch.from_numpy(inv).cuda(), None, out, neighbours)
    real, turn = slots >= 0, lambda x: step.rotate(orc.widen(x), pos, inv, None, neighbours)
    got = from_gpu(out)
    assert np.all(orc.widen(got[~real]) == -3)
    _close(got[real], orc.widen(q)[real], turn(q)[real], d // 2, neighbours)
    ki, vi = pages.image()
    page, at = slots[real] // 16, slots[real] % 16
    _close(ki[page, :, at], orc.widen(k)[real], turn(k)[real], d // 2, neighbours)
    assert np.array_equal(vi[page, :, at], v[real]) and pages.status() == 0
    stored = np.zeros((count, 16), bool)
    stored[page, at] = True
    behind = ~stored & (np.arange(16)[None] > np.where(stored.any(1), 15 - np.argmax(stored[:, ::-1], 1), 16)[:, None])
    in_front = ~stored & ~behind
    for image in (ki.transpose(0, 2, 1, 3), vi.transpose(0, 2, 1, 3)):
        assert np.all(image[behind] == 0) and np.all(image[in_front] == 0x7FC1)
