"""attn_select_pages against the definition in 64 bits (whole numbers: equal)."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import paged_attention as orc
from oracle import paged_step as step
from paper_2607_23815_b200 import kvattn
from step_harness import Pages, guarded, i32, randn_bits, to_gpu

pytestmark = pytest.mark.gpu


def _case(rng, hq, hkv, d, ctx, extra=0):
    need = [max(0, -(-c // 16)) for c in ctx]
    count, width = sum(need) + 1, max(need + [1]) + extra
    ids, tables, at = rng.permutation(count), np.full((len(ctx), width), -1, np.int64), 0
    for i, k in enumerate(need):
        tables[i, :k] = ids[at:at + k]
        at += k
    a, b = randn_bits(rng, 2, count, hkv, d)
    lo, hi = np.minimum(orc.widen(a), orc.widen(b)), np.maximum(orc.widen(a), orc.widen(b))
    return randn_bits(rng, len(ctx), hq, d), np.stack([lo, hi], 2), tables, count


def _bits(bounds):
    return (np.asarray(bounds, np.float32).view(np.uint32) >> 16).astype(np.uint16)


def _run(q, bounds, tables, ctx, hkv, count, n_select, first, last, max_ctx=None, want_status=0):
    B, _, d = q.shape
    pages = Pages(count, hkv, d)
    (lists, c1), (counts, c2) = guarded((B, hkv, n_select), torch.int32, -99), guarded((B, hkv), torch.int32, -99)
    kvattn.attn_select_pages(pages.pool, to_gpu(q), to_gpu(_bits(bounds)), i32(tables), i32(ctx), max(max(ctx), 0) if max_ctx is None else max_ctx,
                             first, last, lists, counts)
    torch.cuda.synchronize()
    assert c1() and c2() and pages.status() == want_status
    return lists.cpu().numpy(), counts.cpu().numpy()


def _check(q, bounds, tables, ctx, hkv, count, n_select, first, last):
    lists, counts = _run(q, bounds, tables, ctx, hkv, count, n_select, first, last)
    want, wcounts = step.select_pages(q, bounds, tables, ctx, hkv, n_select, first, last)
    assert np.array_equal(counts, wcounts)
    assert np.array_equal(lists, want), np.argwhere(np.any(lists != want, -1))[:5]


@pytest.mark.parametrize("hq,hkv,d", [(32, 8, 128), (64, 8, 128), (8, 8, 128), (4, 2, 128), (4, 2, 64), (8, 1, 64), (12, 3, 64), (3, 3, 64)])
@pytest.mark.parametrize("n_select,first,last", [(1, 0, 0), (8, 1, 2), (32, 0, 4), (5, 2, 3)])
def test_the_pages_with_the_largest_scores(hq, hkv, d, n_select, first, last):
    rng = np.random.default_rng(hq * d + n_select)
    ctx = [0, 1, 15, 16, 17, n_select * 16 - 1, n_select * 16, n_select * 16 + 1, 700, 1999, 33]
    q, bounds, tables, count = _case(rng, hq, hkv, d, ctx, extra=3)
    _check(q, bounds, tables, ctx, hkv, count, n_select, first, last)


@pytest.mark.parametrize("hq,hkv,d,ctx,n_select", [(32, 8, 128, [15731], 64), (4, 1, 64, [24576 * 16], 100), (8, 1, 128, [60001, 3], 128), (16, 2, 64, [9000] * 5, 40),
                                                   (32, 8, 64, [5000] * 30, 16), (32, 8, 128, [257] * 64, 16)])
def test_long_contexts_and_many_rows(hq, hkv, d, ctx, n_select):
    rng = np.random.default_rng(len(ctx))
    q, bounds, tables, count = _case(rng, hq, hkv, d, ctx)
    _check(q, bounds, tables, ctx, hkv, count, n_select, 1, 2)


@pytest.mark.parametrize("batch", [1, 40])
@pytest.mark.parametrize("what", ["equal", "zero", "few_values", "last_bits", "wide", "infinite", "not_numbers", "overflow", "tiny", "negative_zero"])
def test_the_order_is_that_of_exact_scores(what, batch):
    rng = np.random.default_rng(11)
    hq, hkv, d, ctx = 8, 2, 64, [3000, 2000, 500] * batch
    ctx = ctx[:batch * 3]
    q, bounds, tables, count = _case(rng, hq, hkv, d, ctx)
    if what == "equal":
        bounds[:] = bounds[:1]
    if what == "zero":
        q[:] = 0
    if what == "few_values":                                                    # many equal scores, a few steps apart
        bounds = np.sign(bounds) * (rng.integers(0, 2, (count, 1, 1, 1)) + 1.0)
        bounds = np.broadcast_to(bounds[:, :, :, :1], bounds.shape).copy()
        bounds = np.stack([bounds.min(2), bounds.max(2)], 2)
    if what == "last_bits":                                                     # pages differ by one step of one element, far below 32 bits of the sum
        bounds[:] = bounds[:1] * 0 + np.where(np.arange(d) < 32, 96.0, 1e-3).astype(np.float32).view(np.uint32).__and__(0xffff0000).astype(np.uint32).view(np.float32)
        bounds[:, :, :, -1] = (2.0 ** -12 * (1 + rng.integers(0, 128, (count, hkv)) / 128))[..., None]
    if what == "wide":                                                          # a few elements dwarf the others
        bounds *= 2.0 ** rng.integers(-30, 30, (count, hkv, 1, 1))
        bounds = orc.widen(_bits(bounds))
    if what == "infinite":
        bounds[rng.integers(0, count, 40), :, 1, rng.integers(0, d, 40)] = np.inf
        bounds[rng.integers(0, count, 40), :, 0, rng.integers(0, d, 40)] = -np.inf
    if what == "not_numbers":
        bounds[rng.integers(0, count, 9), :, :, 5] = np.nan
        q[0, 3, 9] = 0x7FC0
    if what == "overflow":
        bounds *= 2.0 ** 120
        q = (q & 0x807F) | (254 << 7)
    if what == "tiny":
        bounds *= 2.0 ** -120
        bounds, q = orc.widen(_bits(bounds)), (q & 0x807F) | (20 << 7)
    if what == "negative_zero":
        bounds[:], q = np.array([-0.0, 0.0])[None, None, :, None] * np.where(rng.random((count, hkv, 1, 1)) < 0.5, -1.0, 1.0), q
    bounds = orc.widen(_bits(bounds))
    for n_select, first, last in ((20, 0, 0), (31, 1, 4)):
        _check(q, bounds, tables, ctx, hkv, count, n_select, first, last)


def test_longer_than_stated_and_pages_outside():
    rng = np.random.default_rng(3)
    ctx = [400, 900, 640]
    q, bounds, tables, count = _case(rng, 4, 2, 64, ctx)
    want, wcounts = step.select_pages(q, bounds, tables, ctx, 2, 8, 1, 1)
    lists, counts = _run(q, bounds, tables, ctx, 2, count, 8, 1, 1, max_ctx=640, want_status=kvattn.KV_ERR_BOUNDS)
    assert np.all(lists[1] == -99) and np.all(counts[1] == -99)
    assert np.array_equal(lists[[0, 2]], want[[0, 2]]) and np.array_equal(counts[[0, 2]], wcounts[[0, 2]])
    bad = tables.copy()
    bad[1, 7], bad[1, 20] = count, -3
    lists, counts = _run(q, bounds, bad, ctx, 2, count, 8, 1, 1, want_status=kvattn.KV_ERR_BOUNDS)
    assert np.array_equal(lists[[0, 2]], want[[0, 2]]) and np.all(counts == 8) and np.all(np.diff(lists[1], axis=-1) > 0)


def test_entries_past_the_context_are_not_read():
    rng = np.random.default_rng(4)
    ctx = [300, 170]
    q, bounds, tables, count = _case(rng, 4, 2, 64, ctx, extra=2)
    bounds[~np.isin(np.arange(count), tables[tables >= 0])] = np.nan
    tables[tables < 0] = 1 << 30
    _check(q, bounds, tables, ctx, 2, count, 6, 1, 1)


def test_refusals():
    pages, lib = Pages(3, 2, 64), kvattn.lib()
    t = torch.zeros(8192, dtype=torch.bfloat16, device="cuda")
    p = lambda off=0: C.c_void_p(t.data_ptr() + off)
    good = dict(pool=pages.pool.handle, q=p(), hq=4, b=p(), bt=p(), width=2, ctx=p(), batch=1, mc=32, n=2, first=0, last=1, lists=p(8192), counts=p(12000))
    call = lambda **kw: lib.attn_select_pages(*{**good, **kw}.values(), None)
    inv, uns = kvattn.KV_ERR_INVALID, kvattn.KV_ERR_UNSUPPORTED
    n0 = kvattn.kvattn_launch_count()
    for kw in (dict(pool=None), dict(q=None), dict(b=None), dict(bt=None), dict(ctx=None), dict(lists=None), dict(counts=None), dict(batch=-1), dict(width=-1),
               dict(mc=-1), dict(mc=33), dict(n=0), dict(first=-1), dict(last=-1), dict(first=2), dict(q=p(8)), dict(b=p(4))):
        assert call(**kw) == inv, kw
    for kw in (dict(hq=3), dict(hq=0), dict(hq=32), dict(width=1 << 20, mc=24577 * 16)):
        assert call(**kw) == uns, kw
    assert call(batch=0) == 0 and kvattn.kvattn_launch_count() == n0
    assert call() == 0
    q, b, bt = torch.zeros(1, 4, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(3, 2, 2, 64, dtype=torch.bfloat16, device="cuda"), i32([[0, 1]])
    ok = [q, b, bt, i32([20]), 32, 0, 0, i32(np.zeros((1, 2, 2))), i32([[0, 0]])]
    for i, bad in ((0, q[0]), (1, b[:2]), (2, i32([[0, 1]] * 2)), (3, i32([1, 2])), (7, i32(np.zeros((1, 3, 2)))), (8, i32([0]))):
        with pytest.raises(ValueError):
            kvattn.attn_select_pages(pages.pool, *[bad if j == i else x for j, x in enumerate(ok)])
    kvattn.attn_select_pages(pages.pool, *ok)
    assert ok[7].flatten().tolist() == [0, 1, 0, 1] and pages.status() == 0


@pytest.mark.parametrize("hq,hkv,d,n,ctx", [(32, 8, 128, 90, (300, 900)), (8, 8, 64, 100, (17, 3000)), (64, 8, 128, 80, (2900, 3200))])
def test_more_rows_than_the_device_holds(hq, hkv, d, n, ctx):
    rng = np.random.default_rng(n)
    lens = rng.integers(ctx[0], ctx[1] + 1, n).tolist()
    q, bounds, tables, count = _case(rng, hq, hkv, d, lens)
    _check(q, bounds, tables, lens, hkv, count, 7, 1, 1)


@pytest.mark.parametrize("what", ["normal", "equal", "few_values", "not_numbers"])
def test_many_rows_of_few_pages(what):
    rng = np.random.default_rng(6)
    hq, hkv, d = 16, 8, 64
    lens = rng.integers(1, 190 * 16, 90).tolist()
    lens[:12] = [16 * n for n in (8, 9, 39, 40, 41, 71, 72, 73, 134, 135, 136, 137)]   # (up to 128 pages in question, and more)
    q, bounds, tables, count = _case(rng, hq, hkv, d, lens)
    if what == "equal":
        bounds[:] = bounds[:1]
    if what == "few_values":
        bounds = np.sign(bounds) * (rng.integers(0, 3, (count, 1, 1, 1)) + 1.0)
        bounds = np.stack([bounds.min(2), bounds.max(2)], 2)
    if what == "not_numbers":
        bounds[rng.integers(0, count, count // 9), :, 1, 3] = np.nan
        bounds[rng.integers(0, count, count // 9), :, 0, 4] = -np.inf
    for n_select, first, last in ((8, 1, 2), (40, 0, 0), (5, 3, 2)):
        _check(q, orc.widen(_bits(bounds)), tables, lens, hkv, count, n_select, first, last)
