"""attn_decode_selected against the definition in 64 bits.

Tolerance: O is rounded to bf16 once (2^-8 of it) and every weight once before it multiplies a value (2^-8 of sum p |v|); scores of up to 2^6 are summed
in 32 bits and exponentiated with a relative error of 2^-22 or less (2^-16 of sum p |v|, with room).  LSE: those scores' 2^-18 and a logarithm."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import paged_attention as orc
from oracle import paged_step as step
from paper_2607_23815_b200 import kvattn
from step_harness import Pages, from_gpu, guarded, i32, randn_bits, to_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(params=[0, 1, 2])
def impl(request):
    kvattn.kvattn_set_decode_impl(request.param)
    yield request.param
    kvattn.kvattn_set_decode_impl(0)


def _state(rng, hkv, d, ctx, extra=0):
    need = [max(0, -(-c // 16)) for c in ctx]
    count, width = sum(need) + 1, max(need + [1]) + extra
    ids, tables, at = rng.permutation(count), np.full((len(ctx), width), -1, np.int64), 0
    pages = Pages(count, hkv, d)
    for i, c in enumerate(ctx):
        k = need[i]
        tables[i, :k] = ids[at:at + k]
        at += k
        for b in range(k):
            n = min(16, c - 16 * b)
            pages.host.k[tables[i, b], :, :n], pages.host.v[tables[i, b], :, :n] = randn_bits(rng, 2, hkv, n, d)
    pages.upload()
    return pages, tables


def _lists(rng, ctx, hkv, width, how):
    lists, counts = np.full((len(ctx), hkv, width), -1, np.int64), np.zeros((len(ctx), hkv), np.int64)
    for i, c in enumerate(ctx):
        nb = max(0, -(-c // 16))
        for h in range(hkv):
            k = min(nb, width) if how != "ragged" else int(rng.integers(0, min(nb, width) + 1))
            pick = rng.permutation(nb)[:k]
            lists[i, h, :k] = pick if how == "unordered" else np.sort(pick)
            counts[i, h] = k
    return lists, counts


def _run(pages, q, tables, ctx, lists, counts, scale, max_ctx=None):
    B, hq, d = q.shape
    (out, c1), (lse, c2) = guarded((B, hq, d), torch.bfloat16, -7.0), guarded((B, hq), torch.float32, -7.0)
    kvattn.attn_decode_selected(pages.pool, to_gpu(q), i32(tables), i32(ctx), max(max(ctx), 0) if max_ctx is None else max_ctx, i32(lists), i32(counts),
                                scale, out, lse)
    torch.cuda.synchronize()
    assert c1() and c2()
    return orc.widen(from_gpu(out)), lse.cpu().numpy().astype(np.float64)


def _close(got, pages, q, tables, ctx, lists, counts, scale):
    hq = q.shape[1]
    o, l = step.decode_selected(pages.host, q, hq, tables, ctx, lists, counts, scale)
    v, pages.host.v = pages.host.v, pages.host.v & 0x7FFF
    reach = step.decode_selected(pages.host, q, hq, tables, ctx, lists, counts, scale)[0]
    pages.host.v = v
    d = np.abs(got[0] - o)
    assert np.all(d <= 2.0 ** -8 * (np.abs(o) + reach) + 2.0 ** -15 * reach), float(d.max())
    assert np.array_equal(np.isneginf(got[1]), np.isneginf(l))
    fin = np.isfinite(l)
    assert np.all(np.abs(got[1][fin] - l[fin]) <= 1e-4)


@pytest.mark.parametrize("hq,hkv,d,ctx,width", [
    (32, 8, 128, [15731], 64), (4, 2, 64, [0, 1, 15, 16, 17, 300], 4), (8, 1, 128, [33, 512, 700], 9), (3, 3, 64, [257] * 5, 1), (16, 8, 64, [400] * 40, 8),
    (64, 8, 128, [900, 77, 2000], 40), (32, 8, 128, [150] * 120, 6), (32, 8, 64, [1000] * 90, 33)])
@pytest.mark.parametrize("how", ["full", "ragged", "unordered"])
def test_attention_over_the_listed_pages(hq, hkv, d, ctx, width, how, impl):
    rng = np.random.default_rng(hq + d + width)
    pages, tables = _state(rng, hkv, d, ctx, extra=2)
    q, scale = randn_bits(rng, len(ctx), hq, d), float(np.float32(d ** -0.5))
    lists, counts = _lists(rng, ctx, hkv, width, how)
    _close(_run(pages, q, tables, ctx, lists, counts, scale), pages, q, tables, ctx, lists, counts, scale)
    assert pages.status() == 0


@pytest.mark.parametrize("hq,hkv,d,ctx", [(32, 8, 128, [517]), (32, 8, 64, [1300, 2000, 64]), (8, 2, 128, [200] * 50), (16, 8, 64, [90] * 100)])
def test_all_pages_are_the_same_bits_as_attn_decode(hq, hkv, d, ctx, impl):
    rng = np.random.default_rng(1)
    pages, tables = _state(rng, hkv, d, ctx)
    q, width = randn_bits(rng, len(ctx), hq, d), tables.shape[1]
    lists = np.broadcast_to(np.arange(width), (len(ctx), hkv, width))
    counts = np.broadcast_to(-(-np.array(ctx) // 16)[:, None], (len(ctx), hkv))
    out, lse = torch.empty(len(ctx), hq, d, dtype=torch.bfloat16, device="cuda"), torch.empty(len(ctx), hq, device="cuda")
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    kvattn.attn_decode(pages.pool, to_gpu(q), i32(tables), i32(ctx), max(ctx), 0.1, out, lse, ws)
    got = _run(pages, q, tables, ctx, lists, counts, 0.1)
    assert np.array_equal(got[0], orc.widen(from_gpu(out))) and np.array_equal(got[1], lse.cpu().numpy().astype(np.float64))


def test_lists_that_do_not_fit_the_sequence_are_recorded(impl):
    rng = np.random.default_rng(2)
    ctx, hq, hkv, d = [100, 250, 80, 33], 8, 2, 64
    pages, tables = _state(rng, hkv, d, ctx)
    q = randn_bits(rng, 4, hq, d)
    lists, counts = _lists(rng, ctx, hkv, 6, "full")
    scale = 0.125
    assert pages.status() == 0
    odd = lists.copy()
    odd[0, 0, 1], odd[1, 1, 3], odd[2, 0, 0] = 7, -1, 0x7fffffff                # blocks that the sequence has not got are passed over
    _close(_run(pages, q, tables, ctx, odd, counts, scale), pages, q, tables, ctx, odd, counts, scale)
    assert pages.status() == kvattn.KV_ERR_BOUNDS
    wrong = counts.copy()
    wrong[1, 0], wrong[3, 1] = 7, -1
    o, l = _run(pages, q, tables, ctx, lists, wrong, scale)
    assert pages.status() == kvattn.KV_ERR_BOUNDS
    left = np.zeros((4, hq), bool)
    left[1, :4] = left[3, 4:] = True
    assert np.all(o[left] == -7) and np.all(l[left] == -7) and not np.any(o[~left] == -7)
    o, l = _run(pages, q, tables, ctx, lists, counts, scale, max_ctx=64)        # bounds are looked at in steps of 1024 tokens
    assert pages.status() == 0
    lists[0, 0, 0], tables[0, 0] = 0, pages.n                                   # a page outside the pool, in the table
    _run(pages, q, tables, ctx, lists, counts, scale)
    assert pages.status() == kvattn.KV_ERR_BOUNDS


def test_slots_behind_the_context_and_unlisted_pages_are_hidden(impl):
    rng = np.random.default_rng(6)
    ctx, hq, hkv, d = [1, 9, 24, 55], 4, 2, 128
    pages, tables = _state(rng, hkv, d, ctx)                                    # (slots behind the end are not numbers)
    for i, c in enumerate(ctx):
        if c > 32:
            pages.host.k[tables[i, 1]] = pages.host.v[tables[i, 1]] = 0x7FC0    # an unlisted page of such values
    pages.upload()
    q, lists, counts = randn_bits(rng, 4, hq, d), np.full((4, 2, 3), -1), np.ones((4, 2), np.int64)
    lists[:, :, 0] = (-(-np.array(ctx) // 16) - 1)[:, None]                     # the newest page alone
    _close(_run(pages, q, tables, ctx, lists, counts, 0.3), pages, q, tables, ctx, lists, counts, 0.3)
    assert pages.status() == 0


def test_refusals():
    pages, lib = Pages(3, 2, 64), kvattn.lib()
    t = torch.zeros(8192, dtype=torch.bfloat16, device="cuda")
    p = lambda off=0: C.c_void_p(t.data_ptr() + off)
    good = dict(pool=pages.pool.handle, q=p(), hq=4, bt=p(), width=2, ctx=p(), batch=1, mc=32, lists=p(), counts=p(), n=2, scale=1.0, out=p(8192), lse=p(12000))
    call = lambda **kw: lib.attn_decode_selected(*{**good, **kw}.values(), None)
    inv, uns = kvattn.KV_ERR_INVALID, kvattn.KV_ERR_UNSUPPORTED
    n0 = kvattn.kvattn_launch_count()
    for kw in (dict(pool=None), dict(q=None), dict(bt=None), dict(ctx=None), dict(lists=None), dict(counts=None), dict(out=None), dict(lse=None), dict(batch=-1),
               dict(width=-1), dict(mc=-1), dict(mc=33), dict(n=0), dict(q=p(8)), dict(out=p(8194))):
        assert call(**kw) == inv, kw
    for kw in (dict(hq=3), dict(hq=0), dict(hq=32)):
        assert call(**kw) == uns, kw
    assert call(batch=0) == 0 and kvattn.kvattn_launch_count() == n0
    assert call() == 0 and call(mc=0) == 0
    q = torch.zeros(1, 4, 64, dtype=torch.bfloat16, device="cuda")
    ok = [q, i32([[0, 1]]), i32([20]), 32, i32(np.zeros((1, 2, 2))), i32([[2, 2]]), 1.0, q.clone(), torch.zeros(1, 4, device="cuda")]
    for i, bad in ((0, q[0]), (1, i32([[0, 1]] * 2)), (2, i32([1, 2])), (4, i32(np.zeros((1, 3, 2)))), (5, i32([0])), (7, q[:, :2]), (8, torch.zeros(3, device="cuda"))):
        with pytest.raises((ValueError, AssertionError)):
            kvattn.attn_decode_selected(pages.pool, *[bad if j == i else x for j, x in enumerate(ok)])
    torch.cuda.synchronize()
    assert pages.status() == 0
