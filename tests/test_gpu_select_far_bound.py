"""The page choice with a bound far above the lengths, as a captured step passes it for its whole life: the same lists, whatever the bound makes of the launch."""
import numpy as np
import pytest
import torch

from oracle import paged_step as step
from paper_2607_23815_b200 import kvattn
from step_harness import guarded, i32, to_gpu
from test_gpu_select_pages import Pages, _bits, _case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,hkv,d,ctx", [
    (32, 8, 128, [700]), (4, 2, 64, [0, 15, 1000, 333]), (64, 8, 128, [2900, 3200, 40, 900, 1600]), (32, 8, 64, [200 + 37 * i for i in range(30)]),
    (16, 8, 64, [17 + 29 * i for i in range(90)]), (32, 8, 128, [512 + 11 * i for i in range(120)])])
@pytest.mark.parametrize("times", [1, 4, 16, 0])
def test_lists_do_not_depend_on_the_bound(hq, hkv, d, ctx, times):
    rng = np.random.default_rng(len(ctx))
    q, bounds, tables, count = _case(rng, hq, hkv, d, ctx)
    most = 24576 * 16                                                          # (0: the largest there is)
    max_ctx = min(most, max(ctx) * times) if times else most
    wide = np.full((len(ctx), -(-max_ctx // 16)), -1, np.int64)
    wide[:, :tables.shape[1]] = tables
    pages = Pages(count, hkv, d)
    lists, lists_ok = guarded((len(ctx), hkv, 9), torch.int32, -99)
    counts, counts_ok = guarded((len(ctx), hkv), torch.int32, -99)
    call = lambda: kvattn.attn_select_pages(pages.pool, tq, tb, tt, tc, max_ctx, 1, 2, lists, counts)
    tq, tb, tt, tc = to_gpu(q), to_gpu(_bits(bounds)), i32(wide), i32(ctx)
    call()
    want, wcounts = step.select_pages(q, bounds, tables, ctx, hkv, 9, 1, 2)
    assert np.array_equal(lists.cpu().numpy(), want) and np.array_equal(counts.cpu().numpy(), wcounts)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    lists.fill_(-99), counts.fill_(-99)
    graph.replay()
    assert np.array_equal(lists.cpu().numpy(), want) and np.array_equal(counts.cpu().numpy(), wcounts)
    assert lists_ok() and counts_ok() and pages.status() == 0


@pytest.mark.parametrize("times", [1, 4, 16])
def test_a_growing_step_replayed_under_one_bound(times):
    rng = np.random.default_rng(times)
    hq, hkv, d, n = 16, 4, 64, 40
    last = rng.integers(300, 900, n)
    q, bounds, tables, count = _case(rng, hq, hkv, d, last.tolist())
    max_ctx = 900 * times
    wide = np.full((n, -(-max_ctx // 16)), -1, np.int64)
    wide[:, :tables.shape[1]] = tables
    pages = Pages(count, hkv, d)
    lens, lists, counts = i32(np.zeros(n)), i32(np.zeros((n, hkv, 7))), i32(np.zeros((n, hkv)))
    tq, tb, tt = to_gpu(q), to_gpu(_bits(bounds)), i32(wide)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kvattn.attn_select_pages(pages.pool, tq, tb, tt, lens, max_ctx, 0, 1, lists, counts)
    for part in (0, 1, 40, 120, 500, 900):
        ctx = np.minimum(last, part)
        lens.copy_(i32(ctx))
        graph.replay()
        want, wcounts = step.select_pages(q, bounds, tables, ctx, hkv, 7, 0, 1)
        assert np.array_equal(lists.cpu().numpy(), want) and np.array_equal(counts.cpu().numpy(), wcounts)
    assert pages.status() == 0
