"""Decode over block tables of more than 2^27 entries a row, whose tokens pass 31 bits: lengths up to 2^31 - 1 are served, the last block among the listed.

Tolerance: as for attn_decode_selected elsewhere, 2^-8 for the rounding of O, 2^-8 for that of the weights, 2^-15 for sums and exponentials in 32 bits."""
import numpy as np
import pytest
import torch

from oracle import paged_attention as orc
from oracle import paged_step as step
from paper_2607_23815_b200 import kvattn
from step_harness import Pages, from_gpu, guarded, i32, randn_bits, to_gpu

pytestmark = pytest.mark.gpu

WIDTH = (1 << 27) + 2                                                         # 0.5 GB


@pytest.fixture(params=[0, 1, 2])
def impl(request):
    kvattn.kvattn_set_decode_impl(request.param)
    yield request.param
    kvattn.kvattn_set_decode_impl(0)


@pytest.fixture(scope="module")
def table():
    return torch.full((1, WIDTH), -1, dtype=torch.int32, device="cuda")


def _selected(pages, q, bt, ctx, lists, max_ctx):
    _, hq, d = q.shape
    (out, c1), (lse, c2) = guarded((1, hq, d), torch.bfloat16, -7.0), guarded((1, hq), torch.float32, -7.0)
    counts = torch.full((1, pages.heads), len(lists), dtype=torch.int32, device="cuda")
    kvattn.attn_decode_selected(pages.pool, to_gpu(q), bt, i32([ctx]), max_ctx, i32(np.broadcast_to(lists, (1, pages.heads, len(lists)))), counts, 0.125, out, lse)
    torch.cuda.synchronize()
    assert c1() and c2()
    return out, lse


def _pages(rng, hkv, d):
    pages = Pages(4, hkv, d)
    pages.host.k[:], pages.host.v[:] = randn_bits(rng, 2, 4, hkv, 16, d)
    return pages


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (8, 2, 64), (500, 500, 64)])
def test_a_short_sequence_of_a_wide_table(hq, hkv, d, table, impl):
    rng = np.random.default_rng(d)
    pages, ctx = _pages(rng, hkv, d), 40
    pages.upload()
    q = randn_bits(rng, 1, hq, d)
    table[0, :3] = i32([2, 0, 3])
    near = table[:, :3].contiguous()
    got, want = (_selected(pages, q, bt, ctx, [2, 0], ctx) for bt in (table, near))
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and float(want[0].float().norm()) > 0
    got, want = ([torch.full((1, hq, d), -7.0, dtype=torch.bfloat16, device="cuda"), torch.full((1, hq), -7.0, device="cuda")] for _ in range(2))
    for bt, (o, l) in ((table, got), (near, want)):
        kvattn.attn_decode(pages.pool, to_gpu(q), bt, i32([ctx]), ctx, 0.125, o, l, None)
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and pages.status() == 0


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (8, 2, 64), (500, 500, 64)])
@pytest.mark.parametrize("ctx", [0x7fffffff, 0x7ffffff1, 0x7ffffff0])
def test_the_longest_sequences(hq, hkv, d, ctx, table, impl):
    rng = np.random.default_rng(ctx & 15)
    pages, last = _pages(rng, hkv, d), (ctx - 1) // 16
    for slots in (pages.host.k, pages.host.v):                                 # what lies behind the last token is no number
        slots[1, :, (ctx - 1) % 16 + 1:] = 0x7FC0
    pages.upload()
    q, ids = randn_bits(rng, 1, hq, d), {0: 2, 5: 0, last: 1}
    for block, page in ids.items():
        table[0, block] = page
    for lists, status in (([last], 0), ([last, 5, 0], 0), ([0, -1, last, 1 << 27, 5, last + 1, 0x7fffffff], kvattn.KV_ERR_BOUNDS)):
        got = _selected(pages, q, table, ctx, lists, 0x7fffffff)
        assert pages.status() == status
        all_lists, counts = np.broadcast_to(lists, (1, hkv, len(lists))), np.full((1, hkv), len(lists))
        o, l = step.decode_selected(pages.host, q, hq, [ids], [ctx], all_lists, counts, 0.125)
        v, pages.host.v = pages.host.v, pages.host.v & 0x7FFF
        reach = step.decode_selected(pages.host, q, hq, [ids], [ctx], all_lists, counts, 0.125)[0]
        pages.host.v = v
        assert np.all(np.abs(orc.widen(from_gpu(got[0])) - o) <= 2.0 ** -8 * (np.abs(o) + reach) + 2.0 ** -15 * reach)
        assert np.all(np.abs(got[1].cpu().numpy() - l) <= 1e-4)
    table[0, list(ids)] = -1
