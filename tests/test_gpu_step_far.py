"""The calls around attention where byte and element offsets pass 32 bits, and on tensors that are not on the current device."""
import numpy as np
import pytest
import torch

from oracle import paged_attention as orc
from oracle import paged_step as step
from paper_2607_23815_b200 import kvattn
from step_harness import from_gpu, i32, randn_bits, to_gpu

pytestmark = pytest.mark.gpu

_GB = 1 << 30


def _room(gb):
    if torch.cuda.mem_get_info()[0] < gb * _GB:
        pytest.skip("not enough free device memory")


def test_pages_whose_bytes_and_bounds_lie_beyond_32_bits():
    _room(60)
    H, D, N = 8, 128, (1 << 20) + 4096                            # 34 GB of pages, 4.3 GB of bounds
    buf = torch.empty((N, H, 16 * D), dtype=torch.bfloat16, device="cuda")     # keys and values share them here: their rows are the same
    bounds = torch.empty((N, H, 2, D), dtype=torch.bfloat16, device="cuda")
    pool = kvattn.kv_pool_create_ex(N, 16, H, D, buf, buf)
    assert kvattn.kv_page_bounds_bytes(pool) == bounds.nbytes > 1 << 32
    rng = np.random.default_rng(0)
    far = [N - 1, 3, N - 4000, (1 << 20) + 1, 1 << 19, N // 3, 0, N - 2, (1 << 20) - 1, 77]
    T, hq = 16 * len(far) - 5, 32
    rows, q = randn_bits(rng, T, H, D), randn_bits(rng, T, hq, D)
    z = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    bt, cu, pos, slots, nxt, qo = z(1, len(far)), z(2), z(T), z(T), z(1), torch.empty(T, hq, D, dtype=torch.bfloat16, device="cuda")
    kvattn.kv_step_tables(pool, z(1), i32([T]), i32(far), bt, cu, pos, slots, nxt)
    assert bt.tolist() == [far] and slots.tolist() == [far[t // 16] * 16 + t % 16 for t in range(T)]
    kvattn.kv_append_rotary(pool, to_gpu(q), to_gpu(rows), to_gpu(rows), slots, pos * 0, torch.ones(D // 2, device="cuda"), None, qo)
    assert np.array_equal(from_gpu(qo), q)
    kvattn.kv_page_bounds(pool, slots, bounds)
    host = orc.PagePool(len(far), 16, H, D)                      # the same pages, numbered 0, 1, ...
    host.append(list(range(len(far))), 0, rows, rows)
    near = step.page_bounds(host, np.arange(T), np.zeros((len(far), H, 2, D)))
    assert np.array_equal(orc.widen(from_gpu(bounds[far])), near)
    qd, lists, counts, tables = q[-1:], z(1, H, 4), z(1, H), [list(range(len(far)))]
    out, lse = torch.empty(1, hq, D, dtype=torch.bfloat16, device="cuda"), torch.empty(1, hq, device="cuda")
    kvattn.attn_select_pages(pool, to_gpu(qd), bounds, bt, nxt, T, 1, 1, lists, counts)
    kvattn.attn_decode_selected(pool, to_gpu(qd), bt, nxt, T, lists, counts, 0.088, out, lse)
    want, wc = step.select_pages(qd, near, tables, [T], H, 4, 1, 1)
    assert np.array_equal(lists.cpu().numpy(), want) and np.array_equal(counts.cpu().numpy(), wc) and kvattn.kv_last_async_status(pool) == 0
    o, l = step.decode_selected(host, qd, hq, tables, [T], want, wc, np.float32(0.088))
    host.v = host.v & 0x7FFF
    reach = step.decode_selected(host, qd, hq, tables, [T], want, wc, np.float32(0.088))[0]
    assert np.all(np.abs(orc.widen(from_gpu(out)) - o) <= 2.0 ** -8 * (np.abs(o) + reach) + 2.0 ** -15 * reach)
    assert np.all(np.abs(lse.cpu().numpy() - l) <= 1e-4)
    pool.destroy()


def test_rows_that_lie_more_than_32_bits_apart():
    _room(20)
    D, hq, T, stride = 64, 2, 18, 1 << 27                         # 4.8 GB from the first token to the last
    whole = torch.empty(stride * (T - 1) + 4 * hq * D, dtype=torch.bfloat16, device="cuda")
    part = lambda at: whole.as_strided((T, hq, D), (stride, D, 1), at)
    q, out, k, v = (part(i * hq * D) for i in range(4))
    rng = np.random.default_rng(1)
    rows = [randn_bits(rng, T, hq, D) for _ in range(3)]
    for x, r in zip((q, k, v), rows):
        x.copy_(to_gpu(r))
    pages = [torch.zeros(2, hq, 16 * D, dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    near = torch.empty(T, hq, D, dtype=torch.bfloat16, device="cuda")
    pos, inv = i32(np.arange(T) + 99), torch.rand(D // 2, device="cuda")
    for (kb, vb), args in ((pages[:2], (q, k, v, out)), (pages[2:], (*map(to_gpu, rows), near))):
        pool = kvattn.kv_pool_create_ex(2, 16, hq, D, kb, vb)
        kvattn.kv_append_rotary(pool, *args[:3], i32(np.arange(T)), pos, inv, None, args[3])
        assert kvattn.kv_last_async_status(pool) == 0
    assert torch.equal(out, near) and torch.equal(pages[0], pages[2]) and torch.equal(pages[1], pages[3]) and float(near.float().norm()) > 0


@pytest.mark.skipif(torch.cuda.device_count() < 2, reason="needs a second device")
def test_tensors_on_another_device_are_refused():
    pool = kvattn.kv_pool_create(2, 16, 2, 64)
    there, i = torch.zeros(1, 2, 64, dtype=torch.bfloat16, device="cuda:1"), torch.zeros(1, dtype=torch.int32, device="cuda:1")
    here, n = torch.zeros(1, 2, 64, dtype=torch.bfloat16, device="cuda"), i32([0])
    n0 = kvattn.kvattn_launch_count()
    for call in (lambda: kvattn.kv_append_rotary(pool, there, None, None, None, n, torch.zeros(32, device="cuda"), None, here),
                 lambda: kvattn.kv_append_rotary(pool, here, None, None, None, i, torch.zeros(32, device="cuda"), None, here),
                 lambda: kvattn.kv_page_bounds(pool, i, here),
                 lambda: kvattn.kv_step_tables(pool, i, n, n, n.view(1, 1), i32([0, 0]), n, n)):
        with pytest.raises(ValueError, match="another device"):
            call()
    assert kvattn.kvattn_launch_count() == n0
