"""kv_step_tables at the longest lengths: the page of a sequence's last tokens is the one it has, and none is taken from the list for them."""
import pytest
import torch

from paper_2607_23815_b200 import kvattn
from step_harness import Pages, i32

pytestmark = pytest.mark.gpu


def test_tokens_of_the_last_page_there_is():
    width = 1 << 27                                                           # 2^31 tokens, one more than a length holds
    pages, bt = Pages(4, 1, 64), torch.full((1, width), -1, dtype=torch.int32, device="cuda")
    for ctx, new in ((0x7ffffff1, 14), (0x7ffffff2, 13), (0x7ffffffe, 1), (0x7ffffff0, 15), (0x7fffffef, 16), (0x7fffffdf, 18)):
        owned, end = (ctx + 15) // 16, (ctx + new + 15) // 16
        held = {b: page for b, page in zip(range(width - 3, width), (1, 3, 1)) if b < owned}
        for b in range(width - 3, width):
            bt[0, b] = held.get(b, -1)
        z = lambda n: i32([-9] * n)
        cu, pos, slots, nxt, cur = z(2), z(new), z(new), z(1), z(1)
        kvattn.kv_step_tables(pages.pool, i32([ctx]), i32([new]), i32([0, 2]), bt, cu, pos, slots, nxt, None, cur)
        held.update(zip(range(owned, end), (0, 2)))
        assert pages.status() == 0 and slots.tolist() == [held[p // 16] * 16 + p % 16 for p in range(ctx, ctx + new)]
        assert pos.tolist() == list(range(ctx, ctx + new)) and cu.tolist() == [0, new]
        assert int(cur) == end - owned and int(nxt) == ctx + new and bt[0, -3:].tolist() == [held.get(b, -1) for b in range(width - 3, width)]
