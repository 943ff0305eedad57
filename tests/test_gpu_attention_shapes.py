"""Rows of another size than the pool's, and results smaller than their queries, are refused by the attention calls before anything is launched: the kernels go by
the pool's head_dim alone, and would read and write past the ends of such tensors."""
import pytest
import torch

from paper_2607_23815_b200 import kvattn
from step_harness import Pages, i32

pytestmark = pytest.mark.gpu


def _calls(pool, dev="cuda"):
    ws, bt, one, cu = torch.empty(1 << 22, dtype=torch.uint8, device="cuda"), i32([[0, 1]]), i32([4]), i32([0, 4])
    staging = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    h = lambda x: x.cpu()
    return {
        "decode": lambda q, k, v, o, l: kvattn.attn_decode(pool, q[:1], bt, i32([20]), 32, 1.0, o[:1], l[:1], ws),
        "static": lambda q, k, v, o, l: kvattn.attn_decode_static(pool, q[:1], bt, i32([20]), 32, 1.0, o[:1], l[:1]),
        "extend": lambda q, k, v, o, l: kvattn.attn_extend(pool, q, cu, bt, i32([16]), one, 4, 20, 1.0, o, l, ws),
        "planned": lambda q, k, v, o, l: (kvattn.attn_extend_plan(pool, q.shape[1], cu, bt, i32([16]), one, 4, 4, 20, ws),
                                          kvattn.attn_extend_planned(pool, q, cu, bt, i32([16]), one, 4, 20, 1.0, o, l, ws)),
        "append": lambda q, k, v, o, l: kvattn.kv_append(pool, k, v, cu, i32([16]), None, bt),
        "extend_append": lambda q, k, v, o, l: kvattn.attn_extend_append(pool, q, k, v, cu, bt, i32([16]), one, 4, 20, 1.0, o, l, ws),
        "host": lambda q, k, v, o, l: kvattn.attn_extend_host(pool, h(q), h(k), h(v), h(cu), h(bt), torch.tensor([16], dtype=torch.int32), h(one), 4, 20, 1.0, h(o),
                                                              h(l), staging),
    }


NEEDS = {"decode": "qol", "static": "qol", "extend": "qol", "planned": "qol", "append": "kv", "extend_append": "qkvol", "host": "qkvol"}


@pytest.mark.parametrize("name", sorted(NEEDS))
@pytest.mark.parametrize("d,other", [(128, 64), (64, 128), (64, 63)])
def test_rows_and_results_that_do_not_fit(name, d, other):
    pages = Pages(2, 2, d, fill=0)
    rows = lambda heads, x=d: torch.zeros(4, heads, x, dtype=torch.bfloat16, device="cuda")
    call, good = _calls(pages.pool)[name], dict(q=rows(4), k=rows(2), v=rows(2), o=rows(4), l=torch.zeros(4, 4, device="cuda"))
    assert kvattn.kv_last_async_status(pages.pool) == 0
    bad = []
    if "q" in NEEDS[name]:
        bad += [dict(q=rows(4, other), o=rows(4, other)), dict(q=rows(4, other)), dict(o=rows(4)[:, :3]), dict(o=rows(3)), dict(l=good["l"][:, :3].contiguous())]
    if "k" in NEEDS[name]:
        bad += [dict(k=rows(2, other), v=rows(2, other)), dict(k=rows(2, other)), dict(v=rows(1)), dict(v=rows(2)[:3])]
    plans = 1 if name == "planned" else 0                                       # (the plan, which takes no rows)
    for change in bad:
        n0 = kvattn.kvattn_launch_count()
        with pytest.raises((ValueError, AssertionError)):
            call(*{**good, **{key: x.contiguous() for key, x in change.items()}}.values())
        assert kvattn.kvattn_launch_count() - n0 <= plans, change
    call(*good.values())
    larger = dict(o=torch.zeros(6, 4, d, dtype=torch.bfloat16, device="cuda"), l=torch.zeros(6, 4, device="cuda"))   # buffers of a larger step
    call(*{**good, **larger}.values())
    torch.cuda.synchronize()
    assert kvattn.kv_last_async_status(pages.pool) == 0


def test_fan_out():
    pages = Pages(4, 2, 128, fill=0)
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    def call(q, o, l):
        kvattn.attn_extend_shared(pages.pool, q, i32([0, 2, 4]), i32([0, 2]), i32([[0, 1]]), i32([20]), i32([[2], [3]]), i32([2, 2]), 2, 4, 20, 1.0, o, l, ws)
    rows = lambda heads, x=128, n=4: torch.zeros(n, heads, x, dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros(4, 4, device="cuda")
    n0 = kvattn.kvattn_launch_count()
    for bad in ((rows(4, 64), rows(4, 64), lse), (rows(4, 64), rows(4), lse), (rows(4), rows(3), lse), (rows(4), rows(4), lse[:3])):
        with pytest.raises(ValueError):
            call(*bad)
    assert kvattn.kvattn_launch_count() == n0
    call(rows(4), rows(4), lse)
    torch.cuda.synchronize()
    assert kvattn.kv_last_async_status(pages.pool) == 0
