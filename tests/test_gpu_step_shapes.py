"""Rows of another size than the pool's are refused by the calls around attention before anything is launched: the kernels go by the pool's head_dim alone."""
import pytest
import torch

from paper_2607_23815_b200 import kvattn
from step_harness import Pages, i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,other", [(128, 64), (64, 128), (128, 127), (64, 1), (128, 0)])
def test_queries_of_another_head_size_are_refused(d, other):
    pages = Pages(3, 2, d)
    bounds, lists, counts = torch.zeros(3, 2, 2, d, dtype=torch.bfloat16, device="cuda"), i32([[[0, 1]] * 2]), i32([[2, 2]])
    rows = lambda x: torch.zeros(1, 4, x, dtype=torch.bfloat16, device="cuda")
    bt, ctx, lse = i32([[0, 1]]), i32([20]), torch.zeros(1, 4, device="cuda")
    n0 = kvattn.kvattn_launch_count()
    with pytest.raises(ValueError, match="head_dim"):
        kvattn.attn_select_pages(pages.pool, rows(other), bounds, bt, ctx, 32, 0, 0, lists, counts)
    with pytest.raises(ValueError, match="head_dim"):
        kvattn.attn_decode_selected(pages.pool, rows(other), bt, ctx, 32, lists, counts, 1.0, rows(other), lse)
    assert kvattn.kvattn_launch_count() == n0
    kvattn.attn_select_pages(pages.pool, rows(d), bounds, bt, ctx, 32, 0, 0, lists, counts)
    kvattn.attn_decode_selected(pages.pool, rows(d), bt, ctx, 32, lists, counts, 1.0, rows(d), lse)
    torch.cuda.synchronize()
    assert pages.status() == 0
