"""New keys and values of other heads than the pool's, or fewer than the queries' tokens, are refused before anything is launched: the kernels read as many as the pool has."""
import pytest
import torch

from paper_2607_23815_b200 import kvattn
from step_harness import Pages, i32
from test_gpu_attention_shapes import _calls

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["append", "extend_append", "host"])
@pytest.mark.parametrize("d", [64, 128])
def test_new_rows_that_do_not_fit(name, d):
    pages = Pages(2, 2, d, fill=0)
    rows = lambda heads, n=4: torch.zeros(n, heads, d, dtype=torch.bfloat16, device="cuda")
    call, good = _calls(pages.pool)[name], dict(q=rows(4), k=rows(2), v=rows(2), o=rows(4), l=torch.zeros(4, 4, device="cuda"))
    bad = [dict(k=rows(n), v=rows(n)) for n in (1, 3, 4, 0)]
    if name != "append":                                                        # (which takes the number of rows from k_new)
        bad.append(dict(k=rows(2, 3), v=rows(2, 3)))
    n0 = kvattn.kvattn_launch_count()
    for change in bad:
        with pytest.raises(ValueError, match="k_new"):
            call(*{**good, **change}.values())
    assert kvattn.kvattn_launch_count() == n0
    call(*good.values())
    torch.cuda.synchronize()
    assert pages.status() == 0
