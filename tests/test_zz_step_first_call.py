"""The calls around attention may be captured into a graph before they have run: in a process of its own each is captured as its first call.

(attn_decode_selected prepares as attn_decode does: one call of either beforehand.)"""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

_SCRIPT = """
import torch
from paper_2607_23815_b200 import kvattn
i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
ok = []
for d, hq, hkv, batch, width in ((128, 8, 2, 2, 8), (64, 8, 8, 60, 8), (64, 4, 4, 2, 300)):
    k, v = (torch.randn(batch * width, hkv, 16, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    pool = kvattn.kv_pool_create_ex(batch * width, 16, hkv, d, k, v)
    free, bt = torch.arange(batch * width, dtype=torch.int32, device="cuda"), i32(batch, width)
    n = width * 16 - 3
    lens, new, cu, pos, slots = i32(batch), torch.full((batch,), n, dtype=torch.int32, device="cuda"), i32(batch + 1), i32(batch * n), i32(batch * n)
    nxt = i32(batch)
    q, kv = torch.randn(batch * n, hq, d, dtype=torch.bfloat16, device="cuda"), torch.randn(batch * n, hkv, d, dtype=torch.bfloat16, device="cuda")
    qo, inv, bounds = torch.zeros_like(q), torch.rand(d // 2, device="cuda"), torch.zeros(batch * width, hkv, 2, d, dtype=torch.bfloat16, device="cuda")
    lists, counts = i32(batch, hkv, 4), i32(batch, hkv)
    out, lse, qd = torch.zeros(batch, hq, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(batch, hq, device="cuda"), q[:batch].contiguous()
    kvattn.attn_decode_static(pool, qd, bt, lens, n, 0.1, out, lse)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        kvattn.kv_step_tables(pool, lens, new, free, bt, cu, pos, slots, nxt)
        kvattn.kv_append_rotary(pool, q, kv, kv, slots, pos, inv, None, qo)
        kvattn.kv_page_bounds(pool, slots, bounds)
        kvattn.attn_select_pages(pool, qd, bounds, bt, nxt, n, 1, 1, lists, counts)
        kvattn.attn_decode_selected(pool, qd, bt, nxt, n, lists, counts, 0.1, out, lse)
    g.replay()
    torch.cuda.synchronize()
    assert counts.unique().tolist() == [4] and kvattn.kv_last_async_status(pool) == 0 and bool(torch.isfinite(lse).all()) and float(qo.float().norm()) > 0
    first = [x.clone() for x in (lists, out, lse, qo, bounds)]
    kvattn.kv_page_bounds(pool, slots, bounds)
    kvattn.attn_select_pages(pool, qd, bounds, bt, nxt, n, 1, 1, lists, counts)
    kvattn.attn_decode_selected(pool, qd, bt, nxt, n, lists, counts, 0.1, out, lse)
    assert all(torch.equal(a, b) for a, b in zip(first, (lists, out, lse, qo, bounds)))
print("done")
"""


def test_the_first_call_may_be_a_captured_one():
    r = subprocess.run([sys.executable, "-c", _SCRIPT], capture_output=True, text=True, cwd=ROOT, timeout=600, env=dict(os.environ, CUDA_MODULE_LOADING="LAZY"))
    assert r.returncode == 0 and "done" in r.stdout, (r.stdout, r.stderr[-3000:])
