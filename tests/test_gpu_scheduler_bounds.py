"""The bounds that the scheduler's executor keeps: at every decode step those of the pages its tasks attend over are what their keys give, pages that were
freed, evicted and handed out again among them, and the chosen pages are the ones that these bounds make the best."""
import numpy as np
import pytest
import torch

from oracle import paged_attention as orc
from oracle import paged_step as step
from paper_2607_23815_b200 import kvattn, synth
from paper_2607_23815_b200.scheduler import LibraryEngine, LibraryExecutor, Scheduler, StageSpec
from step_harness import from_gpu, _places

pytestmark = pytest.mark.gpu

PLAN = [StageSpec("sem_filter", (300, 700), (1, 1), 8, 0.7, 3), StageSpec("join + sem_map", (20, 50), (3, 9), 16, 1.0, 1)]


class _Checked(LibraryExecutor):
    def __init__(self, pool, geom, keys, **more):
        super().__init__(pool, geom, **more)
        self.bounds.fill_(float("nan"))                                       # (what no append has renewed is no bound)
        self.keys, self.first_owner, self.again, self.choices = keys, {}, 0, 0
        self.calls_seen = 0

    def decode(self, tasks):
        seen = {}
        whole = self.kv.attn_select_pages

        def select(pool, q, bounds, bt, ctx, max_ctx, first, last, pages, counts):
            whole(pool, q, bounds, bt, ctx, max_ctx, first, last, pages, counts)
            seen.update(q=q, bounds=bounds, bt=bt, ctx=ctx, first=first, last=last, pages=pages, counts=counts)

        self.kv = type("Seen", (), {**{n: staticmethod(getattr(kvattn, n)) for n in ("kv_append", "kv_page_bounds", "attn_decode_selected")},
                                    "attn_select_pages": staticmethod(select)})
        try:
            super().decode(tasks)
        finally:
            self.kv = kvattn
        self._check(tasks, **seen)

    def _check(self, tasks, q, bounds, bt, ctx, first, last, pages, counts):
        g = self.geom
        tables, lens = bt.cpu().numpy(), ctx.cpu().numpy()
        assert bounds.data_ptr() == self.bounds.data_ptr()
        kept = orc.widen(from_gpu(bounds)).reshape(-1, g.n_kv_heads, 2, g.head_dim)
        place = _places(g.head_dim).reshape(-1)
        ids = np.unique(np.concatenate([row[:-(-int(n) // 16)] for row, n in zip(tables, lens)]))
        raw = orc.widen(self.keys[torch.as_tensor(ids, device="cuda").long()].view(torch.int16).cpu().numpy().view(np.uint16))
        image = raw.reshape(len(ids), g.n_kv_heads, -1)[:, :, place].reshape(len(ids), g.n_kv_heads, 16, g.head_dim)
        for task, row, n in zip(tasks, tables, lens):
            for b in range(-(-int(n) // 16)):
                page, held = int(row[b]), min(16, int(n) - 16 * b)
                k = image[np.searchsorted(ids, page), :, :held]
                assert np.array_equal(kept[page, :, 0], k.min(1)) and np.array_equal(kept[page, :, 1], k.max(1)), (task.uid, b, page)
                if b * 16 >= task.reuse_tokens:                               # a page of its own
                    self.again += self.first_owner.setdefault(page, task.uid) != task.uid
        if self.calls_seen % 7 == 0:
            want, wcounts = step.select_pages(from_gpu(q), kept, tables, lens, g.n_kv_heads, pages.shape[2], first, last)
            assert np.array_equal(pages.cpu().numpy(), want) and np.array_equal(counts.cpu().numpy(), wcounts)
            self.choices += int((wcounts < -(-lens // 16)[:, None]).sum())
        self.calls_seen += 1


@pytest.mark.parametrize("pinning,policy,pages", [("explicit", "memory_aware", 800), ("virtual", "breadth_first", 400)])
@pytest.mark.parametrize("head_dim", [64, 128])
def test_bounds_are_those_of_the_keys(pinning, policy, pages, head_dim):
    geom = synth.Geometry(8, 2, head_dim)
    k, v = (torch.empty(pages, 2, 16 * head_dim, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    pool = kvattn.kv_pool_create_ex(pages, 16, 2, head_dim, k, v)
    ex = _Checked(pool, geom, k, seed=5, decode_pages=6)
    Scheduler(PLAN, 12, LibraryEngine(pool), pinning=pinning, policy=policy, seed=5, executor=ex, tokens_per_tick=4096).run()
    assert kvattn.kv_last_async_status(pool) == kvattn.KV_OK
    assert ex.calls_seen == ex.calls["decode"] > 7 and ex.choices > 0
    assert ex.again > 0, "no page was handed out again"
    pool.destroy()
