"""The scheduler's executor with decode over chosen pages: with room for all of them, the results of decode over the whole context, bit for bit, step by
step; with less, finite results of as many pages as it was given, over pages that come and go."""
import pytest
import torch

from paper_2607_23815_b200 import kvattn, synth
from paper_2607_23815_b200.scheduler import LibraryEngine, LibraryExecutor, Scheduler, StageSpec

pytestmark = pytest.mark.gpu

PLAN = [StageSpec("sem_filter", (300, 700), (1, 1), 8, 0.7, 3), StageSpec("join + sem_map", (20, 50), (3, 9), 16, 1.0, 1)]


class _Kept(LibraryExecutor):
    def __init__(self, *a, **k):
        super().__init__(*a, **k)
        self.outs, self.seen = [], []

    def decode(self, tasks):
        super().decode(tasks)
        self.outs.append(self.last_out)
        if self.bounds is not None:
            ctx = torch.tensor([t.reuse_tokens + t.extend_tokens + t.generated for t in tasks], device="cuda")
            self.seen.append(((ctx + 15) // 16, self.last_counts))


def _run(pages, pinning, policy, decode_pages):
    geom = synth.Geometry(8, 2, 128)
    pool = kvattn.kv_pool_create(pages, 16, geom.n_kv_heads, geom.head_dim)
    ex = _Kept(pool, geom, seed=5, decode_pages=decode_pages)
    Scheduler(PLAN, 12, LibraryEngine(pool), pinning=pinning, policy=policy, seed=5, executor=ex, tokens_per_tick=4096).run()
    torch.cuda.synchronize()
    assert kvattn.kv_last_async_status(pool) == kvattn.KV_OK and ex.calls["decode"] > 0
    pool.destroy()
    return ex


@pytest.mark.parametrize("pinning,policy,pages", [("explicit", "memory_aware", 800), ("virtual", "breadth_first", 400)])
def test_decode_over_chosen_pages(pinning, policy, pages):
    whole, every, few = (_run(pages, pinning, policy, n) for n in (None, 100000, 6))
    assert len(whole.outs) == len(every.outs) == len(few.outs)
    assert all(torch.equal(a, b) for a, b in zip(whole.outs, every.outs))
    assert all(bool((c == n[:, None]).all()) for n, c in every.seen)
    assert all(bool((c == n.clamp(max=6)[:, None]).all()) for n, c in few.seen) and max(int(n.max()) for n, _ in few.seen) > 6
    assert all(bool(torch.isfinite(o.float()).all()) for o in few.outs) and not all(torch.equal(a, b) for a, b in zip(whole.outs, few.outs))


def test_too_few_pages_are_refused():
    pool = kvattn.kv_pool_create(4, 16, 2, 128)
    with pytest.raises(ValueError):
        LibraryExecutor(pool, synth.Geometry(8, 2, 128), decode_pages=1)
