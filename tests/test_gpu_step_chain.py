"""The calls around attention as a step uses them: lengths to tables and slots, projected rows rotated into their pages, the pages' bounds, the choice of pages
and attention over them; prefill, then decode steps, on several streams, captured and replayed."""
import numpy as np
import pytest
import torch

from oracle import paged_attention as orc
from oracle import paged_step as step
from paper_2607_23815_b200 import kvattn
from step_harness import Pages, from_gpu, i32, randn_bits, to_gpu

pytestmark = pytest.mark.gpu


class _Run:
    """A batch that grows step by step, on the device and in the oracle."""

    def __init__(self, hq, hkv, d, ctx, steps, n_select, first, last, rows, seed, width=24):
        self.rng = np.random.default_rng(seed)
        self.hq, self.hkv, self.d, self.B, self.width = hq, hkv, d, len(ctx), width
        self.n_select, self.first, self.last = n_select, first, last
        count = self.B * width
        self.pages = Pages(count, hkv, d)
        self.free = self.rng.permutation(count).tolist()
        self.tables, self.ctx, self.cursor = np.full((self.B, width), -1, np.int64), [0] * self.B, 0
        self.max_ctx = max(ctx) + steps
        self.inv = (10000.0 ** (-np.arange(d // 2) * 2 / d)).astype(np.float32)
        self.axis = np.arange(d // 2) % 3
        z = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
        self.g = dict(lens=z(self.B), new=z(self.B), free=i32(self.free), bt=i32(self.tables), cu=z(self.B + 1), pos=z(rows), slots=z(rows), cur=z(1),
                      pos3=z(3, rows), inv=torch.from_numpy(self.inv).cuda(), axis=i32(self.axis), lists=z(self.B, hkv, n_select), counts=z(self.B, hkv),
                      qkv=torch.zeros(rows, (hq + 2 * hkv) * d, dtype=torch.bfloat16, device="cuda"),
                      q=torch.zeros(rows, hq, d, dtype=torch.bfloat16, device="cuda"),
                      bounds=torch.full((count, hkv, 2, d), float("nan"), dtype=torch.bfloat16, device="cuda"),
                      out=torch.zeros(self.B, hq, d, dtype=torch.bfloat16, device="cuda"), lse=torch.zeros(self.B, hq, device="cuda"))
        self.bounds = np.full((count, hkv, 2, d), np.nan)
        self.scale = float(np.float32(d ** -0.5))

    def rows(self, n, total):
        """New projected rows, for both sides."""
        qkv = randn_bits(self.rng, total, (self.hq + 2 * self.hkv) * self.d)
        self.g["qkv"][:total].copy_(to_gpu(qkv))
        self.g["new"].copy_(i32(n))
        return qkv

    def store(self, total, stream=None):
        g, d = self.g, self.d
        kvattn.kv_step_tables(self.pages.pool, g["lens"], g["new"], g["free"], g["bt"], g["cu"], g["pos"][:total], g["slots"][:total], g["lens"], g["cur"],
                              g["cur"], stream)
        q, k, v = (x.unflatten(1, (-1, d)) for x in g["qkv"][:total].split([self.hq * d, self.hkv * d, self.hkv * d], 1))
        g["pos3"][:, :total].copy_(g["pos"][:total].expand(3, -1))                # (text: the axes go together)
        kvattn.kv_append_rotary(self.pages.pool, q, k, v, g["slots"][:total], g["pos3"][:, :total].contiguous(), g["inv"], g["axis"], g["q"][:total], False, stream)
        kvattn.kv_page_bounds(self.pages.pool, g["slots"][:total], g["bounds"], stream)

    def attend(self, stream=None):
        g, q = self.g, self.g["q"][:self.B]
        kvattn.attn_select_pages(self.pages.pool, q, g["bounds"], g["bt"], g["lens"], self.max_ctx, self.first, self.last, g["lists"], g["counts"], stream)
        kvattn.attn_decode_selected(self.pages.pool, q, g["bt"], g["lens"], self.max_ctx, g["lists"], g["counts"], self.scale, g["out"], g["lse"], stream)

    def check_store(self, n, qkv, total):
        self.tables, cu, pos, slots, self.ctx, self.cursor, ok = step.step_tables(self.ctx, n, self.free, self.tables, total, self.pages.n, self.cursor)
        assert ok
        g, hq, hkv, d = self.g, self.hq, self.hkv, self.d
        assert np.array_equal(g["bt"].cpu().numpy(), self.tables) and np.array_equal(g["slots"][:total].cpu().numpy(), slots)
        assert np.array_equal(g["lens"].cpu().numpy(), self.ctx) and int(g["cur"]) == self.cursor
        x = orc.widen(qkv).reshape(total, hq + 2 * hkv, d)
        turned = step.rotate(x, np.broadcast_to(pos, (3, total)), self.inv, self.axis)
        real = slots >= 0
        page, at = slots[real] // 16, slots[real] % 16
        ki, vi = self.pages.image()
        got_k, got_q = orc.widen(ki[page, :, at]), orc.widen(from_gpu(g["q"][:total]))[real]
        for got, want in ((got_q, turned[real, :hq]), (got_k, turned[real, hq:hq + hkv])):   # half a step of bf16, and 32 bits of values up to 6
            assert np.all(np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 12 * 2.0 ** -19)
        assert np.array_equal(vi[page, :, at], qkv.reshape(total, -1, d)[real, hq + hkv:])
        self.pages.host.k, self.pages.host.v = ki, vi                                # what follows reads what is stored
        self.bounds = step.page_bounds(self.pages.host, slots, self.bounds)
        assert np.array_equal(orc.widen(from_gpu(g["bounds"])), self.bounds, equal_nan=True)

    def check_attend(self):
        g = self.g
        q = from_gpu(g["q"][:self.B])
        lists, counts = step.select_pages(q, self.bounds, self.tables, self.ctx, self.hkv, self.n_select, self.first, self.last)
        assert np.array_equal(g["lists"].cpu().numpy(), lists) and np.array_equal(g["counts"].cpu().numpy(), counts)
        o, l = step.decode_selected(self.pages.host, q, self.hq, self.tables, self.ctx, lists, counts, self.scale)
        v, self.pages.host.v = self.pages.host.v, self.pages.host.v & 0x7FFF
        reach = step.decode_selected(self.pages.host, q, self.hq, self.tables, self.ctx, lists, counts, self.scale)[0]
        self.pages.host.v = v
        assert np.all(np.abs(orc.widen(from_gpu(g["out"])) - o) <= 2.0 ** -8 * (np.abs(o) + reach) + 2.0 ** -15 * reach)
        assert np.all(np.abs(g["lse"].cpu().numpy() - l) <= 1e-4) and self.pages.status() == 0


@pytest.mark.parametrize("hq,hkv,d", [(32, 8, 128), (4, 2, 64), (8, 8, 64)])
@pytest.mark.parametrize("how", ["plain", "stream", "graph"])
def test_prefill_then_decode_steps(hq, hkv, d, how):
    ctx, steps = [1, 16, 131, 300, 47], 20
    r = _Run(hq, hkv, d, ctx, steps, 6, 1, 2, sum(ctx) + 9, seed=d + hq)
    stream = torch.cuda.Stream() if how == "stream" else None
    with torch.cuda.stream(stream) if stream else torch.cuda.stream(torch.cuda.current_stream()):
        total = sum(ctx) + 9
        qkv = r.rows(ctx, total)
        r.store(total)
        torch.cuda.synchronize()
        r.check_store(ctx, qkv, total)
        graph = None
        for i in range(steps):
            qkv = r.rows([1] * r.B, r.B + 2)
            if how == "graph":
                if graph is None:                                                    # (the decode kernels have not run yet: an eager step first)
                    r.store(r.B + 2)
                    r.attend()
                    torch.cuda.synchronize()
                    graph = torch.cuda.CUDAGraph()
                    with torch.cuda.graph(graph):
                        r.store(r.B + 2)
                        r.attend()
                else:
                    graph.replay()
            else:
                r.store(r.B + 2)
                r.attend()
            torch.cuda.synchronize()
            r.check_store([1] * r.B, qkv, r.B + 2)
            r.check_attend()


def test_with_room_for_all_pages_it_is_attn_decode():
    ctx = [40, 333, 7]
    r = _Run(32, 8, 128, ctx, 1, 24, 0, 0, sum(ctx), seed=3)
    r.rows(ctx, sum(ctx))
    r.store(sum(ctx))
    r.rows([1] * 3, 3)
    r.store(3)
    r.attend()
    g = r.g
    out, lse = torch.empty_like(g["out"]), torch.empty_like(g["lse"])
    kvattn.attn_decode(r.pages.pool, g["q"][:3].contiguous(), g["bt"], g["lens"], r.max_ctx, r.scale, out, lse, torch.empty(1 << 20, dtype=torch.uint8, device="cuda"))
    assert g["counts"].tolist() == [[-(-(c + 1) // 16)] * 8 for c in ctx]
    assert torch.equal(out, g["out"]) and torch.equal(lse, g["lse"]) and r.pages.status() == 0


def test_two_batches_on_two_streams_at_once():
    runs = [_Run(16, 4, 128, [90 + 31 * i, 200, 15], 6, 5, 1, 1, 400, seed=i) for i in range(2)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    news = [[90 + 31 * i, 200, 15] for i in range(2)]
    rows = [r.rows(n, sum(n)) for r, n in zip(runs, news)]
    torch.cuda.synchronize()
    for r, s, n in zip(runs, streams, news):
        with torch.cuda.stream(s):
            r.store(sum(n))
    torch.cuda.synchronize()
    for r, n, x in zip(runs, news, rows):
        r.check_store(n, x, sum(n))
    for _ in range(6):
        rows = [r.rows([1] * 3, 3) for r in runs]
        torch.cuda.synchronize()
        for r, s in zip(runs, streams):
            with torch.cuda.stream(s):
                r.store(3)
                r.attend()
        torch.cuda.synchronize()
        for r, x in zip(runs, rows):
            r.check_store([1] * 3, x, 3)
            r.check_attend()


def test_stored_rows_serve_the_other_attention_calls():
    """Rotated suffixes stored through slots, then attn_extend over the same pages, against the oracle on what is stored."""
    rng = np.random.default_rng(9)
    hq, hkv, d, P, E = 8, 2, 128, [30, 0, 64], [20, 40, 3]
    pages, width = Pages(20, hkv, d), 8
    free, tables = i32(rng.permutation(20)), i32(np.full((3, width), -1))
    inv, T = torch.rand(d // 2, device="cuda"), sum(P) + sum(E)
    cursor, lens = i32([0]), i32([0] * 3)
    out = None
    for new in (P, E):
        n = sum(new)
        cu, pos, slots = i32([0] * 4), i32([0] * n), i32([0] * n)
        kvattn.kv_step_tables(pages.pool, lens, i32(new), free, tables, cu, pos, slots, lens, cursor, cursor)
        q, k, v = (to_gpu(randn_bits(rng, n, h, d)) for h in (hq, hkv, hkv))
        kvattn.kv_append_rotary(pages.pool, q, k, v, slots, pos, inv, None, q)
    out, lse = torch.empty_like(q), torch.empty(n, hq, device="cuda")
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    L = max(p + e for p, e in zip(P, E))
    kvattn.attn_extend(pages.pool, q, cu, tables, i32(P), i32(E), max(E), L, 0.1, out, lse, ws)
    torch.cuda.synchronize()
    pages.host.k, pages.host.v = pages.image()
    o, l = orc.attn_extend(pages.host, from_gpu(q), hq, cu.cpu().numpy(), tables.cpu().numpy(), P, E, 0.1)
    assert np.all(np.abs(orc.widen(from_gpu(out)) - o) <= 4e-3 + 2.0 ** -6 * np.abs(o)) and np.all(np.abs(lse.cpu().numpy() - l) <= 1e-3)
    assert pages.status() == 0 and T == 157
