"""kv_step_tables against a token-by-token walk (whole numbers: equal)."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import paged_step as step
from paper_2607_23815_b200 import kvattn
from step_harness import Pages, guarded, i32

pytestmark = pytest.mark.gpu


def _make(rng, ctx, new, width, n_pages):
    """Tables with pages for ctx, -7 elsewhere; a list of the other pages."""
    ids = rng.permutation(n_pages).tolist()
    tables = np.full((len(ctx), width), -7, np.int64)
    for i, c in enumerate(ctx):
        k = max(0, min(width, -(-c // 16)))
        tables[i, :k], ids = ids[:k], ids[k:]
    return tables, ids


def _run(pages, ctx, new, free, tables, total, cursor=None, in_place=False, positions=True):
    B = len(ctx)
    t = {k: guarded(s, torch.int32, -99) for k, s in dict(bt=tables.shape, cu=(B + 1,), pos=(total,), slots=(total,), nxt=(B,), cur=(1,)).items()}
    t["bt"][0].copy_(i32(tables))
    c, n, f = i32(ctx), i32(new), i32(free)
    nxt, cur = t["nxt"][0], t["cur"][0]
    cin = None if cursor is None else i32([cursor])
    if in_place:
        nxt.copy_(c)
        cur.fill_(cursor or 0)
        c, cin = nxt, cur
    kvattn.kv_step_tables(pages.pool, c, n, f, t["bt"][0], t["cu"][0], t["pos"][0] if positions else None, t["slots"][0], nxt, cin, cur)
    torch.cuda.synchronize()
    assert all(check() for _, check in t.values()), "written outside"
    return [t[k][0].cpu().numpy() for k in ("bt", "cu", "pos", "slots", "nxt", "cur")]


def _compare(got, want, positions=True):
    tables, cu, pos, slots, nxt, cur, ok = want
    assert np.array_equal(got[0], tables) and np.array_equal(got[1], cu) and np.array_equal(got[3], slots)
    assert np.array_equal(got[4], nxt) and got[5][0] == cur
    assert not positions or np.array_equal(got[2], pos)


SHAPES = [  # sequences, tokens before, new tokens, rows of padding
    (1, (0, 0), (1, 1), 0), (1, (16, 16), (1, 1), 3), (1, (15, 15), (1, 1), 0), (1, (1483, 1483), (37, 37), 0), (3, (0, 50), (0, 40), 5),
    (251, (1024, 4095), (1, 1), 5), (255, (0, 40), (0, 3), 0), (256, (0, 40), (0, 3), 1), (257, (0, 40), (0, 3), 2), (511, (0, 40), (0, 3), 0), (512, (0, 40), (0, 3), 1), (513, (0, 40), (0, 3), 2), (1600, (0, 33), (0, 40), 7),
    (40, (0, 200), (300, 9000), 64), (7, (5, 5), (0, 0), 0), (7, (5, 5), (0, 0), 9), (1, (3, 3), (200001, 200001), 0)]


@pytest.mark.parametrize("n,before,fresh,pad", SHAPES)
@pytest.mark.parametrize("in_place", [False, True])
def test_tables_positions_and_slots(n, before, fresh, pad, in_place):
    rng = np.random.default_rng(n * 7 + pad)
    ctx, new = rng.integers(before[0], before[1] + 1, n).tolist(), rng.integers(fresh[0], fresh[1] + 1, n).tolist()
    width = max(1, max(-(-(a + b) // 16) for a, b in zip(ctx, new)))
    count = sum(-(-(a + b) // 16) for a, b in zip(ctx, new)) + 5
    pages = Pages(count, 1, 64)
    tables, free = _make(rng, ctx, new, width, count)
    total = sum(new) + pad
    cursor = 2 if n % 2 else None                                              # (three pages are left over)
    want = step.step_tables(ctx, new, free, tables, total, count, cursor or 0)
    assert want[-1]
    _compare(_run(pages, ctx, new, free, tables, total, cursor, in_place), want)
    assert pages.status() == 0


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("what", ["negative", "ctx", "width", "rows", "pages", "page", "tail", "cursor", "no_pages", "huge"])
@pytest.mark.parametrize("n", [9, 700])
def test_what_does_not_fit_gets_nothing_and_is_recorded(what, n, in_place):
    rng = np.random.default_rng(5)
    ctx, new = rng.integers(0, 60, n).tolist(), rng.integers(1, 30, n).tolist()
    width = 8
    count = sum(-(-(a + b) // 16) for a, b in zip(ctx, new)) + 5
    tables, free = _make(rng, ctx, new, width, count)
    total, cursor, at = sum(new) + 3, 0, n // 2
    if what == "negative":
        new[at] = -3
    if what == "ctx":
        ctx[at] = -1
    if what == "width":
        new[at] = width * 16 - ctx[at] + 1
        total += 200
    if what == "huge":
        new[at] = new[at + 1] = 0x7fffffff
    if what == "rows":
        total = sum(new) - 5
    if what == "pages":
        free = free[:len(free) // 3]
    if what == "no_pages":
        free = []
    if what == "page":
        free[1], free[3] = count, -1
    if what == "tail":
        ctx[at], new[at] = 17, 3
        tables[at, :2] = [0, count + 9]
    if what == "cursor":
        cursor = -4
    want = step.step_tables(ctx, new, free, tables, total, count, cursor)
    assert not want[-1]
    pages = Pages(count, 1, 64)
    _compare(_run(pages, ctx, new, free, tables, total, cursor, in_place), want)
    assert pages.status() == kvattn.KV_ERR_BOUNDS and pages.status() == 0


def test_a_length_has_31_bits():
    width = (1 << 27) + 2
    pages, bt = Pages(4, 1, 64), torch.empty((1, width), dtype=torch.int32, device="cuda")
    bt[0, -3:] = 1
    for ctx, new, ok in ((0x7ffffffe, 1, True), (0x7ffffffe, 2, False), (0x7fffffff, 0, True), (0x7ffffff0, 0x7fffffff, False)):
        total = min(new, 40)
        cu, pos, slots, nxt, cur = i32([0, 0]), i32([9] * total), i32([9] * total), i32([5]), i32([0])
        kvattn.kv_step_tables(pages.pool, i32([ctx]), i32([new]), i32([2]), bt, cu, pos, slots, nxt, None, cur)
        assert int(nxt) == ctx + (new if ok else 0) and int(cur) == 0
        assert slots.tolist() == ([16 + 14] * total if ok else [-1] * total) and pos.tolist() == ([ctx] * total if ok else [0] * total)
        assert pages.status() == (0 if ok else kvattn.KV_ERR_BOUNDS)


def test_no_sequences_and_no_positions():
    pages = Pages(4, 1, 64)
    got = _run(pages, [], [], [1, 2], np.zeros((0, 3)), 5)
    assert got[1].tolist() == [0] and got[3].tolist() == [-1] * 5 and got[2].tolist() == [0] * 5 and got[5].tolist() == [0]
    got = _run(pages, [4], [2], [1, 2], np.array([[3]]), 2, positions=False)
    assert got[3].tolist() == [3 * 16 + 4, 3 * 16 + 5] and got[2].tolist() == [-99] * 2 and pages.status() == 0


@pytest.mark.parametrize("n", [5, 600])
def test_a_captured_step_advances_lengths_and_cursor_in_place(n):
    rng = np.random.default_rng(n)
    steps, width = 40, 8
    ctx = rng.integers(0, 60, n).tolist()
    pages = Pages(n * width, 1, 64)
    tables, free = _make(rng, ctx, None, width, n * width)
    bt, lens, cur, new, f = i32(tables), i32(ctx), i32([0]), i32([1] * n), i32(free)
    cu, pos, slots = i32([0] * (n + 1)), i32([0] * n), i32([0] * n)
    call = lambda: kvattn.kv_step_tables(pages.pool, lens, new, f, bt, cu, pos, slots, lens, cur, cur)
    call()                                                                     # (loads the kernel; taken back below)
    bt.copy_(i32(tables)), lens.copy_(i32(ctx)), cur.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    used = 0
    for _ in range(steps):
        graph.replay()
        tables, _, wpos, wslots, ctx, used, ok = step.step_tables(ctx, [1] * n, free, tables, n, n * width, used)
        assert ok and np.array_equal(slots.cpu().numpy(), wslots) and np.array_equal(pos.cpu().numpy(), wpos)
    assert np.array_equal(bt.cpu().numpy(), tables) and np.array_equal(lens.cpu().numpy(), ctx) and int(cur) == used and pages.status() == 0


def test_refusals():
    pages, lib = Pages(4, 1, 64), kvattn.lib()
    a = i32(np.zeros(64))
    p = lambda off=0: C.c_void_p(a.data_ptr() + 4 * off)
    good = dict(pool=pages.pool.handle, ctx=p(), new=p(2), batch=2, free=p(4), n_free=2, bt=p(6), width=1, total=2, cu=p(8), pos=p(11), slots=p(13),
                nxt=p(15), cin=None, cout=p(17))
    call = lambda **kw: lib.kv_step_tables(*{**good, **kw}.values(), None)
    inv, uns = kvattn.KV_ERR_INVALID, kvattn.KV_ERR_UNSUPPORTED
    n0 = kvattn.kvattn_launch_count()
    for kw in (dict(pool=None), dict(batch=-1), dict(n_free=-1), dict(width=-1), dict(total=-1), dict(ctx=None), dict(new=None), dict(free=None),
               dict(bt=None), dict(cu=None), dict(slots=None), dict(nxt=p(1))):
        assert call(**kw) == inv, kw
    assert call(total=(1 << 30) + 1) == uns and call(n_free=(1 << 30) + 1) == uns
    assert kvattn.kvattn_launch_count() == n0
    assert call() == 0 and call(pos=None, nxt=None, cout=None) == 0
    torch.cuda.synchronize()
    t = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")
    ok = [t(2), t(2), t(3), t((2, 1)), t(3), t(2), t(2), t(2), None, t(1)]
    for i, bad in ((0, t(3)), (1, t(1)), (3, t((3, 1))), (3, t(2)), (4, t(2)), (5, t(3)), (7, t(1)), (8, t(2)), (9, t(2))):
        with pytest.raises(ValueError):
            kvattn.kv_step_tables(pages.pool, *[bad if j == i else x for j, x in enumerate(ok)])
    with pytest.raises(TypeError):
        kvattn.kv_step_tables(pages.pool, ok[0].long(), *ok[1:])
