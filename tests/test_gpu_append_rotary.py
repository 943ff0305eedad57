"""kv_append_rotary against the rotation in 64 bits.

Tolerance: the rounding to bf16, 2^-8 of the value; a sine or cosine in 32 bits (the angle is a fraction of a turn formed in 64 bits and rounded to 32:
2 pi 2^-25 at most, the function itself 2^-23) and two products and a sum in 32 bits (3 x 2^-24): below 2^-20 of |x1| + |x2| in all; positions of 2^31 leave
the angle (here and in the oracle) off by 2^-53 of itself, 2^-21 and 2^-22: below 2^-19 altogether."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import paged_attention as orc
from oracle import paged_step as step
from paper_2607_23815_b200 import kvattn
from step_harness import Pages, bits, from_gpu, guarded, i32, randn_bits, to_gpu

pytestmark = pytest.mark.gpu


def _slots(rng, n_pages, ctx, new, pad):
    ids, rows, at = rng.permutation(n_pages), [], 0
    for a, b in zip(ctx, new):
        t = a % 16 + np.arange(b)
        rows += (ids[at + t // 16] * 16 + t % 16).tolist()
        at += -(-(a % 16 + b) // 16)
    return np.array(rows + [-1] * pad)


def _close(got, x, want, half, neighbours):
    """got bf16 bits, x the rows before, want the rows after, float64."""
    j = np.arange(half)
    a, b = (2 * j, 2 * j + 1) if neighbours else (j, j + half)
    reach = np.zeros_like(x)
    reach[..., a] = reach[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    tol = 2.0 ** -8 * np.abs(want) + 2.0 ** -19 * reach
    d = np.abs(orc.widen(got) - want)
    assert np.all(d <= tol), float(np.max(d - tol))


CASES = [  # q heads, kv heads, D, rot, axes, neighbours, sequences' (before, new), padding
    (32, 8, 128, 128, 1, False, [(1483, 1)], 0), (32, 8, 128, 128, 1, False, [(14, 5), (0, 33), (31, 1), (7, 0), (16, 16)], 3),
    (4, 2, 64, 64, 1, True, [(15, 2), (0, 1)], 0), (16, 8, 64, 48, 3, True, [(3, 70), (12, 4)], 1), (8, 1, 128, 96, 2, False, [(9, 40)], 2),
    (64, 8, 128, 16, 1, True, [(0, 17), (5, 11)], 0), (8, 8, 128, 128, 3, True, [(100, 30)], 7), (1, 1, 64, 16, 1, False, [(2, 13), (2, 14), (2, 15)], 0),
    (5, 3, 64, 64, 2, False, [(8, 25)], 1), (32, 8, 64, 32, 1, False, [(0, 200)] * 12, 40)]


@pytest.mark.parametrize("hq,hkv,d,rot,axes,neighbours,seqs,pad", CASES)
@pytest.mark.parametrize("fused", [False, True])
def test_rows_are_rotated_and_stored(hq, hkv, d, rot, axes, neighbours, seqs, pad, fused):
    rng = np.random.default_rng(hq * 31 + d + rot)
    ctx, new = zip(*seqs)
    count = sum(-(-(a % 16 + b) // 16) for a, b in seqs) + 2
    pages = Pages(count, hkv, d)
    slots = _slots(rng, count, ctx, new, pad)
    T = len(slots)
    far = [0, 1, 77, 4095, 131071, 1000003, 2 ** 24 + 1, 2 ** 31 - 1, -5]
    pos = rng.choice(far, (axes, T)) if T > 3 else np.full((axes, T), 16000)
    inv = (500000.0 ** (-np.arange(rot // 2) * 2 / rot)).astype(np.float32)
    axis = rng.integers(0, axes, rot // 2)
    q, k, v = (randn_bits(rng, T, h, d) for h in (hq, hkv, hkv))
    v[0, 0, :3] = [0x7FC0, 0xFF80, 0x8000]                                     # values are copied, whatever they are
    if fused:
        row = to_gpu(np.concatenate([x.reshape(T, -1) for x in (q, k, v)], 1))
        tq, tk, tv = (x.unflatten(1, (-1, d)) for x in row.split([hq * d, hkv * d, hkv * d], 1))
    else:
        tq, tk, tv = to_gpu(q), to_gpu(k), to_gpu(v)
    out, check = guarded((T, hq, d), torch.bfloat16, -3.0)
    kvattn.kv_append_rotary(pages.pool, tq, tk, tv, i32(slots), i32(pos) if axes > 1 else i32(pos[0]), torch.from_numpy(inv).cuda(),
                            i32(axis) if axes > 1 else None, out, neighbours)
    torch.cuda.synchronize()
    assert check() and pages.status() == 0
    turn = lambda x: step.rotate(orc.widen(x), pos, inv, axis if axes > 1 else None, neighbours)
    real = slots >= 0
    got = from_gpu(out)
    assert np.all(got[~real] == bits(-3.0)), "a row of padding was written"
    _close(got[real], orc.widen(q)[real], turn(q)[real], rot // 2, neighbours)
    assert np.array_equal(got[real][..., rot:], q[real][..., rot:])
    ki, vi = pages.image()
    page, at = slots[real] // 16, slots[real] % 16
    _close(ki[page, :, at], orc.widen(k)[real], turn(k)[real], rot // 2, neighbours)
    assert np.array_equal(vi[page, :, at], v[real])
    touched = np.zeros((count, 16), bool)
    touched[page, at] = True
    for p in range(count):
        last = np.where(touched[p])[0]
        tail = np.arange(16) > (last.max() if len(last) else 16)
        for image in (ki, vi):
            assert np.all(image[p][:, tail] == 0), "the slots behind a page's last row are cleared"
            assert np.all(image[p][:, ~tail & ~touched[p]] == 0x7FC1), "a slot in front was written"


@pytest.mark.parametrize("d", [64, 128])
def test_in_place_only_queries_only_keys(d):
    rng = np.random.default_rng(d)
    T, pages = 37, Pages(5, 2, d)
    q, k, v = (randn_bits(rng, T, h, d) for h in (4, 2, 2))
    pos, inv, slots = i32(np.arange(T) + 500), torch.rand(d // 2, device="cuda"), i32(np.arange(T))
    run = lambda tq, tk, tv, s, out: kvattn.kv_append_rotary(pages.pool, tq, tk, tv, s, pos, inv, None, out)
    ref = torch.empty(T, 4, d, dtype=torch.bfloat16, device="cuda")
    run(to_gpu(q), to_gpu(k), to_gpu(v), slots, ref)
    whole = [x.clone() for x in (pages.k, pages.v)]
    pages.k.zero_(), pages.v.zero_()
    same = to_gpu(q)
    run(same, None, None, None, same)
    assert torch.equal(same, ref) and not pages.k.any() and not pages.v.any()
    run(None, to_gpu(k), to_gpu(v), slots, None)
    keep = 16 * 3                                                              # (pages 0-2 hold the rows, with their tail)
    assert all(torch.equal(a[:3], b[:3]) for a, b in zip((pages.k, pages.v), whole)) and pages.status() == 0 and keep >= T
    qkv = to_gpu(np.concatenate([x.reshape(T, -1) for x in (q, k, v)], 1))     # in place inside the projection's rows
    part = qkv[:, :4 * d].unflatten(1, (4, d))
    run(part, None, None, None, part)
    assert torch.equal(part, ref) and torch.equal(qkv[:, 4 * d:], to_gpu(np.concatenate([x.reshape(T, -1) for x in (k, v)], 1)))


def test_the_same_pages_as_kv_append_where_nothing_turns():
    rng = np.random.default_rng(8)
    a, b = Pages(12, 8, 128), Pages(12, 8, 128)
    k, v = to_gpu(randn_bits(rng, 90, 8, 128)), to_gpu(randn_bits(rng, 90, 8, 128))
    bt = i32(rng.permutation(12).reshape(2, 6))
    kvattn.kv_append(a.pool, k, v, i32([0, 40, 90]), i32([5, 20]), None, bt)
    tables, cu, pos, slots = bt.clone(), i32([0] * 3), i32([0] * 90), i32([0] * 90)
    kvattn.kv_step_tables(b.pool, i32([5, 20]), i32([40, 50]), bt.view(-1)[[1, 2, 8, 9, 10]].contiguous(), tables, cu, pos, slots)
    kvattn.kv_append_rotary(b.pool, None, k, v, slots, pos * 0, torch.ones(64, device="cuda"), None, None)
    assert torch.equal(tables, bt) and torch.equal(a.k, b.k) and torch.equal(a.v, b.v) and a.status() == 0 and b.status() == 0


def test_slots_and_axes_outside_are_recorded():
    pages, T = Pages(3, 2, 64), 4
    x = torch.ones(T, 2, 64, dtype=torch.bfloat16, device="cuda")
    inv, pos = torch.zeros(32, device="cuda"), i32(np.zeros((2, T)))
    out = torch.full_like(x, 5.0)
    kvattn.kv_append_rotary(pages.pool, x, x, x, i32([0, 48, 0x7fffffff, -2]), pos, inv, i32(np.zeros(32)), out)
    assert pages.status() == kvattn.KV_ERR_BOUNDS
    assert [float(o) for o in out[:, 0, 0]] == [1.0, 5.0, 5.0, 5.0]
    assert np.all(pages.image()[0][1:] == 0x7FC1)
    for wrong in (2, -1):
        kvattn.kv_append_rotary(pages.pool, x, None, None, None, pos, inv, i32([0] * 31 + [wrong]), out)
        assert pages.status() == kvattn.KV_ERR_BOUNDS and torch.equal(out, x)


def test_refusals():
    pages, lib = Pages(3, 2, 64), kvattn.lib()
    t = torch.zeros(4096, dtype=torch.bfloat16, device="cuda")
    p = lambda off=0: C.c_void_p(t.data_ptr() + off)
    good = dict(pool=pages.pool.handle, q=p(), qs=256, k=p(), ks=128, v=p(), vs=128, hq=4, slots=p(4096), pos=p(4096), axes=1, inv=p(4096),
                axis=None, rot=64, nb=0, total=2, out=p(), os=256)
    call = lambda **kw: lib.kv_append_rotary(*{**good, **kw}.values(), None)
    inv, uns = kvattn.KV_ERR_INVALID, kvattn.KV_ERR_UNSUPPORTED
    n0 = kvattn.kvattn_launch_count()
    for kw in (dict(pool=None), dict(total=-1), dict(axes=0), dict(hq=0), dict(rot=-16), dict(out=None), dict(k=None), dict(v=None), dict(slots=None),
               dict(pos=None), dict(inv=None), dict(axes=2), dict(q=p(2)), dict(k=p(8)), dict(v=p(4)), dict(out=p(2)), dict(qs=255), dict(qs=248),
               dict(ks=120), dict(vs=130), dict(os=0)):
        assert call(**kw) == inv, kw
    for kw in (dict(rot=0), dict(rot=24), dict(rot=80)):
        assert call(**kw) == uns, kw
    assert call(total=0) == 0 and call(q=None, k=None, v=None) == 0 and kvattn.kvattn_launch_count() == n0
    assert call(total=1, qs=3, ks=0, vs=1, os=5) == 0                           # (one row has no next one)
    x = torch.zeros(2, 2, 64, dtype=torch.bfloat16, device="cuda")
    ok = [x, x, x, i32([0, 1]), i32([0, 0]), torch.zeros(32, device="cuda"), None, x.clone()]
    for i, bad in ((0, x[:, :, :32]), (1, x[:, :1]), (2, None), (3, i32([0])), (4, i32([0])), (6, i32([0])), (7, x[:1]), (7, None), (0, x.transpose(0, 1))):
        with pytest.raises(ValueError):
            kvattn.kv_append_rotary(pages.pool, *[bad if j == i else y for j, y in enumerate(ok)])
    with pytest.raises(TypeError):
        kvattn.kv_append_rotary(pages.pool, x.float(), *ok[1:])
    torch.cuda.synchronize()
    assert pages.status() in (0, kvattn.KV_ERR_BOUNDS)
