"""What surrounds attention in a step over the paged KV pool, one operator a case.

The chain of a step: lengths become block tables, positions and slots (kv_step_tables); projected rows are rotated by
their positions and stored at their slots (kv_append_rotary); the pages they touched get new summaries (kv_page_bounds);
a query picks the pages that can matter to it by these summaries (attn_select_pages) and attends over them
(attn_decode_selected).

Sizes are those of the library's own workloads: 8B and 70B head geometry and heads of 64 dims, tuple contexts of a few
hundred to sixteen thousand tokens, suffixes of tens to hundreds, batches of 1 to 256.  Lengths belong to the case (they
are drawn from its `lengths` number), values and page placement come from the seed.

With `own` false, run() computes the plain form with elementary torch operations; with `own` true it calls the library.
"""
import math
import random

import torch

own = False

PAGE = 16
DEVICE = "cuda" if torch.cuda.is_available() else "cpu"

G8B, G70B, G64 = (32, 8, 128), (64, 8, 128), (32, 8, 64)


def _case(name, op, geom, n, ctx=(0, 0), new=(0, 0), pad=0, axes=1, rot=0, neighbours=False, select=0, first=0, last=0, lengths=1):
    hq, hkv, d = geom
    return {"name": name, "op": op, "hq": hq, "hkv": hkv, "d": d, "n": n, "ctx_lo": ctx[0], "ctx_hi": ctx[1], "new_lo": new[0],
            "new_hi": new[1], "pad": pad, "axes": axes, "rot": rot or d, "neighbours": neighbours, "select": select, "first": first,
            "last": last, "lengths": lengths}


def listed():
    return [
        # one token for each answer of a full batch, rows padded to the size that the step was captured with
        _case("tables_decode", "tables", G8B, 251, ctx=(1024, 4095), new=(1, 1), pad=5, lengths=31),
        # a step of from-scratch prefills and suffixes behind reused pages: tens of thousands of slots
        _case("tables_prefill", "tables", G8B, 64, ctx=(0, 2048), new=(419, 2733), lengths=32),
        # the row of a single answer: the smallest call there is
        _case("rotary_one", "rotary", G8B, 1, ctx=(1483, 1483), new=(1, 1), lengths=33),
        # the headline batch's suffixes, as the fused projection leaves them
        _case("rotary_extend_8b", "rotary", G8B, 64, ctx=(512, 2048), new=(64, 256), lengths=34),
        # image tokens: time, height and width rotate 48 of 64 dims, in neighbouring pairs
        _case("rotary_axes_d64", "rotary", G64, 9, ctx=(0, 16384), new=(300, 2000), axes=3, rot=48, neighbours=True, lengths=35),
        # the page of each answer's newest token
        _case("bounds_decode", "bounds", G8B, 256, ctx=(1024, 4095), new=(1, 1), lengths=36),
        # documents that have just been prefilled
        _case("bounds_prefill", "bounds", G8B, 13, new=(8192, 16384), lengths=37),
        # a few answers at the head or the tail of a pipeline
        _case("select_few_d64", "select", G64, 13, ctx=(200, 3000), select=32, first=1, last=2, lengths=38),
        # long documents that are being answered about, 70B heads
        _case("select_long_70b", "select", G70B, 32, ctx=(8192, 16384), select=128, first=1, last=4, lengths=39),
        # one answer about one long document
        _case("selected_one", "selected", G8B, 1, ctx=(15731, 15731), select=64, lengths=40),
        # the answers of a full batch over 1024 tokens each
        _case("selected_8b", "selected", G8B, 256, ctx=(1024, 4096), select=64, lengths=41),
        # long documents, 70B heads, 2048 tokens each
        _case("selected_long_70b", "selected", G70B, 32, ctx=(8192, 16384), select=128, lengths=42),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["tables", "rotary", "rotary", "bounds", "select", "select", "selected", "selected"])
    geom = rng.choice([G8B, G8B, G70B, G64, (8, 8, 128), (16, 8, 64), (16, 4, 128), (8, 1, 128)])
    c = dict(lengths=rng.randrange(1000, 1 << 30))
    decode = rng.random() < 0.4  # one new token for each sequence
    if op in ("tables", "rotary", "bounds"):
        most = {"tables": 120000, "rotary": 16000, "bounds": 150000}[op]
        hi = 1 if decode else _log_int(rng, 2, 4096)
        c.update(new=(1 if decode else rng.randint(1, hi), hi), n=_log_int(rng, 1, max(1, min(256, most // hi))))
        at = _log_int(rng, 1, 16384)
        c.update(ctx=(0 if rng.random() < 0.3 else at // 3, at), pad=rng.choice([0, 0, rng.randint(1, 64)]) if op != "bounds" else 0)
    if op == "rotary":
        d = geom[2]
        c.update(axes=rng.choice([1, 1, 2, 3]), rot=rng.choice([d, d, 16 * rng.randint(1, d // 16)]), neighbours=rng.random() < 0.4)
    if op in ("select", "selected"):
        hi = _log_int(rng, 17, 16384)
        lo = max(1, int(hi * rng.uniform(0.25, 1.0)))
        first, last = rng.randint(0, 2), rng.randint(0, 4)
        c.update(ctx=(lo, hi), n=_log_int(rng, 1, max(1, min(256, 500000 // hi))), select=max(first + last, _log_int(rng, 1, 128)),
                 first=first, last=last)
    n = c.pop("n")
    out = _case("", op, geom, n, **c)
    del out["name"]
    return out


# ---- lengths, pages -------------------------------------------------------------------------------------------------
def _lengths(c):
    r = random.Random(c["lengths"])
    ctx = [r.randint(c["ctx_lo"], c["ctx_hi"]) for _ in range(c["n"])]
    return ctx, [r.randint(c["new_lo"], c["new_hi"]) for _ in range(c["n"])]


def _pages(n):
    return -(-n // PAGE)


def work(c):
    ctx, new = _lengths(c)
    hq, hkv, d, n = c["hq"], c["hkv"], c["d"], c["n"]
    tokens = sum(new)
    need = sum(_pages(a + b) - _pages(a) for a, b in zip(ctx, new))
    touched = sum(_pages(a + b) - a // PAGE for a, b in zip(ctx, new) if b)
    if c["op"] == "tables":  # lengths, new pages and the half-filled pages' ids in; tables, positions, slots, sums, lengths out
        return {"bytes": 4.0 * (2 * n + 2 * need + sum(1 for a in ctx if a % PAGE) + 2 * (tokens + c["pad"]) + 2 * n + 2), "flops": 0}
    if c["op"] == "rotary":  # q, k, v in; q, k, v out; slots, positions, frequencies
        row = (2 * hq + 4 * hkv) * d * 2 + 4 * (1 + c["axes"])
        return {"bytes": float(tokens * row + c["rot"] * 4), "flops": 3.0 * tokens * (hq + hkv) * c["rot"]}
    if c["op"] == "bounds":  # the stored keys of the touched pages in, two rows a page and head out
        keys = sum(a + b - a // PAGE * PAGE for a, b in zip(ctx, new) if b)
        return {"bytes": float(hkv * d * 2 * (keys + 2 * touched) + 4 * tokens), "flops": 2.0 * hkv * d * keys}
    nb = [_pages(a) for a in ctx]
    if c["op"] == "select":
        return {"bytes": float(hkv * d * 4 * sum(nb) + 4 * sum(nb) + n * (hq * d * 2 + 4 + hkv * (c["select"] + 1) * 4)),
                "flops": 2.0 * hq * d * sum(nb)}
    # (the listed pages are any of the sequence's: a last page that is not full weighs by its share)
    seen = sum(a if b <= c["select"] else c["select"] * PAGE for a, b in zip(ctx, nb))
    listed_pages = sum(min(b, c["select"]) for b in nb)
    return {"bytes": float(seen * hkv * d * 4 + n * hq * (d * 4 + 4) + (hkv + 1) * 4 * listed_pages), "flops": 4.0 * hq * d * seen}


# ---- states ---------------------------------------------------------------------------------------------------------
def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEVICE)


def _table(lens, ids, width):
    """A block table [len(lens)][width] whose rows take their pages from `ids` one after the other; the rest is -1."""
    need = torch.tensor([_pages(x) for x in lens], device=DEVICE)
    first = torch.cumsum(need, 0) - need
    b = torch.arange(width, device=DEVICE)[None, :]
    at = (first[:, None] + b).clamp(max=max(ids.numel() - 1, 0))
    return torch.where(b < need[:, None], ids[at], torch.full_like(at, -1, dtype=torch.int32)), int(need.sum())


def _slots(c, ctx, new, ids):
    """Slots of the new tokens (then `pad` rows of -1), pages of every sequence counted from its first touched one."""
    rows, at = [], 0
    for a, b in zip(ctx, new):
        t = torch.arange(a % PAGE, a % PAGE + b, device=DEVICE)
        rows.append(ids[at + t // PAGE] * PAGE + t % PAGE)
        at += _pages(a % PAGE + b)
    rows.append(torch.full((c["pad"],), -1, device=DEVICE))
    return torch.cat(rows).to(torch.int32)


def _positions(c, ctx, new):
    """[axes][tokens]: the token's place; with several axes, frames of an image or a film of 16 x 24 patches."""
    rows = []
    for a, b in zip(ctx, new):
        t = torch.arange(b, device=DEVICE)
        rows.append(torch.stack([a + t // 384, a + t // 24 % 16, a + t % 24][:c["axes"]]) if c["axes"] > 1 else (a + t)[None])
    rows.append(torch.zeros(c["axes"], c["pad"], dtype=torch.int64, device=DEVICE))
    return torch.cat(rows, 1).to(torch.int32)


def prepare(c, seed):
    ctx, new = _lengths(c)
    hq, hkv, d, n, op = c["hq"], c["hkv"], c["d"], c["n"], c["op"]
    gen = torch.Generator(device=DEVICE).manual_seed(seed * 1000003 + c["lengths"] % 1000003)

    def randn(*shape):
        return torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.bfloat16)

    def pages_of(count, heads=hkv, dim=d, like=randn):
        return [like(count, heads, PAGE, dim) for _ in range(2)]

    def ids_of(count):
        return torch.randperm(count, generator=gen, device=DEVICE).to(torch.int32)

    def none(*shape):
        return torch.empty(shape, dtype=torch.bfloat16, device=DEVICE)

    s = {"c": c, "scale": 1.0 / math.sqrt(d), "max_ctx": max(ctx)}
    if op == "tables":
        total = [a + b for a, b in zip(ctx, new)]
        count = sum(_pages(x) for x in total) + 7
        ids = ids_of(count)
        bt, used = _table(ctx, ids, max(_pages(x) for x in total))
        tokens = sum(new) + c["pad"]
        s.update(ctx=_i32(ctx), new=_i32(new), bt=bt, new_pages=ids[used:].contiguous(), cu=_i32([0] * (n + 1)), next=_i32([0] * n),
                 positions=_i32([0] * tokens), slots=_i32([0] * tokens), cursor=_i32([0]), pages=pages_of(count, 1, 64, none))
    elif op in ("rotary", "bounds"):
        count = sum(_pages(a % PAGE + b) for a, b in zip(ctx, new)) + 3
        s.update(slots=_slots(c, ctx, new, ids_of(count).long()), pages=pages_of(count))
        tokens = sum(new) + c["pad"]
        if op == "bounds":
            s["bounds"] = torch.zeros(count, hkv, 2, d, dtype=torch.bfloat16, device=DEVICE)
        else:
            rot = c["rot"]
            s["qkv"] = randn(tokens, (hq + 2 * hkv) * d)  # a fused projection's rows
            s["positions"] = _positions(c, ctx, new)
            s["inv_freq"] = 500000.0 ** (-torch.arange(0, rot, 2, device=DEVICE, dtype=torch.float32) / rot)
            s["freq_axis"] = (torch.arange(rot // 2, device=DEVICE) * c["axes"] // (rot // 2)).to(torch.int32)
            s["q_out"] = torch.zeros(tokens, hq, d, dtype=torch.bfloat16, device=DEVICE)
    else:
        count = sum(_pages(x) for x in ctx)
        width = max(_pages(x) for x in ctx)
        s["bt"], _ = _table(ctx, ids_of(count), width)
        s.update(ctx=_i32(ctx), q=randn(n, hq, d), list=torch.full((n, hkv, c["select"]), -1, dtype=torch.int32, device=DEVICE),
                 counts=torch.zeros(n, hkv, dtype=torch.int32, device=DEVICE))
        if op == "select":
            s["pages"] = pages_of(count, like=none)
            # summaries of pages whose keys have a direction in common, as neighbouring tokens' keys do
            mean, spread = randn(count, hkv, 1, d), randn(count, hkv, 2, d).abs()
            s["bounds"] = mean + torch.cat([-spread[:, :, :1], spread[:, :, 1:]], 2)
        else:
            s["pages"] = pages_of(count)
            # a list of distinct pages in ascending order, the newest among them
            nb = (s["ctx"] + PAGE - 1) // PAGE
            b = torch.arange(width, device=DEVICE)
            rank = torch.rand(n, hkv, width, generator=gen, device=DEVICE)
            rank = torch.where(b == nb[:, None, None] - 1, 2.0, torch.where(b < nb[:, None, None], rank, -1.0))
            take = min(c["select"], width)
            top, at = rank.topk(take, dim=-1)
            at = torch.where(top >= 0, at, width).sort(-1).values
            s["list"][:, :, :take] = torch.where(at < width, at, -1).to(torch.int32)
            s["counts"].copy_((s["list"] >= 0).sum(-1))
            s.update(out=torch.zeros_like(s["q"]), lse=torch.zeros(n, hq, device=DEVICE))
    if own:
        from paper_2607_23815_b200 import kvattn
        k, v = s["pages"]
        s["pool"] = kvattn.kv_pool_create_ex(k.shape[0], PAGE, k.shape[1], k.shape[3], k, v)
    return s


# ---- the plain forms ------------------------------------------------------------------------------------------------
def _in_block(d):
    """Element (slot, dim) of a page's block lies at this place of it: [16 * d] indices (the library's documented layout)."""
    slot, x = torch.arange(PAGE, device=DEVICE)[:, None], torch.arange(d, device=DEVICE)[None, :]
    place = slot // 8 * (8 * d) + x // 64 * 512 + slot % 8 * 64 + ((x % 64 // 8) ^ (slot % 8)) * 8 + x % 8
    return place


def _plain_tables(s):
    ctx, new, bt = s["ctx"].long(), s["new"].long(), s["bt"]
    n, width = bt.shape
    have = (ctx + PAGE - 1) // PAGE
    need = (ctx + new + PAGE - 1) // PAGE - have
    after = torch.cumsum(need, 0)
    cu = torch.cat([torch.zeros_like(ctx[:1]), torch.cumsum(new, 0)])
    j = torch.arange(width, device=bt.device)[None, :] - have[:, None]
    taken = s["new_pages"][((after - need)[:, None] + j).clamp(0, s["new_pages"].numel() - 1)]
    bt = torch.where((j >= 0) & (j < need[:, None]), taken, bt)
    t = torch.arange(s["slots"].numel(), device=bt.device)
    seq = torch.searchsorted(cu[1:], t, right=True).clamp(max=n - 1)
    real = t < cu[-1]
    pos = torch.where(real, ctx[seq] + t - cu[seq], 0)
    slots = torch.where(real, bt[seq, pos // PAGE] * PAGE + pos % PAGE, -1)
    i32 = torch.int32
    return bt, cu.to(i32), pos.to(i32), slots.to(i32), (ctx + new).to(i32), after[-1:].to(i32)


def _rotated(x, cos, sin, rot, neighbours):
    """x [tokens][heads][d] in 32 bits, cos / sin [tokens][1][rot / 2]."""
    y = x[..., :rot]
    a, b = (y[..., 0::2], y[..., 1::2]) if neighbours else (y[..., :rot // 2], y[..., rot // 2:])
    p, q = a * cos - b * sin, b * cos + a * sin
    y = torch.stack([p, q], -1).flatten(-2) if neighbours else torch.cat([p, q], -1)
    return torch.cat([y, x[..., rot:]], -1)


def _plain_rotary(s):
    c, slots = s["c"], s["slots"].long()
    hq, hkv, d, rot = c["hq"], c["hkv"], c["d"], c["rot"]
    q, k, v = (x.unflatten(1, (-1, d)).float() for x in s["qkv"].split([hq * d, hkv * d, hkv * d], 1))
    angle = s["positions"].long()[s["freq_axis"].long()].t().double() * s["inv_freq"].double()  # a far position's angle needs 64 bits
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    real = slots >= 0
    q = torch.where(real[:, None, None], _rotated(q, cos, sin, rot, c["neighbours"]).bfloat16(), s["q_out"])
    k, v = _rotated(k, cos, sin, rot, c["neighbours"]).bfloat16(), v.bfloat16()
    # padding rows repeat the first row's store
    slots, k, v = (torch.where(real.view(-1, *[1] * (x.dim() - 1)), x, x[:1]) for x in (slots, k, v))
    page, at = slots // PAGE, slots % PAGE
    follow = torch.cat([s["slots"].long()[1:], torch.full_like(slots[:1], -1)])
    clears = (real & (follow != slots + 1))[:, None] & (torch.arange(PAGE, device=slots.device) > at[:, None])
    place = _in_block(d)
    block = (page[:, None] * hkv + torch.arange(hkv, device=slots.device)) * (PAGE * d)  # [tokens][heads]
    behind = torch.where(clears, torch.arange(PAGE, device=slots.device), at[:, None])   # slots behind a page's last token, or its own
    for buf, rows in zip(s["pages"], (k, v)):
        flat = buf.view(-1)
        flat[block[:, None, :, None] + place[behind][:, :, None, :]] = 0
        flat[block[:, :, None] + place[at][:, None, :]] = rows
    return q, s["pages"]


def _plain_bounds(s):
    c, slots = s["c"], s["slots"].long()
    follow = torch.cat([slots[1:], torch.full_like(slots[:1], -1)])
    last = slots[(slots >= 0) & ((follow != slots + 1) | (slots % PAGE == PAGE - 1))]
    page, n = last // PAGE, last % PAGE + 1
    keys = s["pages"][0].view(-1, c["hkv"], PAGE * c["d"])[page][:, :, _in_block(c["d"])].float()  # [pages][heads][16][d]
    hidden = (torch.arange(PAGE, device=slots.device) >= n[:, None])[:, None, :, None]
    s["bounds"][page] = torch.stack([keys.masked_fill(hidden, math.inf).amin(2), keys.masked_fill(hidden, -math.inf).amax(2)], 2).bfloat16()
    return s["bounds"]


def _plain_select(s):
    c, bt = s["c"], s["bt"]
    n, width = bt.shape
    hkv, d = c["hkv"], c["d"]
    q = s["q"].double().view(n, hkv, -1, d)  # neighbours at the border of the choice differ by less than 32 bits show
    bounds = s["bounds"][bt.clamp(min=0).long()].double()  # [n][pages][heads][lo, hi][d]
    score = torch.matmul(q.clamp(max=0), bounds[:, :, :, 0].permute(0, 2, 3, 1)) + torch.matmul(q.clamp(min=0), bounds[:, :, :, 1].permute(0, 2, 3, 1))
    score = score.amax(2)  # [n][heads][pages]
    nb = ((s["ctx"].long() + PAGE - 1) // PAGE)[:, None, None]
    b = torch.arange(width, device=bt.device)
    score = torch.where((b < c["first"]) | (b >= nb - c["last"]), math.inf, score)
    score = torch.where(b < nb, score, -math.inf)
    order = score.sort(dim=-1, descending=True, stable=True).indices[..., :c["select"]]
    counts = nb[..., 0].clamp(max=c["select"]).expand(n, hkv)
    picked = torch.where(torch.arange(order.shape[-1], device=bt.device) < counts[..., None], order, width).sort(-1).values
    pages = torch.full((n, hkv, c["select"]), -1, dtype=torch.int32, device=bt.device)
    pages[..., :picked.shape[-1]] = torch.where(picked < width, picked, -1)
    return pages, counts.to(torch.int32)


def _plain_selected(s):
    c, bt, listed_pages = s["c"], s["bt"], s["list"].long()
    n, hkv, m = listed_pages.shape
    d = c["d"]
    in_list = (torch.arange(m, device=bt.device) < s["counts"][..., None]) & (listed_pages >= 0)
    phys = bt.long()[torch.arange(n, device=bt.device)[:, None, None], listed_pages.clamp(min=0)]
    heads = torch.arange(hkv, device=bt.device)[None, :, None]
    place = _in_block(d)
    k, v = (x.view(-1, hkv, PAGE * d)[phys, heads][..., place].view(n, hkv, m * PAGE, d).float() for x in s["pages"])
    at = listed_pages[..., None] * PAGE + torch.arange(PAGE, device=bt.device)
    seen = (in_list[..., None] & (at < s["ctx"].long()[:, None, None, None])).view(n, hkv, 1, m * PAGE)
    score = torch.matmul(s["q"].float().view(n, hkv, -1, d), k.transpose(2, 3)) * s["scale"]
    score = torch.where(seen, score, -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(score - top)
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, v) / torch.where(total > 0, total, 1.0)
    return out.reshape(n, -1, d).bfloat16(), (top + torch.log(total)).reshape(n, -1)


PLAIN = {"tables": _plain_tables, "rotary": _plain_rotary, "bounds": _plain_bounds, "select": _plain_select, "selected": _plain_selected}


# ---- one pass -------------------------------------------------------------------------------------------------------
def run(s):
    c, op = s["c"], s["c"]["op"]
    if not own:
        return PLAIN[op](s)
    from paper_2607_23815_b200 import kvattn
    pool = s["pool"]
    if op == "tables":
        kvattn.kv_step_tables(pool, s["ctx"], s["new"], s["new_pages"], s["bt"], s["cu"], s["positions"], s["slots"], s["next"], None,
                              s["cursor"])
        return s["bt"], s["cu"], s["positions"], s["slots"], s["next"], s["cursor"]
    if op == "rotary":
        hq, hkv, d = c["hq"], c["hkv"], c["d"]
        q, k, v = (x.unflatten(1, (-1, d)) for x in s["qkv"].split([hq * d, hkv * d, hkv * d], 1))
        kvattn.kv_append_rotary(pool, q, k, v, s["slots"], s["positions"], s["inv_freq"], s["freq_axis"], s["q_out"], c["neighbours"])
        return s["q_out"], s["pages"]
    if op == "bounds":
        kvattn.kv_page_bounds(pool, s["slots"], s["bounds"])
        return s["bounds"]
    if op == "select":
        kvattn.attn_select_pages(pool, s["q"], s["bounds"], s["bt"], s["ctx"], s["max_ctx"], c["first"], c["last"], s["list"], s["counts"])
        return s["list"], s["counts"]
    kvattn.attn_decode_selected(pool, s["q"], s["bt"], s["ctx"], s["max_ctx"], s["list"], s["counts"], s["scale"], s["out"], s["lse"])
    return s["out"], s["lse"]


# ---- from the definitions, in 64 bits -------------------------------------------------------------------------------
def _logical(blocks, d):
    """Blocks [..., 16 * d] as [..., slot, dim], by walking the layout's tiles: 8 rows of 64 dims whose 16-byte pieces are
    crossed with the row's number."""
    tiles = blocks.double().unflatten(-1, (2, d // 64, 8, 8, 8))  # [group][half][row][piece][8]
    rows = [torch.stack([tiles[..., r, piece ^ r, :] for piece in range(8)], -2) for r in range(8)]  # each [group][half][piece][8]
    return torch.stack(rows, -4).flatten(-3).flatten(-3, -2)  # [group][row][half * piece * 8] -> [slot][dim]


def _physical(rows, d):
    """The inverse of _logical: [..., slot, dim] as [..., 16 * d]."""
    tiles = rows.unflatten(-1, (d // 64, 8, 8)).unflatten(-4, (2, 8))  # [group][row][half][piece][8]
    crossed = [torch.stack([tiles[..., r, :, piece ^ r, :] for piece in range(8)], -2) for r in range(8)]
    return torch.stack(crossed, -3).flatten(-5)


def _exact_tables(s, ctx, new):
    free, bt, c = s["new_pages"].tolist(), s["bt"].tolist(), s["c"]
    cu, pos, slots, used = [0], [], [], 0
    for i, (a, b) in enumerate(zip(ctx, new)):
        for t in range(a, a + b):
            if t % PAGE == 0:
                bt[i][t // PAGE] = free[used]
                used += 1
            pos.append(t)
            slots.append(bt[i][t // PAGE] * PAGE + t % PAGE)
        cu.append(cu[-1] + b)
    pos, slots = pos + [0] * c["pad"], slots + [-1] * c["pad"]
    return tuple(_i32(x) for x in (bt, cu, pos, slots, [a + b for a, b in zip(ctx, new)], [used]))


def _exact_rotary(s):
    c = s["c"]
    hq, hkv, d, rot = c["hq"], c["hkv"], c["d"], c["rot"]
    axis = s["freq_axis"].tolist()
    theta = torch.stack([s["positions"][axis[j]].double() * float(s["inv_freq"][j]) for j in range(rot // 2)], 1)
    turn = torch.polar(torch.ones_like(theta), theta)[:, None]
    rows = s["qkv"].double().unflatten(1, (-1, d))

    def turned(x):
        y = x[..., :rot]
        pair = (y.unflatten(-1, (rot // 2, 2)) if c["neighbours"] else y.unflatten(-1, (2, rot // 2)).transpose(-1, -2)).contiguous()
        z = torch.view_as_real(torch.view_as_complex(pair) * turn)
        return torch.cat([(z if c["neighbours"] else z.transpose(-1, -2)).flatten(-2), x[..., rot:]], -1)

    slots = s["slots"].tolist()
    q = torch.where((s["slots"] >= 0)[:, None, None], turned(rows[:, :hq]), s["q_out"].double())
    pages = [_logical(x.flatten(-2), d) for x in s["pages"]]
    real = [t for t, x in enumerate(slots) if x >= 0]
    ends = [t for t in real if t + 1 == len(slots) or slots[t + 1] != slots[t] + 1]
    for image, new in zip(pages, (turned(rows[:, hq:hq + hkv]), rows[:, hq + hkv:])):
        for t in ends:
            image[slots[t] // PAGE, :, slots[t] % PAGE + 1:] = 0
        where = s["slots"].long()[real]
        image[where // PAGE, :, where % PAGE] = new[real]
    return q, [_physical(x, d).view_as(y) for x, y in zip(pages, s["pages"])]


def _exact_bounds(s):
    c = s["c"]
    slots, keys, out = s["slots"].tolist(), _logical(s["pages"][0].flatten(-2), c["d"]), s["bounds"].double()
    count = {}
    for x in slots:
        count[x // PAGE] = max(count.get(x // PAGE, 0), x % PAGE + 1)
    pages, counts = torch.tensor(list(count), device=DEVICE), torch.tensor(list(count.values()), device=DEVICE)
    lo = hi = keys[pages, :, 0]
    for t in range(1, PAGE):
        there = (counts > t)[:, None, None]
        lo = torch.where(there, torch.minimum(lo, keys[pages, :, t]), lo)
        hi = torch.where(there, torch.maximum(hi, keys[pages, :, t]), hi)
    out[pages, :, 0], out[pages, :, 1] = lo, hi
    return out


def _exact_select(s, ctx):
    c = s["c"]
    n, hkv, d, m = c["n"], c["hkv"], c["d"], c["select"]
    pages, counts = torch.full((n, hkv, m), -1, dtype=torch.int32), torch.zeros(n, hkv, dtype=torch.int32)
    for i, length in enumerate(ctx):
        nb = _pages(length)
        forced = [b for b in range(nb) if b < c["first"] or b >= nb - c["last"]]
        own_bounds = s["bounds"][s["bt"][i, :nb].long()].double()  # [pages][heads][2][d]
        q = s["q"][i].double().view(hkv, -1, 1, d)
        for h in range(hkv):
            lo, hi = own_bounds[:, h, 0], own_bounds[:, h, 1]
            best = torch.maximum(q[h] * lo, q[h] * hi).sum(-1).amax(0).tolist()
            others = sorted((b for b in range(nb) if c["first"] <= b < nb - c["last"]), key=lambda b: (-best[b], b))
            chosen = sorted((forced + others)[:m])
            pages[i, h, :len(chosen)] = torch.tensor(chosen, dtype=torch.int32)
            counts[i, h] = len(chosen)
    return pages.to(DEVICE), counts.to(DEVICE)


def _exact_selected(s, ctx):
    c = s["c"]
    n, hq, hkv, d = c["n"], c["hq"], c["hkv"], c["d"]
    out, lse = torch.zeros(n, hq, d, dtype=torch.float64, device=DEVICE), torch.full((n, hq), -math.inf, dtype=torch.float64, device=DEVICE)
    g, scale = hq // hkv, s["scale"]
    lists, bt = s["list"].cpu(), s["bt"].cpu()
    for i, length in enumerate(ctx):
        for h in range(hkv):
            blocks = [b for b in lists[i, h].tolist() if b >= 0]
            if not blocks:
                continue
            phys = [int(bt[i, b]) for b in blocks]
            seen = torch.tensor([b * PAGE + t < length for b in blocks for t in range(PAGE)], device=DEVICE)
            k, v = (_logical(x[phys, h].flatten(-2), d).flatten(0, 1)[seen] for x in s["pages"])
            logits = s["q"][i, h * g:(h + 1) * g].double() @ k.t() * scale
            lse[i, h * g:(h + 1) * g] = torch.logsumexp(logits, -1)
            out[i, h * g:(h + 1) * g] = torch.softmax(logits, -1) @ v
    return out, lse


def exact(c, seed):
    """The operators' results by their definitions, in 64 bits (whole numbers as they are)."""
    s, (ctx, new) = prepare(c, seed), _lengths(c)
    if c["op"] == "tables":
        return _exact_tables(s, ctx, new)
    if c["op"] == "rotary":
        return _exact_rotary(s)
    if c["op"] == "bounds":
        return _exact_bounds(s)
    return _exact_select(s, ctx) if c["op"] == "select" else _exact_selected(s, ctx)
