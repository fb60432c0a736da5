"""The operators on a paged cache of keys and values in 8 bits, as cases that can be timed.

  fork       sequences that take the beginning of others (whole pages shared, the last one copied), grow or are cut
  append     new keys and values rotated, rounded to 8 bits and written into a layer's pages, the queries rotated with them
  attention  queries over a layer's pages: single tokens, verified blocks and token trees, chunks of prompts
  compact    the tokens that a sequence keeps, moved together in all layers

The cache: codes in e4m3 [layers][pages][kv_heads][page][head_dim] with a power-of-two scale for every page, layer and KV head, of K
and of V; a table [sequences][blocks] of page numbers (-1: none) and the number of table entries that name each page.
"""
from __future__ import annotations

import math
import random

import torch

own = False

E4M3 = torch.float8_e4m3fn
_TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
# the drafters that the workloads of this repository have (heads, KV heads, head size, layers), and a target of ordinary shape
_SMALL = dict(layers=4, heads=12, kv_heads=12, hd=64)
_WIDE = dict(layers=12, heads=14, kv_heads=2, hd=64)
_TINY = dict(layers=2, heads=4, kv_heads=4, hd=32)
_TARGET = dict(layers=2, heads=32, kv_heads=8, hd=128)


def listed():
    return [
        # the three inputs of one chat request set up from its image prompt: latency of the bookkeeping
        dict(name="fork_chat", op="fork", **_SMALL, page=64, sources=1, each=2, low=704, high=704, room=64),
        # 32 requests give their prompts to two more inputs each, and make room for the next tokens themselves
        dict(name="fork_serving", op="fork", **_WIDE, page=64, sources=32, each=2, low=256, high=4096, room=128),
        # one decoding step of 32 requests with three inputs: a token each
        dict(name="append_step", op="append", **_SMALL, page=64, seqs=96, low=256, high=4096, new_low=1, new_high=1, axes=1, dtype="bf16"),
        # prompts with images under three axes of positions (time, height, width), of ragged lengths
        dict(name="append_images", op="append", **_TARGET, page=64, seqs=8, low=0, high=131, new_low=577, new_high=4127, axes=3, dtype="bf16"),
        # the smallest call: the three inputs of one chat request
        dict(name="attention_chat", op="attention", **_SMALL, page=64, seqs=3, low=128, high=704, new=1, dtype="bf16", cap=0.0, slope=False,
             prefix=0, tree=1),
        # serving: 32 requests of three inputs with contexts of all lengths
        dict(name="attention_serving", op="attention", **_SMALL, page=64, seqs=96, low=256, high=4096, new=1, dtype="bf16", cap=0.0,
             slope=False, prefix=0, tree=1),
        # a few documents of great length, grouped queries
        dict(name="attention_long", op="attention", **_WIDE, page=128, seqs=4, low=65537, high=262144, new=1, dtype="bf16", cap=0.0,
             slope=False, prefix=0, tree=1),
        # a target model verifies the token trees (gamma 5, width 3: 16 rows) of 32 requests, with capped scores
        dict(name="attention_tree", op="attention", **_TARGET, page=32, seqs=32, low=500, high=8192, new=16, dtype="bf16", cap=30.0,
             slope=False, prefix=0, tree=3),
        # a chunk of two prompts whose image prefix is seen by all rows
        dict(name="attention_prompt", op="attention", **_TARGET, page=64, seqs=2, low=2111, high=4096, new=2048, dtype="bf16", cap=0.0,
             slope=False, prefix=576, tree=1),
        # an fp32 drafter with biases by distance, a handful of rows each
        dict(name="attention_fp32", op="attention", **_TINY, page=16, seqs=24, low=80, high=1000, new=4, dtype="fp32", cap=0.0, slope=True,
             prefix=0, tree=1),
        # after the verification of 32 token trees: the accepted sibling moves behind the accepted chain
        dict(name="compact_tree", op="compact", **_WIDE, page=64, seqs=32, low=300, high=4096, keep=6, among=16),
        # long contexts that lose three quarters of their image tokens (2 x 2 pooled)
        dict(name="compact_images", op="compact", **_SMALL, page=64, seqs=8, low=33, high=700, keep=1024, among=4096),
    ]


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["fork", "append", "append", "attention", "attention", "attention", "attention", "compact"])
    hd = rng.choice([32, 64, 64, 128, 128])
    kv = rng.randint(1, 8)
    c = dict(op=op, layers=rng.randint(1, 4), heads=kv * rng.choice([1, 1, 2, 3, 4, 7, 8]), kv_heads=kv, hd=hd, page=rng.choice([16, 32, 64, 64, 128]))
    row = kv * hd                                              # values of a token's K
    if op == "fork":
        c.update(sources=_log_int(rng, 1, 48), each=rng.randint(1, 3), high=_log_int(rng, 20, 4096), room=_log_int(rng, 1, 300))
        c["low"] = max(1, c["high"] // rng.choice([1, 3, 20]))
    elif op == "append":
        c.update(seqs=_log_int(rng, 1, 100), axes=rng.choice([0, 1, 1, 2, 3]), dtype=rng.choice(["bf16", "bf16", "fp32"]))
        most = 8_000_000 // (c["seqs"] * (c["heads"] + kv) * hd)
        c["new_high"] = 1 if rng.random() < 0.4 else _log_int(rng, 1, max(1, min(4000, most)))
        c["new_low"] = max(1, c["new_high"] // rng.choice([1, 4]))
        c["high"] = _log_int(rng, 1, 3000)
        c["low"] = c["high"] // rng.choice([1, 5])
    elif op == "compact":
        c.update(seqs=_log_int(rng, 1, 40), among=_log_int(rng, 2, 2500), high=_log_int(rng, 1, 2000))
        c["among"] = max(2, min(c["among"], 30_000_000 // (c["seqs"] * c["layers"] * row)))
        c["keep"] = max(1, int(c["among"] * rng.uniform(0.2, 0.9)))
        c["low"] = max(0, c["high"] // rng.choice([1, 5]))
    else:
        kind = rng.choice(["step", "step", "block", "tree", "prompt"])
        c.update(dtype=rng.choice(["bf16", "bf16", "bf16", "fp32"]), cap=rng.choice([0.0, 0.0, 20.0, 50.0]), slope=False, prefix=0, tree=1)
        if kind == "tree":
            gamma, c["tree"] = rng.choice([3, 5, 7]), rng.choice([2, 3, 4])
            c["new"] = gamma + 1 + gamma * (c["tree"] - 1)
        else:
            c["new"] = 1 if kind == "step" else rng.randint(2, 17) if kind == "block" else _log_int(rng, 40, 1500)
            c["slope"] = rng.random() < 0.25
            c["prefix"] = rng.choice([0, 0, 0, _log_int(rng, 1, 700)])
        c["seqs"] = _log_int(rng, 1, 3 if kind == "prompt" else 100)
        most = 100_000_000 // (c["seqs"] * row)                 # no more cache than the largest listed case reads
        if kind == "prompt":
            most = min(most, 4096)
        else:
            most = min(most, 400_000_000 // (c["seqs"] * c["new"] * c["heads"]))
        c["high"] = max(c["new"], _log_int(rng, 4, max(8, most)))
        c["low"] = max(c["new"], c["high"] // rng.choice([1, 2, 16]))
    return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _ceil(a, b):
    return -(-a // b)


def _spread(rng, n, low, high):
    got = [low + (high - low) * i // max(1, n - 1) for i in range(n)]
    rng.shuffle(got)
    return got


def _paired(rng, a, b):
    """The same pairs whatever the seed, in an order of its own."""
    both = list(zip(a, b))
    rng.shuffle(both)
    return [x for x, _ in both], [y for _, y in both]


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _pool(c, g, rng, held, n_seqs, extra=0):
    """A cache in which sequence i has pages for held[i] tokens; the pages lie in no order, some are free."""
    ps = c["page"]
    blocks = [_ceil(h, ps) for h in held]
    used = sum(blocks)
    n_pages = used + extra + 3
    max_pages = max(blocks) + _ceil(c.get("room", 0), ps) + 1
    order = torch.randperm(n_pages, generator=g, device="cuda", dtype=torch.int64).to(torch.int32)
    at = torch.full((n_seqs, max_pages), -1, dtype=torch.int64)
    first = 0
    for i, b in enumerate(blocks):
        at[i, :b] = torch.arange(first, first + b)
        first += b
    at = at.cuda()
    table = torch.where(at >= 0, order[at.clamp(min=0)], -1).to(torch.int32)
    ref = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    ref[order[:used].long()] = 1
    shape = (c["layers"], n_pages, c["kv_heads"], ps, c["hd"])
    pool = {"table": table, "ref": ref}
    for x in ("k", "v"):
        # standard deviations of about one, amplitudes that fill the range of a page
        codes = torch.empty(shape, dtype=E4M3, device="cuda")
        for layer in range(c["layers"]):
            codes[layer] = (100.0 * torch.randn(shape[1:], generator=g, device="cuda", dtype=torch.float16)).clamp(-448, 448).to(E4M3)
        pool[x] = codes
        pool[x + "_scale"] = 2.0 ** -torch.randint(6, 9, shape[:3], generator=g, device="cuda").float()
    return pool


def _tree_masks(gamma, d):
    """Row masks of a verified token tree: the chain's gamma + 1 positions, then the leaf of every sibling candidate."""
    rows = [(1 << (i + 1)) - 1 for i in range(gamma + 1)]
    leaf = gamma + 1
    for depth in range(gamma):
        for _ in range(d - 1):
            rows.append(((1 << (depth + 1)) - 1) | (1 << leaf))
            leaf += 1
    return rows


def _inputs(c, seed):
    rng = random.Random(seed)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = {"case": c}
    H, hd, Hkv, L = c["heads"], c["hd"], c["kv_heads"], c["layers"]
    s["layer"] = L - 1
    if c["op"] == "fork":
        n, each = c["sources"], c["each"]
        lens = _spread(rng, n, c["low"], c["high"])
        kids = n * each
        # every source's copies, and the source itself, which stays and gets room
        s["pool"] = _pool(c, g, rng, lens + [0] * kids, n + kids, sum(_ceil(c["room"], c["page"]) + 2 for _ in range(n + kids)))
        src, dst, keep = list(range(n)), list(range(n)), list(lens)
        for i in range(kids):
            src.append(i // each)
            dst.append(n + i)
            keep.append(max(0, lens[i // each] - rng.randrange(0, 1 + min(lens[i // each], 40))))
        s.update(src=_ints(src), dst=_ints(dst), keep=_ints(keep), length=_ints([k + rng.randint(1, c["room"]) for k in keep]))
    elif c["op"] == "append":
        n = c["seqs"]
        start, new = _paired(rng, _spread(random.Random(n), n, c["low"], c["high"]), _spread(random.Random(n + 1), n, c["new_low"], c["new_high"]))
        T = sum(new)
        s["pool"] = _pool(c, g, rng, [a + b for a, b in zip(start, new)], n)
        dt = _TYPES[c["dtype"]]
        # a fused projection's rows [q | k | v], as the caller has them
        s["qkv"] = torch.randn((T, H + 2 * Hkv, hd), generator=g, device="cuda", dtype=torch.float32).to(dt)
        cu = [0]
        for x in new:
            cu.append(cu[-1] + x)
        s.update(seq=_ints(list(range(n))), first=_ints(cu), start=_ints(start), max_new=max(new), total=T)
        s["q_out"] = torch.empty((T, H, hd), dtype=dt, device="cuda")
        axes = c["axes"]
        if axes:
            pos = torch.cat([torch.arange(a, a + b) for a, b in zip(start, new)])
            grid = [pos] + [torch.where(pos % 600 < 576, pos // 600 * 600 + (pos % 600 // 24 if a == 1 else pos % 24), pos) for a in range(1, axes)]
            s["positions"] = torch.stack(grid).to(torch.int32).cuda().contiguous()
            part = hd // 2 // axes // 2
            s["sections"] = tuple([hd // 2 - part * (axes - 1)] + [part] * (axes - 1))
    elif c["op"] == "compact":
        n, ps = c["seqs"], c["page"]
        start = _spread(rng, n, c["low"], c["high"])
        s["pool"] = _pool(c, g, rng, [a + c["among"] for a in start], n)
        index = torch.full((n, c["keep"]), 0, dtype=torch.int32)
        count = []
        for i in range(n):
            k = rng.randint(max(1, c["keep"] // 2), c["keep"])
            count.append(k)
            index[i, :k] = torch.tensor(sorted(rng.sample(range(c["among"]), k)), dtype=torch.int32) + start[i]
        s.update(seq=_ints(list(range(n))), start=_ints(start), count=_ints(count), index=index.cuda())
    else:
        n, new = c["seqs"], c["new"]
        # every third sequence of a block or a prompt has fewer rows than the others
        fewer = random.Random(n)
        rows = [new if c["tree"] > 1 or i % 3 != 1 else max(1, new - fewer.randrange(0, 1 + new // 2)) for i in range(n)]
        lens, rows = _paired(rng, _spread(fewer, n, c["low"], c["high"]), rows)
        s["pool"] = _pool(c, g, rng, lens, n)
        dt = _TYPES[c["dtype"]]
        cu = [0]
        for x in rows:
            cu.append(cu[-1] + x)
        s["q"] = (1.5 * torch.randn((cu[-1], H, hd), generator=g, device="cuda")).to(dt)
        s["out"] = torch.empty_like(s["q"])
        s.update(seq=_ints(list(range(n))), first=_ints(cu), length=_ints(lens), max_new=max(rows), scale=1.0 / math.sqrt(hd))
        s["slopes"] = torch.tensor([2.0 ** (-8.0 * (h + 1) / H) for h in range(H)], device="cuda") if c["slope"] else None
        s["prefix"] = _ints([min(c["prefix"], x) for x in lens]) if c["prefix"] else None
        s["tree"] = None
        if c["tree"] > 1:
            gamma = (new - 1) // c["tree"]
            masks = _tree_masks(gamma, c["tree"])
            s["tree"] = torch.tensor(masks * n, dtype=torch.int64, device="cuda")
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_2601_20357_b200 import binding
        s["pages"] = binding.Pages(**s["pool"])
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(s):
    op = s["case"]["op"]
    p = s["pool"]
    if own:
        pages = s["pages"]
        if op == "fork":
            pages.fork(s["src"], s["dst"], s["keep"], s["length"])
        elif op == "append":
            H, Hkv = s["case"]["heads"], s["case"]["kv_heads"]
            q, k, v = s["qkv"][:, :H], s["qkv"][:, H:H + Hkv], s["qkv"][:, H + Hkv:]
            more = dict(q=q, q_out=s["q_out"], positions=s["positions"], sections=s["sections"], theta=10000.0) if s["case"]["axes"] else {}
            pages.append(s["layer"], k, v, s["seq"], s["first"], s["start"], s["max_new"], **more)
        elif op == "compact":
            pages.compact(s["seq"], s["start"], s["count"], s["index"])
        else:
            pages.attention(s["layer"], s["q"], s["out"], s["seq"], s["first"], s["length"], s["max_new"], scale=s["scale"],
                            softcap=s["case"]["cap"], slopes=s["slopes"], prefix=s["prefix"], tree=s["tree"])
            return s["out"]
    else:
        out = {"fork": _fork, "append": _append, "compact": _compact, "attention": _attention}[op](s)
        if op == "attention":
            return out
    if op == "append":
        layer = s["layer"]
        got = {x: p[x][layer] for x in ("k", "v", "k_scale", "v_scale")}
        if s["case"]["axes"]:
            got["q"] = s["q_out"]
        return got
    return dict(p)


def _rotated(x, positions, sections, theta):
    half = x.shape[-1] // 2
    axis = torch.repeat_interleave(torch.arange(len(sections), device="cuda"), torch.tensor(sections, device="cuda"), output_size=half)
    inv = theta ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
    angle = positions.double()[axis].T * inv                    # [T][half]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    a, b = x.float()[..., :half], x.float()[..., half:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)


def _least_scale(amax):
    m, e = torch.frexp(amax)
    e = torch.where(amax > 0, e - 9 + (m > 0.875), -126).clamp(-126, 120)
    return torch.ldexp(torch.ones_like(amax, dtype=torch.float64), e).float()


def _append(s):
    p, layer, ps = s["pool"], s["layer"], s["case"]["page"]
    H, Hkv = s["case"]["heads"], s["case"]["kv_heads"]
    q, k, v = s["qkv"][:, :H], s["qkv"][:, H:H + Hkv].float(), s["qkv"][:, H + Hkv:].float()
    if s["case"]["axes"]:
        k = _rotated(k, s["positions"], s["sections"], 10000.0)
        s["q_out"].copy_(_rotated(q, s["positions"], s["sections"], 10000.0))
    first, start, seq = s["first"].long(), s["start"].long(), s["seq"].long()
    e = torch.repeat_interleave(torch.arange(seq.numel(), device="cuda"), first[1:] - first[:-1], output_size=s["total"])
    pos = start[e] + torch.arange(s["total"], device="cuda") - first[e]
    page, off = p["table"][seq[e], pos // ps].long(), pos % ps
    old_page, old_n = p["table"][seq, start // ps].long().clamp(min=0), start % ps
    kept = (old_n > 0) & (first[1:] > first[:-1])
    lane = torch.arange(ps, device="cuda")
    for x, name in ((k, "k"), (v, "v")):
        codes, scale = p[name][layer].view(torch.uint8), p[name + "_scale"][layer]
        x = torch.where(x.isnan(), 0.0, x)
        amax = torch.where(x.isfinite(), x.abs(), 0.0).amax(-1)
        block = torch.zeros_like(scale).scatter_reduce(0, page[:, None].expand_as(amax), amax, "amax")
        need = _least_scale(block)
        was = torch.zeros_like(scale).index_put((old_page,), torch.where(kept[:, None], scale[old_page], 0.0), accumulate=True)
        need = torch.maximum(need, was)
        before = codes[old_page]                                # [n][Hkv][ps][hd]
        ratio = (scale[old_page] / need[old_page])[:, :, None, None]
        moved = (before.view(E4M3).float() * ratio).to(E4M3).view(torch.uint8)
        stay = (kept[:, None] & (lane < old_n[:, None]))[:, None, :, None]
        codes[old_page[:, None], :, lane[None]] = torch.where(stay, moved, before).transpose(1, 2)
        scale[page] = need[page]
        codes[page, :, off] = (x / need[page][..., None]).clamp(-448, 448).to(E4M3).view(torch.uint8)


def _attention(s):
    p, layer, c = s["pool"], s["layer"], s["case"]
    ps, H, Hkv, hd = c["page"], c["heads"], c["kv_heads"], c["hd"]
    seq, first, length = s["seq"].long(), s["first"].long(), s["length"].long()
    n = seq.numel()
    pages = p["table"][seq].long().clamp(min=0)
    most = pages.shape[1] * ps

    def whole(name):
        x = p[name][layer].view(torch.uint8)[pages].view(E4M3).float() * p[name + "_scale"][layer][pages][..., None, None]
        return x.permute(0, 2, 1, 3, 4).reshape(n, Hkv, most, hd)

    row = torch.arange(s["max_new"], device="cuda")
    rows = first[1:] - first[:-1]
    live = row < rows[:, None]                                  # [n][R]
    at = (first[:-1, None] + row).clamp(max=s["q"].shape[0] - 1)
    q = s["q"][at].float().view(n, s["max_new"], Hkv, H // Hkv, hd).permute(0, 2, 3, 1, 4)
    score = torch.matmul(q.reshape(n, Hkv, -1, hd), whole("k").transpose(-1, -2)).mul_(s["scale"])
    score = score.view(n, H, s["max_new"], most)
    if c["cap"]:
        score = score.div_(c["cap"]).tanh_().mul_(c["cap"])
    j = torch.arange(most, device="cuda")
    here = length[:, None] - rows[:, None] + row                # [n][R]
    if s["slopes"] is not None:
        score -= s["slopes"][None, :, None, None] * (here[:, :, None] - j).abs()[:, None].float()
    if s["tree"] is not None:
        new = j - (length - rows)[:, None]                      # [n][most]
        seen = (new < 0)[:, None] | (((s["tree"][at][..., None] >> new.clamp(0, 63)[:, None]) & 1) > 0) & (new < 64)[:, None]
    else:
        seen = j <= here[..., None]
    if s["prefix"] is not None:
        seen = seen | (j < s["prefix"].long()[:, None])[:, None]
    seen = (seen & (j < length[:, None])[:, None])[:, None]     # [n][1][R][most]
    score.masked_fill_(~seen, -math.inf)
    top = score.amax(-1, keepdim=True)
    w = score.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = w.sum(-1, keepdim=True)
    o = torch.matmul(w.view(n, Hkv, -1, most), whole("v")).view(n, H, s["max_new"], hd)
    o = torch.where(total > 0, o / total, 0.0).transpose(1, 2)  # [n][R][H][hd]
    back = torch.repeat_interleave(torch.arange(n, device="cuda"), rows, output_size=s["q"].shape[0])
    s["out"].copy_(o[back, torch.arange(s["q"].shape[0], device="cuda") - first[back]])
    return s["out"]


def _fork(s):
    p, ps = s["pool"], s["case"]["page"]
    table, ref = p["table"], p["ref"]
    src, dst, keep = s["src"].long(), s["dst"].long(), s["keep"].long()
    blocks = (s["length"].long() + ps - 1) // ps
    full, part = keep // ps, keep % ps
    b = torch.arange(table.shape[1], device="cuda")
    from_, to = table[src].long(), table[dst].long()
    share = b < full[:, None]
    count = torch.zeros(ref.numel() + 1, dtype=torch.int64, device="cuda")
    one = torch.ones_like(from_)
    count.scatter_add_(0, torch.where(share, from_ + 1, 0).view(-1), one.view(-1))
    count.scatter_add_(0, (to + 1).view(-1), -one.view(-1))
    left = ref.long() + count[1:]
    tail = from_.gather(1, full.clamp(max=b.numel() - 1)[:, None])[:, 0].clamp(min=0)
    stays = (part > 0) & (src == dst) & (left[tail] == 0)
    left.index_put_((tail,), stays.long(), accumulate=True)
    copied = (part > 0) & ~stays
    pinned = torch.zeros_like(left).index_put_((tail,), copied.long(), accumulate=True)
    free = torch.argsort(((left > 0) | (pinned > 0)).to(torch.int8), stable=True)
    fresh = (b >= (full + stays.long())[:, None]) & (b < blocks[:, None])
    number = (fresh.view(-1).cumsum(0) - 1).view_as(fresh).clamp(min=0)
    new = free[number.clamp(max=free.numel() - 1)]
    row = torch.where(share | (stays[:, None] & (b == full[:, None])), from_, torch.where(fresh, new, -1))
    left.index_put_((torch.where(fresh, new, 0).view(-1),), fresh.long().view(-1), accumulate=True)
    table[dst] = row.to(torch.int32)
    ref.copy_(left)
    target = row.gather(1, full.clamp(max=b.numel() - 1)[:, None])[:, 0].clamp(min=0)
    # (an entry that copies nothing does what the first that copies does; where none does, a page is copied onto itself)
    one = torch.where(copied, torch.arange(copied.numel(), device="cuda"), copied.to(torch.int8).argmax())
    spare, tail, copied, part = torch.where(copied, target, tail)[one], tail[one], copied[one], part[one]
    lane = torch.arange(ps, device="cuda")
    moves = (copied[:, None] & (lane < part[:, None]))[None, :, None, :, None]
    for x in ("k", "v"):
        codes, scale = p[x].view(torch.uint8), p[x + "_scale"]
        codes[:, spare] = torch.where(moves, codes[:, tail], codes[:, spare])
        scale[:, spare] = scale[:, tail]


def _compact(s):
    p, ps = s["pool"], s["case"]["page"]
    seq, start, count, index = s["seq"].long(), s["start"].long(), s["count"].long(), s["index"].long()
    n, most = index.shape
    i = torch.arange(most, device="cuda")
    live = i < count[:, None]
    to = torch.where(live, start[:, None] + i, start[:, None])
    of = torch.where(live, index, start[:, None])
    page_to, page_of = p["table"][seq[:, None], to // ps].long(), p["table"][seq[:, None], of // ps].long()
    old_page, old_n = p["table"][seq, start // ps].long(), start % ps
    lane = torch.arange(ps, device="cuda")
    stay = (lane < old_n[:, None])[None, :, None, :, None]
    for x in ("k", "v"):
        codes, scale = p[x].view(torch.uint8), p[x + "_scale"]
        value = codes[:, page_of, :, of % ps].view(E4M3)        # [n][most][L][Hkv][hd]
        weight = scale[:, page_of]                              # [L][n][most][Hkv]
        at = torch.where(live, page_to, scale.shape[1]).view(1, -1, 1).expand(weight.shape[0], -1, weight.shape[3])
        need = torch.zeros((weight.shape[0], scale.shape[1] + 1, weight.shape[3]), device="cuda")
        need.scatter_reduce_(1, at, weight.reshape(at.shape), "amax")
        need = need[:, :-1]
        was = torch.where((old_n > 0)[None, :, None], scale[:, old_page], 0.0)
        need[:, old_page] = torch.maximum(need[:, old_page], was)
        before = codes[:, old_page]                             # [L][n][Hkv][ps][hd]
        ratio = torch.where(need[:, old_page] > 0, scale[:, old_page] / need[:, old_page], 1.0)[..., None, None]
        moved = (before.view(E4M3).float() * ratio).to(E4M3).view(torch.uint8)
        codes[:, old_page] = torch.where(stay, moved, before)
        ratio = (weight / need[:, page_to]).permute(1, 2, 0, 3)[..., None]
        new = (value.float() * ratio).to(E4M3).view(torch.uint8)
        # (an entry with fewer tokens writes its first one again)
        first = new[:, :1].expand_as(new)
        codes[:, page_to, :, to % ps] = torch.where(live[:, :, None, None, None], new, first)
        scale.copy_(torch.where(need > 0, need, scale))


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    c = case
    rng = random.Random(0)
    L, H, Hkv, hd, ps = c["layers"], c["heads"], c["kv_heads"], c["hd"], c["page"]
    token = 2 * Hkv * hd                                        # bytes of a token's K and V in one layer
    if c["op"] == "fork":
        lens = _spread(rng, c["sources"], c["low"], c["high"])
        n = c["sources"] * (1 + c["each"])
        entries = sum(_ceil(x, ps) * (1 + c["each"]) for x in lens)
        return {"bytes": 8.0 * entries + 4.0 * n * 4 + L * c["sources"] * c["each"] * (ps // 2) * token * 2.0, "flops": 0.0}
    if c["op"] == "append":
        T = sum(_spread(rng, c["seqs"], c["new_low"], c["new_high"]))
        wide = 2 if c["dtype"] == "bf16" else 4
        turned = H if c["axes"] else 0
        return {"bytes": float(T) * ((2 * Hkv + 2 * turned) * hd * wide + token), "flops": 6.0 * T * (turned + 2 * Hkv) * hd}
    if c["op"] == "compact":
        return {"bytes": 1.5 * c["seqs"] * c["keep"] * L * token, "flops": 0.0}
    lens = _spread(rng, c["seqs"], c["low"], c["high"])
    rows = c["new"] if c["tree"] > 1 else c["new"] * (11 / 12)
    wide = 2 if c["dtype"] == "bf16" else 4
    seen = sum(x - (c["new"] - 1) / 2 for x in lens)
    return {"bytes": float(sum(lens)) * token + 2.0 * rows * c["seqs"] * H * hd * wide, "flops": 4.0 * rows * seen * H * hd}


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------

def _e4m3_nearest(x):
    """The e4m3 value nearest to x (ties to even), for |x| <= 448."""
    _, e = torch.frexp(x)
    step = torch.ldexp(torch.ones_like(x), (e - 1).clamp(min=-6) - 3)
    return torch.round(x / step) * step


def _exact_scale(amax):
    e = torch.ceil(torch.log2(amax.clamp(min=1e-300) / 448.0))
    s = torch.pow(2.0, e)
    s = torch.where(s * 448.0 < amax, s * 2, torch.where(s * 224.0 >= amax, s / 2, s))
    return s.clamp(2.0 ** -126, 2.0 ** 120)


def exact(case, seed):
    s = _inputs(case, seed)
    p, ps, layer = s["pool"], case["page"], s["layer"]
    H, Hkv, hd = case["heads"], case["kv_heads"], case["hd"]
    table = p["table"].cpu()
    if case["op"] == "fork":
        return None
    if case["op"] == "append":
        got = {}
        first, start, seq = s["first"].tolist(), s["start"].tolist(), s["seq"].tolist()
        qkv = s["qkv"].double()
        if case["axes"]:
            axis = [a for a, n in enumerate(s["sections"]) for _ in range(n)]
            half = hd // 2
            inv = torch.tensor([10000.0 ** (-i / half) for i in range(half)], dtype=torch.float64, device="cuda")
            turn = torch.polar(torch.ones_like(s["positions"][axis].double().T), s["positions"][axis].double().T * inv)[:, None]
            z = torch.complex(qkv[:, :H + Hkv, :half], qkv[:, :H + Hkv, half:]) * turn
            qkv[:, :H + Hkv] = torch.cat([z.real, z.imag], dim=-1)
            got["q"] = qkv[:, :H]
        for x, lo in (("k", H), ("v", H + Hkv)):
            codes, scale = p[x][layer].double(), p[x + "_scale"][layer].double()
            for e, sq in enumerate(seq):
                t, pos = first[e], start[e]
                while t < first[e + 1]:
                    off = pos % ps
                    n = min(ps - off, first[e + 1] - t)
                    pg = int(table[sq, pos // ps])
                    new = qkv[t:t + n, lo:lo + Hkv].transpose(0, 1)         # [Hkv][n][hd]
                    sc = _exact_scale(new.abs().amax((1, 2)))
                    if off:
                        sc = torch.maximum(sc, scale[pg])
                        codes[pg, :, :off] = _e4m3_nearest(codes[pg, :, :off] * (scale[pg] / sc)[:, None, None])
                    codes[pg, :, off:off + n] = _e4m3_nearest(new / sc[:, None, None])
                    scale[pg] = sc
                    t, pos = t + n, pos + n
            got[x], got[x + "_scale"] = codes, scale
        return got
    if case["op"] == "compact":
        if s["seq"].numel() * case["keep"] > 200_000:
            return None
        got = {"table": None, "ref": None}
        start, count, seq, index = s["start"].tolist(), s["count"].tolist(), s["seq"].tolist(), s["index"].cpu()
        for x in ("k", "v"):
            codes, scale = p[x].double(), p[x + "_scale"].double()
            for e, sq in enumerate(seq):
                i = 0
                while i < count[e]:
                    to = start[e] + i
                    off = to % ps
                    n = min(ps - off, count[e] - i)
                    pg = int(table[sq, to // ps])
                    of = index[e, i:i + n].long()
                    pages = table[sq][of // ps].long().cuda()
                    value = codes[:, pages, :, (of % ps).cuda()].permute(1, 2, 0, 3)      # [L][Hkv][n][hd]
                    sc_of = scale[:, pages].permute(0, 2, 1)                              # [L][Hkv][n]
                    sc = sc_of.amax(-1)
                    if off:
                        sc = torch.maximum(sc, scale[:, pg])
                        codes[:, pg, :, :off] = _e4m3_nearest(codes[:, pg, :, :off] * (scale[:, pg] / sc)[..., None, None])
                    codes[:, pg, :, off:off + n] = _e4m3_nearest(value * (sc_of / sc[..., None])[..., None])
                    scale[:, pg] = sc
                    i += n
            got[x], got[x + "_scale"] = codes, scale
        return got
    first, length, seq = s["first"].tolist(), s["length"].tolist(), s["seq"].tolist()
    if sum((b - a) * n for a, b, n in zip(first, first[1:], length)) * H * hd > 10 ** 12:
        return None
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    for e, sq in enumerate(seq):
        n, rows = length[e], first[e + 1] - first[e]
        pg = table[sq, :_ceil(n, ps)].long().cuda()
        K, V = ((p[x][layer][pg].double() * p[x + "_scale"][layer][pg].double()[..., None, None]).transpose(0, 1).reshape(Hkv, -1, hd)[:, :n] for x in "kv")
        i = torch.arange(n - rows, n, device="cuda")[:, None]
        j = torch.arange(n, device="cuda")[None]
        if s["tree"] is not None:
            bits = s["tree"][first[e]:first[e + 1]].cpu().tolist()
            seen = torch.tensor([[jj < n - rows or bool(b >> (jj - n + rows) & 1) for jj in range(max(0, n - rows), n)] for b in bits], device="cuda")
            seen = torch.cat([torch.ones((rows, max(0, n - rows)), dtype=torch.bool, device="cuda"), seen], dim=1)
        else:
            seen = j <= i
        if s["prefix"] is not None:
            seen = seen | (j < int(s["prefix"][e]))
        for h in range(H):
            x = s["q"][first[e]:first[e + 1], h].double() @ K[h // (H // Hkv)].T * s["scale"]
            if case["cap"]:
                x = case["cap"] * torch.tanh(x / case["cap"])
            if s["slopes"] is not None:
                x = x - s["slopes"][h].double() * (i - j).abs()
            out[first[e]:first[e + 1], h] = torch.softmax(x.masked_fill(~seen, -math.inf), dim=-1) @ V[h // (H // Hkv)]
    return out
