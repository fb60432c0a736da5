"""The paged 8-bit caches on the GPU against their definitions in 64 bits (oracle/pages.py): append, fork, compact and
attention, each at the sizes and masks where it can go wrong, what they refuse, and a run of them together."""
import ctypes as C
import math
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from oracle import pages as O
from paper_2601_20357_b200 import binding as TB

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda", 0)
NAMES = ("k", "v", "k_scale", "v_scale", "table", "ref")
HALF = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}              # half a step, relative
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def make(held, *, L=2, Hkv=2, ps=64, hd=64, spare=3, blocks=0, seqs=0, seed=0, nan_tail=False):
    """A cache in which sequence i has pages of its own for held[i] tokens, in no order."""
    r = np.random.default_rng(seed)
    need = [-(-h // ps) for h in held]
    n_pages, n_seqs = sum(need) + spare, max(seqs, len(held))
    order = r.permutation(n_pages)
    c = {"table": np.full((n_seqs, max(max(need, default=0) + 1, blocks)), -1, np.int32), "ref": np.zeros(n_pages, np.int32)}
    at = 0
    for i, b in enumerate(need):
        c["table"][i, :b] = order[at:at + b]
        at += b
    c["ref"][order[:at]] = 1
    for x in ("k", "v"):
        c[x] = O.encode(r.standard_normal((L, n_pages, Hkv, ps, hd)) * 90)
        c[x + "_scale"] = (2.0 ** r.integers(-9, -5, (L, n_pages, Hkv))).astype(np.float32)
        if nan_tail:                                        # what lies behind the sequences' ends may be anything
            for i, h in enumerate(held):
                if h % ps:
                    c[x][:, c["table"][i, h // ps], :, h % ps:] = r.choice([0x7F, 0xFF, 0x7E, 0], (L, Hkv, ps - h % ps, hd))
            c[x][:, c["ref"] == 0] = 0x7F
    return c


def to_gpu(c, **kw):
    t = {x: torch.from_numpy(c[x].copy()).to(DEV) for x in NAMES}
    t["k"], t["v"] = t["k"].view(torch.float8_e4m3fn), t["v"].view(torch.float8_e4m3fn)
    return TB.Pages(**t, **kw)


def from_gpu(p):
    torch.cuda.synchronize()
    return {x: getattr(p, x).view(torch.uint8).cpu().numpy() if x in ("k", "v") else getattr(p, x).cpu().numpy() for x in NAMES}


def same(a, b, names=NAMES):
    for x in names:
        assert np.array_equal(a[x], b[x]), f"{x}: {np.argwhere(a[x] != b[x])[:5].tolist()}"


# ---- append ----------------------------------------------------------------------------------------------------

APPEND = [
    # (starts, counts): single tokens, inside and at the ends of pages; nothing at all; over several pages
    ([0, 1, 63, 64, 127], [1, 1, 1, 1, 1]),
    ([5, 0, 130], [0, 1, 0]),
    ([0, 3, 64, 17], [200, 130, 64, 47]),
    ([250], [7]),
    ([10, 0], [3, 150]),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("hd,ps,Hkv", [(64, 64, 2), (32, 16, 3), (128, 128, 1), (128, 32, 2), (32, 128, 1), (64, 16, 5)])
@pytest.mark.parametrize("case", range(len(APPEND)))
def test_append_without_rotation_is_the_definition_to_the_bit(case, hd, ps, Hkv, dtype):
    """x 2^-e is exact and the rounding is one: codes and scales are equal, old tokens brought to a larger scale too."""
    start, count = APPEND[case]
    c = make([a + b for a, b in zip(start, count)], hd=hd, ps=ps, Hkv=Hkv, seed=case, seqs=len(start) + 2)
    first = np.concatenate([[0], np.cumsum(count)]).tolist()
    r = np.random.default_rng(case + 100)
    x = r.standard_normal((2, first[-1], Hkv, hd)) * np.exp2(r.integers(-12, 9, (2, first[-1], Hkv, 1)))
    x[:, ::5, 0] = 0.0
    k, v = (torch.from_numpy(y).to(DEV, TYPES[dtype]) for y in x)
    p = to_gpu(c)
    p.append(1, k, v, ints(list(range(len(start)))), ints(first), ints(start), max(count))
    O.append(c, 1, k.double().cpu().numpy(), v.double().cpu().numpy(), list(range(len(start))), first, start)
    got = from_gpu(p)
    for x in ("k", "v"):                                    # tokens behind the new ones in their block are not kept: not looked at
        for s, (a, n) in enumerate(zip(start, count)):
            end = a + n
            if n and end % ps:
                for d in (got, c):
                    d[x][1, c["table"][s, end // ps], :, end % ps:] = 0
    same(got, c)
    assert p.last_error() == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("hd,ps,H,Hkv,sections", [(64, 64, 6, 2, (32,)), (64, 16, 3, 3, (16, 8, 8)), (128, 32, 8, 1, (40, 0, 24)), (32, 128, 4, 2, (4, 4, 4, 4))])
@pytest.mark.parametrize("counts", [[1, 1, 1, 1], [70, 1, 33, 0]])
def test_append_rotates_by_several_axes(counts, hd, ps, H, Hkv, sections, dtype):
    """Far positions too.  The fp32 rotation y c - z s is off by at most 2^-21 (|y| + |z|): two roundings of 2^-24 for the products
    and the sum each, 2^-23 for cosine and sine each (angle reduced in fp64, then one rounding and sincospif).  A code is
    then off by its half step and that."""
    start = [0, 13, 100, 7]
    c = make([a + b for a, b in zip(start, counts)], hd=hd, ps=ps, Hkv=Hkv, seed=hd)
    first = np.concatenate([[0], np.cumsum(counts)]).tolist()
    T = first[-1]
    r = np.random.default_rng(5)
    qkv = torch.from_numpy(r.standard_normal((T, H + 2 * Hkv, hd))).to(DEV, TYPES[dtype])
    q, k, v = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
    pos = r.integers(0, 2 ** 31 - 1, (len(sections), T)).astype(np.int32)
    pos[:, ::2] = r.integers(0, 3000, pos[:, ::2].shape)
    q_out = torch.full((T, H, hd), 7.0, device=DEV, dtype=TYPES[dtype])
    p = to_gpu(c)
    before = from_gpu(p)
    p.append(0, k, v, None, ints(first), ints(start), max(counts), positions=torch.from_numpy(pos).to(DEV), sections=sections, theta=10000.0, q=q, q_out=q_out)
    got = from_gpu(p)
    kd, qd = k.double().cpu().numpy(), q.double().cpu().numpy()
    kr, qr = O.rotate(kd, pos, sections, 1e4), O.rotate(qd, pos, sections, 1e4)
    pair = lambda x: np.concatenate([np.abs(x[..., :hd // 2]) + np.abs(x[..., hd // 2:])] * 2, axis=-1)
    assert (np.abs(q_out.double().cpu().numpy() - qr) <= HALF[dtype] * np.abs(qr) + 2.0 ** -21 * pair(qd)).all()
    O.append(c, 0, kr, v.double().cpu().numpy(), list(range(4)), first, start)
    for s, (a, n) in enumerate(zip(start, counts)):
        if not n:
            continue
        for name, x, slack in (("k", kr, 2.0 ** -21 * pair(kd)), ("v", v.double().cpu().numpy(), 0 * kd)):
            new = O.gather(got, 0, s, a + n, name)[:, a:].transpose(1, 0, 2)
            want, sl = x[first[s]:first[s + 1]], slack[first[s]:first[s + 1]]
            sc = np.stack([got[name + "_scale"][0, got["table"][s, j // ps]] for j in range(a, a + n)])[..., None]
            step = np.maximum(np.exp2(np.floor(np.log2(np.maximum(np.abs(want) / sc, 1e-30)))), 2.0 ** -6) * 2.0 ** -3 * sc
            assert (np.abs(new - want) <= step / 2 + sl).all()
        same({"s": got["k_scale"][0, got["table"][s, (a + n - 1) // ps]]}, {"s": c["k_scale"][0, c["table"][s, (a + n - 1) // ps]]}, ["s"])
    for x in ("k", "v", "k_scale", "v_scale"):
        assert np.array_equal(got[x][1], before[x][1]) and np.array_equal(got[x][:, c["ref"] == 0], before[x][:, c["ref"] == 0])
    # rotated in place, from rows that start anywhere, keys alone
    wide = torch.zeros((T, (H + 2 * Hkv) * hd + 3), device=DEV, dtype=TYPES[dtype])
    rows = wide[:, 1:1 + (H + 2 * Hkv) * hd].unflatten(1, (H + 2 * Hkv, hd))
    rows.copy_(qkv)
    p2 = to_gpu(make([a + b for a, b in zip(start, counts)], hd=hd, ps=ps, Hkv=Hkv, seed=hd))
    p2.append(0, rows[:, H:H + Hkv], rows[:, H + Hkv:], ints([0, 1, 2, 3]), ints(first), ints(start), max(counts) + 5, positions=torch.from_numpy(pos).to(DEV), sections=sections,
              q=rows[:, :H], q_out=rows[:, :H])
    same(from_gpu(p2), got)
    assert torch.equal(rows[:, :H], q_out) and torch.equal(rows[:, H:], qkv[:, H:])
    p2.append(0, k, v, None, ints(first), ints(start), max(counts), positions=torch.from_numpy(pos).to(DEV), sections=sections)
    same(from_gpu(p2), got)
    assert p.last_error() == 0 and p2.last_error() == 0


def test_append_turns_by_the_whole_angle():
    """Unit vectors come back as (cos, sin) themselves.  Allowed: 1 ulp of the fp32 function (2^-24 below 1), half a step of its correction (2^-25), and
    2^-35 for the correction's own roundings and the reference's angle (turns up to 2^15 in 53 bits: 2^-38 times 2 pi)."""
    hd, T = 64, 4000
    p = to_gpu(make([1, 4100], L=1, Hkv=1, ps=64, hd=hd))
    pos = np.random.default_rng(9).integers(0, 1 << 17, T)
    q = torch.zeros((T, 1, hd), device=DEV)
    q[..., :hd // 2] = 1.0
    out = torch.empty_like(q)
    p.append(0, q, q, ints([1]), ints([0, T]), ints([0]), T, positions=ints([pos.tolist()]), sections=(hd // 2,), q=q, q_out=out)
    assert p.last_error() == 0
    angle = pos[:, None] * 10000.0 ** (-2.0 * np.arange(hd // 2) / hd)
    want = np.concatenate([np.cos(angle), np.sin(angle)], -1)
    assert np.abs(out[:, 0].double().cpu().numpy() - want).max() <= 1.5 * 2.0 ** -24 + 2.0 ** -35


def test_append_scales_at_the_borders():
    """Maxima at 448 2^e and just behind, subnormal and the largest values, zeros; NaN is stored as 0 and infinities saturate, and
    both are reported."""
    big = float(torch.finfo(torch.float32).max)
    tops = [448.0, float(np.nextafter(np.float32(448), np.float32(1e9))), 447.0, 2.0 ** -130, 2.0 ** -149, 0.0, big, -big, 1.75 * 2.0 ** -126, 1.7500001]
    c = make([16 * len(tops)], L=1, Hkv=1, ps=16, hd=32)
    x = np.zeros((16 * len(tops), 1, 32))
    r = np.random.default_rng(0)
    for i, t in enumerate(tops):
        x[16 * i:16 * i + 16] = r.uniform(-1, 1, (16, 1, 32)) * abs(t) * 0.99
        x[16 * i + 3, 0, 5] = t
    x = torch.from_numpy(x).to(DEV, torch.float32)
    p = to_gpu(c)
    p.append(0, x, -x, None, ints([0, len(x)]), ints([0]), len(x))
    O.append(c, 0, x.double().cpu().numpy(), -x.double().cpu().numpy(), [0], [0, len(x)], [0])
    same(from_gpu(p), c)
    assert p.last_error() == 0
    y = x[:20].clone()
    y[2, 0, 1], y[18, 0, 0], y[19, 0, 7] = math.nan, math.inf, -math.inf
    p.append(0, y, x[:20], None, ints([0, 20]), ints([0]), 20)
    O.append(c, 0, y.double().cpu().numpy(), x[:20].double().cpu().numpy(), [0], [0, 20], [0])
    got = from_gpu(p)
    same(got, c)
    assert p.last_error() == TB.ERR_NUMERIC and p.last_error() == 0


def test_append_refuses_on_the_device_what_it_cannot_do():
    c = make([100, 100, 100, 100], ps=64, seqs=5)
    c["ref"][c["table"][1, 1]] = 2                          # shared
    c["table"][2, 0] = 10 ** 6                              # no such page
    p = to_gpu(c)
    before = from_gpu(p)
    x = torch.ones((4, 2, 64), device=DEV)
    call = lambda seq, first, start, n=4: p.append(0, x[:n], x[:n], ints(seq), ints(first), ints(start), 4)
    for seq, first, start, code in [([1], [0, 4], [70], TB.ERR_INVALID_ARG), ([2], [0, 4], [0], TB.ERR_INVALID_ARG), ([7], [0, 4], [0], TB.ERR_INVALID_ARG),
                                    ([-1], [0, 4], [0], TB.ERR_INVALID_ARG), ([0], [0, 4], [-1], TB.ERR_INVALID_ARG), ([0], [0, 5], [0], TB.ERR_INVALID_ARG),
                                    ([0], [3, 2], [0], TB.ERR_INVALID_ARG), ([0, 0], [0, 2, 4], [0, 10], TB.ERR_INVALID_ARG), ([4], [0, 4], [0], TB.ERR_INVALID_ARG),
                                    ([0], [0, 4], [190], TB.ERR_KV_OVERFLOW), ([0], [0, 4], [2 ** 31 - 2], TB.ERR_KV_OVERFLOW)]:
        call(seq, first, start)
        assert p.last_error() == code, (seq, first, start)
        same(from_gpu(p), before)
    # more tokens than max_new said; then: the good entry of a call is done although the other is not
    p.append(0, x, x, ints([0]), ints([0, 4]), ints([0]), 3)
    assert p.last_error() == TB.ERR_INVALID_ARG
    same(from_gpu(p), before)
    call([3, 1], [0, 2, 4], [0, 64])
    assert p.last_error() == TB.ERR_INVALID_ARG
    O.append(c, 0, x[:2].double().cpu().numpy(), x[:2].double().cpu().numpy(), [3], [0, 2], [0])
    got = from_gpu(p)
    for d in (got, c):
        for name in ("k", "v"):
            d[name][0, c["table"][3, 0], :, 2:] = 0
    same(got, c)


# ---- fork ------------------------------------------------------------------------------------------------------

def forked(c, p, src, dst, keep, length):
    p.fork(ints(src), ints(dst), ints(keep), ints(length))
    enough = O.fork(c, src, dst, keep, length)
    same(from_gpu(p), c)
    assert p.last_error() == (0 if enough else TB.ERR_KV_OVERFLOW)


@pytest.mark.parametrize("hd,ps,Hkv,L", [(64, 64, 2, 2), (32, 16, 1, 3), (128, 128, 3, 1)])
def test_fork_follows_the_definition_over_many_calls(hd, ps, Hkv, L):
    """Random batches: forks, cuts inside shared pages, sequences that change places, growth beyond the free pages, frees."""
    r = np.random.default_rng(hd)
    blocks, seqs = 7, 9
    c = make([], L=L, Hkv=Hkv, ps=ps, hd=hd, spare=30, blocks=blocks, seqs=seqs, seed=hd)
    p = to_gpu(c)
    held = [0] * seqs
    for step in range(40):
        n = int(r.integers(1, seqs + 1))
        dst = r.permutation(seqs)[:n].tolist()
        src = [d if r.random() < 0.4 else int(r.integers(seqs)) for d in dst]
        keep = [int(r.integers(0, held[s] + 1)) if r.random() < 0.7 else held[s] for s in src]
        room = [min(blocks * ps, k + int(r.integers(0, 2 * ps))) if r.random() < 0.8 else k for k in keep]
        forked(c, p, src, dst, keep, room)
        for d, m in zip(dst, room):
            held[d] = m
        for s in range(seqs):                               # (what ran out of pages holds less)
            named = int((c["table"][s] >= 0).sum())
            have = 0
            while have < blocks and c["table"][s, have] >= 0:
                have += 1
            held[s] = min(held[s], have * ps)
        for s in range(seqs):
            if (c["table"][s] >= 0).sum() * ps > held[s] + ps - 1:       # a hole: give the sequence back before it is used
                forked(c, p, [s], [s], [0], [0])
                held[s] = 0
    forked(c, p, list(range(seqs)), list(range(seqs)), [0] * seqs, [0] * seqs)
    assert not c["ref"].any()


def test_fork_of_many_sequences_and_pages():
    """More entries than threads of the page search's first scan, pages beyond its first round, one source for all."""
    c = make([100], L=1, Hkv=1, ps=16, hd=32, spare=12000, seqs=1500, blocks=8)
    c["ref"][:9000] |= 1 << 3                               # (pages that others hold)
    c["ref"][::7] = np.where(c["ref"][::7] == 8, 0, c["ref"][::7])
    p = to_gpu(c)
    n = 1499
    forked(c, p, [0] * n, list(range(1, n + 1)), [100] * n, [100 + (i % 25) for i in range(n)])
    forked(c, p, list(range(n + 1)), list(range(n + 1)), [0] * (n + 1), [0] * (n + 1))


def test_fork_refuses_on_the_device_what_it_cannot_do():
    c = make([100, 100], ps=64, seqs=4, blocks=3)
    c["table"][3, 0] = 77
    p = to_gpu(c)
    before = from_gpu(p)
    for src, dst, keep, length, code in [([4], [0], [0], [0], TB.ERR_INVALID_ARG), ([0], [-1], [0], [0], TB.ERR_INVALID_ARG), ([0], [1], [-1], [5], TB.ERR_INVALID_ARG),
                                         ([0], [1], [9], [8], TB.ERR_INVALID_ARG), ([0], [2], [129], [129], TB.ERR_INVALID_ARG), ([3], [2], [1], [1], TB.ERR_INVALID_ARG),
                                         ([0, 1], [2, 2], [5, 5], [9, 9], TB.ERR_INVALID_ARG), ([0], [2], [10], [193], TB.ERR_KV_OVERFLOW)]:
        p.fork(ints(src), ints(dst), ints(keep), ints(length))
        assert p.last_error() == code, (src, dst, keep, length)
        same(from_gpu(p), before)
    p.fork(ints([0, 9]), ints([2, 1]), ints([70, 0]), ints([70, 0]))
    assert p.last_error() == TB.ERR_INVALID_ARG
    O.fork(c, [0], [2], [70], [70])
    same(from_gpu(p), c)


# ---- compact ---------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("hd,ps,Hkv,L", [(64, 64, 2, 2), (32, 16, 3, 1), (128, 128, 1, 2)])
def test_compact_follows_the_definition(hd, ps, Hkv, L):
    held = [300, 90, 41, 260, 17]
    c = make(held, L=L, Hkv=Hkv, ps=ps, hd=hd, seed=hd + 1)
    p = to_gpu(c)
    r = np.random.default_rng(3)
    index = [[20, 21, 25, 40, 41, 60, 77, 89, 255, 256, 299], sorted(r.choice(np.arange(9, 90), 40, replace=False).tolist()), [], list(range(3, 260)), [16]]
    start, count = [20, 9, 5, 3, 0], [len(x) for x in index]
    width = max(count) + 2
    table = torch.tensor([x + [-9] * (width - len(x)) for x in index], dtype=torch.int32, device=DEV)
    p.compact(ints([0, 1, 2, 3, 4]), ints(start), ints(count), table)
    O.compact(c, [0, 1, 2, 3, 4], start, count, index)
    got = from_gpu(p)
    for x in ("k", "v"):                                    # the last block written keeps nothing behind the moved tokens
        for s, (a, n) in enumerate(zip(start, count)):
            if n and (a + n) % ps:
                for d in (got, c):
                    d[x][:, c["table"][s, (a + n) // ps], :, (a + n) % ps:] = 0
    same(got, c)
    assert p.last_error() == 0


def test_compact_of_more_tokens_than_are_looked_up_at_once():
    c = make([4100], L=1, Hkv=1, ps=16, hd=32, seed=8)
    p = to_gpu(c)
    index = sorted(np.random.default_rng(1).choice(np.arange(5, 4100), 2900, replace=False).tolist())
    p.compact(ints([0]), ints([5]), ints([2900]), ints([index]))
    O.compact(c, [0], [5], [2900], [index])
    got = from_gpu(p)
    for d in (got, c):
        for x in ("k", "v"):
            d[x][:, c["table"][0, 2905 // 16], :, 2905 % 16:] = 0
    same(got, c)


def test_compact_refuses_on_the_device_what_it_cannot_do():
    c = make([100, 100, 100], ps=64, seqs=4)
    c["ref"][c["table"][1, 0]] = 2
    p = to_gpu(c)
    before = from_gpu(p)
    for seq, start, count, index in [([0], [5], [2], [[6, 6]]), ([0], [5], [2], [[7, 6]]), ([0], [5], [2], [[4, 9]]), ([0], [5], [2], [[6, 500]]), ([0], [5], [2], [[6, 191]]),
                                     ([0], [5], [3], [[6, 8]]), ([0], [5], [-1], [[6, 8]]), ([0], [-2], [2], [[6, 8]]), ([4], [5], [2], [[6, 8]]), ([1], [5], [2], [[6, 8]]),
                                     ([3], [5], [2], [[6, 8]]), ([0, 0], [5, 70], [1, 1], [[6, 0], [71, 0]]), ([0], [2 ** 31 - 1], [2], [[6, 8]])]:
        p.compact(ints(seq), ints(start), ints(count), ints(index))
        assert p.last_error() == TB.ERR_INVALID_ARG, (seq, start, count, index)
        same(from_gpu(p), before)
    p.compact(ints([1, 2]), ints([5, 5]), ints([1, 1]), ints([[9], [9]]))       # (the other entry is done)
    assert p.last_error() == TB.ERR_INVALID_ARG
    got = from_gpu(p)
    assert np.array_equal(O.gather(got, 0, 2, 6, "k")[:, 5], O.gather(before, 0, 2, 10, "k")[:, 9])
    assert np.array_equal(got["k"][:, c["table"][1, 0]], before["k"][:, c["table"][1, 0]])


# ---- attention -------------------------------------------------------------------------------------------------

def check_attention(c, p, layer, q, first, length, *, seq=None, dtype="bf16", scale=None, softcap=0.0, slopes=None, prefix=None, tree=None, max_new=None, out=None):
    """Against 64 bits, element by element.  Allowed: half a step of the output's type; of the weights' mean of |V| (`size`),
      the rounding of a weight to 11 bits (2^-11; fp32 rows: 22 bits) and, below 2^-14 of 2^15, of a flushed one;
      exponents: scores off by 2^-20 of their terms (fp32 sums of up to 128 exact products, cut off at 2^-23 and more;
      fp16 terms of q: 2^-22), base-2 exponential 2^-22; the sums over n positions 2^-22 (32 partial sums of n / 32
      terms of 2^-24 each stay below that for n up to 128, and grow as sqrt(n): n 2^-27 is added).
    """
    H, hd = q.shape[1], q.shape[2]
    scale = scale or hd ** -0.5
    qg = torch.from_numpy(q).to(DEV, TYPES[dtype])
    fresh = out is None
    if fresh:
        out = torch.full_like(qg, 7.0)
    seqs = list(range(len(length))) if seq is None else seq
    rows = [b - a for a, b in zip(first, first[1:])]
    p.attention(layer, qg, out, None if seq is None else ints(seq), ints(first), ints(length), max_new or max(rows), scale=scale, softcap=softcap,
                slopes=None if slopes is None else torch.from_numpy(slopes).to(DEV, torch.float32), prefix=None if prefix is None else ints(prefix),
                tree=None if tree is None else torch.tensor([int(b) - (1 << 64 if int(b) >> 63 else 0) for b in tree], dtype=torch.int64, device=DEV))
    got = out.double().cpu().numpy()
    qd = qg.double().cpu().numpy()
    for e, s in enumerate(seqs):
        a, b, n = first[e], first[e + 1], length[e]
        if a == b:
            continue
        mask = O.seen(b - a, n, 0 if prefix is None else prefix[e], None if tree is None else tree[a:b])
        K, V = O.gather(c, layer, s, n, "k"), O.gather(c, layer, s, n, "v")
        want, size, terms = O.attention(qd[a:b], K, V, scale, mask, softcap, None if slopes is None else slopes.astype(np.float32))
        weight = 2.0 ** -11 if dtype == "bf16" else 2.0 ** -22
        tol = HALF[dtype] * np.abs(want) + size * (weight + 2 * (terms + 8) * 2.0 ** -20 + 2.0 ** -22 + n * 2.0 ** -27)
        bad = ~(np.abs(got[a:b] - want) <= tol)
        assert not bad.any(), (e, s, n, b - a, np.argwhere(bad)[:4].tolist(), got[a:b][bad][:4], want[bad][:4], tol[bad][:4])
        assert (got[a:b][~mask.any(1)] == 0).all()
    if fresh:                                               # rows of no entry are left as they are
        assert (got[:first[0]] == 7.0).all() and (got[first[-1]:] == 7.0).all()
    return out


def queries(T, H, hd, seed=0, size=1.5):
    return np.random.default_rng(seed).standard_normal((T, H, hd)) * size


ROWS = [
    # (lengths, rows): single tokens at the ends of pages and chunks, sequences of length 1 and 0 (of no rows, too)
    ([1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 300], [1] * 12),
    ([5, 0, 40, 0, 130, 7], [1, 1, 0, 0, 1, 1]),
    ([3, 16, 70, 129, 200], [3, 2, 5, 4, 5]),
    ([2, 0, 1, 90], [5, 3, 4, 33]),                         # more rows than tokens
    ([777], [1]),
    ([260, 100], [130, 41]),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("hd,ps,H,Hkv", [(64, 64, 4, 4), (64, 16, 14, 2), (32, 128, 6, 2), (32, 16, 3, 3), (128, 64, 8, 1), (128, 128, 4, 2), (128, 16, 5, 5), (128, 32, 12, 3)])
@pytest.mark.parametrize("case", range(len(ROWS)))
def test_attention_of_ragged_rows(case, hd, ps, H, Hkv, dtype):
    length, rows = ROWS[case]
    c = make(length, Hkv=Hkv, ps=ps, hd=hd, seed=case, nan_tail=True)
    p = to_gpu(c)
    lead = 2                                                # rows of no entry in front and behind
    first = (lead + np.concatenate([[0], np.cumsum(rows)])).tolist()
    check_attention(c, p, 1, queries(first[-1] + 3, H, hd, case), first, length, dtype=dtype)
    assert p.last_error() == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("hd,ps,H,Hkv", [(64, 64, 4, 2), (32, 16, 4, 4), (128, 32, 8, 1)])
@pytest.mark.parametrize("kind", ["cap", "slopes", "prefix", "tree", "cap slopes prefix", "cap tree prefix"])
def test_attention_of_capped_biased_and_masked_scores(kind, hd, ps, H, Hkv, dtype):
    length, rows = [150, 16, 70, 4, 301], [16, 16, 9, 6, 1]
    if "tree" in kind:
        length, rows = length + [90], rows + [64]
    c = make(length, Hkv=Hkv, ps=ps, hd=hd, seed=9, nan_tail=True)
    p = to_gpu(c)
    first = np.concatenate([[0], np.cumsum(rows)]).tolist()
    r = np.random.default_rng(1)
    tree = None
    if "tree" in kind:
        tree = [int(r.integers(0, 2 ** 63)) * 2 + int(r.integers(2)) for _ in range(first[-1])]
        tree[3], tree[5] = 0, 2 ** 64 - 1
        # (rows of a sequence without anything before it: the fourth has as many rows as tokens and more)
    check_attention(c, p, 0, queries(first[-1], H, hd, 2, 3.0), first, length, dtype=dtype, softcap=5.0 if "cap" in kind else 0.0,
                    slopes=2.0 ** -np.arange(1, H + 1) if "slopes" in kind else None,
                    prefix=[0, 16, 100, 2, 77, 5][:len(rows)] if "prefix" in kind else None, tree=tree)
    assert p.last_error() == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [1, 4, 40, 100])
@pytest.mark.parametrize("cap", [1e3, 1e6])
def test_attention_caps_far_above_the_scores(cap, rows, dtype):
    """Such a cap changes little, and what it costs must not grow with it: check_attention's bound without the cap among its terms, and as
    much again of the scores for tanh (2^-21 of its value) and the four products around it (2^-24 each)."""
    H, hd, length = 4, 64, [300, 117]
    c = make(length, L=1, Hkv=1, seed=6, nan_tail=True)
    p = to_gpu(c)
    q = torch.from_numpy(queries(2 * rows, H, hd, 4)).to(DEV, TYPES[dtype])
    out = torch.empty_like(q)
    p.attention(0, q, out, None, ints([0, rows, 2 * rows]), ints(length), rows, scale=0.125, softcap=cap)
    for e, n in enumerate(length):
        a, b = e * rows, (e + 1) * rows
        want, size, terms = O.attention(q[a:b].double().cpu().numpy(), O.gather(c, 0, e, n, "k"), O.gather(c, 0, e, n, "v"), 0.125, O.seen(rows, n, 0, None), cap)
        weight = 2.0 ** -11 if dtype == "bf16" else 2.0 ** -22
        tol = HALF[dtype] * np.abs(want) + size * (weight + 4 * (terms - cap) * 2.0 ** -20 + 2.0 ** -22 + n * 2.0 ** -27)
        assert (np.abs(out[a:b].double().cpu().numpy() - want) <= tol).all(), (e, float((np.abs(out[a:b].double().cpu().numpy() - want) / tol).max()))
    assert p.last_error() == 0


def test_attention_where_scales_differ_widely_between_pages():
    """K and V of some pages a thousand times those of others, scores far apart, and a scale that is no power of two."""
    c = make([500], Hkv=2, ps=16, hd=64, seed=4)
    r = np.random.default_rng(5)
    for x in ("k_scale", "v_scale"):
        c[x] = (c[x] * np.exp(r.uniform(-7, 3, c[x].shape))).astype(np.float32)
    for dtype in ("bf16", "fp32"):
        check_attention(c, to_gpu(c), 1, queries(7, 4, 64, 3), [0, 7], [500], dtype=dtype)
        check_attention(c, to_gpu(c), 0, queries(7, 4, 64, 3, 1e-20), [0, 7], [500], dtype=dtype)
    # weights of a page of large V all but vanish: the others' must not be lost
    c["k"][:], c["k_scale"][:] = 0, 1.0
    page = c["table"][0, 3]
    c["k"][:, page], c["v_scale"][:, page] = O.encode(np.full(64, -8.0)), 2.0 ** 9
    q = np.abs(queries(2, 4, 64, 6))
    for dtype in ("bf16", "fp32"):
        check_attention(c, to_gpu(c), 1, q, [0, 2], [500], dtype=dtype)


def test_attention_of_one_long_sequence_among_short_ones():
    c = make([9000, 3, 40], L=1, Hkv=2, ps=64, hd=64, seed=6)
    p = to_gpu(c)
    for rows in ([1, 1, 1], [6, 2, 6], [40, 3, 1]):
        first = np.concatenate([[0], np.cumsum(rows)]).tolist()
        check_attention(c, p, 0, queries(first[-1], 4, 64, 7), first, [9000, 3, 40])


def test_attention_of_many_items_of_one_chunk():
    """Every item (sequence and KV head) is one chunk, and a CTA has several: their rows differ in size by powers of two, so that an
    item that took another's scale would show."""
    n = 120
    length, rows = [100 + i % 29 for i in range(n)], [17 + i % 4 for i in range(n)]
    c = make(length, L=1, Hkv=8, ps=128, hd=64, seed=12)
    first = np.concatenate([[0], np.cumsum(rows)]).tolist()
    q = queries(first[-1], 8, 64, 11)
    for e in range(n):
        q[first[e]:first[e + 1]] *= 2.0 ** -(e % 7) * np.exp2(-np.arange(8) % 5)[None, :, None]
    p = to_gpu(c)
    for _ in range(3):
        check_attention(c, p, 0, q, first, length)


def test_attention_names_a_sequence_more_than_once_and_in_any_order():
    c = make([100, 50, 7], Hkv=1, ps=16, hd=32, seed=3)
    p = to_gpu(c)
    check_attention(c, p, 0, queries(6, 4, 32), [0, 2, 3, 3, 6], [80, 7, 20, 100], seq=[0, 2, 1, 0])


def test_attention_of_rows_that_start_anywhere():
    for dtype in ("bf16", "fp32"):
        c = make([100, 33], Hkv=2, ps=16, hd=32, seed=3)
        p = to_gpu(c)
        q = queries(5, 4, 32)
        want = check_attention(c, p, 0, q, [0, 2, 5], [100, 33], dtype=dtype)
        wide = torch.full((5, 4 * 32 + 5), 3.0, device=DEV, dtype=TYPES[dtype])
        rows = wide[:, 1:1 + 128].unflatten(1, (4, 32))
        rows.copy_(torch.from_numpy(q))
        p.attention(0, rows, rows, None, ints([0, 2, 5]), ints([100, 33]), 3, scale=32 ** -0.5)       # in place
        assert torch.equal(rows, want) and (wide[:, 0] == 3).all() and (wide[:, 129:] == 3).all()


def test_attention_refuses_on_the_device_what_it_cannot_do():
    c = make([100, 100, 100], ps=64, seqs=4)
    c["table"][1, 0] = -1
    c["table"][2, 1] = 500
    p = to_gpu(c)
    q = queries(4, 2, 64)
    good = [1.0]

    def call(seq, first, length, max_new=4, tree=None):
        out = torch.full((4, 2, 64), 7.0, device=DEV, dtype=torch.bfloat16)
        p.attention(0, torch.from_numpy(q).to(DEV, torch.bfloat16), out, ints(seq), ints(first), ints(length), max_new, scale=0.125, tree=tree)
        return out.float().cpu().numpy()

    for seq, first, length, code, rows in [([9], [0, 4], [10], TB.ERR_INVALID_ARG, 4), ([-1], [0, 3], [10], TB.ERR_INVALID_ARG, 3), ([0], [0, 4], [-5], TB.ERR_INVALID_ARG, 4),
                                           ([0], [0, 4], [193], TB.ERR_KV_OVERFLOW, 4), ([0], [0, 4], [2 ** 31 - 1], TB.ERR_KV_OVERFLOW, 4)]:
        got = call(seq, first, length)
        assert p.last_error() == code and (got[:rows] == 0).all() and (got[rows:] == 7).all(), (seq, first, length)
    for first in ([0, 5], [3, 2], [-1, 2]):
        assert (call([0], first, [10]) == 7).all() and p.last_error() == TB.ERR_INVALID_ARG
    assert (call([0], [0, 4], [10], max_new=3) == 0).all() and p.last_error() == TB.ERR_INVALID_ARG
    # blocks without a page count as not seen
    got = call([1], [0, 1], [100])
    assert p.last_error() == TB.ERR_INVALID_ARG
    c["table"][1] = [c["table"][1, 1], -1, -1]
    want, _, _ = O.attention(torch.from_numpy(q[:1]).bfloat16().double().numpy(), O.gather(c, 0, 1, 36, "k"), O.gather(c, 0, 1, 36, "v"), 0.125, O.seen(1, 36))
    assert np.abs(got[:1] - want).max() < 2.0 ** -7 * np.abs(want).max()
    assert (call([1], [0, 1], [0]) != 7)[0].all() and p.last_error() == 0


def test_codes_beyond_four_gigabytes():
    """Pages whose codes lie beyond 2^32 bytes hold and give what pages at the beginning do."""
    L, Hkv, ps, hd = 1, 4, 128, 128
    n_pages = (1 << 32) // (Hkv * ps * hd) + 8
    p = TB.Pages(k=torch.empty((L, n_pages, Hkv, ps, hd), dtype=torch.uint8, device=DEV), v=torch.empty((L, n_pages, Hkv, ps, hd), dtype=torch.uint8, device=DEV),
                 k_scale=torch.ones((L, n_pages, Hkv), device=DEV), v_scale=torch.ones((L, n_pages, Hkv), device=DEV),
                 table=ints([[0, 1, 2, -1], [n_pages - 1, n_pages - 2, n_pages - 3, -1], [-1] * 4]), ref=torch.zeros(n_pages, dtype=torch.int32, device=DEV))
    p.ref[:3] = 1
    p.ref[-3:] = 1
    x = torch.from_numpy(np.random.default_rng(0).standard_normal((2, 300, Hkv, hd))).to(DEV, torch.bfloat16)
    for s in (0, 1):
        p.append(0, x[0], x[1], ints([s]), ints([0, 300]), ints([0]), 300)
    q = torch.from_numpy(queries(8, 8, hd)).to(DEV, torch.bfloat16)
    out = torch.empty_like(q)
    outs = []
    for rows in (1, 8):
        for s in (0, 1):
            p.attention(0, q[:rows], out[:rows], ints([s]), ints([0, rows]), ints([300]), rows, scale=0.1)
            outs.append(out[:rows].clone())
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[2], outs[3])
    p.compact(ints([0, 1]), ints([3, 3]), ints([3, 3]), ints([[4, 130, 280]] * 2))
    p.ref[5:n_pages - 4] = 1                                # the only free pages: 3, 4 and the fourth last
    p.fork(ints([1]), ints([2]), ints([300]), ints([300]))
    assert p.last_error() == 0 and p.table[2].tolist()[:3] == [n_pages - 1, n_pages - 2, 3]
    assert torch.equal(p.k[0, 0], p.k[0, n_pages - 1]) and torch.equal(p.k[0, 3, :, :44], p.k[0, n_pages - 3, :, :44])
    p.attention(0, q, out, ints([2]), ints([0, 8]), ints([300]), 8, scale=0.1)
    one = out.clone()
    p.attention(0, q, out, ints([0]), ints([0, 8]), ints([300]), 8, scale=0.1)
    assert torch.equal(one, out)


# ---- together --------------------------------------------------------------------------------------------------

def test_a_request_from_its_prompt_to_its_verified_tree():
    """As a program uses them: an image prompt with three axes of positions, forked for two more inputs, decoding steps, a token
    tree verified and its accepted path kept, the rest given back; every step's attention against the oracle's own cache."""
    L, H, Hkv, ps, hd = 2, 6, 2, 16, 64
    sections = (16, 8, 8)
    r = np.random.default_rng(0)
    c = make([], L=L, Hkv=Hkv, ps=ps, hd=hd, spare=60, blocks=12, seqs=4)
    p = to_gpu(c)
    held = [0, 0, 0, 0]

    def feed(seqs, counts, tree=None, prefix=None):
        first = np.concatenate([[0], np.cumsum(counts)]).tolist()
        src = [held[s] for s in seqs]
        forked(c, p, seqs, seqs, src, [a + b for a, b in zip(src, counts)])
        T = first[-1]
        pos = np.stack([np.concatenate([np.arange(a, a + b) // d for a, b in zip(src, counts)]) for d in (1, 2, 5)]).astype(np.int32)
        for layer in range(L):
            qkv = torch.from_numpy(r.standard_normal((T, H + 2 * Hkv, hd))).to(DEV, torch.bfloat16)
            q = torch.empty((T, H, hd), device=DEV, dtype=torch.bfloat16)
            p.append(layer, qkv[:, H:H + Hkv], qkv[:, H + Hkv:], ints(seqs), ints(first), ints(src), max(counts), positions=torch.from_numpy(pos).to(DEV),
                     sections=sections, q=qkv[:, :H], q_out=q)
            # (the oracle's cache takes the rounded keys from the GPU: the rounding has its own tests)
            got = from_gpu(p)
            for x in ("k", "v", "k_scale", "v_scale"):
                c[x] = got[x]
            check_attention(c, p, layer, q.double().cpu().numpy(), first, [a + b for a, b in zip(src, counts)], seq=seqs, tree=tree, prefix=prefix)
        for s, n in zip(seqs, counts):
            held[s] += n

    feed([0], [70], prefix=[40])
    forked(c, p, [0, 0], [1, 2], [70, 64], [70, 64])
    held[1], held[2] = 70, 64
    for _ in range(3):
        feed([2, 0, 1], [1, 1, 1])
    gamma, d = 3, 3
    masks = [(1 << (i + 1)) - 1 for i in range(gamma + 1)]
    for depth in range(gamma):
        masks += [((1 << (depth + 1)) - 1) | (1 << (gamma + 1 + depth * (d - 1) + x)) for x in range(d - 1)]
    n = len(masks)
    start = list(held[:3])
    feed([0, 1, 2], [n, n, n], tree=masks * 3)
    # accepted: two of the chain and a sibling; the whole chain; nothing but the first
    keep = [[0, 1, 2, gamma + 1 + 2 * (d - 1) + 1], [0, 1, 2, 3], [0]]
    index = [[a + x for x in k] + [0] * (4 - len(k)) for a, k in zip(start, keep)]
    p.compact(ints([0, 1, 2]), ints(start), ints([len(k) for k in keep]), ints(index))
    O.compact(c, [0, 1, 2], start, [len(k) for k in keep], index)
    for s in range(3):
        held[s] = start[s] + len(keep[s])
    forked(c, p, [0, 1, 2], [0, 1, 2], held[:3], held[:3])
    feed([0, 1, 2], [1, 1, 1])
    forked(c, p, [0, 1, 2, 3], [0, 1, 2, 3], [0] * 4, [0] * 4)
    assert not p.ref.any()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("heads,kv_heads,d,ps", [(4, 2, 256, 16), (4, 4, 128, 64), (2, 1, 256, 32)])
def test_rows_of_a_handle_are_parked_in_pages_and_filled_from_them(heads, kv_heads, d, ps, dtype):
    """A row goes to pages to the bit as the definition has it; two rows filled from a fork of it give the logits, to the bit, of
    rows that were given the same values by tabed_load_prefix_kv."""
    import gpu_harness as H
    from paper_2601_20357_b200 import workloads as W
    hd, L, n, cap = d // heads, 2, 75, 120
    wl = W.Workload(name="pages", config_id=95, drafter=W.DrafterCfg(L, d, heads, kv_heads, 256, 1000, dtype), n_inputs=3, n_requests=1, gamma=2, window_h=4,
                    rounds=1, policy=W.POLICY_STATIC, kv_capacity=cap)
    w = TB.weights_to_device(wl.drafter, W.make_weights(wl), DEV)
    c = make([], L=L, Hkv=kv_heads, ps=ps, hd=hd, spare=40, blocks=8, seqs=3)
    p = to_gpu(c)
    g, plain = H.make_gpu(wl, w), H.make_gpu(wl, w)
    r = np.random.default_rng(4)
    k, v = (torch.from_numpy(r.standard_normal((L, kv_heads, n, hd)) * 0.5).to(DEV, TYPES[dtype]).contiguous() for _ in range(2))
    for row in range(3):
        g.load_prefix_kv(row, k, v)
    forked(c, p, [0], [0], [0], [n])
    g.pages_store_row(p, 1, 0, 0, 40)
    g.pages_store_row(p, 2, 0, 40, n - 40)                  # (in two pieces: the second joins the first one's block)
    for layer in range(L):
        x = [t[layer].transpose(0, 1).double().cpu().numpy() for t in (k, v)]
        O.append(c, layer, x[0][:40], x[1][:40], [0], [0, 40], [0])
        O.append(c, layer, x[0][40:], x[1][40:], [0], [0, n - 40], [40])
    got = from_gpu(p)
    for name in ("k", "v"):
        if n % ps:
            for t in (got, c):
                t[name][:, c["table"][0, n // ps], :, n % ps:] = 0
    same(got, c)
    p.fork(ints([0]), ints([1]), ints([61]), ints([61]))
    for row, (seq, m) in enumerate([(0, n), (1, 61), (1, 33)]):
        g.pages_load_row(p, row, seq, m)
        dense = [torch.from_numpy(np.stack([O.gather(c, layer, 0, m, x) for layer in range(L)])).to(DEV, TYPES[dtype]).contiguous() for x in "kv"]
        plain.load_prefix_kv(row, *dense)
    assert g.debug_view(TB.VIEW_KV_LEN).tolist() == [n, 61, 33] and p.last_error() == 0
    for _ in range(3):
        tok = ints([17])
        a, b = torch.empty((3, 1000), device=DEV), torch.zeros((3, 1000), device=DEV)
        g.decode_step(tok, a)
        plain.decode_step(tok, b)
        assert torch.equal(a, b)
    # what they refuse
    other = to_gpu(make([], L=L + 1, Hkv=kv_heads, ps=ps, hd=hd, spare=4, blocks=8, seqs=3))
    for args, code in [((other, 0, 0, 0, 5), -1), ((p, 3, 0, 0, 5), -1), ((p, -1, 0, 0, 5), -1), ((p, 0, 3, 0, 5), -1), ((p, 0, 0, -1, 5), -1), ((p, 0, 0, 0, 0), -1),
                       ((p, 0, 0, 0, n + 4), -1), ((p, 0, 0, 2 ** 31 - 1, 5), -1)]:
        with pytest.raises(TB.TabedError) as e:
            g.pages_store_row(*args)
        assert e.value.code == code, args[1:]
    for args, code in [((other, 0, 0, 5), -1), ((p, 3, 0, 5), -1), ((p, 0, -1, 5), -1), ((p, 0, 0, 0), -1), ((p, 0, 0, cap + 1), -1)]:
        with pytest.raises(TB.TabedError) as e:
            g.pages_load_row(*args)
        assert e.value.code == code, args[1:]
    g.pages_load_row(p, 0, 2, 20)                           # a sequence without pages: zeros, and a word about it
    assert p.last_error() == TB.ERR_INVALID_ARG
    assert p.last_error() == 0
    for h in (g, plain):
        h.destroy()
    empty = TB.Tabed(n_inputs=2, n_requests=1, gamma=1, window_h=1, policy=TB.POLICY_STATIC, vocab=100)
    with pytest.raises(TB.TabedError) as e:
        empty.pages_load_row(p, 0, 0, 5)
    assert e.value.code == TB.ERR_BAD_STATE
    empty.destroy()


def test_steps_captured_in_graphs_that_share_a_workspace():
    """append + attention of two caches on one stream, captured one graph each over one workspace, replayed in turn: what the
    calls give eagerly.  And a call on a stream of its own waits for nothing else."""
    st = torch.cuda.Stream()
    H, Hkv, ps, hd = 4, 2, 64, 64
    caches = [make([400, 90], L=1, Hkv=Hkv, ps=ps, hd=hd, seed=s) for s in (1, 2)]
    ws = torch.empty(to_gpu(caches[0]).workspace_bytes, dtype=torch.uint8, device=DEV)
    x = [torch.from_numpy(np.random.default_rng(s).standard_normal((2, H + 2 * Hkv, hd))).to(DEV, torch.bfloat16) for s in (3, 4)]
    first, start, length = ints([0, 1, 2]), ints([390, 80]), ints([391, 81])
    pos = ints([[390, 80]])
    torch.cuda.synchronize()

    def step(p, x, q, out):
        p.append(0, x[:, H:H + Hkv], x[:, H + Hkv:], None, first, start, 1, positions=pos, sections=(hd // 2,), q=x[:, :H], q_out=q)
        p.attention(0, q, out, None, first, length, 1, scale=0.125)

    want = []
    for c, y in zip(caches, x):
        p = to_gpu(c)
        q = torch.empty((2, H, hd), device=DEV, dtype=torch.bfloat16)
        out = torch.empty_like(q)
        step(p, y, q, out)
        want.append((out.clone(), from_gpu(p)))
    graphs = []
    for c, y in zip(caches, x):
        p = to_gpu(c, stream=st, workspace=ws)
        q = torch.empty((2, H, hd), device=DEV, dtype=torch.bfloat16)
        out = torch.zeros_like(q)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            step(p, y, q, out)
        graphs.append((g, p, out))
    for _ in range(3):
        for g, p, out in graphs:
            out.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(st):
            for g, _, _ in graphs:
                g.replay()
        torch.cuda.synchronize()
        for (g, p, out), (w, cache) in zip(graphs, want):
            assert torch.equal(out, w)
            same(from_gpu(p), cache)
            assert p.last_error() == 0


FIRST_CALLS = """
import sys
sys.path[:0] = [%r, %r]
import torch
import test_gpu_pages as T
c, st = T.make([400, 190], L=1, Hkv=2, ps=64, hd=64), torch.cuda.Stream()
outs = []
for captured in (True, False):
    p = T.to_gpu(c, stream=st)
    q = (torch.arange(2 * 30 * 4 * 64, device=T.DEV).reshape(60, 4, 64) %% 7 - 3.0).bfloat16()
    out, few = torch.zeros_like(q), torch.zeros_like(q[:2])
    a = [T.ints(x) for x in ([0, 30, 60], [50, 50], [80, 80], [0, 1, 2], [0], [1], [51])]
    kv = q[:, :2].contiguous()
    def run():
        p.append(0, kv, kv, None, a[0], a[1], 30)
        p.attention(0, q, out, None, a[0], a[2], 30, scale=0.1)
        p.attention(0, q[:2], few, None, a[3], a[2], 1, scale=0.1)
        p.compact(a[4], a[1][:1], a[5], a[6].view(1, 1))
        p.fork(a[4], a[4], a[1][:1], a[2][:1])
    torch.cuda.synchronize()
    if captured:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            run()
        g.replay()
    else:
        run()
    torch.cuda.synchronize()
    assert p.last_error() == 0
    outs.append((out, few, T.from_gpu(p)))
assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
T.same(outs[0][2], outs[1][2])
"""


def test_the_first_calls_of_a_process_are_captured():
    here = os.path.dirname(os.path.abspath(__file__))
    r = subprocess.run([sys.executable, "-c", FIRST_CALLS % (os.path.dirname(here), here)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [6, 20, 70, 150])
def test_query_rows_that_are_not_finite_reach_no_others(rows, dtype):
    p = to_gpu(make([700], L=1, Hkv=2))
    q = torch.from_numpy(queries(rows, 4, 64)).to(DEV, TYPES[dtype])
    odd = q.clone()
    odd[1, 0, 3], odd[2, 1, 5] = float("nan"), float("inf")
    outs = []
    for x in (q, odd):
        outs.append(torch.empty_like(x))
        p.attention(0, x, outs[-1], None, ints([0, rows]), ints([700]), rows, scale=0.1)
    differ = (outs[0] != outs[1]).any(-1)
    assert differ[1, 0] and differ[2, 1] and differ.sum() == 2 and outs[1][1, 0].isnan().any() and p.last_error() == 0


def test_empty_batches():
    c = make([100, 30])
    p, z = to_gpu(c), ints([])
    q, k = torch.empty((0, 4, 64), device=DEV), torch.empty((0, 2, 64), device=DEV)
    p.fork(z, z, z, z)
    p.attention(0, q, q, None, ints([0, 0, 0]), ints([100, 30]), 0, scale=0.1)
    p.append(0, k, k, None, ints([0, 0]), ints([0]), 0, positions=z.view(1, 0), sections=(32,), q=q, q_out=q)
    p.compact(z, z, z, z.view(0, 0))
    p.compact(ints([0]), ints([0]), ints([0]), z.view(1, 0))
    assert p.last_error() == 0
    same(from_gpu(p), c)


def test_calls_give_the_same_bits_every_time():
    c = make([3000, 40, 700], L=1, Hkv=2, ps=32, hd=128, seed=2)
    p = to_gpu(c)
    q = torch.from_numpy(queries(9, 8, 128)).to(DEV, torch.bfloat16)
    outs = []
    for _ in range(5):
        out = torch.empty_like(q)
        p.attention(0, q, out, None, ints([0, 4, 5, 9]), ints([3000, 40, 700]), 4, scale=0.1)
        outs.append(out)
    assert all(torch.equal(outs[0], o) for o in outs)


def test_the_binding_refuses_other_tensors():
    c = make([100], ps=64)
    p = to_gpu(c)
    q = torch.zeros((2, 4, 64), device=DEV, dtype=torch.bfloat16)
    f, n = ints([0, 2]), ints([100])
    with pytest.raises(TypeError):
        p.attention(0, q.half(), q.half(), None, f, n, 2, scale=0.1)
    with pytest.raises(TypeError):
        p.attention(0, q, q.float(), None, f, n, 2, scale=0.1)
    with pytest.raises(ValueError):
        p.attention(0, q, q[:1], None, f, n, 2, scale=0.1)
    with pytest.raises(ValueError):
        p.attention(0, q.transpose(0, 1), q.transpose(0, 1), None, ints([0, 4]), n, 4, scale=0.1)
    with pytest.raises(ValueError):
        p.attention(0, q, q, None, f, n.cpu(), 2, scale=0.1)
    with pytest.raises(TB.TabedError):
        p.attention(2, q, q, None, f, n, 2, scale=0.1)
    with pytest.raises(TB.TabedError):
        p.attention(0, q[:, :3], q[:, :3], None, f, n, 2, scale=0.1)
    with pytest.raises(ValueError):
        p.append(0, q[:, :2], q[:, :2], None, f, ints([0]), 2, q=q, q_out=q)
    with pytest.raises(ValueError):
        TB.Pages(**{x: getattr(p, x) for x in NAMES}, workspace=torch.empty(8, dtype=torch.uint8, device=DEV))
    with pytest.raises(TypeError):
        TB.Pages(**{x: getattr(p, x) for x in NAMES if x != "k"}, k=p.k.to(torch.float16))
