"""Sequences that are cut in one call inside a page they share: the definition (oracle/pages.py) against what must hold whatever the rule."""
import numpy as np
import pytest

from oracle import pages as O


def shared(n, blocks, ps=16, spare=60, L=2, Hkv=1, hd=32, others=0):
    """n sequences that share `blocks` pages, and `others` empty ones."""
    r = np.random.default_rng(n)
    pages = blocks + spare
    c = {x: O.encode(r.standard_normal((L, pages, Hkv, ps, hd)) * 50) for x in ("k", "v")}
    c |= {x: (2.0 ** r.integers(-3, 3, (L, pages, Hkv))).astype(np.float32) for x in ("k_scale", "v_scale")}
    c["table"], c["ref"] = np.full((n + others, blocks + 3), -1, np.int32), np.zeros(pages, np.int32)
    own = r.permutation(pages)[:blocks]
    c["table"][:n, :blocks] = own
    c["ref"][own] = n
    return c


def holds(c, held):
    """Every page is named as often as ref says, and the page in which a sequence ends is its own."""
    ps = c["k"].shape[3]
    named = np.bincount(c["table"][c["table"] >= 0], minlength=len(c["ref"]))
    assert np.array_equal(named, c["ref"])
    for s, n in enumerate(held):
        if n % ps:
            assert c["ref"][c["table"][s, n // ps]] == 1, (s, n)


CUTS = [
    # (sequences, blocks, kept tokens, entries that copy into another sequence: (src, keep))
    (2, 1, [10, 10], []),
    (3, 2, [20, 20, 24], []),
    (3, 2, [32, 20, 17], []),
    (3, 3, [20, 40, 24], []),
    (2, 2, [20, 20], [(0, 25), (1, 17)]),
    (40, 2, [17 + i % 15 for i in range(40)], [(3, 20)]),
]


@pytest.mark.parametrize("case", range(len(CUTS)))
@pytest.mark.parametrize("order", ["up", "down"])
def test_joint_cuts_leave_every_sequence_its_own_last_page(case, order):
    n, blocks, keep, more = CUTS[case]
    c = shared(n, blocks, others=len(more))
    before = {x: c[x].copy() for x in c}
    entries = [(s, s, k) for s, k in enumerate(keep)] + [(s, n + i, k) for i, (s, k) in enumerate(more)]
    if order == "down":
        entries = entries[::-1]
    assert O.fork(c, *zip(*entries), [k for _, _, k in entries])
    held = keep + [k for _, k in more]
    holds(c, held)
    for s, d, k in entries:
        for x in ("k", "v"):
            assert np.array_equal(O.gather(c, 1, d, k, x), O.gather(before, 1, s, k, x))
    # the first entry that keeps a part of a page alone keeps the page
    for page in range(blocks):
        inside = [(d, k) for s, d, k in entries if s == d and k // 16 == page and k % 16]
        if inside and all(k < 16 * (page + 1) for _, _, k in entries):
            assert c["table"][inside[0][0], page] == before["table"][0, page]


def test_a_joint_cut_of_the_past_comes_apart_when_the_sequences_grow():
    c = shared(2, 1)
    assert O.fork(c, [0, 1], [0, 1], [10, 10], [12, 30])
    holds(c, [12, 30])
