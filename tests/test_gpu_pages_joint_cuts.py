"""Sequences that are cut in one call inside a page they share, on the GPU: tables, references and copies as the definition has
them, every last page its sequence's own, and tokens appended to all of them."""
import numpy as np
import pytest
import torch

import test_gpu_pages as T
from oracle import pages as O
from test_oracle_pages_joint_cuts import CUTS, holds, shared

pytestmark = pytest.mark.gpu


def grow(c, p, held, ps=16, Hkv=1, hd=32, layer=1):
    """A token for every sequence, in a page that it has or gets."""
    n = len(held)
    x = torch.from_numpy(np.random.default_rng(n).standard_normal((n, Hkv, hd))).to(T.DEV, torch.float32)
    every = list(range(n))
    T.forked(c, p, every, every, held, [h + 1 for h in held])
    p.append(layer, x, x, T.ints(every), T.ints(list(range(n + 1))), T.ints(held), 1)
    assert p.last_error() == 0
    O.append(c, layer, x.double().cpu().numpy(), x.double().cpu().numpy(), every, list(range(n + 1)), held)
    got = T.from_gpu(p)
    for s, h in enumerate(held):
        for name in ("k", "v"):
            assert np.array_equal(O.gather(got, layer, s, h + 1, name), O.gather(c, layer, s, h + 1, name)), s
    holds(got, [h + 1 for h in held])


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("case", range(len(CUTS)))
def test_joint_cuts_leave_every_sequence_its_own_last_page(case, wide):
    """wide: tables of more blocks than the one-launch planning takes."""
    n, blocks, keep, more = CUTS[case]
    c = shared(n, blocks, others=len(more), spare=100)
    if wide:
        c["table"] = np.concatenate([c["table"], np.full((len(c["table"]), 1100), -1, np.int32)], axis=1)
    p = T.to_gpu(c)
    entries = [(s, s, k) for s, k in enumerate(keep)] + [(s, n + i, k) for i, (s, k) in enumerate(more)]
    entries = [entries[i] for i in np.random.default_rng(case).permutation(len(entries))]
    T.forked(c, p, *zip(*entries), [k for _, _, k in entries])
    held = keep + [k for _, k in more]
    holds(T.from_gpu(p), held)
    grow(c, p, held)
    T.forked(c, p, list(range(len(held))), list(range(len(held))), [0] * len(held), [0] * len(held))
    assert not p.ref.any()


def test_more_sequences_than_threads_share_pages_in_groups():
    """1500 sequences: groups of three share a page, the first's entry comes last; entries beyond the first 1024 win their page too."""
    n, ps = 1500, 16
    r = np.random.default_rng(1)
    pages = 2100
    c = {x: O.encode(r.standard_normal((2, pages, 1, ps, 32)) * 50) for x in ("k", "v")}
    c |= {x: (2.0 ** r.integers(-3, 3, (2, pages, 1))).astype(np.float32) for x in ("k_scale", "v_scale")}
    c["table"], c["ref"] = np.full((n, 3), -1, np.int32), np.zeros(pages, np.int32)
    own = r.permutation(pages)[:n // 3]
    group = r.permutation(np.repeat(np.arange(n // 3), 3))
    c["table"][:, 0] = own[group]
    c["ref"][own] = 3
    p = T.to_gpu(c)
    keep = (1 + r.integers(0, 15, n)).tolist()
    order = r.permutation(n).tolist()
    T.forked(c, p, order, order, [keep[s] for s in order], [keep[s] for s in order])
    holds(T.from_gpu(p), keep)
    grow(c, p, keep)


def test_a_joint_cut_of_the_past_comes_apart_when_the_sequences_grow():
    c = shared(2, 1)
    p = T.to_gpu(c)
    T.forked(c, p, [0, 1], [0, 1], [10, 10], [12, 30])
    holds(T.from_gpu(p), [12, 30])
    grow(c, p, [12, 30])
