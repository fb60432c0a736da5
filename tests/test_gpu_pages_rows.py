"""Attention over paged 8-bit caches with 15 to 34 query rows a KV head, where one kernel follows the other, against the definitions in 64 bits."""
import numpy as np
import pytest
import torch

import test_gpu_pages as T

pytestmark = pytest.mark.gpu

SHAPES = [(64, 64, 4, 4), (64, 16, 6, 3), (32, 16, 2, 2), (32, 128, 8, 4), (128, 32, 2, 2)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("hd,ps,H,Hkv", SHAPES)
@pytest.mark.parametrize("rows", [15, 16, 17, 24, 31, 32, 33, 34])
def test_attention_around_the_borders_of_the_kernels(rows, hd, ps, H, Hkv, dtype):
    """rows: of a KV head.  Sequences shorter than their rows, of one chunk and of several."""
    new = max(1, rows // (H // Hkv))
    length, counts = [5, 130, 333, 64], [new, max(1, new - 3), new, 1]
    c = T.make(length, Hkv=Hkv, ps=ps, hd=hd, seed=rows, nan_tail=True)
    p = T.to_gpu(c)
    first = (1 + np.concatenate([[0], np.cumsum(counts)])).tolist()
    T.check_attention(c, p, 1, T.queries(first[-1] + 2, H, hd, rows), first, length, dtype=dtype)
    assert p.last_error() == 0


@pytest.mark.parametrize("hd,ps,H,Hkv", SHAPES)
@pytest.mark.parametrize("rows", [17, 32, 34])
@pytest.mark.parametrize("kind", ["cap slopes prefix", "cap tree prefix"])
def test_masks_around_the_borders_of_the_kernels(kind, rows, hd, ps, H, Hkv):
    new = rows // (H // Hkv)
    length, counts = [150, 16, 70, 4], [new, new, max(1, new - 5), max(1, new - 2)]
    c = T.make(length, Hkv=Hkv, ps=ps, hd=hd, seed=9, nan_tail=True)
    p = T.to_gpu(c)
    first = np.concatenate([[0], np.cumsum(counts)]).tolist()
    r = np.random.default_rng(rows)
    tree = [int(r.integers(0, 2 ** 63)) * 2 + int(r.integers(2)) for _ in range(first[-1])] if "tree" in kind else None
    T.check_attention(c, p, 0, T.queries(first[-1], H, hd, 2, 3.0), first, length, softcap=5.0, slopes=2.0 ** -np.arange(1, H + 1) if "slopes" in kind else None,
                      prefix=[0, 16, 60, 2], tree=tree)
    assert p.last_error() == 0


@pytest.mark.parametrize("rows", [20, 32])
def test_long_sequences_of_blocks_span_ctas(rows):
    c = T.make([9000, 3, 40], L=1, Hkv=2, ps=64, hd=64, seed=6)
    p = T.to_gpu(c)
    first = [0, rows, rows + 1, 2 * rows + 1]
    T.check_attention(c, p, 0, T.queries(first[-1], 2, 64, 7), first, [9000, 3, 40])
    q = torch.from_numpy(T.queries(rows, 2, 64, 8)).to(T.DEV, torch.bfloat16)
    outs = []
    for _ in range(3):
        outs.append(torch.empty_like(q))
        p.attention(0, q, outs[-1], T.ints([0]), T.ints([0, rows]), T.ints([9000]), rows, scale=0.125)
    p.attention(0, q, q, T.ints([0]), T.ints([0, rows]), T.ints([9000]), rows, scale=0.125)       # in place
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2]) and torch.equal(outs[0], q) and p.last_error() == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("max_new", [9, 40, 100, 1000])
def test_more_rows_announced_than_any_entry_has(max_new, dtype):
    """max_new chooses kernel and tile; most of a tile is then empty."""
    length, counts = [1, 200, 333, 0, 64], [1, 3, 0, 2, 1]
    c = T.make(length, Hkv=2, ps=64, hd=64, seed=5, nan_tail=True)
    p = T.to_gpu(c)
    first = (1 + np.concatenate([[0], np.cumsum(counts)])).tolist()
    T.check_attention(c, p, 1, T.queries(first[-1] + 2, 4, 64, 9), first, length, dtype=dtype, max_new=max_new)
    assert p.last_error() == 0
