"""Attention over paged 8-bit caches whose V scales lie far apart: pages of zeros (whose scale is the least there is) among
others, very small and very large V, against the definitions in 64 bits (oracle/pages.py)."""
import numpy as np
import pytest
import torch

import test_gpu_pages as T
from oracle import pages as O

pytestmark = pytest.mark.gpu

SHAPES = [(64, 64, 4, 2), (32, 16, 3, 3), (128, 128, 8, 2)]
LENGTH = 700


def zeroed(c, spans, *, ps, hd, Hkv, layer=1):
    """The cache on the GPU, V of the spans of sequence 0 (whole blocks) written as zeros by an append, and c as it then is."""
    p = T.to_gpu(c)
    r = np.random.default_rng(77)
    for a, b in spans:
        k = torch.from_numpy(r.standard_normal((b - a, Hkv, hd))).to(T.DEV, torch.bfloat16)
        p.append(layer, k, torch.zeros_like(k), T.ints([0]), T.ints([0, b - a]), T.ints([a]), b - a)
    got = T.from_gpu(p)
    for x in T.NAMES:
        c[x] = got[x]
    for a, b in spans:
        assert (c["v_scale"][layer, c["table"][0, a // ps:-(-b // ps)]] == 2.0 ** -126).all()
    assert p.last_error() == 0
    return p


WHERE = {
    "first page": lambda ps: [(0, ps)],
    "first 128": lambda ps: [(0, 128)],
    "first 256": lambda ps: [(0, 256)],
    "middle": lambda ps: [(256, 512)],
    "every other page": lambda ps: [(a, a + ps) for a in range(0, LENGTH - ps, 2 * ps)],
    "all but the end": lambda ps: [(0, LENGTH // ps * ps)],
}


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [1, 8, 16, 40, 64, 100, 300])
@pytest.mark.parametrize("where", WHERE)
@pytest.mark.parametrize("hd,ps,H,Hkv", SHAPES)
def test_attention_where_pages_of_v_are_zeros(hd, ps, H, Hkv, where, rows, dtype):
    """check_attention's bounds as they are: zeros are exact, and their positions' weights count whole in the sum."""
    c = T.make([LENGTH, 90], Hkv=Hkv, ps=ps, hd=hd, seed=21)
    p = zeroed(c, WHERE[where](ps), ps=ps, hd=hd, Hkv=Hkv)
    T.check_attention(c, p, 1, T.queries(rows + 2, H, hd, rows), [0, rows, rows + 2], [LENGTH, 90], dtype=dtype)
    assert p.last_error() == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [1, 6, 40])
@pytest.mark.parametrize("span", [(0, 64), (2048, 7040), (0, 8960), (4096, 8192)])
def test_attention_where_a_long_stretch_of_v_is_zeros(span, rows, dtype):
    """The stretch spans CTAs: some of them see nothing else."""
    c = T.make([9000, 40], L=1, Hkv=2, ps=64, hd=64, seed=22)
    p = zeroed(c, [span], ps=64, hd=64, Hkv=2, layer=0)
    T.check_attention(c, p, 0, T.queries(rows + 1, 4, 64, 3), [0, rows, rows + 1], [9000, 40], dtype=dtype)


def test_attention_where_all_of_v_is_zeros():
    for dtype in ("bf16", "fp32"):
        for rows in (1, 20, 70, 200):
            c = T.make([LENGTH, 90], Hkv=2, ps=64, hd=64, seed=23)
            p = zeroed(c, [(0, LENGTH)], ps=64, hd=64, Hkv=2)
            out = T.check_attention(c, p, 1, T.queries(rows, 4, 64, 3), [0, rows], [LENGTH], dtype=dtype)
            assert (out == 0).all()


def test_positions_of_zeros_keep_weights_far_below_the_largest():
    """One page's scores are up to 2^18 times (in weight) those of 255 pages, whose V is zero; its own V is large.  The others' weights are
    most of the sum, a part of it, or a thousandth."""
    ps, hd, H, Hkv = 16, 64, 2, 1
    for above in (0.0, 5.0, 10.0, 18.0):
        c = T.make([4096], L=1, Hkv=Hkv, ps=ps, hd=hd, seed=24)
        c["k"][:], c["k_scale"][:] = 0, 1.0
        page = c["table"][0, 100]
        c["v"][:], c["v_scale"][:] = 0, 2.0 ** -126
        c["v"][0, page], c["v_scale"][0, page] = O.encode(np.full((Hkv, ps, hd), 448.0)), 2.0 ** 7
        c["k"][0, page, :, :, 0] = O.encode(np.full((Hkv, ps), 8.0))
        q = np.zeros((20, H, hd))
        q[..., 0] = above * np.log(2.0) / 8.0                 # rounded to bf16 with the others
        p = T.to_gpu(c)
        for dtype in ("bf16", "fp32"):
            for rows in (1, 20):
                T.check_attention(c, p, 0, q[:rows], [0, rows], [4096], dtype=dtype, scale=1.0)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [1, 12, 40, 100, 300])
@pytest.mark.parametrize("small,large", [(-126, -6), (-90, -6), (-70, -62), (-126, 20), (-72, 0), (-80, -75), (-64, -56), (-45, 30)])
def test_attention_over_v_of_very_different_sizes(small, large, rows, dtype):
    """check_attention's bounds (its header); V of a scale below 2^-72 (448 2^-72 at most) counts as zero."""
    hd, ps, H, Hkv = 64, 16, 4, 2
    c = T.make([LENGTH], Hkv=Hkv, ps=ps, hd=hd, seed=25)
    r = np.random.default_rng(abs(small) + rows)
    mantissa = r.choice([1.0, 1.0, 1.375], c["v_scale"].shape)
    c["v_scale"] = (np.where(r.random(c["v_scale"].shape) < 0.7, 2.0 ** small, 2.0 ** large) * mantissa).astype(np.float32)
    c["v_scale"][1, c["table"][0, :4]] = 2.0 ** small
    p = T.to_gpu(c)
    q = torch.from_numpy(T.queries(rows, H, hd, rows)).to(T.DEV, T.TYPES[dtype])
    out = torch.empty_like(q)
    p.attention(1, q, out, None, T.ints([0, rows]), T.ints([LENGTH]), rows, scale=hd ** -0.5)
    assert p.last_error() == 0
    K, V = O.gather(c, 1, 0, LENGTH, "k"), O.gather(c, 1, 0, LENGTH, "v")
    want, size, terms = O.attention(q.double().cpu().numpy(), K, V, hd ** -0.5, O.seen(rows, LENGTH))
    weight = 2.0 ** -11 if dtype == "bf16" else 2.0 ** -22
    tol = T.HALF[dtype] * np.abs(want) + size * (weight + 2 * (terms + 8) * 2.0 ** -20 + 2.0 ** -22 + LENGTH * 2.0 ** -27) + (448 * 2.0 ** -72 if small < -72 else 0.0)
    bad = ~(np.abs(out.double().cpu().numpy() - want) <= tol)
    assert not bad.any(), (np.argwhere(bad)[:4].tolist(), out.double().cpu().numpy()[bad][:4], want[bad][:4], tol[bad][:4])
