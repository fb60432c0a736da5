"""The oracle of the paged 8-bit caches against independent restatements."""
import numpy as np
import torch

from oracle import pages as O


def test_codes_are_those_of_e4m3():
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(O.decode(np.arange(256)), want, equal_nan=True)


def test_encode_rounds_to_nearest_even_everywhere():
    pos = O.VALUES[:0x7F]
    mid = (pos[1:] + pos[:-1]) / 2
    x = np.concatenate([pos, mid, np.nextafter(mid, 0), np.nextafter(mid, 1e9), np.random.default_rng(1).uniform(0, 448, 2000)])
    x = np.concatenate([x, -x])
    want = torch.from_numpy(x.astype(np.float32)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    exact = x == x.astype(np.float32)                       # (the others lose their tie or side in fp32)
    assert np.array_equal(O.encode(x)[exact], want[exact])
    for code, v in zip(O.encode(x), np.abs(x)):
        assert abs(abs(O.VALUES[code]) - v) <= np.abs(pos - v).min()
    assert O.encode(np.inf) == 0x7E and O.encode(-1e9) == 0xFE and O.encode(np.nan) == 0x7F


def test_least_scale():
    for e in (-40, 0, 17):
        for a, s in ((448.0, 1.0), (np.nextafter(448.0, 1e9), 2.0), (224.0, 0.5), (225.0, 1.0), (300.0, 1.0)):
            assert O.least_scale(a * 2.0 ** e) == s * 2.0 ** e
    assert O.least_scale(0.0) == 2.0 ** -126 and O.least_scale(3.4e38) == 2.0 ** 120


def test_rotation_of_one_axis_depends_on_distance_alone():
    r = np.random.default_rng(2)
    q, k = r.standard_normal((1, 1, 32)), r.standard_normal((1, 1, 32))
    dot = [float((O.rotate(q, [[a]], (16,), 1e4) * O.rotate(k, [[b]], (16,), 1e4)).sum()) for a, b in ((5, 2), (1005, 1002), (3, 0))]
    assert np.allclose(dot, dot[0], rtol=1e-12)


def test_rotation_sections_follow_their_axis():
    x = np.random.default_rng(3).standard_normal((4, 2, 32))
    pos = np.array([[1, 2, 3, 4], [9, 8, 7, 6]])
    got = O.rotate(x, pos, (10, 6), 1e4)
    a, b = O.rotate(x, pos[:1], (16,), 1e4), O.rotate(x, pos[1:], (16,), 1e4)
    cols = lambda lo, hi: list(range(lo, hi)) + list(range(16 + lo, 16 + hi))
    assert np.array_equal(got[..., cols(0, 10)], a[..., cols(0, 10)]) and np.array_equal(got[..., cols(10, 16)], b[..., cols(10, 16)])


def test_attention_against_torch():
    r = np.random.default_rng(4)
    q, K, V = r.standard_normal((3, 4, 32)), r.standard_normal((2, 9, 32)), r.standard_normal((2, 9, 32))
    mask = O.seen(3, 9, prefix=0)
    got, _, _ = O.attention(q, K, V, 0.2, mask)
    rep = lambda x: torch.from_numpy(np.repeat(x, 2, axis=0))
    want = torch.nn.functional.scaled_dot_product_attention(torch.from_numpy(q).transpose(0, 1), rep(K), rep(V), attn_mask=torch.from_numpy(mask), scale=0.2)
    assert np.allclose(got, want.transpose(0, 1).numpy(), atol=1e-12)


def test_masks():
    assert O.seen(2, 4).tolist() == [[1, 1, 1, 0], [1, 1, 1, 1]]
    assert O.seen(2, 4, prefix=4).all()
    assert O.seen(3, 2).tolist() == [[0, 0], [1, 0], [1, 1]]           # more rows than tokens: the first sees nothing
    assert O.seen(3, 4, tree=[1, 3, 5]).tolist() == [[1, 1, 0, 0], [1, 1, 1, 0], [1, 1, 0, 1]]
    assert O.seen(64, 64, tree=[-1] * 64).all()


def _cache(pages, seqs, blocks, ps=16, L=1, Hkv=1, hd=32, seed=0):
    r = np.random.default_rng(seed)
    c = {x: O.encode(r.standard_normal((L, pages, Hkv, ps, hd)) * 50) for x in ("k", "v")}
    c |= {x: (2.0 ** r.integers(-3, 3, (L, pages, Hkv))).astype(np.float32) for x in ("k_scale", "v_scale")}
    c["table"], c["ref"] = np.full((seqs, blocks), -1, np.int32), np.zeros(pages, np.int32)
    return c


def test_fork_shares_copies_and_frees():
    c = _cache(10, 3, 4)
    assert O.fork(c, [0], [0], [0], [40])
    assert c["table"][0].tolist() == [0, 1, 2, -1] and c["ref"].tolist()[:4] == [1, 1, 1, 0]
    assert O.fork(c, [0], [1], [20], [33])
    assert c["table"][1].tolist() == [0, 3, 4, -1] and c["ref"].tolist()[:5] == [2, 1, 1, 1, 1]
    assert np.array_equal(O.gather(c, 0, 1, 20, "k"), O.gather(c, 0, 0, 20, "k"))
    # cut inside a shared page: it becomes a copy; at a page of its own it stays
    assert O.fork(c, [1, 0], [1, 0], [5, 20], [6, 40])
    assert c["table"][1].tolist()[1:] == [-1, -1, -1] and c["table"][1, 0] == 2      # (given back by sequence 0 in this call)
    assert c["table"][0].tolist()[:2] == [0, 1]
    # the two change places
    a, b = O.gather(c, 0, 0, 20, "v"), O.gather(c, 0, 1, 5, "v")
    assert O.fork(c, [0, 1], [1, 0], [20, 5], [20, 5])
    assert np.array_equal(O.gather(c, 0, 1, 20, "v"), a) and np.array_equal(O.gather(c, 0, 0, 5, "v"), b)
    assert O.fork(c, [0, 1], [0, 1], [0, 0], [0, 0]) and not c["ref"].any() and (c["table"] == -1).all()


def test_appending_in_pieces_is_appending_at_once_but_for_subnormals():
    r = np.random.default_rng(7)
    x = r.standard_normal((30, 1, 32)) * np.exp2(r.integers(-2, 3, (30, 1, 1)))
    one, two = _cache(4, 1, 4), _cache(4, 1, 4)
    for c, cuts in ((one, [0, 30]), (two, [0, 1, 2, 3, 9, 17, 18, 30])):
        O.fork(c, [0], [0], [0], [30])
        for a, b in zip(cuts, cuts[1:]):
            O.append(c, 0, x[a:b], x[a:b], [0], [0, b - a], [a])
    a, b = O.gather(one, 0, 0, 30, "k"), O.gather(two, 0, 0, 30, "k")
    assert np.array_equal(one["k_scale"], two["k_scale"])
    assert np.abs(a - b).max() <= one["k_scale"].max() * 2.0 ** -9      # (a subnormal's step)


def test_compact_moves_the_tokens_that_are_kept():
    c = _cache(6, 1, 6)
    O.fork(c, [0], [0], [0], [90])
    before = O.gather(c, 0, 0, 90, "k")
    keep = [20, 21, 25, 40, 41, 60, 77, 89]
    O.compact(c, [0], [20], [len(keep)], [keep])
    after = O.gather(c, 0, 0, 90, "k")
    step = c["k_scale"].max() * 2.0 ** -9
    assert np.abs(after[:, 20:20 + len(keep)] - before[:, keep]).max() <= step / 2 and np.abs(after[:, :20] - before[:, :20]).max() <= step / 2
