"""What the paged-cache calls refuse on the host, before they touch a device (the addresses here are never dereferenced)."""
import ctypes as C

import pytest

from paper_2601_20357_b200 import binding as B

ADDR = 0x100000


def pages(**kw):
    p = B.TabedPages()
    for n in ("k", "v", "k_scale", "v_scale", "table", "ref", "err", "workspace"):
        setattr(p, n, ADDR)
    p.n_layers, p.n_pages, p.n_kv_heads, p.page_tokens, p.head_dim, p.n_seqs, p.max_pages, p.device = 2, 10, 2, 64, 64, 4, 8, 63
    for n, v in kw.items():
        setattr(p, n, v)
    return p


def new(**kw):
    t = B.TabedPagesNew()
    t.layer, t.n, t.n_tokens, t.max_new, t.dtype = 0, 2, 5, 3, B.DTYPE_BF16
    t.first = t.start = t.k = t.v = t.seq = ADDR
    t.kv_stride, t.n_axes, t.theta, t.positions = 128, 2, 1e4, ADDR
    t.sections[0], t.sections[1] = 20, 12
    t.q = t.q_out = ADDR
    t.n_heads, t.q_stride, t.q_out_stride = 4, 256, 256
    sections = kw.pop("sections", None)
    if sections:
        for i, x in enumerate(sections):
            t.sections[i] = x
    for n, v in kw.items():
        setattr(t, n, v)
    return t


def query(**kw):
    t = B.TabedPagesQuery()
    t.layer, t.n, t.n_tokens, t.max_new, t.dtype, t.n_heads = 0, 2, 5, 3, B.DTYPE_BF16, 4
    t.first = t.length = t.q = t.out = t.seq = ADDR
    t.q_stride = t.out_stride = 256
    t.scale = 0.125
    for n, v in kw.items():
        setattr(t, n, v)
    return t


BAD_PAGES = [dict(k=0), dict(v=0), dict(k_scale=0), dict(table=0), dict(ref=0), dict(err=0), dict(workspace=0)]
BAD_SIZES = [dict(page_tokens=48), dict(page_tokens=0), dict(page_tokens=256), dict(head_dim=96), dict(head_dim=256), dict(n_layers=0), dict(n_pages=0),
             dict(n_kv_heads=0), dict(n_seqs=0), dict(n_seqs=32768), dict(max_pages=0), dict(device=-1), dict(device=64), dict(k=ADDR + 8), dict(v=ADDR + 1),
             dict(workspace=ADDR + 4), dict(max_pages=1 << 26)]


@pytest.mark.parametrize("kw,code", [(k, -2) for k in BAD_PAGES] + [(k, -1) for k in BAD_SIZES])
def test_every_call_refuses_bad_caches(kw, code):
    L, p = B.lib(), C.byref(pages(**kw))
    assert L.tabed_pages_fork(p, ADDR, ADDR, ADDR, ADDR, 1) == code
    assert L.tabed_pages_append(p, C.byref(new())) == code
    assert L.tabed_pages_attention(p, C.byref(query())) == code
    assert L.tabed_pages_compact(p, ADDR, ADDR, ADDR, ADDR, 1, 1) == code


def test_null_pointers():
    L, p = B.lib(), C.byref(pages())
    n = C.c_size_t()
    assert L.tabed_pages_workspace(None, C.byref(n)) == -2 and L.tabed_pages_workspace(p, None) == -2 and L.tabed_pages_last_error(None) == -2
    assert L.tabed_pages_store_row(None, p, 0, 0, 0, 1) == -2 and L.tabed_pages_load_row(None, p, 0, 0, 1) == -2
    for i in range(4):
        a = [ADDR] * 4
        a[i] = None
        assert L.tabed_pages_fork(p, *a, 1) == -2 and L.tabed_pages_compact(p, *a, 1, 1) == -2
    assert L.tabed_pages_append(p, None) == -2 and L.tabed_pages_attention(p, None) == -2
    for f in ("first", "start", "k", "v", "positions", "q_out"):
        assert L.tabed_pages_append(p, C.byref(new(**{f: 0}))) == -2, f
    for f in ("first", "length", "q", "out"):
        assert L.tabed_pages_attention(p, C.byref(query(**{f: 0}))) == -2, f


@pytest.mark.parametrize("kw", [dict(layer=-1), dict(layer=2), dict(n=-1), dict(n=5), dict(n_tokens=-1), dict(max_new=-1), dict(max_new=513), dict(dtype=2),
                                dict(dtype=-1), dict(kv_stride=127), dict(n_axes=-1), dict(n_axes=5), dict(sections=(20, 13)), dict(sections=(-1, 33)),
                                dict(sections=(33, -1)), dict(n_axes=1), dict(theta=0.0), dict(theta=-1.0), dict(theta=float("nan")), dict(theta=float("inf")),
                                dict(n_heads=0), dict(q_stride=255), dict(q_out_stride=0), dict(k=ADDR + 1), dict(q=ADDR + 1), dict(dtype=0, v=ADDR + 2)])
def test_append_refuses(kw):
    assert B.lib().tabed_pages_append(C.byref(pages()), C.byref(new(**kw))) == -1


@pytest.mark.parametrize("kw", [dict(layer=-1), dict(layer=2), dict(n=-1), dict(n_tokens=-1), dict(max_new=-1), dict(dtype=2), dict(n_heads=0), dict(n_heads=3),
                                dict(q_stride=255), dict(out_stride=128), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")),
                                dict(softcap=-1.0), dict(softcap=float("nan")), dict(softcap=float("inf")), dict(q=ADDR + 1), dict(dtype=0, out=ADDR + 2),
                                dict(tree=ADDR, slopes=ADDR), dict(tree=ADDR, max_new=65), dict(tree=ADDR + 4)])
def test_attention_refuses(kw):
    assert B.lib().tabed_pages_attention(C.byref(pages()), C.byref(query(**kw))) == -1


def test_fork_and_compact_refuse_counts():
    L, p = B.lib(), C.byref(pages())
    for n in (-1, 5):
        assert L.tabed_pages_fork(p, ADDR, ADDR, ADDR, ADDR, n) == -1
        assert L.tabed_pages_compact(p, ADDR, ADDR, ADDR, ADDR, n, 1) == -1
    assert L.tabed_pages_compact(p, ADDR, ADDR, ADDR, ADDR, 1, -1) == -1


def test_nothing_to_do_is_done():
    L, p = B.lib(), C.byref(pages())
    assert L.tabed_pages_fork(p, ADDR, ADDR, ADDR, ADDR, 0) == 0
    assert L.tabed_pages_compact(p, ADDR, ADDR, ADDR, ADDR, 0, 4) == 0 and L.tabed_pages_compact(p, ADDR, ADDR, ADDR, ADDR, 1, 0) == 0
    for kw in (dict(n=0), dict(n_tokens=0), dict(max_new=0)):
        assert L.tabed_pages_append(p, C.byref(new(**kw))) == 0
        assert L.tabed_pages_attention(p, C.byref(query(**kw))) == 0


def test_nothing_to_do_needs_no_arrays():
    """The pointer of an empty tensor is null."""
    L, p = B.lib(), C.byref(pages())
    none = [None] * 4
    assert L.tabed_pages_fork(p, *none, 0) == 0 and L.tabed_pages_compact(p, *none, 0, 4) == 0
    assert L.tabed_pages_compact(p, ADDR, ADDR, ADDR, None, 1, 0) == 0
    for kw in (dict(n=0), dict(n_tokens=0), dict(max_new=0)):
        assert L.tabed_pages_append(p, C.byref(new(**kw, k=0, v=0, q=0, q_out=0, positions=0))) == 0
        assert L.tabed_pages_attention(p, C.byref(query(**kw, q=0, out=0))) == 0
    assert L.tabed_pages_append(p, C.byref(new(n=0, layer=-1, k=0))) == -1 and L.tabed_pages_fork(p, *none, -1) == -1


def test_workspace_grows_with_the_sizes_it_depends_on():
    n = C.c_size_t()
    sizes = []
    for kw in (dict(), dict(head_dim=128), dict(n_seqs=30000, max_pages=5000)):
        assert B.lib().tabed_pages_workspace(C.byref(pages(**kw)), C.byref(n)) == 0
        sizes.append(n.value)
    assert sizes == sorted(sizes) and sizes[0] < sizes[1] < sizes[2]
    assert B.lib().tabed_pages_workspace(C.byref(pages(n_seqs=0)), C.byref(n)) == -1
