"""What the calls around a decode step refuse, on the host: nothing is launched here."""
import ctypes as C

import pytest


def _heads(b, **over):
    h = b.Heads(4096, 8192, 0, 512, 128, 0, 512, 128, None, 4)
    for k, v in over.items():
        setattr(h, k, v)
    return h


def _rotation(b, **over):
    r = b.Rotation(b.ROPE_HALVES, 128, 4096, 1e-6)
    for k, v in over.items():
        setattr(r, k, v)
    return r


def _pages(b, **over):
    p = b.Pages(4, 128, b.DTYPE_BF16, 10, 16, 1, 8, 4096, 8192, 4096)
    for k, v in over.items():
        setattr(p, k, v)
    return p


def test_struct_layouts_match_the_header(lazyev_lib):
    b = lazyev_lib
    assert C.sizeof(b.Heads) == 9 * 8 + 8 and C.sizeof(b.Rotation) == 8 + 8 + 8 and C.sizeof(b.Pages) == 7 * 4 + 4 + 3 * 8


def test_norm_rope(lazyev_lib):
    b = lazyev_lib

    def call(q=None, k=None, r=None, seqs=1, n=4, d=128, dtype=b.DTYPE_BF16, positions=None, no_rotation=False):
        return b.lib.lazyev_norm_rope(seqs, n, d, dtype, q, k, None if no_rotation else r or _rotation(b), positions, 0, None)
    assert call() == b.EINVAL and call(_heads(b), no_rotation=True) == b.EINVAL
    assert call(_heads(b), n=0) == b.OK and call(_heads(b, rows=None, to=None), seqs=0) == b.OK      # nothing to do
    for bad in (dict(seqs=-1), dict(n=-1), dict(d=96), dict(d=0), dict(dtype=2), dict(seqs=1 << 20, n=1 << 20), dict(positions=4097)):
        assert call(_heads(b), **bad) == b.EINVAL, bad
    for bad in (dict(rows=None), dict(to=None), dict(n_heads=0), dict(rows=4097), dict(to=8193), dict(weight=4097), dict(seq_stride=1 << 50),
                dict(to_head_stride=-(1 << 50)), dict(n_heads=70000)):
        assert call(_heads(b, **bad)) == b.EINVAL and call(_heads(b), _heads(b, **bad)) == b.EINVAL, bad
    for bad in (dict(dims=24), dict(dims=0), dict(dims=144), dict(dims=-16), dict(inv_freq=None), dict(inv_freq=4098), dict(layout=3),
                dict(layout=-1)):
        assert call(_heads(b), r=_rotation(b, **bad)) == b.EINVAL, bad
    for eps in (-1.0, float("nan"), float("inf")):
        assert call(_heads(b, weight=4096), r=_rotation(b, eps=eps)) == b.EINVAL
        assert call(_heads(b), r=_rotation(b, eps=eps), n=0) == b.OK                                    # nothing is normed
    assert call(_heads(b), r=_rotation(b, dims=128), d=64) == b.EINVAL


BAD_PAGES = [dict(n_kv_heads=0), dict(head_dim=96), dict(dtype=7), dict(n_pages=0), dict(page_size=0), dict(page_size=(1 << 20) + 1),
             dict(n_seqs=0), dict(table_stride=0), dict(k_pages=None), dict(v_pages=None), dict(table=None), dict(k_pages=4104),
             dict(v_pages=8200), dict(table=4098), dict(n_kv_heads=-4), dict(n_pages=-1)]


def test_pages_append(lazyev_lib):
    b = lazyev_lib

    def call(p=None, start=0, n=4, k=None, v=None, r=None):
        return b.lib.lazyev_pages_append(p or _pages(b), start, n, k or _heads(b, to=None), v or _heads(b, to=None), r or _rotation(b), 0, None)
    assert call(n=0) == b.OK and call(start=128, n=0) == b.OK
    assert b.lib.lazyev_pages_append(None, 0, 4, _heads(b), _heads(b), _rotation(b), 0, None) == b.EINVAL
    assert b.lib.lazyev_pages_append(_pages(b), 0, 4, None, _heads(b), _rotation(b), 0, None) == b.EINVAL
    assert b.lib.lazyev_pages_append(_pages(b), 0, 4, _heads(b), _heads(b), None, 0, None) == b.EINVAL
    for bad in BAD_PAGES:
        assert call(_pages(b, **bad)) == b.EINVAL, bad
    for bad in (dict(start=-1), dict(n=-1), dict(start=125), dict(n=129), dict(start=2 ** 31 - 1, n=2 ** 31 - 1)):
        assert call(**bad) == b.EINVAL, bad
    for bad in (dict(n_heads=3), dict(n_heads=5), dict(rows=None)):
        assert call(k=_heads(b, **bad)) == b.EINVAL and call(v=_heads(b, **bad)) == b.EINVAL, bad
    assert call(v=_heads(b, weight=4096)) == b.EINVAL
    assert call(r=_rotation(b, dims=20)) == b.EINVAL


def test_pages_attend(lazyev_lib):
    b = lazyev_lib
    ws = b.lib.lazyev_pages_attend_workspace(_pages(b), 100, 4, 28)

    def call(p=None, length=100, n=4, heads=28, visible=None, q=4096, jo=None, jl=None, out=1 << 20, lse=None, scale=0.0, w=1 << 24, wb=None):
        return b.lib.lazyev_pages_attend(p or _pages(b), length, n, heads, visible, q, jo, jl, out, lse, scale, w, ws if wb is None else wb, None)
    assert call(n=0) == b.OK and call(n=0, q=None, out=None) == b.OK
    assert b.lib.lazyev_pages_attend(None, 1, 1, 4, None, 4096, None, None, 8192, None, 0.0, None, 0, None) == b.EINVAL
    assert b.lib.lazyev_pages_attend_workspace(None, 1, 1, 4) == 0
    for bad in BAD_PAGES:
        assert call(_pages(b, **bad)) == b.EINVAL, bad
        assert b.lib.lazyev_pages_attend_workspace(_pages(b, **bad), 100, 4, 28) == 0
    for bad in (dict(length=-1), dict(length=129), dict(n=-1), dict(heads=0), dict(heads=27), dict(heads=4 * 65), dict(q=None), dict(out=None),
                dict(out=4096), dict(q=4097), dict(out=(1 << 20) + 1), dict(visible=4097), dict(lse=4098), dict(jo=4096), dict(jl=4096),
                dict(jo=4097, jl=4096), dict(jo=4096, jl=4098), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(n=1 << 28)):
        assert call(**bad) == b.EINVAL, bad
    long = _pages(b, page_size=1 << 20)            # a context that several blocks share
    need = b.lib.lazyev_pages_attend_workspace(long, 1 << 20, 4, 28)
    if need:
        for bad in (dict(w=None), dict(wb=need - 1), dict(w=(1 << 24) + 16)):
            assert call(long, length=1 << 20, **{"wb": need, **bad}) == b.EWORKSPACE, bad


def test_shared_step_needs_a_context_and_a_prefix(lazyev_lib):
    b = lazyev_lib
    f = b.lib.lazyev_decode_step_shared
    assert f(None, 0, 1, 1, 1, 1, 1, _pages(b), 10, None, 0, None, None) == b.EINVAL
    assert f(None, 0, 1, 1, 1, 1, 1, None, 10, None, 0, None, None) == b.EINVAL


@pytest.mark.parametrize("size", [1, 2, 3, 7, 16, 24, 100, 127, 128, 1000, 4097, 1 << 20, (1 << 20) - 1, 699051])
def test_division_by_the_page_size(size):
    """The kernels' division: (n + floor(n magic / 2^32)) >> shift, for every place next to a multiple."""
    shift = 0
    while (1 << shift) < size:
        shift += 1
    magic = (((1 << shift) - size) << 32) // size + 1
    assert magic < 1 << 32
    n = set()
    for m in list(range(0, 200)) + [(1 << 30) // size - 1, (1 << 30) // size, ((1 << 31) - 1) // size]:
        n |= {x for x in (m * size - 1, m * size, m * size + 1) if 0 <= x < 1 << 31}
    for x in n:
        assert (x + (x * magic >> 32)) >> shift == x // size and x + (x * magic >> 32) < 1 << 32


def test_pools_of_more_rows_than_32_bits_number(lazyev_lib):
    b = lazyev_lib
    fits, beyond = dict(n_kv_heads=1 << 10, page_size=1 << 20, n_pages=4), dict(n_kv_heads=1 << 10, page_size=1 << 20, n_pages=5)
    for over, code in ((fits, b.OK), (beyond, b.EINVAL), (dict(n_kv_heads=65535, page_size=1 << 20, n_pages=0x7FFFFFFF), b.EINVAL)):
        pages, n = _pages(b, **over), over["n_kv_heads"]
        assert b.lib.lazyev_pages_attend(pages, 0, 0, n, None, None, None, None, None, None, 0.0, None, 0, None) == code, over
        heads = _heads(b, n_heads=n)
        if 2 * n <= 65535:
            assert b.lib.lazyev_pages_append(pages, 0, 0, heads, heads, _rotation(b), 0, None) == code, over


def test_more_blocks_than_a_launch_has(lazyev_lib):
    b = lazyev_lib
    for seqs, code in ((1 << 20, b.OK), ((1 << 20) + 1, b.EINVAL)):
        pages = _pages(b, n_seqs=seqs)
        assert b.lib.lazyev_pages_attend(pages, 1, 0, 4, None, None, None, None, None, None, 0.0, None, 0, None) == code
