"""What the calls around a long cache in pages refuse, on the host: nothing is launched here."""
import ctypes as C

import pytest

from test_pages_refusals import BAD_PAGES, _pages


def _blocks(b, **over):
    x = b.Blocks(4, 128, b.DTYPE_BF16, 1, 8, 16, 4096)
    for k, v in over.items():
        setattr(x, k, v)
    return x


BAD_BLOCKS = [dict(n_kv_heads=0), dict(n_kv_heads=-1), dict(n_kv_heads=70000), dict(head_dim=96), dict(head_dim=0), dict(dtype=2), dict(n_seqs=0),
              dict(n_blocks=0), dict(block=0), dict(block=24), dict(block=8), dict(block=256), dict(block=-16), dict(bounds=None), dict(bounds=4104),
              dict(n_seqs=1 << 21)]


def test_struct_layout_matches_the_header(lazyev_lib):
    assert C.sizeof(lazyev_lib.Blocks) == 6 * 4 + 8


def test_bound(lazyev_lib):
    b = lazyev_lib

    def call(p=None, x=None, start=0, n=4):
        return b.lib.lazyev_blocks_bound(p or _pages(b), x or _blocks(b), start, n, None)
    assert call(n=0) == b.OK and call(start=128, n=0) == b.OK
    assert b.lib.lazyev_blocks_bound(None, _blocks(b), 0, 4, None) == b.EINVAL
    assert b.lib.lazyev_blocks_bound(_pages(b), None, 0, 4, None) == b.EINVAL
    for bad in BAD_PAGES:
        assert call(_pages(b, **bad)) == b.EINVAL, bad
    for bad in BAD_BLOCKS + [dict(n_kv_heads=2), dict(head_dim=64), dict(dtype=b.DTYPE_FP32), dict(n_seqs=2)]:
        assert call(x=_blocks(b, **bad)) == b.EINVAL, bad
    for bad in (dict(start=-1), dict(n=-1), dict(start=125), dict(n=129), dict(start=2 ** 31 - 1, n=2 ** 31 - 1)):
        assert call(**bad) == b.EINVAL, bad
    assert call(x=_blocks(b, n_blocks=7), n=113) == b.EINVAL                      # no room in the bounds


def test_choose(lazyev_lib):
    b = lazyev_lib
    ws = b.lib.lazyev_blocks_choose_workspace(_blocks(b), 128, 4, 28, 1, 3)
    assert ws > 0

    def call(x=None, length=128, n=4, heads=28, visible=None, q=4096, first=1, last=1, chosen=3, to=8192, w=1 << 24, wb=None):
        return b.lib.lazyev_blocks_choose(x or _blocks(b), length, n, heads, visible, q, first, last, chosen, to, w, ws if wb is None else wb, None)
    assert call(n=0) == b.OK and call(n=0, q=None, to=None) == b.OK
    assert b.lib.lazyev_blocks_choose(None, 1, 1, 4, None, 4096, 0, 1, 1, 8192, None, 0, None) == b.EINVAL
    for bad in BAD_BLOCKS:
        assert call(_blocks(b, **bad)) == b.EINVAL, bad
        assert b.lib.lazyev_blocks_choose_workspace(_blocks(b, **bad), 128, 4, 28, 1, 3) == 0
    for bad in (dict(length=-1), dict(length=129), dict(n=-1), dict(heads=0), dict(heads=27), dict(heads=4 * 65), dict(q=None), dict(to=None),
                dict(q=4097), dict(to=8194), dict(visible=4097), dict(first=-1), dict(last=0), dict(first=2, last=2), dict(chosen=0),
                dict(chosen=(1 << 20) + 1), dict(n=1 << 28), dict(last=4)):
        assert call(**bad) == b.EINVAL, bad
    for bad in (dict(w=None), dict(wb=ws - 1), dict(w=(1 << 24) + 16)):
        assert call(**bad) == b.EWORKSPACE, bad
    assert b.lib.lazyev_blocks_choose_workspace(_blocks(b), 128, 4, 28, 1, 8) == 0  # nobody has to choose
    many = _blocks(b, n_seqs=1 << 10, n_kv_heads=1 << 10, n_blocks=1 << 20)
    assert b.lib.lazyev_blocks_choose(many, 1 << 24, 1, 1 << 10, None, 4096, 0, 1, 3, 8192, 1 << 24, 1 << 60, None) == b.EINVAL


def test_attend(lazyev_lib):
    b = lazyev_lib
    size = b.lib.lazyev_blocks_attend_workspace

    def call(p=None, length=100, block=16, m=4, list=4096, n=4, heads=28, visible=None, q=4096, jo=None, jl=None, out=1 << 20, lse=None, scale=0.0,
             w=1 << 24, wb=1 << 30):
        return b.lib.lazyev_blocks_attend(p or _pages(b), length, block, m, list, n, heads, visible, q, jo, jl, out, lse, scale, w, wb, None)
    assert call(n=0) == b.OK and call(n=0, q=None, out=None, list=None) == b.OK
    assert b.lib.lazyev_blocks_attend(None, 1, 16, 1, 4096, 1, 4, None, 4096, None, None, 8192, None, 0.0, None, 0, None) == b.EINVAL
    for bad in BAD_PAGES:
        assert call(_pages(b, **bad)) == b.EINVAL, bad
        assert size(_pages(b, **bad), 100, 16, 4, 4, 28) == 0
    for bad in (dict(length=-1), dict(length=129), dict(n=-1), dict(heads=0), dict(heads=27), dict(heads=4 * 65), dict(q=None), dict(out=None),
                dict(out=4096), dict(q=4097), dict(out=(1 << 20) + 1), dict(visible=4097), dict(lse=4098), dict(jo=4096), dict(jl=4096),
                dict(jo=4097, jl=4096), dict(jo=4096, jl=4098), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")),
                dict(list=None), dict(list=4098), dict(block=24), dict(block=0), dict(block=256), dict(m=0), dict(m=-1), dict(m=1 << 27), dict(n=1 << 21)):
        assert call(**bad) == b.EINVAL, bad
    need = size(_pages(b), 128, 128, 1000, 1, 28)
    assert need > 0
    for bad in (dict(w=None), dict(wb=need - 1), dict(w=(1 << 24) + 16)):
        assert call(length=128, block=128, m=1000, n=1, **{"wb": need, **bad}) == b.EWORKSPACE, bad
    # the row number 2^32 - 1 stands for none here
    assert call(_pages(b, n_kv_heads=1 << 10, page_size=1 << 20, n_pages=4), n=0, heads=1 << 10) == b.EINVAL
    assert call(_pages(b, n_kv_heads=1 << 10, page_size=1 << 20, n_pages=3), n=0, heads=1 << 10) == b.OK


def test_weigh(lazyev_lib):
    b = lazyev_lib
    ws = b.lib.lazyev_pages_weigh_workspace(_pages(b), 128, 64, 28)
    assert ws > 0

    def call(p=None, length=128, n=64, heads=28, visible=None, q=4096, lse=4096, scale=0.0, old=None, known=0, decay=1.0, to=8192, stride=128,
             w=1 << 24, wb=None):
        return b.lib.lazyev_pages_weigh(p or _pages(b), length, n, heads, visible, q, lse, scale, old, known, decay, to, stride, w,
                                        ws if wb is None else wb, None)
    assert call(length=0) == b.OK and call(length=0, q=None, to=None) == b.OK
    assert b.lib.lazyev_pages_weigh(None, 1, 1, 4, None, 4096, 4096, 0.0, None, 0, 1.0, 8192, 128, None, 0, None) == b.EINVAL
    for bad in BAD_PAGES:
        assert call(_pages(b, **bad)) == b.EINVAL, bad
        assert b.lib.lazyev_pages_weigh_workspace(_pages(b, **bad), 128, 64, 28) == 0
    nan, inf = float("nan"), float("inf")
    for bad in (dict(length=-1), dict(length=129, stride=129), dict(n=-1), dict(heads=0), dict(heads=27), dict(heads=4 * 65), dict(q=None), dict(lse=None),
                dict(to=None), dict(q=4097), dict(lse=4098), dict(to=8194), dict(visible=4097), dict(old=4098, known=1), dict(known=1), dict(known=-1),
                dict(known=129, old=4096), dict(stride=127), dict(stride=-1), dict(stride=1 << 50), dict(scale=-1.0), dict(scale=nan), dict(scale=inf),
                dict(decay=nan), dict(decay=inf), dict(n=1 << 28)):
        assert call(**bad) == b.EINVAL, bad
    for bad in (dict(w=None), dict(wb=ws - 1), dict(w=(1 << 24) + 16)):
        assert call(**bad) == b.EWORKSPACE, bad


def test_evict(lazyev_lib):
    b = lazyev_lib
    ws = b.lib.lazyev_pages_evict_workspace(_pages(b), 64)
    assert ws > 0 and b.lib.lazyev_pages_evict_workspace(None, 64) == 0 and b.lib.lazyev_pages_evict_workspace(_pages(b), 0) == 0

    def call(p=None, length=128, lengths=None, keep=64, recent=8, first=4, weights=4096, positions=None, stride=128, sources=4096, wt=8192, pt=8192,
             to_stride=64, w=1 << 24, wb=None):
        return b.lib.lazyev_pages_evict(p or _pages(b), length, lengths, keep, recent, first, weights, positions, stride, sources, wt, pt, to_stride, w,
                                        ws if wb is None else wb, None)
    assert b.lib.lazyev_pages_evict(None, 1, None, 1, 0, 0, 4096, None, 1, 4096, None, None, 1, 1 << 24, 256, None) == b.EINVAL
    for bad in BAD_PAGES:
        assert call(_pages(b, **bad)) == b.EINVAL, bad
        assert b.lib.lazyev_pages_evict_workspace(_pages(b, **bad), 64) == 0
    for bad in (dict(length=-1), dict(length=129, stride=129), dict(lengths=4097), dict(keep=0), dict(keep=-1), dict(recent=-1), dict(first=-1),
                dict(recent=65), dict(recent=61), dict(first=57), dict(weights=None), dict(weights=4098), dict(positions=4098), dict(stride=127),
                dict(stride=1 << 50), dict(sources=None), dict(sources=4098), dict(wt=8194), dict(pt=8194), dict(to_stride=63),
                dict(to_stride=1 << 50), dict(pt=None, to_stride=63)):
        assert call(**bad) == b.EINVAL, bad
    for bad in (dict(w=None), dict(wb=ws - 1), dict(w=(1 << 24) + 16)):
        assert call(**bad) == b.EWORKSPACE, bad
    assert call(_pages(b, n_seqs=1 << 20)) == b.EINVAL


def test_binding_needs_a_gpu_tensor(lazyev_lib):
    import torch
    with pytest.raises(ValueError):
        lazyev_lib.KeyBounds(torch.zeros(1, 2, 3, 2, 64), 16)
