"""What the decoding entry points refuse on the host, before anything is launched; no GPU."""
import ctypes as C

import pytest
import torch

from paper_2609_31395_b200 import binding as B

P = C.c_void_p(1 << 20)          # a well-aligned address that is never read
ODD = C.c_void_p((1 << 20) + 2)
N = C.c_void_p(None)


def _pool(**kw):
    d = dict(base=1 << 20, n_layers=4, n_pages=10, page_size=16, n_kv_heads=2, head_dim=64, stride_layer=81920, stride_kv=40960,
             stride_page=2048, stride_slot=128, stride_head=64)
    d.update(kw)
    return B.PoolDesc(**d)


def _tab(**kw):
    d = dict(n_req=2, max_pages=4, page_table=1 << 20, seq_len=1 << 20, free_list=1 << 20, free_count=1 << 20)
    d.update(kw)
    return B.TablesDesc(**d)


def _attend(pool=None, tab=None, l0=0, l1=1, q=P, win=P, hq=8, left=0, out=C.c_void_p(1 << 21), rows=4, max_win=2, max_tok=50,
            ws=P, ws_bytes=None):
    lib, pool, tab = B.load(), pool or _pool(), tab or _tab()
    if ws_bytes is None:
        ws_bytes = lib.actkv_attend_workspace_bytes(pool, max(0, tab.n_req), max(0, l1 - l0), max(1, hq), max(0, max_win), max(0, max_tok))
    return lib.actkv_attend(pool, tab, l0, l1, q, win, hq, 0.1, 1, left, out, N, rows, max_win, max_tok, ws, ws_bytes, N, N)


@pytest.mark.parametrize("kw", [
    dict(pool=_pool(base=0)), dict(pool=_pool(base=(1 << 20) + 8)), dict(pool=_pool(head_dim=12)), dict(pool=_pool(head_dim=264)),
    dict(pool=_pool(page_size=0)), dict(pool=_pool(stride_slot=100)), dict(pool=_pool(stride_kv=4)), dict(pool=_pool(n_pages=0)),
    dict(l0=3, l1=5), dict(l0=2, l1=1), dict(l0=-1), dict(hq=7), dict(hq=0), dict(hq=66), dict(q=N), dict(q=ODD), dict(out=ODD),
    dict(out=P), dict(win=N), dict(rows=-1), dict(max_win=0), dict(max_win=-1), dict(max_tok=-1), dict(left=-1),
    dict(tab=_tab(n_req=-1)), dict(tab=_tab(seq_len=0)), dict(tab=_tab(page_table=0))])
def test_attend_refuses(kw):
    assert _attend(**kw) == B.E_INVALID


def test_attend_refuses_a_short_workspace_and_takes_empty_calls():
    assert _attend(ws_bytes=100) == B.E_WORKSPACE
    assert _attend(ws=N) == B.E_WORKSPACE
    assert _attend(rows=0) == B.OK and _attend(l1=0) == B.OK and _attend(tab=_tab(n_req=0)) == B.OK
    assert B.actkv_attend_workspace_bytes(_pool(), 2, 1, 8, 2, 50) > 0


def test_sizes_beyond_the_index_types_are_refused():
    assert _attend(max_tok=(1 << 30) + 1) == B.E_TOOBIG
    assert _attend(max_win=1 << 23, rows=1 << 23) == B.E_TOOBIG
    assert _attend(tab=_tab(n_req=4096), max_tok=1 << 30) == B.E_TOOBIG
    assert B.load().actkv_resize(_pool(), _tab(n_req=1 << 16, max_pages=1 << 16), P, N, N) == B.E_TOOBIG


def test_attend_workspace_of_a_layer_range_serves_fewer_layers():
    size = [B.actkv_attend_workspace_bytes(_pool(), 3, n, 8, 5, 50) for n in (1, 2, 4)]
    assert size == sorted(size)


def _rows(**kw):
    d = dict(base=1 << 20, stride_layer=4096, stride_row=512, stride_head=64)
    d.update(kw)
    return B.RowsDesc(**d)


def _rope(**kw):
    d = dict(rotary_dim=64, interleaved=0, n_axes=2, section=(C.c_int32 * 4)(12, 20, 0, 0), inv_freq=1 << 20)
    d.update(kw)
    return B.RopeDesc(**d)


def _append(pool=None, tab=None, l0=0, l1=1, q=_rows(), k=_rows(), v=_rows(), win=P, hq=8, rope=_rope(), pos=P, out=P, rows=4):
    return B.load().actkv_append(pool or _pool(), tab or _tab(), l0, l1, q, k, v, win, hq, rope, pos, out, rows, N, N)


@pytest.mark.parametrize("kw", [
    dict(pool=_pool(base=0)), dict(pool=_pool(head_dim=12)), dict(l1=5), dict(k=None), dict(v=None), dict(win=N), dict(out=N),
    dict(hq=0), dict(rows=-1), dict(pos=N), dict(rope=_rope(rotary_dim=63)), dict(rope=_rope(rotary_dim=66)),
    dict(rope=_rope(n_axes=0)), dict(rope=_rope(n_axes=5)), dict(rope=_rope(section=(C.c_int32 * 4)(12, 19, 0, 0))),
    dict(rope=_rope(section=(C.c_int32 * 4)(-1, 33, 0, 0))), dict(rope=_rope(inv_freq=0)), dict(k=_rows(base=0)),
    dict(tab=_tab(page_table=0))])
def test_append_refuses(kw):
    assert _append(**kw) == B.E_INVALID


def test_append_takes_empty_calls():
    assert _append(rows=0) == B.OK and _append(l1=0) == B.OK and _append(tab=_tab(n_req=0)) == B.OK


def test_resize_and_copy_refuse():
    lib = B.load()
    assert lib.actkv_resize(None, _tab(), P, N, N) == B.E_INVALID
    assert lib.actkv_resize(_pool(page_size=0), _tab(), P, N, N) == B.E_INVALID
    assert lib.actkv_resize(_pool(), _tab(), N, N, N) == B.E_INVALID
    assert lib.actkv_resize(_pool(), _tab(free_list=0), P, N, N) == B.E_INVALID
    assert lib.actkv_resize(_pool(), _tab(n_req=0), P, N, N) == B.OK
    copy = lambda pool=_pool(), tab=_tab(), l0=0, l1=1, src=P, n=2, m=9: lib.actkv_copy(pool, tab, l0, l1, src, P, P, n, m, N, N)
    assert copy(pool=_pool(base=0)) == copy(l1=5) == copy(src=N) == copy(n=-1) == copy(m=-1) == B.E_INVALID
    assert copy(tab=_tab(seq_len=0)) == B.E_INVALID
    assert copy(n=65536) == B.E_TOOBIG
    assert copy(n=0) == copy(m=0) == copy(l1=0) == B.OK


def test_logprob_refuses():
    lib = B.load()

    def call(z=P, dtype=0, n=2, vocab=100, stride=100, given=P, n_given=1, k=5, lp=P, tl=P, ti=P):
        return lib.actkv_logprob(z, dtype, n, vocab, stride, given, n_given, k, lp, P, P, tl, ti, N, N)
    bad = [dict(z=N), dict(z=ODD), dict(dtype=2), dict(n=-1), dict(vocab=0), dict(stride=99), dict(given=N), dict(n_given=-1),
           dict(k=-1), dict(k=65), dict(lp=N), dict(tl=N), dict(ti=N)]
    assert [call(**kw) for kw in bad] == [B.E_INVALID] * len(bad)
    assert call(n=0) == B.OK and call(n=1 << 30) == B.E_TOOBIG


def test_the_binding_refuses_cpu_tensors_and_wrong_shapes():
    z = torch.zeros(2, 10)
    with pytest.raises(TypeError):
        B.actkv_logprob(z, None, None, None, None, None, None, None)
    with pytest.raises(TypeError):
        B.rows_desc(torch.zeros(1, 2, 3, 8, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        B.rope_desc(None, [1, 1, 1, 1, 1])
    with pytest.raises(ValueError):
        B.rope_desc(torch.zeros(3), [1, 1])
    with pytest.raises(TypeError):
        B.rope_desc(torch.zeros(2), [1, 1])
