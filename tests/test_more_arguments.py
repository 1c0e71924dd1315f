"""What actkv_reposition, actkv_penalize and actkv_sample refuse on the host, before anything is launched; no GPU."""
import ctypes as C

import pytest
import torch

from paper_2609_31395_b200 import binding as B
from paper_2609_31395_b200 import harness as H

P = C.c_void_p(1 << 20)          # a well-aligned address that is never read
ODD = C.c_void_p((1 << 20) + 1)
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


def _rope(**kw):
    d = dict(rotary_dim=64, interleaved=0, n_axes=2, section=(C.c_int32 * 4)(12, 20, 0, 0), inv_freq=1 << 20)
    d.update(kw)
    return B.RopeDesc(**d)


def _reposition(pool=None, tab=None, l0=0, l1=1, rope=_rope(), to_freq=N, frm=B.PositionsDesc(1 << 20, 0, 0), to=None, ind=P, sum_tok=50, max_tok=50):
    return B.load().actkv_reposition(pool or _pool(), tab or _tab(), l0, l1, rope, to_freq, frm, to, ind, sum_tok, max_tok, N, N)


@pytest.mark.parametrize("kw", [
    dict(pool=_pool(base=0)), dict(pool=_pool(head_dim=12)), dict(pool=_pool(head_dim=264)), dict(pool=_pool(page_size=0)),
    dict(pool=_pool(n_pages=0)), dict(pool=_pool(n_kv_heads=0)), dict(l1=5), dict(l0=2), dict(l0=-1), dict(rope=None), dict(rope=_rope(rotary_dim=63)),
    dict(rope=_rope(rotary_dim=66)), dict(rope=_rope(rotary_dim=-2)), dict(rope=_rope(n_axes=0)), dict(rope=_rope(n_axes=5)),
    dict(rope=_rope(section=(C.c_int32 * 4)(12, 19, 0, 0))), dict(rope=_rope(section=(C.c_int32 * 4)(-1, 33, 0, 0))), dict(rope=_rope(inv_freq=0)),
    dict(ind=N), dict(sum_tok=-1), dict(max_tok=-1), dict(tab=_tab(n_req=-1)), dict(tab=_tab(seq_len=0)), dict(tab=_tab(page_table=0)),
    dict(tab=_tab(max_pages=-1))])
def test_reposition_refuses(kw):
    assert _reposition(**kw) == B.E_INVALID


def test_reposition_takes_calls_that_move_nothing():
    assert _reposition(l1=0) == _reposition(tab=_tab(n_req=0)) == _reposition(max_tok=0) == B.OK
    assert _reposition(frm=None) == _reposition(frm=B.PositionsDesc(0, 7, 7)) == B.OK
    assert _reposition(rope=_rope(rotary_dim=0, n_axes=1, section=(C.c_int32 * 4)(0, 0, 0, 0), inv_freq=0)) == B.OK


def test_reposition_refuses_what_a_launch_cannot_hold():
    assert _reposition(tab=_tab(n_req=65536)) == B.E_TOOBIG
    assert _reposition(max_tok=(1 << 30) + 1) == B.E_TOOBIG
    assert _reposition(pool=_pool(n_layers=40000), l1=40000) == B.E_TOOBIG


def _rules(**kw):
    d = dict(tokens=1 << 20, token_stride=100, hist_len=1 << 20, repetition=1 << 20, bias_indptr=1 << 20, bias_token=1 << 20, bias_value=1 << 20,
             n_bias=4, allow=1 << 20, allow_stride=32, n_allow=5)
    d.update(kw)
    return B.LogitRulesDesc(**d)


def _penalize(z=P, dtype=0, vocab=1000, stride=1000, win=P, n_req=2, rows=4, max_win=2, max_hist=90, rules=_rules(), out=P, out_stride=1000):
    return B.load().actkv_penalize(z, dtype, vocab, stride, win, n_req, rows, max_win, max_hist, rules, out, out_stride, N, N)


@pytest.mark.parametrize("kw", [
    dict(z=N), dict(z=ODD), dict(out=N), dict(out=ODD), dict(dtype=2), dict(dtype=-1), dict(vocab=0), dict(stride=999), dict(out_stride=999),
    dict(out_stride=1001), dict(win=N), dict(n_req=-1), dict(rows=-1), dict(max_win=-1), dict(max_win=0), dict(max_hist=-1), dict(rules=None),
    dict(rules=_rules(hist_len=0)), dict(rules=_rules(token_stride=-1)), dict(rules=_rules(bias_token=0)), dict(rules=_rules(bias_value=0)),
    dict(rules=_rules(n_bias=-1)), dict(rules=_rules(allow_stride=31)), dict(rules=_rules(n_allow=-1))])
def test_penalize_refuses(kw):
    assert _penalize(**kw) == B.E_INVALID


def test_penalize_takes_empty_calls():
    assert _penalize(n_req=0) == _penalize(rows=0) == B.OK
    assert _penalize(max_hist=1 << 30) == B.E_TOOBIG
    assert _penalize(n_req=0x7fffffff, vocab=100000, stride=100000, out_stride=100000, rules=_rules(allow=0)) == B.E_TOOBIG


def _sample(z=P, dtype=0, n=2, vocab=100, stride=100, u=P, token=P):
    return B.load().actkv_sample(z, dtype, n, vocab, stride, u, P, P, P, P, token, P, P, N, N)


def test_sample_refuses():
    bad = [dict(z=N), dict(z=ODD), dict(dtype=2), dict(n=-1), dict(vocab=0), dict(vocab=-3), dict(stride=99), dict(u=N), dict(token=N)]
    assert [_sample(**kw) for kw in bad] == [B.E_INVALID] * len(bad)
    assert _sample(n=0) == B.OK
    assert _sample(vocab=344065, stride=344065) == _sample(n=(1 << 27) + 1) == B.E_TOOBIG


def test_the_binding_refuses_cpu_tensors():
    z = torch.zeros(2, 10)
    with pytest.raises(TypeError):
        B.actkv_sample(z, None, None, None, None, None, None, None, None, None)
    with pytest.raises(TypeError):
        B.actkv_penalize(z, None, 1, B.LogitRulesDesc(), 1, 1, z, None)
    with pytest.raises(TypeError):
        B.actkv_reposition(_pool(), _tab(), 0, 1, _rope(), None, None, None, torch.zeros(3, dtype=torch.int32), 5, None)
    with pytest.raises(TypeError):
        H.LogitRules(torch.zeros((1, 4), dtype=torch.int32), torch.zeros(1, dtype=torch.int32))


def test_positions_of_every_shape():
    t = lambda *s: torch.zeros(s, dtype=torch.int32)
    get = lambda x, a=2, u=6: (lambda d: (d[0].stride_axis, d[0].stride_unit, d[1]))(B.positions_desc(x, a, u))
    assert get(t(9)) == (0, 0, 9) and get(t(2, 9)) == (9, 0, 9) and get(t(1, 9)) == (0, 0, 9)
    assert get(t(2, 6, 9)) == (54, 9, 9) and get(t(1, 6, 9)) == (0, 9, 9) and get(t(2, 1, 9)) == (9, 0, 9)
    assert get(t(2, 8, 9)[:, 1:7, 2:]) == (72, 9, 7) and get(t(9)[None].expand(2, 9)) == (0, 0, 9)
    for bad in (t(3, 9), t(2, 5, 9), t(1, 2, 6, 9), t(2, 6, 9).transpose(1, 2).contiguous().transpose(1, 2)):
        with pytest.raises((ValueError, TypeError)):
            get(bad)
    with pytest.raises(TypeError):
        B.positions_desc(torch.zeros(9), 1, 1)
