"""actkv_resize and actkv_copy against the oracle: whole numbers and bytes, so everything is compared exactly."""
import numpy as np
import pytest
import torch

from oracle import actkv_oracle as O
from paper_2609_31395_b200 import binding as B
from paper_2609_31395_b200 import harness as H

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _decoder(lens, page=16, spare=20, width=None, seed=0, layers=1, hk=1, D=8, head_major=False, offset=0):
    need = [-(-n // page) for n in lens]
    n_pages = sum(need) + spare
    perm = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    width = max(need + [1]) if width is None else width
    pt = torch.full((len(lens), width), -1, dtype=torch.int32)
    at = 0
    for r, n in enumerate(need):
        pt[r, :n] = perm[at:at + n]
        at += n
    free = torch.full((n_pages,), -1, dtype=torch.int32)
    free[:spare] = perm[at:]
    shape = (layers, 2, n_pages, hk, page, D) if head_major else (layers, 2, n_pages, page, hk, D)
    pool = torch.randn(int(np.prod(shape)) + offset, device=DEV, generator=torch.Generator(device=DEV).manual_seed(seed))
    pool = pool.to(torch.bfloat16)[offset:].view(shape)
    if head_major:
        pool = pool.transpose(3, 4)
    return H.Decoder(pool, pt.to(DEV), _i32(lens), free.to(DEV), _i32([spare]), hk, layers_per_call=layers)


def _tables(d):
    return O.Tables(d.page_table.cpu().numpy().copy(), d.seq_len.cpu().numpy().copy(), d.free_list.cpu().numpy().copy(), int(d.free_count.cpu()))


def _same(a, b):
    assert np.array_equal(a.page_table, b.page_table) and np.array_equal(a.seq_len, b.seq_len)
    assert a.free_count == b.free_count and np.array_equal(a.free_list, b.free_list)


@pytest.mark.parametrize("lens,new,page", [
    ([0], [1], 16), ([5], [5], 16), ([16, 17], [17, 16], 16), ([100, 0, 33, 64], [0, 100, -1, 65], 16),
    ([100, 200, 300], [0, 0, 0], 16), ([1, 2, 3], [9, 0, 17], 1), ([50, 60], [71, 12], 7)])
def test_resize_by_hand_picked_lengths(lens, new, page):
    d = _decoder(lens, page, spare=40, width=80)
    want = O.resize(_tables(d), new, page)
    d.resize(_i32(new))
    d.check_status()
    _same(_tables(d), want)


@pytest.mark.parametrize("R,seed", [(7, 0), (64, 1), (300, 2), (1024, 3), (1025, 4), (2500, 5)])
def test_resize_of_many_requests(R, seed):
    g = np.random.default_rng(seed)
    lens, new = g.integers(0, 400, R).tolist(), g.integers(-60, 500, R).tolist()
    d = _decoder(lens, 16, spare=32 * R, width=32, seed=seed)
    want = O.resize(_tables(d), new, 16)
    d.resize(_i32(new))
    d.check_status()
    _same(_tables(d), want)
    # and back: what was popped last comes first
    d.resize(_i32(lens))
    d.check_status()
    assert d.seq_len.cpu().tolist() == lens
    used = torch.cat([d.page_table[d.page_table >= 0].flatten(), d.free_list[: int(d.free_count)]]).cpu()
    assert sorted(used.tolist()) == list(range(d.pd.n_pages))


def test_resize_is_all_or_nothing():
    def refused(change, code, lens=(100, 50), new=(200, 0), spare=3, width=14):
        d = _decoder(list(lens), 16, spare=spare, width=width)
        change(d)
        before = _tables(d)
        d.resize(_i32(list(new)))
        assert d.status.cpu().tolist()[0] == code
        _same(_tables(d), before)
    refused(lambda d: None, B.E_NOFREE)                                   # 6 pages wanted, 3 free, freed ones do not serve
    refused(lambda d: None, B.E_INVALID, new=(300, 0), spare=40)          # beyond the table row
    refused(lambda d: d.free_count.fill_(-1), B.E_INVALID)
    refused(lambda d: d.free_count.fill_(10 ** 6), B.E_INVALID)
    refused(lambda d: d.free_list.fill_(10 ** 6), B.E_BADPAGE, spare=40)
    refused(lambda d: d.page_table[1].fill_(-7), B.E_BADPAGE, new=(100, 0))
    refused(lambda d: d.seq_len.fill_(-3), B.E_INVALID)
    refused(lambda d: d.status.copy_(_i32([B.E_BADPAGE, 1, 2, 0])), B.E_BADPAGE, new=(100, 0))
    # a list that would not hold what is pushed (a page both free and in use)
    refused(lambda d: d.free_count.fill_(d.pd.n_pages), B.E_INVALID, new=(100, 0))


def test_resize_in_a_captured_graph():
    d = _decoder([0, 5], 16, spare=40, width=20)
    new = _i32([1, 6])
    g = torch.cuda.CUDAGraph()
    s = torch.cuda.Stream()
    with torch.cuda.graph(g, stream=s):
        d.resize(new)
    want = _tables(d)
    for step in range(1, 40):
        new.copy_(_i32([step * 7, 6 + step]))
        g.replay()
        want = O.resize(want, [step * 7, 6 + step], 16)
    d.check_status()
    _same(_tables(d), want)


def _expect_copy(d, pairs, l0, l1):
    want = d.pool.clone()
    P, pt = d.pd.page_size, d.page_table.cpu()
    for s, t, n in pairs:
        for j in range(n):
            want[l0:l1, :, pt[t, j // P], j % P] = d.pool[l0:l1, :, pt[s, j // P], j % P]
    return want


@pytest.mark.parametrize("lens,pairs", [
    ([33, 33], [(0, 1, 33)]), ([1, 1], [(0, 1, 1)]), ([40, 100, 17], [(1, 0, 40), (1, 2, 16)]), ([40, 100], [(0, 1, 0)]),
    ([70, 70, 70, 64, 30, 100], [(0, 1, 70), (0, 2, 3), (5, 3, 50), (0, 4, 30)])])
@pytest.mark.parametrize("kw", [dict(), dict(page=5, hk=3, D=24, layers=3), dict(page=32, hk=4, D=128, layers=2),
                                dict(hk=2, D=64, head_major=True), dict(hk=2, D=12), dict(hk=1, D=64, offset=1)])
def test_copies(lens, pairs, kw):
    d = _decoder(lens, seed=len(lens), **kw)
    want = _expect_copy(d, pairs, 0, d.pd.n_layers)
    src, dst, n = (_i32(x) for x in zip(*pairs))
    d.copy(src, dst, n, max(p[2] for p in pairs))
    d.check_status()
    assert torch.equal(d.pool.view(torch.int16) if d.pool.is_contiguous() else d.pool.contiguous().view(torch.int16),
                       want.contiguous().view(torch.int16))


def test_copy_of_a_layer_range_into_many_branches():
    lens = [100] + [100] * 150
    d = _decoder(lens, layers=4, hk=2, D=64)
    pairs = [(0, i, 100 - i % 40) for i in range(1, 151)]
    want = _expect_copy(d, pairs, 1, 3)
    src, dst, n = (_i32(x) for x in zip(*pairs))
    d.copy(src, dst, n, 120, l0=1, l1=3)
    d.check_status()
    assert torch.equal(d.pool, want)


def test_copy_reports_what_it_drops():
    def run(pairs, code, max_len=64, change=lambda d: None, kept=()):
        d = _decoder([60, 60, 60, 20], hk=1, D=16)
        change(d)
        want = _expect_copy(d, kept, 0, 1)
        src, dst, n = (_i32(x) for x in zip(*pairs))
        d.copy(src, dst, n, max_len)
        assert d.status.cpu().tolist()[0] == code
        assert torch.equal(d.pool, want)
    run([(0, 9, 5), (0, 1, 60)], B.E_INVALID, kept=[(0, 1, 60)])
    run([(-1, 1, 5), (0, 2, 60)], B.E_INVALID, kept=[(0, 2, 60)])
    run([(0, 0, 5)], B.E_INVALID)
    run([(0, 3, 60), (0, 1, 60)], B.E_INVALID, kept=[(0, 1, 60)])        # longer than the destination
    run([(3, 0, 21)], B.E_INVALID)                                       # longer than the source
    run([(0, 1, 60)], B.E_INVALID, max_len=50)
    run([(0, 1, -2), (0, 2, 20)], B.E_INVALID, kept=[(0, 2, 20)])

    def bad_page(d):
        d.page_table[1, 0] = 12345
    d = _decoder([60, 60, 60], hk=1, D=16)
    bad_page(d)
    before = d.pool.clone()
    d.copy(_i32([0, 0]), _i32([1, 2]), _i32([60, 60]), 60)
    assert d.status.cpu().tolist()[:3] == [B.E_BADPAGE, 1, 12345]
    P = 16
    for j in range(60):                                                  # the other branch is whole, the other pages of this one too
        assert torch.equal(d.pool[0, :, d.page_table[2, j // P], j % P], before[0, :, d.page_table[0, j // P], j % P])
        if j >= P:
            assert torch.equal(d.pool[0, :, d.page_table[1, j // P], j % P], before[0, :, d.page_table[0, j // P], j % P])
    d = _decoder([60, 60, 60], hk=1, D=16)
    d.copy(_i32([0, 1]), _i32([1, 2]), _i32([60, 60]), 60)               # request 1 as destination and source
    assert d.status.cpu().tolist()[0] == B.E_INVALID
