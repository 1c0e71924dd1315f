"""actkv_reposition behind a compaction, through the public classes and with no look at a status in between: what a compaction that was refused leaves."""
import numpy as np
import pytest
import torch

from oracle import actkv_oracle as O
from paper_2609_31395_b200 import binding as B
from paper_2609_31395_b200 import harness as H

import parity_util as U

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NL, HK, HQ, D, P, W = 2, 2, 4, 64, 16, 8
LENS, BUDGET = [100, 61, 128], [40, 61, 33]      # (the second request keeps everything)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Cache:
    def __init__(self, seed, lens=LENS, budget=BUDGET, spare=12):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.lens, self.budget, R = lens, budget, len(lens)
        need = [-(-n // P) for n in lens]
        n_pages = sum(need) + spare
        perm = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).tolist()
        table = [[perm.pop() for _ in range(n)] + [-1] * (max(need) - n) for n in need]
        self.pool = torch.randn((NL, 2, n_pages, P, HK, D), generator=g, device=DEV).to(torch.bfloat16)
        self.table, self.seq_len, self.free, self.fc = _i32(table), _i32(lens), _i32(perm + [0] * sum(need)), _i32([spare])
        self.dec = H.Decoder(self.pool, self.table, self.seq_len, self.free, self.fc, HQ)
        self.comp = H.Compressor(self.pool, self.table, self.seq_len, self.free, self.fc, HQ,
                                 H.StepSizes(R, R * W, W, sum(lens), max(lens), sum(budget), max(budget)))
        self.freq = 1.0 / 10000.0 ** (torch.arange(D // 2, device=DEV) / (D // 2))
        self.rope = H.Rope(self.freq, [D // 2])
        self.q = torch.randn((NL, R * W, HQ, D), generator=g, device=DEV).to(torch.bfloat16)
        self.win, self.tok, self.limit = _i32(range(0, R * W + 1, W)), _i32([0] + np.cumsum(lens).tolist()), _i32(budget)
        self.before, self.old = self.keys(), self.table.cpu().numpy()

    def keys(self):
        return self.pool[:, 0].double().cpu().numpy()

    def rows(self, keys, table, l, h, r, n):
        j = np.arange(n)
        return keys[l, table[r, j // P], j % P, h]

    def step(self, **kw):
        self.comp.step(self.q, self.win, self.tok, self.limit, D ** -0.5, True, **kw)

    def up(self):
        """What the README has behind a step."""
        comp = self.comp
        self.dec.reposition(self.rope, comp.keep_indptr, max(self.budget), from_pos=comp.sel_idx[None], status=comp.status)

    def check(self, order):
        """Every cached key is the one of token order(unit, r)[slot], turned to place(unit, r)[slot]."""
        now, table, f = self.keys(), self.table.cpu().numpy(), self.freq.cpu().numpy()
        assert self.seq_len.cpu().tolist() == self.budget
        for l in range(NL):
            for h in range(HK):
                for r, n in enumerate(self.budget):
                    was, will = order(l * HK + h, r)
                    raw = self.rows(self.before, self.old, l, h, r, self.lens[r])[was]
                    want = O.reposition_unit(raw, was[None], will[None], f, f, [D // 2], False)
                    # half a step of bf16, and 2^-19 of the pair for the angle, sine and cosine
                    tol = 2.0 ** -8 * np.abs(want) + 2.0 ** -19 * 2 * np.abs(raw).max(initial=0.0)
                    assert (np.abs(self.rows(now, table, l, h, r, n) - want) <= tol).all()


def _lists(c):
    sel, ind = c.comp.sel_idx.cpu().numpy(), c.comp.keep_indptr.cpu().tolist()
    return lambda unit, r: sel[unit, ind[r]:ind[r + 1]]


@pytest.mark.parametrize("captured", [False, True])
def test_keys_are_left_alone_behind_a_compaction_that_was_refused(captured):
    c = Cache(1)
    c.fc.fill_(5)                                # (ten pages are needed)
    bits = U.bits(c.pool)

    def both():
        c.step()
        c.up()
    both()
    if captured:
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            both()
        both = g.replay
        for _ in range(2):
            both()
    assert c.comp.status[0].item() == B.E_NOFREE and np.array_equal(U.bits(c.pool), bits) and c.seq_len.cpu().tolist() == c.lens
    with pytest.raises(B.ActKVError):
        c.comp.check_status()
    c.dec.check_status()
    c.fc.fill_(12)                               # room is made, the status cleared: the same calls are carried out
    c.comp.status.zero_()
    both()
    c.comp.check_status()
    of = _lists(c)
    c.check(lambda unit, r: (of(unit, r), np.arange(c.budget[r])))


def test_an_error_of_the_call_goes_to_the_words_that_it_was_given():
    c = Cache(2)
    bits = U.bits(c.pool)
    c.dec.reposition(c.rope, _i32([0, 101, 162, 290]), 128, from_pos=_i32(range(1, 291)), status=c.comp.status)
    assert c.comp.status.tolist()[:2] == [B.E_INVALID, 0] and c.dec.status.tolist() == [0] * 4 and np.array_equal(U.bits(c.pool), bits)
    c.dec.reposition(c.rope, _i32([0, 100, 161, 289]), 128, from_pos=_i32(range(1, 290)))          # (the Decoder's own, which are clean)
    assert c.dec.status.tolist() == [0] * 4 and not np.array_equal(U.bits(c.pool), bits)


def _ranks(comp, n, longest):
    """The recipe of Decoder.reposition's documentation."""
    request = torch.searchsorted(comp.keep_indptr[1:], torch.arange(n, device=DEV), right=True)
    order = comp.new_order[:, :n] + longest * request
    return order.argsort(1).argsort(1) - comp.keep_indptr[request]


@pytest.mark.parametrize("lens,budget", [(LENS, BUDGET), ([300], [111]), ([33, 0, 16, 200], [1, 0, 16, 130]), ([70, 80], [70, 80])])
def test_behind_a_compaction_in_place(lens, budget):
    c = Cache(3, lens, budget)
    c.step(inplace=True, want_order=True)
    n = sum(budget)
    c.dec.reposition(c.rope, c.comp.keep_indptr, max(budget), from_pos=c.comp.new_order[None], to_pos=_ranks(c.comp, n, 1 << 20)[None].int(), status=c.comp.status)
    c.comp.check_status()
    order, ind = c.comp.new_order.cpu().numpy(), c.comp.keep_indptr.cpu().tolist()
    of, disordered = _lists(c), 0

    def lies(unit, r):
        nonlocal disordered
        was = order[unit, ind[r]:ind[r + 1]]
        assert np.array_equal(np.sort(was), of(unit, r))
        disordered += int((np.diff(was) < 0).any())
        return was, np.searchsorted(of(unit, r), was)
    c.check(lies)
    assert (disordered > 0) == any(b < n for b, n in zip(budget, lens))


def test_a_step_in_place_without_the_order_is_as_before():
    a, b = Cache(4), Cache(4)
    a.step(inplace=True)
    b.step(inplace=True, want_order=True)
    assert getattr(a.comp, "new_order", None) is None and np.array_equal(U.bits(a.pool), U.bits(b.pool)) and torch.equal(a.table, b.table)


def test_behind_a_compaction_in_place_that_was_refused():
    c = Cache(5)
    c.table[1, 2] = 10000                        # (a page that is not there)
    c.step(inplace=True, want_order=True)
    bits = U.bits(c.pool)
    c.dec.reposition(c.rope, c.comp.keep_indptr, max(BUDGET), from_pos=c.comp.new_order[None], to_pos=_ranks(c.comp, sum(BUDGET), 1 << 20)[None].int(),
                     status=c.comp.status)
    assert c.comp.status[0].item() == B.E_BADPAGE and c.seq_len.cpu().tolist() == LENS and np.array_equal(U.bits(c.pool), bits)
