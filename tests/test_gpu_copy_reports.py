"""actkv_copy reports every pair that it drops, wherever the pair stands among others of its source."""
import pytest
import torch

from paper_2609_31395_b200 import binding as B
from paper_2609_31395_b200 import harness as H

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
N = 300


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _decoder(head_major):
    lens = [40] * N + [20]                             # the last one is shorter
    need = [3] * N + [2]
    pt = torch.full((N + 1, 3), -1, dtype=torch.int32)
    at = 0
    for r, n in enumerate(need):
        pt[r, :n] = torch.arange(at, at + n)
        at += n
    shape = (1, 2, at, 2, 16, 16) if head_major else (1, 2, at, 16, 2, 16)
    pool = torch.randn(shape, device=DEV, generator=torch.Generator(device=DEV).manual_seed(4)).to(torch.bfloat16)
    if head_major:                                     # (the kernel for any layout; the other pool takes bulk copies)
        pool = pool.transpose(3, 4)
    return H.Decoder(pool, pt.to(DEV), _i32(lens), _i32([0] * at), _i32([0]), 2)


@pytest.mark.parametrize("head_major", [False, True])
@pytest.mark.parametrize("at", [1, 31, 32, 40, 127, 128, 200, 260])
@pytest.mark.parametrize("bad", ["destination out of range", "longer than the destination", "longer than the bound",
                                 "longer than the source", "negative", "onto itself"])
def test_an_unsound_pair_behind_sound_ones(head_major, at, bad):
    d = _decoder(head_major)
    pairs = [[0, i, 40] for i in range(1, 281)]        # request 0 into 280 branches
    bound = 40
    if bad == "destination out of range":
        pairs[at][1] = N + 7
    elif bad == "longer than the destination":
        pairs[at][1] = N
    elif bad == "longer than the bound":
        pairs[at][2], bound = 40, 39
        for i, p in enumerate(pairs):
            p[2] = 40 if i == at else 39
    elif bad == "longer than the source":
        pairs[at][2], bound = 41, 48
    elif bad == "negative":
        pairs[at][2] = -1
    else:
        pairs[at][1] = 0
    want = d.pool.clone()
    pt = d.page_table.cpu()
    for i, (s, t, n) in enumerate(pairs):
        if i != at:
            for c in range(3):
                slots = max(0, min(16, n - 16 * c))
                want[:, :, pt[t, c], :slots] = d.pool[:, :, pt[s, c], :slots]
    src, dst, n = (_i32(x) for x in zip(*pairs))
    d.copy(src, dst, n, bound)
    st = d.status.cpu().tolist()
    assert st[0] == B.E_INVALID
    if bad != "onto itself":                           # (every other pair has that request as its source: any of them may come first)
        assert st[1] == at
    assert torch.equal(d.pool, want)


def test_sound_pairs_report_nothing():
    d = _decoder(False)
    d.copy(_i32([0] * 280), _i32(list(range(1, 281))), _i32([i % 41 for i in range(280)]), 40)
    d.check_status()


def test_a_source_out_of_range_among_many():
    d = _decoder(False)
    src = [0] * 200
    src[150] = N + 1
    d.copy(_i32(src), _i32(list(range(1, 201))), _i32([40] * 200), 40)
    assert d.status.cpu().tolist()[:3] == [B.E_INVALID, 150, N + 1]
