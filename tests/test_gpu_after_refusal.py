"""actkv_append and actkv_copy behind an actkv_resize that was refused: what the cache holds stays as it was, bit for bit.  Any other error
(rows and pages that these two calls drop themselves, a request that attention leaves out) stops nothing else: the tokens of the other
requests are written, in this call and in those on the next layers."""
import pytest
import torch

from paper_2609_31395_b200 import binding as B
from paper_2609_31395_b200 import harness as H

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _decoder(lens, spare, width, layers=1, hk=2, G=2, D=16, P=16, rows=64, head_major=False):
    need = [-(-n // P) for n in lens]
    n_pages = sum(need) + spare
    perm = torch.randperm(n_pages, generator=torch.Generator().manual_seed(1)).to(torch.int32)
    pt = torch.full((len(lens), width), -1, dtype=torch.int32)
    at = 0
    for r, n in enumerate(need):
        pt[r, :n] = perm[at:at + n]
        at += n
    free = torch.full((n_pages,), -1, dtype=torch.int32)
    free[:spare] = perm[at:]
    shape = (layers, 2, n_pages, hk, P, D) if head_major else (layers, 2, n_pages, P, hk, D)
    pool = torch.randn(shape, device=DEV, generator=torch.Generator(device=DEV).manual_seed(2)).to(torch.bfloat16)
    if head_major:
        pool = pool.transpose(3, 4)
    return H.Decoder(pool, pt.to(DEV), _i32(lens), free.to(DEV), _i32([spare]), hk * G, rows, rows, P * width, layers)


def _new_rows(d, rows, layers=1, seed=3):
    hk, D, hq = d.pd.n_kv_heads, d.pd.head_dim, d.n_q_heads
    x = torch.randn((layers, rows, hq + 2 * hk, D), device=DEV, generator=torch.Generator(device=DEV).manual_seed(seed)).to(torch.bfloat16)
    return x[:, :, :hq], x[:, :, hq:hq + hk], x[:, :, hq + hk:]


def _state(d):
    return [t.clone() for t in (d.pool, d.page_table, d.seq_len, d.free_list, d.free_count)]


def _same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("cause", ["pages", "table", "free page id"])
def test_a_refused_step_leaves_the_cache_alone(cause, captured):
    # 16 and 40 tokens: the first request needs a page for its new one
    d = _decoder([16, 40], spare=0 if cause == "pages" else 3, width=1 if cause == "table" else 4) if cause != "table" else \
        _decoder([48, 40], spare=3, width=3)
    if cause == "free page id":
        d.free_list.fill_(1 << 20)
    code = {"pages": B.E_NOFREE, "table": B.E_INVALID, "free page id": B.E_BADPAGE}[cause]
    q, k, v = _new_rows(d, 2)
    wi, new = _i32([0, 1, 2]), d.seq_len + 1
    q_out, out = torch.empty(q.shape, dtype=torch.bfloat16, device=DEV), torch.empty(q.shape, dtype=torch.bfloat16, device=DEV)

    def step():
        d.resize(new)
        d.append(k, v, wi, q=q, q_out=q_out)
        d.attend(q_out, wi, 0.25, True, out)
    before = _state(d)
    if captured:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        for _ in range(3):
            g.replay()
    else:
        step()
    assert d.status.cpu().tolist()[0] == code
    assert _same(_state(d), before)
    # the caller makes room, clears the status and tries again
    if cause == "pages":
        d.resize(_i32([-1, -1]))                       # (status is set: does nothing)
        d.append(k, v, wi)
        assert _same(_state(d), before)
        d.status.zero_()
        d.resize(_i32([-1, 10]))                       # two pages given back
        new.copy_(_i32([17, 11]))
    elif cause == "table":
        d.status.zero_()
        new.copy_(_i32([48, 41]))
        d.seq_len.copy_(_i32([47, 40]))
    else:
        d.status.zero_()
        used = set(d.page_table.flatten().tolist())
        d.free_list.copy_(_i32([p for p in range(d.pd.n_pages) if p not in used] + [-1] * (d.pd.n_pages - 3)))
    if captured:
        g.replay()
    else:
        step()
    d.check_status()
    for r in range(2):
        j = int(d.seq_len[r]) - 1
        page = int(d.page_table[r, j // 16])
        assert torch.equal(d.pool[0, 0, page, j % 16], k[0, r]) and torch.equal(d.pool[0, 1, page, j % 16], v[0, r])


@pytest.mark.parametrize("code", [B.E_INVALID, B.E_BADPAGE, B.E_NOFREE, B.E_TIMEOUT])
def test_a_resize_that_finds_an_error_stops_both(code):
    # whatever call it comes from: the lengths are not the ones that were asked for
    d = _decoder([30, 30, 20], spare=2, width=4)
    q, k, v = _new_rows(d, 3)
    q_out = torch.zeros(q.shape, dtype=torch.bfloat16, device=DEV)
    d.status.copy_(_i32([code, 5, 6, 0]))
    before = _state(d)
    for _ in range(2):
        d.resize(d.seq_len + 1)
        d.append(k, v, _i32([0, 1, 2, 3]), q=q, q_out=q_out)
        d.copy(_i32([0]), _i32([1]), _i32([30]), 30)
    assert _same(_state(d), before) and d.status.cpu().tolist()[:3] == [code, 5, 6]
    assert torch.equal(q_out, q)                       # (the queries are the caller's, not the cache's)
    d.status.zero_()
    d.resize(d.seq_len + 1)
    d.append(k, v, _i32([0, 1, 2, 3]))
    d.check_status()
    assert torch.equal(d.pool[0, 1, d.page_table[0, 1], 30 % 16], v[0, 0])


@pytest.mark.parametrize("damage", ["length", "page"])
def test_an_error_of_attention_in_one_layer_leaves_the_next_layers_alone(damage):
    # three requests, two layers; attend reports request 1 in layer 0, the tokens of the others belong into layer 1 all the same
    d = _decoder([30, 30, 20], spare=2, width=4, layers=2)
    q, k, v = _new_rows(d, 3, 2)
    q, wi = q.contiguous(), _i32([0, 1, 2, 3])
    out = torch.empty_like(q[:1])
    d.resize(d.seq_len + 1)
    if damage == "page":
        d.page_table[1, 0] = 1 << 20                   # (token 0's; the new one is on page 1)
    else:
        d.max_tok = 30
    for l in range(2):
        d.append(k[l:l + 1], v[l:l + 1], wi, l0=l)
        d.attend(q[l:l + 1], wi, 0.25, True, out, l0=l)
    assert d.status.cpu().tolist()[0] == (B.E_BADPAGE if damage == "page" else B.E_INVALID)
    for l in range(2):
        for r, n in enumerate([30, 30, 20]):
            assert torch.equal(d.pool[l, 0, d.page_table[r, 1], n % 16], k[l, r]) and torch.equal(d.pool[l, 1, d.page_table[r, 1], n % 16], v[l, r])


@pytest.mark.parametrize("head_major", [False, True])
def test_a_refused_fork_leaves_the_other_request_alone(head_major):
    # request 1 is to become a branch of request 0: it has 30 entries, 60 are wanted and there is no page
    d = _decoder([60, 30], spare=0, width=4, D=64, head_major=head_major)
    before = _state(d)
    d.resize(_i32([-1, 60]))
    d.copy(_i32([0]), _i32([1]), _i32([20]), 60)
    assert d.status.cpu().tolist()[0] == B.E_NOFREE and _same(_state(d), before)


def test_rows_that_are_dropped_stop_no_others():
    # 1200 rows of 300 requests in two layers; the pages of requests 0 and 150 are damaged
    R, W = 300, 4
    d = _decoder([20] * R, spare=5, width=2, layers=2, rows=R * W)
    good = [r for r in range(R) if r not in (0, 150)]
    table = d.page_table.cpu()
    d.page_table[0, 1] = 1 << 20
    d.page_table[150, 1] = -1
    wi = _i32([W * r for r in range(R + 1)])
    _, k, v = _new_rows(d, R * W, 2)
    want = d.pool.clone()
    for r in good:                                     # tokens 16 .. 19
        for l in range(2):
            want[l, 0, table[r, 1], :W], want[l, 1, table[r, 1], :W] = k[l, W * r:W * (r + 1)], v[l, W * r:W * (r + 1)]
    for l in range(2):                                 # the second call finds the first one's report
        d.append(k[l:l + 1], v[l:l + 1], wi, l0=l)
    assert d.status.cpu().tolist()[0] == B.E_BADPAGE and d.status.cpu().tolist()[1] in (0, 150)
    assert torch.equal(d.pool, want)
    # but pages are no longer handed out, and what relied on them is not written
    d.resize(d.seq_len + 13)
    before = _state(d)
    d.append(k[:1], v[:1], wi)
    d.copy(_i32([1]), _i32([2]), _i32([20]), 20)
    assert _same(_state(d), before)


def test_pairs_that_are_dropped_stop_no_others():
    n = 100
    d = _decoder([40] * (n + 1), spare=0, width=3, D=64)
    d.page_table[7, 0] = -5
    before = d.pool.clone()
    src, dst = _i32([0] * n), _i32(list(range(1, n + 1)))
    for _ in range(2):
        d.copy(src, dst, _i32([40] * n), 40)
    assert d.status.cpu().tolist()[:3] == [B.E_BADPAGE, 7, -5]
    pt = d.page_table.cpu()
    for r in range(1, n + 1):
        for c in range(3):
            if (r, c) != (7, 0):
                slots = 16 if c < 2 else 8
                assert torch.equal(d.pool[:, :, pt[r, c], :slots], before[:, :, pt[0, c], :slots])
