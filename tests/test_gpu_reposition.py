"""GPU parity of actkv_reposition against the float64 oracle.

Tolerance: the angle as a float32 of 2^-32 turns (24 bits: pi 2^-24) times 2 pi 2^-32 (a rounding more) is off by at most 2^-21.3; sine and cosine
of the special function units by 2^-21.1 in [-pi, pi]; the products and their sum by 2^-23: together below 2^-19 (|x| + |y|).  The frequency in
turns is a float64 product, off by 2^-54: at the positions here (below 2^20) nothing; at 2^31 2^-23 turns, below 2^-20 rad.  Rounded once to bf16:
2^-8 relative, half a step."""
import numpy as np
import pytest
import torch

from oracle import actkv_oracle as O
from paper_2609_31395_b200 import binding as B
from paper_2609_31395_b200 import harness as H

import parity_util as U

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _case(lens, moved=None, layers=1, l0=0, hk=2, D=64, page=16, rotary=None, sections=None, interleaved=False, per_unit=True, frm=True, to=False,
          rescale=False, head_major=False, far=1 << 20, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    rotary = D if rotary is None else rotary
    moved = lens if moved is None else moved
    need = [-(-n // page) for n in lens]
    n_pages = sum(need) + 3
    perm = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    pt = torch.full((len(lens), max(need + [1])), -1, dtype=torch.int32)
    at = 0
    for r, n in enumerate(need):
        pt[r, :n] = perm[at:at + n]
        at += n
    shape = (layers + l0, 2, n_pages, hk, page, D) if head_major else (layers + l0, 2, n_pages, page, hk, D)
    pool = torch.randn(shape, generator=g, device=DEV).to(torch.bfloat16)
    if head_major:
        pool = pool.transpose(3, 4)
    sections = [rotary // 2] if sections is None else sections
    ind = [3] + (3 + np.cumsum(moved)).tolist()                  # (the positions need not begin at 0)
    shape = (len(sections), layers * hk, ind[-1]) if per_unit else (len(sections), ind[-1])
    pos = lambda: torch.randint(0, far, shape, generator=g, device=DEV).to(torch.int32)
    freq = torch.tensor([1e4 ** (-i / max(1, rotary // 2)) for i in range(rotary // 2)], dtype=torch.float32, device=DEV)
    return dict(dec=H.Decoder(pool, pt.to(DEV), _i32(lens), _i32([0] * n_pages), _i32([0]), hk, layers_per_call=layers), pool=pool, pt=pt.numpy(),
                lens=lens, moved=moved, ind=ind, page=page, layers=layers, l0=l0, hk=hk, freq=freq, sections=sections, interleaved=interleaved,
                rope=H.Rope(freq, sections, interleaved), frm=pos() if frm else None, to=pos() if to else None,
                to_freq=freq * torch.linspace(1, 0.2, rotary // 2, device=DEV) if rescale else None)


def _run(c, **kw):
    c["dec"].reposition(c["rope"], _i32(c["ind"]), max(c["moved"] + [1]), c["frm"], c["to"], c["to_freq"], l0=c["l0"], l1=c["l0"] + c["layers"], **kw)


def _check(c, before, near=2.0 ** -19):
    want, tol = before.double().cpu().numpy(), np.zeros(before.shape)
    f0 = c["freq"].cpu().numpy()
    f1 = f0 if c["to_freq"] is None else c["to_freq"].cpu().numpy()

    def places(p, unit, r, n):
        if p is None:
            return np.tile(np.arange(n), (len(c["sections"]), 1))
        p = p.cpu().numpy()
        return (p[:, unit] if p.ndim == 3 else p)[:, c["ind"][r]:c["ind"][r] + n]
    for r, n in enumerate(c["moved"]):
        j = np.arange(n)
        page, slot = c["pt"][r, j // c["page"]], j % c["page"]
        for l in range(c["layers"]):
            for h in range(c["hk"]):
                unit = l * c["hk"] + h
                a, b = places(c["frm"], unit, r, n), places(c["to"], unit, r, n)
                k = want[c["l0"] + l, 0, page, slot, h]
                y = O.reposition_unit(k, a, b, f0, f1, c["sections"], c["interleaved"])
                stays = (a == b).all(axis=0) & (c["to_freq"] is None)
                turned = 2 * len(f0)
                room = 2.0 ** -8 * np.abs(y) + near * 2 * np.abs(k).max(initial=0.0)
                room[:, turned:] = 0.0
                room[stays] = 0.0
                y[stays] = k[stays]
                want[c["l0"] + l, 0, page, slot, h], tol[c["l0"] + l, 0, page, slot, h] = y, room
    got = c["pool"].double().cpu().numpy()
    assert (np.abs(got - want) <= tol).all(), float((np.abs(got - want) - tol).max())   # V, other dims and other tokens as they were
    c["dec"].check_status()


@pytest.mark.parametrize("kw", [
    dict(lens=[1]), dict(lens=[0]), dict(lens=[17, 0, 1, 300]), dict(lens=[40], D=128, hk=8), dict(lens=[33, 70], D=128, hk=4, layers=3, l0=1),
    dict(lens=[50], interleaved=True), dict(lens=[50], D=128, interleaved=True, hk=5), dict(lens=[50], D=80), dict(lens=[50, 9], D=80, rotary=40),
    dict(lens=[50], D=80, rotary=40, interleaved=True), dict(lens=[50], D=128, rotary=64), dict(lens=[50], D=256, hk=1), dict(lens=[30], D=8),
    dict(lens=[30], D=16, rotary=2), dict(lens=[30], rotary=6, interleaved=True), dict(lens=[30], rotary=62), dict(lens=[30], D=24, rotary=24),
    dict(lens=[200, 31], sections=[8, 12, 12]), dict(lens=[60], sections=[0, 16, 0, 16], interleaved=True), dict(lens=[60], D=128, sections=[64, 0]),
    dict(lens=[60], sections=[1, 31], per_unit=False), dict(lens=[60, 44], per_unit=False, hk=7, layers=2), dict(lens=[60], per_unit=False, interleaved=True, hk=3),
    dict(lens=[90, 5], to=True), dict(lens=[90, 5], frm=False, to=True), dict(lens=[90, 5], to=True, sections=[10, 22], rescale=True),
    dict(lens=[90, 5], frm=False, rescale=True), dict(lens=[90], rescale=True, interleaved=True, D=128), dict(lens=[90], rescale=True, rotary=30),
    dict(lens=[90], rescale=True, rotary=32, sections=[4, 12], interleaved=True), dict(lens=[90, 20], frm=False, rescale=True, hk=6, D=128),
    dict(lens=[77], page=5), dict(lens=[77], page=1), dict(lens=[200], page=64), dict(lens=[77, 40], head_major=True, hk=3), dict(lens=[77], page=7, rotary=10),
    dict(lens=[100, 64, 32], moved=[60, 0, 32]), dict(lens=[100, 64], moved=[0, 0]), dict(lens=[3000, 100, 1700], D=128, hk=4, layers=2),
    dict(lens=[40] * 70, hk=1), dict(lens=[9000], per_unit=False, hk=8, D=128, layers=2)])
def test_parity(kw):
    c = _case(**kw)
    before = c["pool"].clone()
    _run(c)
    _check(c, before)


@pytest.mark.parametrize("interleaved", [False, True])
def test_positions_at_the_ends_of_their_type(interleaved):
    c = _case([64], D=128, to=True, interleaved=interleaved, seed=3)
    ends = torch.tensor([0, -1, 1, 2 ** 31 - 1, -2 ** 31, -2 ** 31 + 1, 2 ** 30, 12345], dtype=torch.int32, device=DEV)
    c["frm"][..., 3:] = ends[torch.arange(64, device=DEV) % 8]
    c["to"][..., 3:] = ends[torch.arange(64, device=DEV) // 8]
    before = c["pool"].clone()
    _run(c)
    _check(c, before, near=2.0 ** -17)


def test_keys_that_stay_keep_their_bits():
    c = _case([50, 40], D=128, hk=3, to=True)
    c["to"].copy_(c["frm"])
    c["pool"][:, 0, :, :, 1, 5] = float("nan")
    c["pool"][:, 0, :, :, 2, 70] = float("inf")
    before = U.bits(c["pool"])
    _run(c)
    assert np.array_equal(U.bits(c["pool"]), before)
    c["to"][:, 1, 3 + 50 + 7] += 1                               # one key of one unit moves
    _run(c)
    changed = (U.bits(c["pool"]) != before).any(axis=-1)
    assert changed.sum() == 1 and changed[0, 0, c["pt"][1, 0], 7, 1]


def test_appended_there_or_moved_there():
    """A key appended at p and moved to q lies within its roundings of one appended at q: 2^-8 more for the second rounding."""
    n, hk, D = 48, 2, 64
    a, b = _case([n], hk=hk, D=D, sections=[12, 20], per_unit=False, seed=5), _case([n], hk=hk, D=D, sections=[12, 20], per_unit=False, seed=5)
    g = torch.Generator(device=DEV).manual_seed(1)
    kv = torch.randn((1, n, 2 * hk, D), generator=g, device=DEV).to(torch.bfloat16)
    p, q = (torch.randint(0, 100000, (2, n), generator=g, device=DEV).to(torch.int32) for _ in range(2))
    for c, pos in ((a, p), (b, q)):
        c["dec"].append(kv[:, :, :hk], kv[:, :, hk:], _i32([0, n]), rope=c["rope"], positions=pos)
    a["dec"].reposition(a["rope"], _i32([0, n]), n, p, q)
    j = np.arange(n)
    x, y = (c["pool"][0, :, c["pt"][0, j // 16], j % 16].double() for c in (a, b))
    size = torch.hypot(y[0][..., :D // 2], y[0][..., D // 2:]).repeat(1, 1, 2)
    assert ((x[0] - y[0]).abs() <= 2.0 ** -8 * (2.5 * size)).all() and torch.equal(x[1], y[1])


def test_back_and_forth_returns():
    c = _case([100], D=128, hk=4, to=True)
    before = c["pool"].clone()
    _run(c)
    assert not torch.equal(c["pool"], before)
    c["frm"], c["to"] = c["to"], c["frm"]
    _run(c)
    x, y = c["pool"].double(), before.double()
    size = torch.hypot(y[..., :64], y[..., 64:]).repeat(1, 1, 1, 1, 1, 2)
    assert ((x - y).abs() <= 2.0 ** -8 * 2.1 * size + 1e-6).all()       # two roundings, each of at most 2^-8 of its pair's size (and its partner's)


@pytest.mark.parametrize("cause,code", [("length", B.E_INVALID), ("too long", B.E_INVALID), ("negative", B.E_INVALID), ("page", B.E_BADPAGE),
                                        ("positions", B.E_INVALID), ("status", B.E_NOFREE)])
@pytest.mark.parametrize("rotary", [64, 6])
def test_all_or_nothing(cause, code, rotary):
    c = _case([500, 40, 300], rotary=rotary)
    d, ind, max_tok = c["dec"], list(c["ind"]), 500
    if cause == "length":
        d.seq_len[1] = 39
    elif cause == "too long":
        max_tok = 400
    elif cause == "negative":
        ind[2] = ind[1] - 1
    elif cause == "page":
        d.page_table[2, 18] = -1
    elif cause == "positions":
        c["frm"] = c["frm"][..., :ind[-1] - 1]
    else:
        d.status[0] = code
    before = U.bits(c["pool"])
    d.reposition(c["rope"], _i32(ind), max_tok, c["frm"])
    assert np.array_equal(U.bits(c["pool"]), before) and d.status[0].item() == code
    if cause == "page":
        assert d.status.tolist()[:3] == [code, 2, -1]


def test_a_captured_call_on_another_stream():
    c = _case([130, 60], D=128, hk=4, to=True)
    ind = _i32(c["ind"])
    first = c["pool"].clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        c["dec"].reposition(c["rope"], ind, 130, c["frm"], c["to"])
    torch.cuda.synchronize()
    assert torch.equal(c["pool"], first)
    g.replay()
    torch.cuda.synchronize()
    _check(c, first)
    again = c["pool"].clone()
    with torch.cuda.stream(s):
        _run(c)
    s.synchronize()
    _check(c, again)


def test_positions_of_a_wrong_shape_are_refused():
    c = _case([20], sections=[10, 22])
    ok = c["frm"]
    for bad in (ok[:, :1].repeat(1, 3, 1), ok.repeat(2, 1, 1)[:3], ok[None]):
        with pytest.raises(ValueError):
            c["dec"].reposition(c["rope"], _i32([0, 20]), 20, bad)
    for bad in (ok.long(), ok.cpu(), ok.transpose(1, 2).contiguous().transpose(1, 2)):
        with pytest.raises(TypeError):
            c["dec"].reposition(c["rope"], _i32([0, 20]), 20, bad)
    with pytest.raises(ValueError):
        c["dec"].reposition(c["rope"], _i32([0, 20]), 20, ok, to_inv_freq=c["freq"][:-1])
    with pytest.raises(ValueError):
        c["dec"].reposition(c["rope"], _i32([0]), 20, ok)
