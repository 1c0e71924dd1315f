"""GPU parity of actkv_append against the float64 oracle.

Tolerance: x cos t - y sin t with sine and cosine of float32 (argument in half turns rounded at 2^-25: 2^-23 after pi; 2 ulp) and
products in float32: at most 2^-21 (|x| + |y|); rounded once to bf16: 2^-8 relative, half a step."""
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


def _case(ctx, wins, layers=1, hk=2, G=3, D=64, page=16, rotary=64, sections=None, interleaved=False, seed=0, shift=0, layer0=0):
    """shift: elements that q, k, v lie off a 16-byte boundary."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    R, hq = len(wins), hk * G
    L = [a + b for a, b in zip(ctx, wins)]
    need = [-(-n // page) for n in L]
    n_pages = sum(need) + 3
    perm = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    pt = torch.full((R, max(need + [1])), -1, dtype=torch.int32)
    at = 0
    for r, n in enumerate(need):
        pt[r, :n] = perm[at:at + n]
        at += n
    pool = torch.randn((layers + layer0, 2, n_pages, page, hk, D), generator=g, device=DEV, dtype=torch.bfloat16)
    rows = sum(wins)
    width = (hq + 2 * hk) * D + shift
    qkv = torch.randn((layers, rows, width), generator=g, device=DEV, dtype=torch.bfloat16)[:, :, shift:].unflatten(2, (hq + 2 * hk, D))
    sections = [rotary // 2] if sections is None else sections
    pos = torch.randint(0, 1000000, (len(sections), rows), generator=g, device=DEV).to(torch.int32)
    freq = torch.tensor([1e6 ** (-i / max(1, rotary // 2)) for i in range(rotary // 2)], dtype=torch.float32, device=DEV)
    dec = H.Decoder(pool, pt.to(DEV), _i32(L), _i32([0] * n_pages), _i32([0]), hq, max(1, rows), max(wins), max(L), layers)
    return dict(dec=dec, pool=pool, qkv=qkv, pos=pos, freq=freq, wi=_i32([0] + np.cumsum(wins).tolist()), L=L, wins=wins, hq=hq, hk=hk,
                D=D, page=page, sections=sections, interleaved=interleaved, pt=pt.numpy(), layers=layers, layer0=layer0,
                rope=H.Rope(freq, sections, interleaved) if rotary else None)


def _run(c, q_out=None, q="q"):
    hq, hk = c["hq"], c["hk"]
    x = c["qkv"]
    out = torch.full((c["layers"], x.shape[1], hq, c["D"]), 9.0, dtype=torch.bfloat16, device=DEV) if q_out is None else q_out
    c["dec"].append(x[:, :, hq:hq + hk], x[:, :, hq + hk:], c["wi"], q=None if q is None else x[:, :, :hq],
                    q_out=None if q is None else out, rope=c["rope"], positions=c["pos"], l0=c["layer0"], l1=c["layer0"] + c["layers"])
    return out


def _check(c, out, before):
    hq, hk = c["hq"], c["hk"]
    x = O.bf16_bits_to_f64(U.bits(c["qkv"]))
    y = np.array(x)
    if c["rope"] is not None:
        y[:, :, :hq + hk] = O.rotate(x[:, :, :hq + hk], c["pos"].cpu().numpy(), c["freq"].cpu().numpy(), c["sections"], c["interleaved"])
    room = 2.0 ** -8 * np.abs(y) + (0 if c["rope"] is None else 2.0 ** -20 * np.abs(x).max())
    if out is not None:
        assert (np.abs(out.double().cpu().numpy() - y[:, :, :hq]) <= room[:, :, :hq]).all()
    want, tol = before.double().cpu().numpy(), np.zeros(before.shape)
    row = 0
    for r, w in enumerate(c["wins"]):
        for j in range(c["L"][r] - w, c["L"][r]):
            p, s = c["pt"][r, j // c["page"]], j % c["page"]
            for l in range(c["layers"]):
                want[c["layer0"] + l, 0, p, s], tol[c["layer0"] + l, 0, p, s] = y[l, row, hq:hq + hk], room[l, row, hq:hq + hk]
                want[c["layer0"] + l, 1, p, s] = y[l, row, hq + hk:]
            row += 1
    assert (np.abs(c["pool"].double().cpu().numpy() - want) <= tol).all()        # the rest of the pool as it was
    c["dec"].check_status()


@pytest.mark.parametrize("kw", [
    dict(ctx=[0], wins=[1]), dict(ctx=[5, 100, 31, 16], wins=[1, 1, 1, 1]), dict(ctx=[3, 0, 40], wins=[17, 0, 60]),
    dict(ctx=[7, 9], wins=[4, 5], layers=3, layer0=1), dict(ctx=[7, 9], wins=[4, 5], D=128, rotary=128, sections=[16, 24, 24]),
    dict(ctx=[7, 9], wins=[4, 5], D=128, rotary=64, sections=[10, 0, 22]), dict(ctx=[7, 9], wins=[4, 5], D=80, rotary=40),
    dict(ctx=[7, 9], wins=[4, 5], D=80, rotary=80, sections=[10, 10, 10, 10], interleaved=True),
    dict(ctx=[7, 9], wins=[4, 5], D=64, rotary=24, interleaved=True), dict(ctx=[7, 9], wins=[4, 5], D=64, rotary=6),
    dict(ctx=[7, 9], wins=[4, 5], D=64, rotary=6, interleaved=True), dict(ctx=[7, 9], wins=[4, 5], rotary=0),
    dict(ctx=[7, 9], wins=[4, 5], D=256, rotary=256), dict(ctx=[7, 9], wins=[4, 5], D=8, rotary=8, hk=1, G=1),
    dict(ctx=[7, 9], wins=[4, 5], page=5), dict(ctx=[7, 9], wins=[4, 5], shift=1), dict(ctx=[7, 9], wins=[4, 5], shift=8, hk=1, G=8)])
def test_rows_turn_and_land_in_their_slots(kw):
    c = _case(seed=len(str(kw)), **kw)
    before = c["pool"].clone()
    out = _run(c)
    _check(c, out, before)


def test_many_requests():
    g = np.random.default_rng(2)
    c = _case(g.integers(0, 40, 100).tolist(), g.integers(0, 4, 100).tolist())
    before = c["pool"].clone()
    _check(c, _run(c), before)


def test_without_q_and_in_place():
    c = _case([7, 9], [4, 5])
    before = c["pool"].clone()
    _run(c, q=None)
    _check(c, None, before)
    # q_out may be q's own memory when q lies as q_out does
    c = _case([7, 9], [4, 5], seed=3)
    want = _run(c)
    q = c["qkv"][:, :, :c["hq"]].contiguous()
    c["dec"].append(c["qkv"][:, :, c["hq"]:c["hq"] + c["hk"]], c["qkv"][:, :, c["hq"] + c["hk"]:], c["wi"], q=q, q_out=q, rope=c["rope"],
                    positions=c["pos"])
    assert torch.equal(q, want)


def test_far_positions_keep_their_angle():
    c = _case([0], [3])
    c["pos"].copy_(torch.tensor([[2 ** 31 - 1, 123456789, -5]], dtype=torch.int32))
    before = c["pool"].clone()
    _check(c, _run(c), before)


def test_rows_that_fit_nowhere_are_reported_and_dropped():
    c = _case([7, 9], [4, 5], seed=1)
    c["dec"].page_table[1, 0] = 99999
    before = c["pool"].clone()
    _run(c)
    assert c["dec"].status.cpu().tolist()[:3] == [B.E_BADPAGE, 1, 99999]
    assert int((c["pool"] != before).flatten(3).any(-1).sum()) <= 2 * 1 * 1      # request 0's page only, K and V
    c = _case([0, 9], [4, 5], seed=1)
    c["dec"].seq_len[0] = 2                                                      # two of its four rows fall before token 0
    _run(c)
    assert c["dec"].status.cpu().tolist()[:2] == [B.E_INVALID, 0]
    c = _case([7, 9], [4, 5], seed=1)
    c["dec"].seq_len[1] = 1 << 20                                                # beyond the table
    _run(c)
    assert c["dec"].status.cpu().tolist()[:2] == [B.E_INVALID, 1]


def test_the_binding_checks_shapes():
    c = _case([7, 9], [4, 5])
    k = c["qkv"][:, :, :c["hk"]]
    with pytest.raises(ValueError):
        c["dec"].append(k, k[:, :, :1], c["wi"])
    with pytest.raises(ValueError):
        c["dec"].append(k, k, c["wi"], q=c["qkv"][:, :, :c["hq"]], q_out=k.contiguous())
    with pytest.raises(ValueError):
        c["dec"].append(k, k, c["wi"], rope=c["rope"])
