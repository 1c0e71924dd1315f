"""The decoding calls as they are used: decode steps that append to a paged cache and attend over it, the LSE handed to the
streaming score, a compression step in between, branches that go on alone, and the log probabilities beside the monitor."""
import numpy as np
import pytest
import torch

from oracle import actkv_oracle as O
from paper_2609_31395_b200 import binding as B
from paper_2609_31395_b200 import harness as H
from paper_2609_31395_b200 import synth

import parity_util as U

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _close(got, want, scale=1.0):
    got = got.float().cpu().numpy()
    # half a bf16 step of the value and float32 noise of sums over values of order 1
    assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 2e-4 * scale).all()


def test_decode_compress_branch_and_go_on():
    NL, hk, G, D, P, R = 2, 2, 4, 64, 16, 3
    hq, width = hk * G, 40
    gen = torch.Generator(device=DEV).manual_seed(0)
    pool = torch.randn((NL, 2, 120, P, hk, D), generator=gen, device=DEV, dtype=torch.bfloat16)
    table = torch.full((R, width), -1, dtype=torch.int32, device=DEV)
    seq_len, free, fc = _i32([0] * R), torch.randperm(120, generator=torch.Generator().manual_seed(1)).to(torch.int32).to(DEV), _i32([120])
    dec = H.Decoder(pool, table, seq_len, free, fc, hq, 420, 300, 600, NL)
    freq = 1.0 / 10000.0 ** (torch.arange(D // 2, device=DEV) / (D // 2))
    rope = H.Rope(freq, [D // 2])
    lens, pos0 = [0] * R, [0] * R
    scale = D ** -0.5

    def step(wins):
        """Every request's new tokens: pages, rows, attention; checked against the oracle on what the cache then holds."""
        rows = sum(wins)
        wi = _i32([0] + np.cumsum(wins).tolist())
        for r in range(R):
            lens[r] += wins[r]
        dec.resize(_i32(lens))
        qkv = torch.randn((NL, rows, hq + 2 * hk, D), generator=gen, device=DEV, dtype=torch.bfloat16)
        pos = _i32([[pos0[r] + w for r in range(R) for w in range(wins[r])]])
        for r in range(R):
            pos0[r] += wins[r]
        q = torch.empty((NL, rows, hq, D), dtype=torch.bfloat16, device=DEV)
        dec.append(qkv[:, :, hq:hq + hk], qkv[:, :, hq + hk:], wi, q=qkv[:, :, :hq], q_out=q, rope=rope, positions=pos)
        out, lse = torch.empty_like(q), torch.empty(q.shape[:3], device=DEV)
        for l in range(NL):                                                 # layer by layer, as a model does
            dec.attend(q[l:l + 1], wi, scale, True, out[l:l + 1], lse[l:l + 1], l0=l)
        dec.check_status()
        want, wl = O.attend(U.bits(pool), table.cpu().numpy(), seq_len.cpu().numpy(), U.bits(q), wi.cpu().numpy(), hq, scale, True)
        _close(out, want)
        assert np.abs(lse.cpu().numpy() - wl).max() <= 1e-4
        return q, wi, lse

    step([200, 90, 130])                                                    # prompts
    for _ in range(3):
        step([1, 1, 1])
    # the LSE of a window is the one that the score takes: same scores as with the LSE computed there
    q, wi, lse = step([8, 8, 8])
    tok = _i32([0] + np.cumsum(lens).tolist())
    budget = _i32([60, 90, 50])
    sz = H.StepSizes(R, 24, 8, sum(lens), max(lens), 200, 90)
    comp = H.Compressor(pool, table, seq_len, free, fc, hq, sz, want_lse=True)
    comp.run_score(q, wi, tok, scale, True)
    own = comp.score.clone()
    comp.run_score(q, wi, tok, scale, True, lse_in=lse)
    assert U.max_rel(comp.score.cpu().numpy(), own.cpu().numpy()) < 1e-4
    assert (comp.lse - lse).abs().max().item() < 1e-4
    comp.step(q, wi, tok, budget, scale, True, lse_in=lse)                  # the cache is cut
    comp.check_status()
    lens[:] = [min(a, b) for a, b in zip(lens, [60, 90, 50])]
    assert seq_len.cpu().tolist() == lens
    step([1, 0, 2])                                                         # and decoding goes on, positions where they were
    # request 0 goes on in request 2's place as a branch
    lens[2] = 0
    dec.resize(_i32(lens))
    lens[2], pos0[2] = lens[0], pos0[0]
    dec.resize(_i32(lens))
    dec.copy(_i32([0]), _i32([2]), _i32([lens[0]]), lens[0])
    a = [U.bits(pool[:, :, table[r, j // P].item(), j % P]) for r in (0, 2) for j in (0, lens[0] // 2, lens[0] - 1)]
    assert all(np.array_equal(x, y) for x, y in zip(a[:3], a[3:]))
    step([2, 1, 1])
    # everything is given back
    dec.resize(_i32([0] * R))
    dec.check_status()
    assert int(fc) == 120 and sorted(free.cpu().tolist()) == list(range(120))


def test_logprob_beside_the_monitor():
    logits, tind = synth.confidence_logits(2, 40, 4096, seed=1, device=DEV)
    hist, hlen = torch.zeros((2, 256), device=DEV), _i32([0, 0])
    ws = torch.empty(B.actkv_budget_workspace_bytes(80, 2, 256) + 256, dtype=torch.uint8, device=DEV)
    status = _i32([0] * 4)
    B.actkv_budget(logits, tind, 80, 4096, hist, hlen, 256, B.BudgetParams.paper_defaults(), None, _i32([5, 5]), _i32([0, 0]), None, 2, ws, status)
    o = H.LogprobBuffers(80, 0, 20, DEV)
    B.actkv_logprob(logits, None, None, o.entropy, o.lse, o.top_logprob, o.top_index, o.status)
    # the monitor's confidence is minus the mean of the 20 largest log probabilities
    T = -o.top_logprob.double().mean(1).cpu()
    assert (T - hist[:, :40].reshape(-1).double().cpu()).abs().max().item() < 2e-5


def test_a_decode_step_in_one_graph():
    NL, hk, G, D, P, R = 1, 2, 4, 128, 16, 4
    hq = hk * G
    gen = torch.Generator(device=DEV).manual_seed(3)
    lens = [100, 31, 47, 15]
    need = [-(-n // P) for n in lens]
    pool = torch.randn((NL, 2, 60, P, hk, D), generator=gen, device=DEV, dtype=torch.bfloat16)
    perm = torch.randperm(60, generator=torch.Generator().manual_seed(1)).to(torch.int32)
    table = torch.full((R, 12), -1, dtype=torch.int32)
    at = 0
    for r, n in enumerate(need):
        table[r, :n] = perm[at:at + n]
        at += n
    free = torch.full((60,), -1, dtype=torch.int32)
    free[:60 - at] = perm[at:]
    table, free = table.to(DEV), free.to(DEV)
    dec = H.Decoder(pool, table, _i32(lens), free, _i32([60 - at]), hq, R, 1, 190)
    wi = _i32(list(range(R + 1)))
    new_len, pos = _i32(lens), _i32([lens])
    qkv = torch.randn((NL, R, hq + 2 * hk, D), generator=gen, device=DEV, dtype=torch.bfloat16)
    q, out, lse = (torch.empty((NL, R, hq, D), dtype=torch.bfloat16, device=DEV) for _ in range(2)), None, None
    q, out = q
    lse = torch.empty((NL, R, hq), device=DEV)
    rope = H.Rope(torch.rand(D // 2, device=DEV), [D // 2])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        new_len.add_(1)
        dec.resize(new_len)
        dec.append(qkv[:, :, hq:hq + hk], qkv[:, :, hq + hk:], wi, q=qkv[:, :, :hq], q_out=q, rope=rope, positions=pos)
        dec.attend(q, wi, D ** -0.5, True, out, lse)
    for step in range(20):
        qkv.normal_(generator=gen)
        g.replay()
        torch.cuda.synchronize()
        if step % 6 == 5:
            want, wl = O.attend(U.bits(pool), table.cpu().numpy(), dec.seq_len.cpu().numpy(), U.bits(q), wi.cpu().numpy(), hq, D ** -0.5, True)
            _close(out, want)
            assert np.abs(lse.cpu().numpy() - wl).max() <= 1e-4
    dec.check_status()
    assert dec.seq_len.cpu().tolist() == [n + 20 for n in lens]
