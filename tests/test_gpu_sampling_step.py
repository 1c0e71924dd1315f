"""The calls around a model's logits as they are used: a cache is cut, its keys move to the positions that are left, decoding goes on there, the
logits are put under rules, a token is drawn, scored, and fed back; by calls of their own and as one captured graph."""
import numpy as np
import pytest
import torch

from oracle import actkv_oracle as O
from paper_2609_31395_b200 import binding as B
from paper_2609_31395_b200 import harness as H

import parity_util as U

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NL, HK, G, D, P, R, VOCAB = 2, 2, 2, 64, 16, 3, 1003
HQ, SCALE = HK * G, D ** -0.5


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _f32(x):
    return torch.tensor(x, dtype=torch.float32, device=DEV)


class Model:
    """Two layers that only look, random weights: token -> q, k, v per layer; logits from what the layers saw."""

    def __init__(self, seed):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.qkv = torch.randn((NL, VOCAB, HQ + 2 * HK, D), generator=g, device=DEV).to(torch.bfloat16)
        self.out = torch.randn((NL * HQ * D, VOCAB), generator=g, device=DEV) * 0.35
        self.pool = torch.randn((NL, 2, 60, P, HK, D), generator=g, device=DEV).to(torch.bfloat16)
        self.table = torch.full((R, 20), -1, dtype=torch.int32, device=DEV)
        self.seq_len, self.fc = _i32([0] * R), _i32([60])
        self.free = torch.randperm(60, generator=torch.Generator().manual_seed(seed)).to(torch.int32).to(DEV)
        self.dec = H.Decoder(self.pool, self.table, self.seq_len, self.free, self.fc, HQ, 256, 128, 320, NL)
        self.freq = 1.0 / 10000.0 ** (torch.arange(D // 2, device=DEV) / (D // 2))
        self.rope = H.Rope(self.freq, [16, 16])                             # two axes
        cap = 200
        self.tokens, self.hist, self.prompt = torch.zeros((R, cap), dtype=torch.int32, device=DEV), _i32([0] * R), _i32([0] * R)
        self.words = torch.randint(-2 ** 31, 2 ** 31 - 1, (2, (VOCAB + 31) // 32), generator=g, device=DEV).to(torch.int32)
        self.allow_row = _i32([-1, 0, 1])
        self.rules = H.LogitRules(self.tokens, self.hist, self.prompt, _f32([1.1, 1.0, 1.3]), _f32([0.0, 0.4, 0.2]), _f32([0.3, 0.0, -0.1]), _i32([0, 2, 2, 3]),
                                  _i32([5, 900, 17]), _f32([2.0, -np.inf, 1.5]), self.words, self.allow_row)
        self.sampler = H.Sampler(R, DEV)
        self.t, self.k, self.p, self.m = _f32([0.8, 1.0, 0.0]), _i32([40, 0, 0]), _f32([0.9, 0.95, 1.0]), _f32([0.0, 0.01, 0.0])
        self.one = _i32(range(R + 1))
        self.new_len = _i32([0] * R)
        self.q = torch.empty((NL, R, HQ, D), dtype=torch.bfloat16, device=DEV)
        self.seen = torch.empty_like(self.q)
        self.lse = torch.empty((NL, R, HQ), device=DEV)
        self.logits, self.raw = torch.empty((R, VOCAB), device=DEV), torch.empty((R, VOCAB), device=DEV)
        self.pos = torch.empty((2, R), dtype=torch.int32, device=DEV)

    def prompts(self, lens, seed):
        """Prompts into the cache; the token's index is its position on both axes."""
        g = torch.Generator(device=DEV).manual_seed(seed)
        rows = sum(lens)
        tok = torch.randint(0, VOCAB, (rows,), generator=g, device=DEV)
        wi = _i32([0] + np.cumsum(lens).tolist())
        self.dec.resize(_i32(lens))
        x = self.qkv[:, tok]
        pos = _i32(np.tile(np.concatenate([np.arange(n) for n in lens]), (2, 1)))
        q = torch.empty((NL, rows, HQ, D), dtype=torch.bfloat16, device=DEV)
        self.dec.append(x[:, :, HQ:HQ + HK], x[:, :, HQ + HK:], wi, q=x[:, :, :HQ], q_out=q, rope=self.rope, positions=pos)
        for r, n in enumerate(lens):
            self.tokens[r, :n] = tok[wi[r]:wi[r + 1]].to(torch.int32)
        self.hist.copy_(_i32(lens))
        self.prompt.copy_(_i32(lens))
        self.dec.check_status()
        return x[:, :, HQ:HQ + HK], q, wi

    def cut(self, q, wi, lens, budget):
        """The cache down to the budget, and the surviving keys to positions 0, 1, ...; returns the survivors per (layer, KV head) and request."""
        sz = H.StepSizes(R, 3 * 8, 8, sum(lens), max(lens), sum(budget), max(budget))
        comp = H.Compressor(self.pool, self.table, self.seq_len, self.free, self.fc, HQ, sz)
        last = torch.cat([q[:, wi[r + 1] - 8:wi[r + 1]] for r in range(R)], 1)
        comp.step(last, _i32([0, 8, 16, 24]), wi, _i32(budget), SCALE, True)
        comp.check_status()
        was = comp.sel_idx[None].expand(2, -1, -1)                          # both axes had the index
        self.dec.reposition(self.rope, comp.keep_indptr, max(budget), was)
        self.dec.check_status()
        return comp.sel_idx.cpu().numpy(), comp.keep_indptr.cpu().tolist()

    def step(self, u):
        """One token per request: all of it on the device, so that it can be captured."""
        self.new_len.copy_(self.seq_len + 1)
        self.pos.copy_(self.seq_len.expand(2, R))
        token = self.tokens.gather(1, self.hist.long()[:, None] - 1)[:, 0].long()
        x = self.qkv[:, token]
        self.dec.resize(self.new_len)
        self.dec.append(x[:, :, HQ:HQ + HK], x[:, :, HQ + HK:], self.one, q=x[:, :, :HQ], q_out=self.q, rope=self.rope, positions=self.pos)
        self.dec.attend(self.q, self.one, SCALE, True, self.seen, self.lse)
        torch.mm(self.seen.transpose(0, 1).reshape(R, -1).float(), self.out, out=self.raw)
        self.sampler.penalize(self.raw, self.one, self.rules, max_hist=self.tokens.shape[1], out=self.logits)
        self.sampler.sample(self.logits, u, self.t, self.k, self.p, self.m)
        self.tokens.scatter_(1, self.hist.long()[:, None], self.sampler.token[:, None])
        self.hist.add_(1)


def test_cut_move_and_go_on():
    lens, budget = [100, 61, 128], [40, 61, 33]                             # (the second keeps everything)
    m = Model(0)
    k, q, wi = m.prompts(lens, 1)
    sel, ind = m.cut(q, wi, lens, budget)
    assert m.seq_len.cpu().tolist() == budget
    # the keys are the prompts' own, turned to where they now are.  Two roundings to bf16 (append, reposition; half a step of the larger of a pair each:
    # 2^-8 of its length twice) and the angles' part, 2^-19 twice.
    f = m.freq.cpu().numpy()
    kk = k.double().cpu().numpy()
    table = m.table.cpu().numpy()
    for l in range(NL):
        for h in range(HK):
            for r in range(R):
                idx = sel[l * HK + h, ind[r]:ind[r + 1]]
                n = len(idx)
                raw = kk[l, wi[r].item() + idx, h]
                want = O.reposition_unit(raw, np.zeros((2, n)), np.tile(np.arange(n), (2, 1)), f, f, [16, 16], False)
                got = m.pool[l, 0, table[r, np.arange(n) // P].tolist(), (np.arange(n) % P).tolist(), h].double().cpu().numpy()
                size = np.hypot(raw[:, :D // 2], raw[:, D // 2:])
                tol = np.concatenate([size, size], 1) * (2 * 2.0 ** -8 + 2.0 ** -16 + 4 * 2.0 ** -19)
                assert (np.abs(got - want) <= tol).all()
    gen = torch.Generator(device=DEV).manual_seed(5)
    allowed = np.unpackbits(m.words.cpu().numpy().view(np.uint8), axis=1, bitorder="little")[:, :VOCAB].astype(bool)
    o = H.LogprobBuffers(R, 1, 1, DEV)
    for _ in range(6):
        u = torch.rand(R, generator=gen, device=DEV)
        m.step(u)
        m.dec.check_status()
        m.sampler.check_status()
        # attention over moved and new keys, from what the cache holds
        want, _ = O.attend(U.bits(m.pool), m.table.cpu().numpy(), m.seq_len.cpu().numpy(), U.bits(m.q), m.one.cpu().numpy(), HQ, SCALE, True)
        assert (np.abs(m.seen.float().cpu().numpy() - want) <= 2.0 ** -8 * np.abs(want) + 2e-4).all()
        hist, tokens, raw, z = m.hist.cpu().tolist(), m.tokens.cpu().numpy(), m.raw.double().cpu().numpy(), m.logits.double().cpu().numpy()
        rep, freq, pres, bias = [1.1, 1.0, 1.3], [0.0, 0.4, 0.2], [0.3, 0.0, -0.1], [{5: 2.0, 900: -np.inf}, {}, {17: 1.5}]
        f32 = lambda x: float(np.float32(x))
        B.actkv_logprob(m.logits, m.sampler.token[:, None], o.logprob, o.entropy, o.lse, o.top_logprob, o.top_index, o.status)
        for r in range(R):
            past = tokens[r, :hist[r] - 1]
            ok = None if r == 0 else allowed[r - 1]
            w = O.penalize_row(raw[r], past, lens[r], f32(rep[r]), f32(freq[r]), f32(pres[r]), {t: f32(b) for t, b in bias[r].items()}, ok)
            fin = np.isfinite(w)
            assert (np.isfinite(z[r]) == fin).all()
            size = np.abs(raw[r][fin]) * 1.3 + 2.6 + 0.4 * 7 + 0.3          # (a bias of 2 times 1.3; at most 6 own tokens)
            assert (np.abs(z[r][fin] - w[fin]) <= 5 * 2.0 ** -24 * size).all()
            got = (int(m.sampler.token[r]), int(m.sampler.kept[r]))
            token, logprob, kept = O.sample_row(z[r], float(u[r]), float(m.t[r]), int(m.k[r]), float(m.p[r]), float(m.m[r]))
            assert got == (token, kept)
            assert abs(float(m.sampler.logprob[r]) - logprob) <= 2.0 ** -23 * abs(logprob) + 2.0 ** -26
            assert tokens[r, hist[r] - 1] == token and z[r][token] > -np.inf
            # the score of the drawn token under the whole distribution
            whole = z[r][token] - z[r][fin].max() - np.log(np.exp(z[r][fin] - z[r][fin].max()).sum())
            assert abs(float(o.logprob[r, 0]) - whole) <= 1e-5 * max(1.0, abs(whole))
    assert m.seq_len.cpu().tolist() == [b + 6 for b in budget]


def test_one_graph_per_token():
    lens, budget = [60, 44, 31], [20, 30, 31]
    us = torch.rand((20, R), generator=torch.Generator(device=DEV).manual_seed(2), device=DEV)

    def start():
        m = Model(3)
        _, q, wi = m.prompts(lens, 4)
        m.cut(q, wi, lens, budget)
        return m
    a, b = start(), start()
    for u in us:
        a.step(u)
    a.dec.check_status()
    a.sampler.check_status()
    u = us[0].clone()
    b.step(u)                                                               # (the first token by itself: libraries are loaded)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.step(u)
    for x in us[1:]:
        u.copy_(x)
        g.replay()
    b.dec.check_status()
    b.sampler.check_status()
    assert torch.equal(a.hist, b.hist) and torch.equal(a.tokens, b.tokens) and torch.equal(a.seq_len, b.seq_len)
    assert a.seq_len.cpu().tolist() == [n + 20 for n in budget]
    assert torch.equal(a.pool, b.pool) and torch.equal(a.logits, b.logits) and torch.equal(a.sampler.logprob, b.sampler.logprob)
