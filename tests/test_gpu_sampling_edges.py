"""Calls of actkv_reposition, actkv_penalize and actkv_sample at the ends of their ranges: rows and pages that lie further than 32 bits apart, the largest
vocabulary, logits and temperatures at the ends of float32, one token all through a history, calls on two streams at once, graphs that take turns."""
import numpy as np
import pytest
import torch

from oracle import actkv_oracle as O
from paper_2609_31395_b200 import binding as B
from paper_2609_31395_b200 import harness as H

import parity_util as U

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
INF = float("inf")


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _f32(x):
    return torch.tensor(x, dtype=torch.float32, device=DEV)


def _drawn(z, s, u, t=1.0, k=0, p=1.0, m=0.0):
    for i, row in enumerate(z.double().cpu().numpy()):
        token, logprob, kept = O.sample_row(row, float(u[i]), t, k, p, m)
        assert (int(s.token[i]), int(s.kept[i])) == (token, kept)
        assert float(s.logprob[i]) == logprob or abs(float(s.logprob[i]) - logprob) <= 2.0 ** -23 * abs(logprob) + 2.0 ** -26


def test_rows_further_apart_than_32_bits():
    vocab, apart = 1000, (1 << 30) + 8
    full = torch.empty(2 * apart + vocab, dtype=torch.bfloat16, device=DEV)
    z = full.as_strided((3, vocab), (apart, 1))
    g = torch.Generator(device=DEV).manual_seed(0)
    z.copy_(torch.randn((3, vocab), generator=g, device=DEV) * 3)
    was = z.double().cpu().numpy()
    hist = torch.randint(0, vocab, (3, 50), generator=g, device=DEV).to(torch.int32)
    rules = H.LogitRules(hist, _i32([50] * 3), None, _f32([1.25] * 3), _f32([0.5] * 3))
    s = H.Sampler(3, DEV)
    s.penalize(z, _i32([0, 1, 2, 3]), rules, 1, 50)
    u = torch.rand(3, generator=g, device=DEV)
    s.sample(z, u)
    s.check_status()
    for r in range(3):
        want = O.penalize_row(was[r], hist[r].cpu().numpy(), 0, 1.25, 0.5, 0.0, {}, None)
        # float32 as in the parity tests, and one rounding to bf16
        assert (np.abs(z[r].double().cpu().numpy() - want) <= 2.0 ** -8 * np.abs(want) + 5 * 2.0 ** -24 * (1.25 * np.abs(was[r]) + 4)).all()
    _drawn(z, s, u)


def test_pages_further_apart_than_32_bits():
    P, hk, D = 16, 2, 64
    page = P * hk * D
    full = torch.empty((1 << 31) + 8 * page, dtype=torch.bfloat16, device=DEV)
    pool = full.as_strided((1, 2, 2, P, hk, D), ((1 << 31) + 6 * page, 3 * page, 1 << 31, hk * D, D, 1))
    k = torch.randn((2, P, hk, D), generator=torch.Generator(device=DEV).manual_seed(1), device=DEV).to(torch.bfloat16)
    pool[0, 0].copy_(k)
    freq = 1.0 / 10000.0 ** (torch.arange(D // 2, device=DEV) / (D // 2))
    dec = H.Decoder(pool, _i32([[0, 1]]), _i32([30]), _i32([0, 0]), _i32([0]), hk)
    to = torch.arange(100, 130, device=DEV, dtype=torch.int32)
    dec.reposition(H.Rope(freq, [D // 2]), _i32([0, 30]), 30, None, to)
    dec.check_status()
    raw = k.reshape(2 * P, hk, D).double().cpu().numpy()
    got = pool[0, 0].reshape(2 * P, hk, D).double().cpu().numpy()
    f = freq.cpu().numpy()
    for h in range(hk):
        want = O.reposition_unit(raw[:30, h], np.arange(30)[None], np.arange(100, 130)[None], f, f, [D // 2], False)
        size = np.abs(raw[:30, h, :D // 2]) + np.abs(raw[:30, h, D // 2:])
        assert (np.abs(got[:30, h] - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -19 * np.concatenate([size, size], 1)).all()
    assert np.array_equal(got[30:], raw[30:])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows", [1, 40])
def test_the_largest_vocabulary(rows, dtype):
    vocab = 344064
    g = torch.Generator(device=DEV).manual_seed(rows)
    z = (torch.randn((rows, vocab), generator=g, device=DEV) * 2).to(dtype)
    u = torch.rand(rows, generator=g, device=DEV)
    s = H.Sampler(rows, DEV)
    take = [0, rows - 1]
    for kw in (dict(), dict(k=50), dict(p=0.9), dict(k=5000, p=0.7), dict(t=0.0)):
        full = lambda name, d: None if name not in kw else torch.full((rows,), kw[name], dtype=d, device=DEV)
        s.sample(z, u, full("t", torch.float32), full("k", torch.int32), full("p", torch.float32))
        s.check_status()
        for i in take:
            token, logprob, kept = O.sample_row(z[i].double().cpu().numpy(), float(u[i]), kw.get("t", 1.0), kw.get("k", 0), float(np.float32(kw.get("p", 1.0))), 0.0)
            assert (int(s.token[i]), int(s.kept[i])) == (token, kept)
    with pytest.raises(B.ActKVError):
        s.sample(torch.zeros((1, vocab + 1), device=DEV), u[:1])


@pytest.mark.parametrize("vocab", [3001, 40963])
def test_logits_and_temperatures_at_the_ends_of_float32(vocab):
    g = torch.Generator(device=DEV).manual_seed(2)
    z = (torch.rand((6, vocab), generator=g, device=DEV) * 2 - 1) * 3.3e38
    u = torch.rand(6, generator=g, device=DEV)
    s = H.Sampler(6, DEV)
    for t, k, p, m in ((1e38, 0, 1.0, 0.0), (1e38, 0, 0.5, 0.0), (1e38, 200, 0.75, 0.0), (3e38, 0, 0.75, 0.25), (1.0, 20, 0.75, 0.0), (1.0, 0, 0.75, 0.0), (3e38, 40, 1.0, 0.0)):
        s.sample(z, u, _f32([t] * 6), _i32([k] * 6), _f32([p] * 6), _f32([m] * 6))
        s.check_status()
        _drawn(z, s, u, float(np.float32(t)), k, p, m)


def test_one_token_all_through_a_history():
    n, vocab = 1 << 20, 70
    tokens = torch.full((2, n), 33, dtype=torch.int32, device=DEV)
    tokens[1, n // 2:] = 66
    z = torch.randn((2, vocab), generator=torch.Generator(device=DEV).manual_seed(3), device=DEV)
    was = z.double().cpu().numpy()
    s = H.Sampler(2, DEV)
    s.penalize(z, _i32([0, 1, 2]), H.LogitRules(tokens, _i32([n, n]), _i32([7, n // 2 + 1]), _f32([1.5, 1.5]), _f32([2.0 ** -6] * 2), _f32([0.25] * 2)), 1, n)
    s.check_status()
    for r in range(2):
        want = O.penalize_row(was[r], tokens[r].cpu().numpy(), [7, n // 2 + 1][r], 1.5, 2.0 ** -6, 0.25, {}, None)
        made = [n - 7, n // 2 - 1][r] * 2.0 ** -6                           # what is subtracted: three roundings of it, two of the rest
        assert (np.abs(z[r].double().cpu().numpy() - want) <= 2.0 ** -24 * (5 * 1.5 * np.abs(was[r]) + 3 * (made + 1) * (want != was[r]))).all()


def test_on_two_streams_at_once():
    g = torch.Generator(device=DEV).manual_seed(4)
    z = [torch.randn((64, 151936), generator=g, device=DEV) * 2.5 for _ in range(2)]
    u = [torch.rand(64, generator=g, device=DEV) for _ in range(2)]
    p = _f32([0.9] * 64)
    hist = torch.randint(0, 151936, (64, 3000), generator=g, device=DEV).to(torch.int32)
    wi = _i32(range(65))
    rules = H.LogitRules(hist, _i32([3000] * 64), None, _f32([1.1] * 64))

    def once(x, uu, s, out):
        s.penalize(x, wi, rules, 1, 3000, out=out)
        s.sample(out, uu, None, None, p)
    alone = []
    for x, uu in zip(z, u):
        s, out = H.Sampler(64, DEV), torch.empty_like(x)
        once(x, uu, s, out)
        alone.append((s, out))
    torch.cuda.synchronize()
    streams, both = [torch.cuda.Stream() for _ in range(2)], [(H.Sampler(64, DEV), torch.empty_like(z[0])) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for st, x, uu, (s, out) in zip(streams, z, u, both):
            with torch.cuda.stream(st):
                once(x, uu, s, out)
    torch.cuda.synchronize()
    for (s, out), (s1, out1) in zip(alone, both):
        s1.check_status()
        assert torch.equal(s.token, s1.token) and torch.equal(s.logprob, s1.logprob) and torch.equal(s.kept, s1.kept) and torch.equal(out, out1)


def test_graphs_that_take_turns():
    g = torch.Generator(device=DEV).manual_seed(5)
    z, u, s = torch.randn((5, 5003), generator=g, device=DEV), torch.rand(5, generator=g, device=DEV), H.Sampler(5, DEV)
    few, many = _i32([5] * 5), _i32([3000] * 5)
    graphs = []
    for k in (few, many):
        graphs.append(torch.cuda.CUDAGraph())
        s.sample(z, u, None, k)
        with torch.cuda.graph(graphs[-1]):
            s.sample(z, u, None, k)
    for k, at in ((5, 0), (3000, 1), (5, 0)):
        z.copy_(torch.randn((5, 5003), generator=g, device=DEV))
        u.copy_(torch.rand(5, generator=g, device=DEV))
        graphs[at].replay()
        s.check_status()
        _drawn(z, s, u, k=k)


def test_rules_of_another_device_or_number_of_requests_are_refused():
    z, wi, s = torch.zeros((2, 64), device=DEV), _i32([0, 1, 2]), H.Sampler(2, DEV)
    rules = H.LogitRules(_i32([[1], [2]]), _i32([1, 1]))
    rules.desc.index = 1
    with pytest.raises(TypeError):
        s.penalize(z, wi, rules, 1, 1)
    rules = H.LogitRules(_i32([[1]]), _i32([1]))
    with pytest.raises(ValueError):
        B.actkv_penalize(z, wi, 2, rules.desc, 1, 1, z, s.status)
    s.penalize(z, wi, H.LogitRules(allow=_i32([[-1, 0], [0, -1]])), 1)      # (masks alone are of no number of requests)
    s.check_status()
    assert torch.isinf(z).sum().item() == 64 and z[0, 0] == 0 and z[1, 63] == 0
