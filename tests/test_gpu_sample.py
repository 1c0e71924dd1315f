"""GPU parity of actkv_sample against the float64 oracle.

Tokens and counts are whole: they are equal unless a random number or a limit falls next to a border, closer than the weights' rounding (2^-45 of the
largest each, 2^-50 relative from the exponential): over 2 * 10^5 tokens a sum is off by at most 2^-27, and by 2^-36 as roundings go, so that one
draw in 10^8 may differ.  Log probabilities: float64 until the rounding to float32, 2^-24 relative, beside 2^-27 of the sum."""
import numpy as np
import pytest
import torch

from oracle import actkv_oracle as O
from paper_2609_31395_b200 import binding as B
from paper_2609_31395_b200 import harness as H

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
INF = float("inf")


def _f32(x):
    return torch.tensor(x, dtype=torch.float32, device=DEV)


def _logits(rows, vocab, seed, dtype=torch.float32, kind="random"):
    g = torch.Generator(device=DEV).manual_seed(seed)
    z = torch.randn((rows, vocab), generator=g, device=DEV) * 2.5
    if kind == "masked":
        z.masked_fill_(torch.rand(z.shape, generator=g, device=DEV) > 0.05, -INF)
    elif kind == "lowest":
        z.masked_fill_(torch.rand(z.shape, generator=g, device=DEV) > 0.05, torch.finfo(torch.float32).min)
    elif kind == "ascending":
        z = z.sort(dim=1).values
    elif kind == "equal":
        z.fill_(-1.25)
    elif kind == "few values":
        z = z.round()
    elif kind == "sure":
        z[:, vocab // 2] += 40.0
    elif kind == "far":
        z += 5000.0
    elif kind == "flat":
        z *= 1e-3
    elif kind == "wide":
        z *= 1e30
    elif kind == "subnormal":
        z *= 1e-39
    elif kind == "alone":
        z.fill_(-INF)
        z[:, -1] = 3.0
    return z.to(dtype)


def _check(z, u, t, k, p, m, s):
    n = z.shape[0]
    col = lambda x, d: [d] * n if x is None else x.cpu().tolist()
    zz = z.double().cpu().numpy()
    got = list(zip(s.token[:n].tolist(), s.logprob[:n].tolist(), s.kept[:n].tolist()))
    for i, (uu, tt, kk, pp, mm) in enumerate(zip(u.cpu().tolist(), col(t, 1.0), col(k, 0), col(p, 1.0), col(m, 0.0))):
        token, logprob, kept = O.sample_row(zz[i], uu, tt, kk, pp, mm)
        assert (got[i][0], got[i][2]) == (token, kept), (i, got[i], (token, logprob, kept), (uu, tt, kk, pp, mm))
        assert got[i][1] == logprob or abs(got[i][1] - logprob) <= 2.0 ** -23 * abs(logprob) + 2.0 ** -26, (i, got[i], logprob)
    s.check_status()


def _run(z, seed=0, t=None, k=None, p=None, m=None, u=None):
    n = z.shape[0]
    g = torch.Generator(device=DEV).manual_seed(seed + 100)
    u = torch.rand(n, generator=g, device=DEV) if u is None else u
    full = lambda x, d: None if x is None else torch.full((n,), x, dtype=d, device=DEV) if not isinstance(x, torch.Tensor) else x
    t, k, p, m = full(t, torch.float32), full(k, torch.int32), full(p, torch.float32), full(m, torch.float32)
    s = H.Sampler(n + 1, DEV)
    s.token.fill_(-7), s.logprob.fill_(-7), s.kept.fill_(-7)
    s.sample(z, u, t, k, p, m)
    _check(z, u, t, k, p, m, s)
    assert s.token[n].item() == -7 and s.logprob[n].item() == -7 and s.kept[n].item() == -7
    return s


@pytest.mark.parametrize("rows,vocab", [(1, 1), (1, 2), (3, 7), (5, 33), (7, 1009), (2, 4096), (9, 8193), (2, 20481), (3, 40963), (2, 151936), (1, 262144),
                                        (1, 344064), (40, 32003), (200, 5000), (600, 130)])
@pytest.mark.parametrize("kw", [dict(), dict(k=1), dict(k=5), dict(p=0.9), dict(k=40, p=0.8, t=0.7), dict(m=0.1), dict(t=0.0), dict(t=1.7, p=0.97, m=0.001)])
def test_parity(rows, vocab, kw):
    _run(_logits(rows, vocab, rows + vocab), seed=vocab, **kw)


KINDS = ["masked", "lowest", "ascending", "equal", "few values", "sure", "far", "flat", "wide", "subnormal", "alone"]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("kw", [dict(), dict(k=3), dict(k=2000), dict(p=0.37), dict(k=300, p=0.61, t=0.5), dict(m=0.3), dict(t=0.0), dict(p=0.9999, t=3.0)])
def test_rows_of_many_kinds(kind, dtype, kw):
    _run(_logits(4, 9001, 5, dtype, kind), seed=3, **kw)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind", ["random", "equal", "few values", "flat", "masked"])
@pytest.mark.parametrize("kw", [dict(k=30000), dict(p=0.73), dict(k=100000, p=0.51, t=2.5), dict(k=1025), dict(p=0.02)])
def test_borders_among_many_tokens(kind, dtype, kw):
    _run(_logits(2, 151936, 6, dtype, kind), seed=4, **kw)


def test_settings_by_row():
    n = 64
    g = torch.Generator(device=DEV).manual_seed(9)
    pick = lambda *v: torch.tensor(v, device=DEV)[torch.randint(len(v), (n,), generator=g, device=DEV)]
    _run(_logits(n, 3001, 2), t=pick(0.0, 0.01, 0.3, 1.0, 30.0), k=pick(-1, 0, 1, 7, 3001, 1 << 30).to(torch.int32), p=pick(0.0, -1.0, 0.4, 0.95, 1.0, 7.0),
         m=pick(-1.0, 0.0, 0.01, 1.0, 5.0))


def test_random_numbers_at_their_ends():
    z = _logits(4, 777, 3)
    z[3, -5:] = -INF
    s = _run(z, u=_f32([0.0, 1.0, 1.0 - 2.0 ** -24, 1.0]))
    assert s.token.tolist()[:2] == [0, 776] and s.token[3].item() == 771
    _run(z, u=_f32([0.0, 1.0, 1.0 - 2.0 ** -24, 1.0]), k=9, p=0.9)


def test_tiny_and_large_temperatures():
    z = _logits(6, 5001, 8)
    t = _f32([1e-45, 1e-30, 1e-3, 1e3, 1e30, 3e38])
    _run(z, t=t)
    _run(z, t=t, k=50, p=0.8)
    _run(z, t=t, p=0.5, m=0.2)


def test_the_drawn_frequencies_are_the_probabilities():
    """20000 draws of 6 tokens: a count is off by at most 5 standard deviations, below 5 * sqrt(n) / 2."""
    n = 20000
    z = _f32([[0.0, 1.0, 2.0, -1.0, 0.5, -INF]]).repeat(n, 1)
    s = H.Sampler(n, DEV)
    s.sample(z, torch.rand(n, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV))
    p = torch.softmax(z[0].double(), 0).cpu()
    got = torch.bincount(s.token.long(), minlength=6).cpu()
    assert ((got - n * p).abs() <= 2.5 * n ** 0.5).all() and got[5] == 0


def test_rows_without_a_token():
    z = _logits(5, 3000, 1)
    z[0] = -INF
    z[1, 2999] = float("nan")
    z[2, 17] = INF
    z[3, 5] = -INF
    for kw in (dict(), dict(k=4), dict(p=0.7), dict(t=0.0)):
        s = _run(z, **kw)
        assert s.token.tolist()[:3] == [-1, -1, -1] and s.kept.tolist()[:3] == [0, 0, 0] and min(s.token.tolist()[3:5]) >= 0


@pytest.mark.parametrize("kw", [dict(t=-1.0), dict(t=INF), dict(t=float("nan")), dict(p=float("nan")), dict(m=float("nan")), dict(u=-0.1), dict(u=1.5),
                                dict(u=float("nan"))])
def test_a_row_with_bad_settings_is_reported(kw):
    z = _logits(3, 4000, 2)
    t, p, m, u = _f32([1.0] * 3), _f32([0.9] * 3), _f32([0.0] * 3), _f32([0.3] * 3)
    for name, x in (("t", t), ("p", p), ("m", m), ("u", u)):
        if name in kw:
            x[1] = kw[name]
    s = H.Sampler(3, DEV)
    s.sample(z, u, t, None, p, m)
    assert s.status.tolist()[:2] == [B.E_INVALID, 1]
    assert (s.token[1].item(), s.logprob[1].item(), s.kept[1].item()) == (-1, -INF, 0)
    s.status.zero_()
    for i in (0, 2):
        want = O.sample_row(z[i].double().cpu().numpy(), float(np.float32(0.3)), 1.0, 0, float(np.float32(0.9)), 0.0)
        assert (s.token[i].item(), s.kept[i].item()) == want[::2]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shift", [1, 2, 3, 5])
def test_rows_off_their_alignment(dtype, shift):
    g = torch.Generator(device=DEV).manual_seed(shift)
    full = (torch.randn((6, 2003 + shift), generator=g, device=DEV) * 3).to(dtype)
    _run(full[:, shift:shift + 2000], k=30, p=0.9)
    _run(full[::2, :2001])


def test_the_same_on_every_split():
    """One row alone has a cluster of eight CTAs, many rows have fewer: the same tokens, bit for bit."""
    z = _logits(1, 20000, 4)
    many, u = z.repeat(300, 1), torch.rand(300, device=DEV)
    a = H.Sampler(300, DEV)
    p = _f32([0.9] * 300)
    a.sample(many, u, None, None, p)
    b = H.Sampler(1, DEV)
    for i in range(0, 300, 23):
        b.sample(z, u[i:i + 1], None, None, p)
        assert (b.token[0], b.logprob[0], b.kept[0]) == (a.token[i], a.logprob[i], a.kept[i])


def test_captured_and_on_another_stream():
    z, u = _logits(20, 32003, 4), torch.rand(20, device=DEV)
    t, k, p, m = _f32([0.8] * 20), torch.full((20,), 50, dtype=torch.int32, device=DEV), _f32([0.95] * 20), _f32([0.0] * 20)
    s, stream, g = H.Sampler(20, DEV), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=stream):
        s.sample(z, u, t, k, p, m)
    for seed in range(3):
        z.copy_(_logits(20, 32003, seed + 40))
        u.uniform_()
        g.replay()
        torch.cuda.synchronize()
        _check(z, u, t, k, p, m, s)


def test_results_that_are_not_asked_for():
    z, u = _logits(4, 500, 4), _f32([0.1, 0.4, 0.6, 0.9])
    s = H.Sampler(4, DEV)
    s.sample(z, u)
    token = torch.full((4,), -9, dtype=torch.int32, device=DEV)
    B.actkv_sample(z, u, None, None, None, None, token, None, None, s.status)
    assert torch.equal(token, s.token)
    z[1] = -INF
    B.actkv_sample(z, u, _f32([0.0, 1.0, 1.0, -1.0]), None, None, None, token, None, None, s.status)
    assert token[1] == -1 and token[3] == -1 and token[0] == z[0].argmax()


def test_shapes_that_do_not_fit_are_refused():
    s, z, u = H.Sampler(4, DEV), _logits(4, 500, 4), torch.rand(4, device=DEV)
    for bad in (dict(u=u[:3]), dict(temperature=u[:2]), dict(top_k=torch.zeros(3, dtype=torch.int32, device=DEV))):
        with pytest.raises(ValueError):
            s.sample(**{**dict(logits=z, u=u), **bad})
    for bad in (dict(u=u.double()), dict(u=u.cpu()), dict(top_k=u), dict(top_p=u.half()), dict(logits=z.half()), dict(logits=z.t().contiguous().t())):
        with pytest.raises(TypeError):
            s.sample(**{**dict(logits=z, u=u), **bad})
    with pytest.raises(ValueError):
        H.Sampler(3, DEV).sample(z, u)
    with pytest.raises(B.ActKVError) as e:
        H.Sampler(1, DEV).sample(torch.zeros((1, 344065), device=DEV), u[:1])
    assert e.value.code == B.E_TOOBIG
