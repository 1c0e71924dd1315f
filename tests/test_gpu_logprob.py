"""GPU parity of actkv_logprob against the float64 oracle.

Tolerance: with n logits, x - m is one rounding (2^-24 of |x - m|, below 2^-24 * range), exp of 2 ulp; sums of n float32 terms over 512
threads a CTA: n / 512 + 32 steps of 2^-24; ln of float32: 2^-21 absolute.  So ln S is off by at most e = 2^-21 + (n / 512 + 40) 2^-24
+ range * 2^-23 (range: where the mass lies, below 32 here), a log probability by e + |value| 2^-22, the lse by e + |m| 2^-23, and the
entropy, a mean of x - m under the same weights, by e (1 + H) + 32 e."""
import numpy as np
import pytest
import torch

from oracle import actkv_oracle as O
from paper_2609_31395_b200 import binding as B
from paper_2609_31395_b200 import harness as H

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _run(z, given, k):
    n_given = 0 if given is None else given.shape[1]
    o = H.LogprobBuffers(z.shape[0], n_given, k, DEV)
    for t in (o.logprob, o.entropy, o.lse, o.top_logprob):
        t.fill_(77.0)
    B.actkv_logprob(z, given, o.logprob, o.entropy, o.lse, o.top_logprob, o.top_index, o.status)
    return o


def _check(z, given, k, o):
    zz = z.double().cpu().numpy()
    lse, logp, ent = O.log_probabilities(zz)
    n = zz.shape[1]
    e = 2.0 ** -21 + (n / 512 + 40) * 2.0 ** -24 + 32 * 2.0 ** -23
    m = np.where(np.isfinite(lse), np.abs(lse), 0.0)

    def near(got, want, tol):
        got = got.double().cpu().numpy()
        fin = np.isfinite(want)
        assert np.array_equal(got[~fin], want[~fin])
        over = np.abs(got[fin] - want[fin]) - np.broadcast_to(tol, want.shape)[fin]
        assert (over <= 0).all(), float(over.max())
    near(o.lse, lse, e + m * 2.0 ** -23)
    near(o.entropy, ent, e * (1 + ent) + 32 * e)
    if given is not None:
        at = np.take_along_axis(logp, given.long().cpu().numpy(), 1)
        near(o.logprob, at, e + np.where(np.isfinite(at), np.abs(at), 0) * 2.0 ** -22)
    if k:
        idx = O.top_tokens(zz, k)
        c = idx.shape[1]
        got = o.top_index.cpu().numpy()
        assert np.array_equal(got[:, :c], idx) and (got[:, c:] == -1).all()
        at = np.take_along_axis(logp, idx, 1)
        near(o.top_logprob[:, :c], at, e + np.where(np.isfinite(at), np.abs(at), 0) * 2.0 ** -22)
        assert torch.isneginf(o.top_logprob[:, c:]).all()
    assert o.status.cpu().tolist()[0] == 0


def _logits(rows, vocab, seed, dtype=torch.float32, kind="random"):
    g = torch.Generator(device=DEV).manual_seed(seed)
    z = torch.randn((rows, vocab), generator=g, device=DEV) * 2.5
    if kind == "masked":
        z.masked_fill_(torch.rand(z.shape, generator=g, device=DEV) > 0.05, -float("inf"))
    elif kind == "lowest":
        z.masked_fill_(torch.rand(z.shape, generator=g, device=DEV) > 0.05, torch.finfo(torch.float32).min)
    elif kind == "ascending":
        z = z.sort(dim=1).values
    elif kind == "descending":
        z = z.sort(dim=1, descending=True).values
    elif kind == "equal":
        z.fill_(1.25)
    elif kind == "few values":
        z = z.round()
    elif kind == "sure":
        z[:, vocab // 2] += 25.0
    elif kind == "far":
        z += 5000.0
    return z.to(dtype)


@pytest.mark.parametrize("rows,vocab", [(1, 1), (1, 3), (3, 7), (5, 64), (2, 1009), (4, 8192), (3, 8193), (1, 151936), (20, 40001), (40, 20000),
                                        (200, 33000), (700, 1000)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_and_vocabularies(rows, vocab, dtype):
    z = _logits(rows, vocab, vocab, dtype)
    given = torch.randint(vocab, (rows, 2), device=DEV, generator=torch.Generator(device=DEV).manual_seed(1)).to(torch.int32)
    _check(z, given, 20, _run(z, given, 20))


@pytest.mark.parametrize("kind", ["masked", "lowest", "ascending", "descending", "equal", "few values", "sure", "far"])
@pytest.mark.parametrize("rows,vocab", [(2, 50003), (300, 50003), (9, 151936)])
def test_orders_ties_and_masks(kind, rows, vocab):
    z = _logits(rows, vocab, 3, kind=kind)
    given = torch.zeros((rows, 1), dtype=torch.int32, device=DEV) + vocab // 2
    o = _run(z, given, 64)
    if kind == "far":                                   # the lse itself has float32's step at 5000; the rest is as good as ever
        zz = z.double().cpu().numpy()
        lse, logp, ent = O.log_probabilities(zz)
        assert np.abs(o.lse.cpu().numpy() - lse).max() <= 5010 * 2.0 ** -23
        z = z - 5000.0
        o.lse.copy_(torch.from_numpy(O.log_probabilities(z.double().cpu().numpy())[0]))
    _check(z, given, 64, o)


@pytest.mark.parametrize("k", [0, 1, 2, 33, 64])
@pytest.mark.parametrize("n_given", [0, 1, 700])
def test_how_many_alternatives_and_tokens(k, n_given):
    z = _logits(6, 10007, 5)
    given = torch.randint(10007, (6, n_given), device=DEV, generator=torch.Generator(device=DEV).manual_seed(2)).to(torch.int32) if n_given else None
    _check(z, given, k, _run(z, given, k))


def test_rows_with_a_stride_and_off_alignment():
    wide = _logits(5, 3001, 6)
    for z in (wide[:, 1:2000], wide[:, 3:3001], wide.to(torch.bfloat16)[:, 5:2007]):
        given = torch.full((5, 1), 17, dtype=torch.int32, device=DEV)
        _check(z, given, 11, _run(z, given, 11))


def test_neighbours_of_a_row_do_not_matter():
    wide = torch.full((4, 1030), float("nan"), device=DEV)
    wide[:, 3:1026] = _logits(4, 1023, 7)
    z = wide[:, 3:1026]
    _check(z, None, 5, _run(z, None, 5))


def test_a_row_with_nothing_allowed():
    z = _logits(3, 9000, 8)
    z[1] = -float("inf")
    given = torch.full((3, 1), 4, dtype=torch.int32, device=DEV)
    o = _run(z, given, 6)
    _check(z, given, 6, o)
    assert o.lse[1].item() == -float("inf") and o.entropy[1].item() == 0 and o.top_index[1].tolist() == [0, 1, 2, 3, 4, 5]


@pytest.mark.parametrize("rows", [2, 300])
def test_logits_near_the_end_of_the_type(rows):
    # differences of such logits are multiples of 2^103 or zero: equal ones share the mass, the others have none
    z = torch.full((rows, 9001), -3.4e38, device=DEV)
    z[:, 700], z[:, 5], z[:, 8000] = 3.0e38, 3.0e38, 1.0e38
    z[1, :] = -3.0e38
    given = torch.tensor([[5, 8000, 9]] * rows, dtype=torch.int32, device=DEV)
    o = _run(z, given, 3)
    # lse 3e38 + ln 2 is 3e38 in float32
    assert (o.lse[0] == 3.0e38).item() and (o.lse[1] == -3.0e38).item()
    got = o.logprob.double().cpu().numpy()
    assert abs(got[0, 0] + np.log(2)) < 1e-6 and got[0, 1] < -1e38 and np.abs(got[1] + np.log(9001)).max() < 1e-5
    assert abs(o.entropy[0].item() - np.log(2)) < 1e-6 and abs(o.entropy[1].item() - np.log(9001)) < 1e-4
    assert o.top_index[0].tolist() == [5, 700, 8000] and o.top_index[1].tolist() == [0, 1, 2]


def test_signed_zeros_are_equal():
    z = torch.full((1, 100), -1.0, device=DEV)
    z[0, 10], z[0, 20], z[0, 30] = -0.0, 0.0, -0.0
    assert _run(z, None, 3).top_index[0].tolist() == [10, 20, 30]


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("rows", [3, 400])
def test_nan_and_infinity_stay_in_their_row(value, rows):
    z = _logits(rows, 30000, 9)
    z[1, 20000] = value
    given = torch.full((rows, 1), 4, dtype=torch.int32, device=DEV)
    o = _run(z, given, 6)
    assert torch.isnan(torch.stack([o.lse[1], o.entropy[1], o.logprob[1, 0], o.top_logprob[1, 0]])).all()
    assert ((o.top_index[1] >= 0) & (o.top_index[1] < 30000)).all()
    ok = [r for r in range(rows) if r != 1][:5]
    keep = H.LogprobBuffers(len(ok), 1, 6, DEV)
    for name in ("logprob", "entropy", "lse", "top_logprob", "top_index"):
        getattr(keep, name).copy_(getattr(o, name)[ok])
    _check(z[ok], given[ok], 6, keep)


def test_given_tokens_out_of_range():
    z = _logits(2, 500, 10)
    given = torch.tensor([[-1, 3], [500, 4]], dtype=torch.int32, device=DEV)
    o = _run(z, given, 2)
    assert o.logprob[0, 0].item() == 0 and torch.isnan(o.logprob[1, 0]).item()
    assert torch.isfinite(o.logprob[:, 1]).all() and o.status.cpu().tolist()[:3] == [B.E_BADINDEX, 1, 500]


def test_optional_results_streams_and_graphs():
    z = _logits(30, 20011, 11)
    given = torch.full((30, 1), 4, dtype=torch.int32, device=DEV)
    want = _run(z, given, 8)
    B.actkv_logprob(z, None, None, None, None, None, None, None)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    o = H.LogprobBuffers(30, 1, 8, DEV)
    torch.cuda.synchronize()
    B.actkv_logprob(z, given, o.logprob, None, None, o.top_logprob, o.top_index, o.status, s)
    s.synchronize()
    assert torch.equal(o.logprob, want.logprob) and torch.equal(o.top_index, want.top_index)
    g = torch.cuda.CUDAGraph()
    o2 = H.LogprobBuffers(30, 1, 8, DEV)
    with torch.cuda.graph(g):
        B.actkv_logprob(z, given, o2.logprob, o2.entropy, o2.lse, o2.top_logprob, o2.top_index, o2.status)
    z2 = _logits(30, 20011, 12)
    z.copy_(z2)
    g.replay()
    torch.cuda.synchronize()
    _check(z, given, 8, o2)


def test_the_binding_checks_shapes():
    z = _logits(3, 100, 1)
    f = torch.empty(3, device=DEV)
    idx = torch.empty((3, 2), dtype=torch.int32, device=DEV)
    with pytest.raises(ValueError):
        B.actkv_logprob(z, idx, f, None, None, None, None, None)
    with pytest.raises(ValueError):
        B.actkv_logprob(z, None, None, f[:2], None, None, None, None)
    with pytest.raises(ValueError):
        B.actkv_logprob(z, None, None, None, None, f, idx, None)
    with pytest.raises(TypeError):
        B.actkv_logprob(z.half(), None, None, None, None, None, None, None)
    with pytest.raises(TypeError):
        B.actkv_logprob(z.t(), None, None, None, None, None, None, None)
