"""GPU parity of actkv_penalize against the float64 oracle.

Tolerance: bias, penalty and subtraction are float32 operations of at most one rounding each (2^-24 of what they work on), the factor f n + p two
more: z' is off by at most 5 * 2^-24 of the largest value on its way, |z| + |bias| times the repetition penalty, plus f n + p; bf16 results are
rounded once more, 2^-8 relative, half a step.  Logits that no rule touches keep their bits."""
import numpy as np
import pytest
import torch

from oracle import actkv_oracle as O
from paper_2609_31395_b200 import binding as B
from paper_2609_31395_b200 import harness as H

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
INF = float("inf")


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _f32(x):
    return torch.tensor(x, dtype=torch.float32, device=DEV)


def _case(hist, win, vocab=1000, biases=0, masks=None, dtype=torch.float32, pitch=0, extra=0, prompt=0.5, seed=0, neutral=False, skew=2.0):
    """masks: share of allowed tokens, or None; pitch: elements between rows beyond the vocabulary; extra: rows of no request."""
    rng = np.random.default_rng(seed)
    g = torch.Generator(device=DEV).manual_seed(seed)
    R, rows = len(hist), sum(win) + extra
    full = (torch.randn((rows, vocab + pitch), generator=g, device=DEV) * 4).to(dtype)
    cap = max(hist + [1]) + 3
    tokens = (rng.random((R, cap)) ** skew * (vocab + 2) - 1).astype(np.int64)      # a few outside the vocabulary
    c = dict(full=full, logits=full[:, :vocab], vocab=vocab, win=win, hist=hist, tokens=tokens, wi=_i32([0] + np.cumsum(win).tolist()),
             prompt=[int(n * prompt) for n in hist], rep=[1.0] * R if neutral else [float(np.float32(x)) for x in rng.uniform(0.7, 1.6, R)],
             freq=[0.0] * R if neutral else [float(np.float32(x)) for x in rng.uniform(-0.3, 0.8, R)],
             pres=[0.0] * R if neutral else [float(np.float32(x)) for x in rng.uniform(0, 1, R)], bias=[{} for _ in hist], allow=None, allow_row=None)
    if biases:
        c["bias"] = [{int(t): float(np.float32(x)) for t, x in zip(np.sort(rng.choice(vocab, min(vocab, biases), replace=False)), rng.normal(size=biases) * 5)}
                     for _ in hist]
        c["bias"][0] = {t: (-INF if i % 3 == 0 else b) for i, (t, b) in enumerate(c["bias"][0].items())}
        if R > 1:
            c["bias"][1] = {}
    if masks is not None:
        words = (vocab + 31) // 32 + (seed % 2)
        c["allow"] = rng.integers(0, 1 << 32, (rows + 2, words), dtype=np.uint32) if masks == 0.5 else \
            np.packbits(rng.random((rows + 2, words * 32)) < masks, axis=1, bitorder="little").view(np.uint32)
        c["allow_row"] = [int(x) for x in rng.integers(-1, rows + 2, rows)]
    return c


def _rules(c):
    ind = [0] + np.cumsum([len(b) for b in c["bias"]]).tolist()
    some = ind[-1] > 0
    return H.LogitRules(_i32(c["tokens"]), _i32(c["hist"]), _i32(c["prompt"]), _f32(c["rep"]), _f32(c["freq"]), _f32(c["pres"]),
                        _i32(ind) if some else None, _i32([t for b in c["bias"] for t in b]) if some else None,
                        _f32([x for b in c["bias"] for x in b.values()]) if some else None,
                        None if c["allow"] is None else torch.from_numpy(c["allow"].view(np.int32)).to(DEV),
                        None if c["allow_row"] is None else _i32(c["allow_row"]))


def _want(c, before):
    z = before.double().cpu().numpy()
    want, tol = z.copy(), np.zeros(z.shape)
    row = 0
    for r, w in enumerate(c["win"]):
        for i in range(w):
            n = max(0, c["hist"][r] - (w - 1 - i))
            past = c["tokens"][r, :n]
            m = -1 if c["allow_row"] is None else c["allow_row"][row]
            allowed = None
            if c["allow"] is not None and m >= 0:
                allowed = np.unpackbits(c["allow"][m:m + 1].view(np.uint8), bitorder="little")[:c["vocab"]].astype(bool)
            want[row] = O.penalize_row(z[row], past, c["prompt"][r], c["rep"][r], c["freq"][r], c["pres"][r], c["bias"][r], allowed)
            touched = np.array(sorted(set(int(t) for t in past if 0 <= t < c["vocab"]) | set(c["bias"][r])), dtype=int)
            b = np.array([abs(c["bias"][r].get(int(t), 0.0)) for t in touched])
            size = (np.abs(z[row, touched]) + np.where(np.isfinite(b), b, 0)) * max(c["rep"][r], 1 / c["rep"][r]) + abs(c["freq"][r]) * n + c["pres"][r]
            tol[row, touched] = 5 * 2.0 ** -24 * size
            if before.dtype is torch.bfloat16:
                tol[row, touched] += 2.0 ** -8 * np.abs(np.where(np.isfinite(want[row, touched]), want[row, touched], 0))
            row += 1
    return want, tol


def _check(got, want, tol):
    got = got.double().cpu().numpy()
    fin = np.isfinite(want)
    assert np.array_equal(got[~fin], want[~fin], equal_nan=True)
    over = np.abs(got - np.where(fin, want, 0))[fin] - tol[fin]
    assert (over <= 0).all(), float(over.max())


CASES = [
    dict(hist=[0], win=[1]), dict(hist=[1], win=[1], vocab=1), dict(hist=[5], win=[1], vocab=3), dict(hist=[300], win=[1]),
    dict(hist=[300, 0, 20], win=[1, 1, 1], biases=5), dict(hist=[40, 50], win=[3, 5], biases=40), dict(hist=[2, 0, 4], win=[4, 2, 4]),
    dict(hist=[100, 10, 60], win=[2, 0, 1], extra=2), dict(hist=[200], win=[1], masks=0.5), dict(hist=[200, 100], win=[2, 3], masks=0.02, biases=9),
    dict(hist=[200, 100], win=[2, 3], masks=0.97, seed=1), dict(hist=[30, 20], win=[1, 1], masks=0.0), dict(hist=[30, 20], win=[1, 1], masks=1.0, neutral=True),
    dict(hist=[30, 20], win=[1, 2], masks=0.5, neutral=True, biases=3), dict(hist=[30], win=[1], neutral=True), dict(hist=[500], win=[1], vocab=33, skew=1.0),
    dict(hist=[500], win=[7], vocab=1009, masks=0.5, biases=300), dict(hist=[20], win=[2], vocab=1001, pitch=7, masks=0.3), dict(hist=[90], win=[2], vocab=4000, pitch=4),
    dict(hist=[3000, 100], win=[1, 2], vocab=151936, masks=0.1), dict(hist=[40000], win=[1], vocab=151936, biases=500, skew=3.0),
    dict(hist=[900, 40, 70], win=[40, 8, 30], vocab=30000, masks=0.4), dict(hist=[60] * 40, win=[1] * 40, vocab=32003, biases=2),
    dict(hist=[5000], win=[1], vocab=70000, skew=9.0), dict(hist=[50], win=[1], prompt=0.0), dict(hist=[50], win=[3], prompt=2.0)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("kw", CASES)
def test_parity(kw, in_place, dtype):
    c = _case(dtype=dtype, **kw)
    before = c["full"].clone()
    s = H.Sampler(1, DEV)
    out = None if in_place else torch.full_like(c["full"], 7.0)
    s.penalize(c["logits"], c["wi"], _rules(c), max(c["win"]), max(c["hist"]), out=None if in_place else out[:, :c["vocab"]])
    s.check_status()
    want, tol = _want(c, before[:, :c["vocab"]])
    rows = sum(c["win"])
    if in_place:
        _check(c["logits"], want, tol)
        assert torch.equal(c["full"][:, c["vocab"]:], before[:, c["vocab"]:])
    else:
        _check(out[:rows, :c["vocab"]], want[:rows], tol[:rows])
        assert (out[rows:] == 7.0).all() and (out[:, c["vocab"]:] == 7.0).all() and torch.equal(c["full"], before)


@pytest.mark.parametrize("in_place", [True, False])
def test_special_logits(in_place):
    c = _case([60, 60], [1, 1], vocab=64, masks=0.5, skew=1.0)
    c["allow_row"] = [0, -1]
    z = c["logits"]
    z[:, 0::8], z[:, 1::8], z[:, 2::8], z[:, 3::8] = -INF, INF, float("nan"), torch.finfo(torch.float32).min
    z[:, 4::8], z[:, 5::8] = 0.0, -0.0
    before = z.clone()
    s = H.Sampler(1, DEV)
    out = z if in_place else torch.empty_like(z)
    c["rep"] = [1.25, 0.75]
    s.penalize(z, c["wi"], _rules(c), 1, 60, out=out)
    with np.errstate(over="ignore"):
        want, tol = _want(c, before)
    want = np.where(want < -3.5e38, -INF, want)                 # past float32's range
    want[np.isnan(before.cpu().numpy()) & (want != -INF)] = np.nan
    big = np.abs(before.cpu().numpy()) > 1e30
    tol[big & np.isfinite(want)] = 1e32
    _check(out, want, np.where(np.isfinite(tol), tol, 0))


def test_rules_one_by_one_and_none():
    z = torch.randn((2, 500), device=DEV)
    wi, tok = _i32([0, 1, 2]), _i32([[3, 3, 4], [9, 9, 9]])
    s = H.Sampler(2, DEV)
    run = lambda **kw: (s.penalize(z, wi, H.LogitRules(**kw), 1, 3, out=out), s.check_status())
    out = torch.empty_like(z)
    run()
    assert torch.equal(out, z)
    run(tokens=tok, hist_len=_i32([3, 2]))
    assert torch.equal(out, z)
    run(tokens=tok, hist_len=_i32([3, 2]), presence=_f32([1.0, 0.5]))
    want = z.clone()
    want[0, [3, 4]] -= 1.0
    want[1, 9] -= 0.5
    assert torch.equal(out, want)
    run(tokens=tok, hist_len=_i32([3, 2]), frequency=_f32([1.0, 0.5]), prompt_len=_i32([1, 0]))
    want = z.clone()
    want[0, [3, 4]] -= 1.0
    want[1, 9] -= 1.0
    assert torch.equal(out, want)
    run(repetition=_f32([2.0, 2.0]))                             # no history
    assert torch.equal(out, z)
    run(bias_indptr=_i32([0, 0, 1]), bias_token=_i32([499]), bias_value=_f32([2.5]))
    want = z.clone()
    want[1, 499] += 2.5
    assert torch.equal(out, want)
    allow = torch.zeros((2, 16), dtype=torch.int32, device=DEV)
    allow[0, 0], allow[1, 15] = 1, 1 << 19
    run(allow=allow)
    want = torch.full_like(z, -INF)
    want[0, 0], want[1, 499] = z[0, 0], z[1, 499]
    assert torch.equal(out, want)


@pytest.mark.parametrize("cause,code", [("repetition", B.E_INVALID), ("frequency", B.E_INVALID), ("history", B.E_INVALID), ("window", B.E_INVALID),
                                        ("order", B.E_BADINDEX), ("twice", B.E_BADINDEX), ("token", B.E_BADINDEX), ("bias range", B.E_INVALID)])
def test_a_request_with_bad_rules_is_reported_and_left_alone(cause, code):
    c = _case([100, 80, 60], [1, 2, 1], vocab=70000, biases=6, masks=0.5)
    c["bias"][1] = {5: 1.0, 60000: 2.0, 65000: 3.0}
    win, max_win, max_hist = c["win"], 2, 100
    if cause == "repetition":
        c["rep"][1] = 0.0
    elif cause == "frequency":
        c["freq"][1] = float("nan")
    elif cause == "history":
        c["hist"][1], max_hist = 101, 100
    rules = _rules(c)
    at = int(rules.tensors[6][1])
    if cause == "order":
        rules.tensors[7][at + 1] = 66000
    elif cause == "twice":
        rules.tensors[7][at + 1] = 5
    elif cause == "token":
        rules.tensors[7][at + 2] = 70000
    elif cause == "bias range":
        rules.tensors[6][2] = rules.tensors[7].numel() + 9
        rules.tensors[6][3] = rules.tensors[6][2]
    elif cause == "window":
        max_win = 1
    before = c["logits"].clone()
    s = H.Sampler(1, DEV)
    s.penalize(c["logits"], c["wi"], rules, max_win, max_hist)
    st = s.status.tolist()
    assert st[0] == code and st[1] in (1, 2)
    assert torch.equal(c["logits"][1:3], before[1:3])
    c["hist"][1], c["rep"][1], c["freq"][1] = 80, 1.0, 0.0       # (the oracle's row of the request, which is not looked at)
    if cause == "bias range":
        c["bias"][2] = None
    want, tol = _want({**c, "bias": [b or {} for b in c["bias"]]}, before)
    _check(c["logits"][:1], want[:1], tol[:1])
    if cause != "bias range":
        _check(c["logits"][3:], want[3:], tol[3:])


def test_a_mask_out_of_range_leaves_its_row():
    c = _case([100, 80], [1, 2], masks=0.5)
    c["allow_row"] = [0, c["allow"].shape[0], 1]
    before = c["logits"].clone()
    s = H.Sampler(1, DEV)
    s.penalize(c["logits"], c["wi"], _rules(c), 2, 100)
    assert s.status.tolist()[:3] == [B.E_BADINDEX, 1, c["allow"].shape[0]]
    assert torch.equal(c["logits"][1], before[1])
    c["allow_row"][1] = -1
    want, tol = _want(c, before)
    _check(c["logits"][[0, 2]], want[[0, 2]], tol[[0, 2]])


def test_captured_with_growing_history_and_another_stream():
    c = _case([20, 30], [1, 1], masks=0.5)
    rules, z = _rules(c), c["logits"].clone()
    s, out = H.Sampler(1, DEV), torch.empty_like(c["logits"])
    stream, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=stream):
        s.penalize(c["logits"], c["wi"], rules, 1, 33, out=out)
    for step in range(3):
        rules.tensors[1].add_(1)
        c["hist"] = [n + 1 for n in c["hist"]]
        with torch.cuda.stream(stream):
            stream.wait_stream(torch.cuda.default_stream())
            g.replay()
        stream.synchronize()
        _check(out, *_want(c, z))
    s.check_status()


def test_shapes_that_do_not_fit_are_refused():
    c = _case([20, 30], [1, 1], masks=0.5)
    s, rules = H.Sampler(1, DEV), _rules(c)
    z = c["logits"]
    with pytest.raises(ValueError):
        s.penalize(z, _i32([0, 1, 2, 2]), rules, 1, 30)
    with pytest.raises(ValueError):
        s.penalize(torch.cat([z, z]), _i32([0, 1, 2]), rules, 1, 30)
    with pytest.raises(ValueError):
        s.penalize(z, c["wi"], rules, 1, 30, out=torch.empty_like(z, dtype=torch.bfloat16))
    with pytest.raises(TypeError):
        s.penalize(z.half(), c["wi"], rules, 1, 30)
    with pytest.raises(TypeError):
        s.penalize(z.t().contiguous().t(), c["wi"], rules, 1, 30)
    with pytest.raises(TypeError):
        H.LogitRules(_i32([[1]]), _i32([1]).long())
    with pytest.raises(ValueError):
        H.LogitRules(_i32([[1]]))
    with pytest.raises(ValueError):
        H.LogitRules(_i32([[1], [2]]), _i32([1]))
    with pytest.raises(B.ActKVError):                            # a mask narrower than the vocabulary
        s.penalize(torch.zeros((2, 1100), device=DEV), c["wi"], rules, 1, 30)
