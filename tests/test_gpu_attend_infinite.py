"""actkv_attend on infinite and NaN keys and values, with the warp-level and the tensor-core kernel: what a row sees decides, not the
probability that the entry gets there nor the key tile in which it lies."""
import math

import numpy as np
import pytest
import torch

from oracle import actkv_oracle as O
from paper_2609_31395_b200 import harness as H
from paper_2609_31395_b200 import synth

import parity_util as U

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
MANY = 1 << 19            # a bound on the lengths by which more than 8 rows are work for the tensor-core kernel
INF, NAN = math.inf, math.nan
L, W, G = 700, 5, 4       # window rows stand at 695 .. 699: 20 rows of a KV head


def _make(D, seed=0):
    wl = synth.Workload("attend", 1, 1, G, [L], [W], [0], head_dim=D, page_size=16, causal=True, table_style="fragmented", plant_frac=0.0,
                        seed=seed, poison_tail=True)
    inst = synth.generate(wl, DEV)
    inst.q.copy_(inst.q.abs() + 0.5)                   # so that the sign of a planted key decides the sign of its logits
    return inst


def _put(inst, c, j, value, dims=slice(None)):
    inst.pool[:, c, inst.page_table[0, j // 16].item(), j % 16, :, dims] = value


def _attend(inst, max_tok, window_left):
    wl = inst.wl
    dec = H.Decoder(inst.pool, inst.page_table, inst.seq_len, inst.free_list, inst.free_count, G, W, W, max_tok)
    out, lse = torch.full_like(inst.q, 7.0), torch.full(inst.q.shape[:3], 7.0, device=DEV)
    dec.attend(inst.q, inst.win_indptr, wl.sm_scale, True, out, lse, window_left)
    dec.check_status()
    return out.float().cpu().numpy()[0], lse.cpu().numpy()[0]


def _sees(w, j, window_left):
    p = L - W + w
    return j <= p and (window_left == 0 or j > p - window_left)


def _oracle(inst, window_left):
    return (x[0] for x in O.attend(U.bits(inst.pool), inst.page_table.cpu().numpy(), [L], U.bits(inst.q), [0, W], G, inst.wl.sm_scale, True,
                                   window_left))


def _near(got, want):
    # one rounding to bf16, and float32 noise of values of order 1
    np.testing.assert_allclose(got, want, rtol=2.0 ** -8, atol=1e-3)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("max_tok", [L, MANY])
# without a sliding window: the first tile, one in the middle, the last one; with one of 400 keys: tiles at its lower end too
@pytest.mark.parametrize("j,window_left", [(0, 0), (130, 0), (400, 0), (690, 0), (695, 0), (697, 0), (699, 0), (298, 400), (302, 400),
                                           (320, 400), (500, 400), (696, 400)])
@pytest.mark.parametrize("value", [INF, -INF, NAN])
@pytest.mark.parametrize("hidden", [True, False])
def test_a_visible_value_reaches_its_dims(D, max_tok, j, window_left, value, hidden):
    inst = _make(D)
    if hidden:                                         # a logit of about -2000: the probability is 0 in float32
        _put(inst, 0, j, -200.0)
    want, wlse = _oracle(inst, window_left)
    _put(inst, 1, j, value, [3, D - 1])
    out, lse = _attend(inst, max_tok, window_left)
    np.testing.assert_allclose(lse, wlse, rtol=1e-5)
    rest = [d for d in range(D) if d not in (3, D - 1)]
    for w in range(W):
        _near(out[w][:, rest], want[w][:, rest])
        if _sees(w, j, window_left):
            assert not np.isfinite(out[w][:, [3, D - 1]]).any()
        else:
            _near(out[w], want[w])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("max_tok", [L, MANY])
@pytest.mark.parametrize("j", [0, 260, 400, 690, 697, 699])
@pytest.mark.parametrize("value", [INF, NAN])
def test_infinite_and_nan_logits_make_the_rows_nan_that_see_them(D, max_tok, j, value):
    inst = _make(D)
    want, wlse = _oracle(inst, 0)
    clean = inst.pool.clone()
    _put(inst, 0, j, 0.0)
    _put(inst, 0, j, value, [0])                       # q > 0: the logit is +inf, or NaN
    out, lse = _attend(inst, max_tok, 0)
    for w in range(W):
        if _sees(w, j, 0):
            assert np.isnan(out[w]).all() and np.isnan(lse[w]).all()
        else:
            _near(out[w], want[w])
            np.testing.assert_allclose(lse[w], wlse[w], rtol=1e-5)
    inst.pool.copy_(clean)
    # two of them, in tiles of different warps
    for i in (5, j):
        _put(inst, 0, i, 0.0)
        _put(inst, 0, i, value, [0])
    out, lse = _attend(inst, max_tok, 0)
    assert np.isnan(out).all() and np.isnan(lse).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("max_tok", [L, MANY])
def test_a_logit_of_minus_infinity_has_no_share(D, max_tok):
    inst = _make(D)
    for j in (0, 15, 16, 128, 300, 690, 698):
        _put(inst, 0, j, 0.0)
        _put(inst, 0, j, -INF, [0])
    want, wlse = _oracle(inst, 0)
    out, lse = _attend(inst, max_tok, 0)
    _near(out, want)
    np.testing.assert_allclose(lse, wlse, rtol=1e-5)
    # all of them: the row is empty
    for j in range(L):
        _put(inst, 0, j, 0.0)
        _put(inst, 0, j, -INF, [0])
    out, lse = _attend(inst, max_tok, 0)
    assert (out == 0).all() and np.isneginf(lse).all()
