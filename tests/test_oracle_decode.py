"""Pins of the decoding oracle: attention, rotation, resize, log probabilities against closed forms and torch."""
import math

import numpy as np
import pytest
import torch

from oracle import actkv_oracle as O


def _rng(seed=0):
    return np.random.default_rng(seed)


def test_attention_of_one_row_is_torch_softmax():
    g = _rng(1)
    q, k, v = g.normal(size=(1, 3, 16)), g.normal(size=(40, 16)), g.normal(size=(40, 16))
    out, lse = O.attend_unit(q, k, v, 0.25, True)
    s = torch.from_numpy(q[0] @ k.T * 0.25)
    np.testing.assert_allclose(out[0], (torch.softmax(s, -1) @ torch.from_numpy(v)).numpy(), rtol=1e-12)
    np.testing.assert_allclose(lse[0], torch.logsumexp(s, -1).numpy(), rtol=1e-12)


def test_causal_rows_are_prefixes_and_sliding_rows_are_tails():
    g = _rng(2)
    q, k, v = g.normal(size=(4, 2, 8)), g.normal(size=(9, 8)), g.normal(size=(9, 8))
    out, lse = O.attend_unit(q, k, v, 0.5, True)
    slid, _ = O.attend_unit(q, k, v, 0.5, True, window_left=3)
    for w in range(4):
        p = 9 - 4 + w
        one, l1 = O.attend_unit(q[w:w + 1], k[:p + 1], v[:p + 1], 0.5, False)
        np.testing.assert_allclose(out[w], one[0])
        np.testing.assert_allclose(lse[w], l1[0])
        tail, _ = O.attend_unit(q[w:w + 1], k[p - 2:p + 1], v[p - 2:p + 1], 0.5, False)
        np.testing.assert_allclose(slid[w], tail[0])


def test_a_row_without_keys_is_empty():
    g = _rng(3)
    out, lse = O.attend_unit(g.normal(size=(3, 1, 8)), g.normal(size=(1, 8)), g.normal(size=(1, 8)), 1.0, True)
    assert np.all(out[:2] == 0) and np.all(np.isneginf(lse[:2])) and np.isfinite(lse[2]).all()


def test_lse_is_the_one_of_the_score():
    g = _rng(4)
    q, k = g.normal(size=(3, 2, 16)), g.normal(size=(20, 16))
    _, lse = O.attend_unit(q, k, k, 0.3, True)
    _, want = O.score_unit(q, k, 0.3, True)[:2]
    np.testing.assert_allclose(lse, want, rtol=1e-12)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_keeps_lengths_and_relative_angles(interleaved):
    g = _rng(5)
    f = 1.0 / 10.0 ** np.arange(4)
    x, y = g.normal(size=(2, 1, 10)), g.normal(size=(2, 1, 10))
    pos = np.array([[3, 7], [11, 2]])
    a, b = (O.rotate(t, pos, f, [2, 2], interleaved) for t in (x, y))
    a2, b2 = (O.rotate(t, pos + 5, f, [2, 2], interleaved) for t in (x, y))
    np.testing.assert_allclose((a * a).sum(-1), (x * x).sum(-1))
    np.testing.assert_allclose((a * b).sum(-1), (a2 * b2).sum(-1))
    np.testing.assert_array_equal(a[..., 8:], x[..., 8:])
    quarter = O.rotate(np.array([[[1.0, 0.0]]]), np.array([[1]]), np.array([math.pi / 2]), [1], interleaved)
    np.testing.assert_allclose(quarter[0, 0], [0.0, 1.0], atol=1e-15)


def test_resize_by_hand():
    t = O.Tables(np.array([[5, 6, -1], [7, 8, 9], [1, -1, -1]]), np.array([6, 12, 2]), np.array([2, 3, 4, -1, -1, -1, -1, -1, -1, -1]), 3)
    n = O.resize(t, [9, 0, -1], 4)
    assert n.page_table.tolist() == [[5, 6, 4], [-1, -1, -1], [1, -1, -1]]
    assert n.seq_len.tolist() == [9, 0, 2]
    assert n.free_count == 5 and n.free_list[:5].tolist() == [2, 3, 7, 8, 9]
    with pytest.raises(ValueError):
        O.resize(t, [6, 12, 20], 4)


def test_log_probabilities_against_torch_and_closed_forms():
    z = _rng(6).normal(size=(5, 33)) * 3
    lse, logp, ent = O.log_probabilities(z)
    np.testing.assert_allclose(logp, torch.log_softmax(torch.from_numpy(z), -1).numpy(), rtol=1e-12)
    np.testing.assert_allclose(ent, torch.distributions.Categorical(logits=torch.from_numpy(z)).entropy().numpy(), rtol=1e-10)
    lse, logp, ent = O.log_probabilities(np.array([[0.0] * 8, [-np.inf] * 8, [-np.inf] * 7 + [3.0]]))
    np.testing.assert_allclose(ent, [math.log(8), 0, 0], atol=1e-15)
    assert lse[1] == -np.inf and np.all(np.isneginf(logp[1])) and logp[2, 7] == 0
    assert O.top_tokens(np.array([[1.0, 3.0, 3.0, 2.0]]), 3).tolist() == [[1, 2, 3]]
