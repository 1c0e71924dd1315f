"""The top alternatives among subnormal logits: they are ordered by their values as any others, ties by token, both signs."""
import numpy as np
import pytest
import torch

from oracle import actkv_oracle as O
from paper_2609_31395_b200 import binding as B
from paper_2609_31395_b200 import harness as H

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _top(z, k):
    o = H.LogprobBuffers(z.shape[0], 0, k, DEV)
    B.actkv_logprob(z, None, None, o.entropy, o.lse, o.top_logprob, o.top_index, o.status)
    return o


def _from_bits(bits, dtype):
    if dtype is torch.float32:
        return torch.from_numpy(bits.astype(np.uint32).view(np.float32)).to(DEV)
    return torch.from_numpy(bits.astype(np.uint16).view(np.int16)).to(DEV).view(torch.bfloat16)


# (a few rows: a cluster per row, several CTAs of 512 threads; many rows: 256 threads; the long rows' candidates do not fit the list)
@pytest.mark.parametrize("rows,vocab", [(1, 5), (2, 1000), (3, 40001), (600, 3001)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind", ["one negative value", "negative", "both signs", "negative, a few zeros", "below normal ones"])
def test_subnormal_logits(rows, vocab, dtype, kind):
    g = np.random.default_rng(vocab)
    mant, sign, low = (23, 1 << 31, 1 << 23) if dtype is torch.float32 else (7, 1 << 15, 1 << 7)
    bits = g.integers(1, 1 << mant, (rows, vocab))
    if kind == "one negative value":
        bits[:] = sign | 12345 % low
    elif kind == "both signs":
        bits |= np.where(g.random((rows, vocab)) < 0.5, sign, 0)
    elif kind == "below normal ones":                      # ten normal ones, the others below zero by less than a normal number
        bits |= sign
        bits[:, :10] = (100 << mant) + g.integers(0, low, (rows, min(10, vocab)))
    else:
        bits |= sign
        if kind == "negative, a few zeros":
            bits[:, :: 97] = np.where(g.random(bits[:, :: 97].shape) < 0.5, sign, 0)
    z = _from_bits(bits, dtype)
    k = 64
    o = _top(z, k)
    idx = O.top_tokens(z.double().cpu().numpy(), k)
    got = o.top_index.cpu().numpy()
    assert np.array_equal(got[:, :idx.shape[1]], idx) and (got[:, idx.shape[1]:] == -1).all()
    # the differences of these logits are below 2^-25: every token is as probable as any other.  ln of float32 sums of vocab ones: e as for
    # the other rows, 2^-21 + (n / 512 + 40) 2^-24
    e = 2.0 ** -21 + (vocab / 512 + 40) * 2.0 ** -24
    assert np.abs(o.lse.double().cpu().numpy() - np.log(vocab)).max() <= e + np.log(vocab) * 2.0 ** -22
    assert int(o.status[0]) == 0
