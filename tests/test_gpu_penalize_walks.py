"""actkv_penalize where logits and output do not lie alike: the output begins at another place of a 16-byte vector, or at the same place in some rows only, so
that rows are walked over by vectors and by single tokens in turn while the counts of one CTA go from row to row."""
import numpy as np
import pytest
import torch

from paper_2609_31395_b200 import harness as H

from test_gpu_penalize import _case, _check, _rules, _want

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _place(x, offset, stride):
    """x at rows of this stride, and the memory around it."""
    rows, vocab = x.shape
    flat = torch.full((offset + rows * stride + 9,), 7.0, dtype=x.dtype, device=DEV)
    view = flat.as_strided((rows, vocab), (stride, 1), offset)
    view.copy_(x)
    return flat, view


def _around(flat, view):
    other = torch.ones(flat.shape, dtype=torch.bool, device=DEV)
    other.as_strided(view.shape, view.stride(), view.storage_offset()).fill_(False)
    return flat[other]


# elements: where logits and output begin, and their row strides, for a vocabulary of 1001
PLACES = [((0, 1008), (1, 1008)),       # never alike
          ((0, 1008), (0, 1009)),       # alike in every fourth or eighth row
          ((3, 1009), (3, 1009)),       # alike, each row elsewhere in a vector
          ((1, 1009), (2, 1011)),
          ((0, 1004), (0, 1008)),       # float32: alike; bf16: every other row
          ((5, 1001), (1, 1005))]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("masks", [None, 0.5])
@pytest.mark.parametrize("biases", [0, 30])
@pytest.mark.parametrize("src,dst", PLACES)
@pytest.mark.parametrize("n_req,win", [(3, 4), (150, 9)])       # (a row per CTA, and three)
def test_out_of_place(n_req, win, src, dst, biases, masks, dtype):
    hist = [(37 * r) % 200 for r in range(n_req)]
    c = _case(hist, [win] * n_req, vocab=1001, biases=biases, masks=masks, dtype=dtype, seed=n_req + biases)
    want, tol = _want(c, c["logits"])
    in_flat, z = _place(c["logits"], *src)
    out_flat, out = _place(torch.full_like(c["logits"], 9.0), *dst)
    before = in_flat.clone()
    s = H.Sampler(1, DEV)
    s.penalize(z, c["wi"], _rules(c), win, max(hist), out=out)
    s.check_status()
    _check(out, want, tol)
    assert torch.equal(in_flat, before) and (_around(out_flat, out) == 7.0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("masks", [None, 0.5])
@pytest.mark.parametrize("biases", [0, 30])
@pytest.mark.parametrize("at", [(3, 1009), (1, 1008), (0, 1001)])
def test_in_place(at, biases, masks, dtype):
    hist = [(37 * r) % 200 for r in range(150)]
    c = _case(hist, [9] * 150, vocab=1001, biases=biases, masks=masks, dtype=dtype, seed=7)
    want, tol = _want(c, c["logits"])
    flat, z = _place(c["logits"], *at)
    s = H.Sampler(1, DEV)
    s.penalize(z, c["wi"], _rules(c), 9, max(hist))
    s.check_status()
    _check(z, want, tol)
    assert (_around(flat, z) == 7.0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("masks", [None, 0.3])
@pytest.mark.parametrize("src,dst", [((0, 20004), (1, 20004)), ((0, 20008), (0, 20001)), ((3, 20001), (3, 20001))])
def test_long_rows(src, dst, masks, dtype):
    """More vectors than a CTA has in flight at once, a slice boundary within the row."""
    hist = [900, 40, 70] * 7
    c = _case(hist, [9, 2, 8] * 7, vocab=20001, biases=20, masks=masks, dtype=dtype, seed=1)
    want, tol = _want(c, c["logits"])
    _, z = _place(c["logits"], *src)
    flat, out = _place(torch.full_like(c["logits"], 9.0), *dst)
    s = H.Sampler(1, DEV)
    s.penalize(z, c["wi"], _rules(c), 9, 900, out=out)
    s.check_status()
    _check(out, want, tol)
    assert (_around(flat, out) == 7.0).all()
