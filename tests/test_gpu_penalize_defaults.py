"""Sampler.penalize without the bounds that LogitRules knows by itself."""
import pytest
import torch

from paper_2609_31395_b200 import binding as B
from paper_2609_31395_b200 import harness as H

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def test_a_history_needs_no_bound():
    g = torch.Generator(device=DEV).manual_seed(0)
    z = torch.randn((2, 300), generator=g, device=DEV)
    tokens = torch.randint(0, 300, (2, 90), generator=g, device=DEV).to(torch.int32)
    rules = H.LogitRules(tokens, _i32([90, 17]), None, None, None, torch.tensor([1.0, 0.5], device=DEV))
    s, a, b = H.Sampler(2, DEV), torch.empty_like(z), torch.empty_like(z)
    s.penalize(z, _i32([0, 1, 2]), rules, out=a)
    s.check_status()
    s.penalize(z, _i32([0, 1, 2]), rules, 1, 90, out=b)
    s.check_status()
    want = z.clone()
    want[0, tokens[0].long().unique()] -= 1.0
    want[1, tokens[1, :17].long().unique()] -= 0.5
    assert torch.equal(a, want) and torch.equal(b, want)


def test_a_bound_that_is_given_is_the_bound():
    z, s = torch.zeros((1, 8), device=DEV), H.Sampler(1, DEV)
    rules = H.LogitRules(_i32([[1, 2, 3]]), _i32([3]), presence=torch.ones(1, device=DEV))
    for bound, code in ((0, B.E_INVALID), (2, B.E_INVALID), (3, 0), (1000, 0)):
        s.status.zero_()
        s.penalize(z, _i32([0, 1]), rules, 1, bound)
        assert s.status[0].item() == code


def test_buffers_wider_than_a_history_may_be():
    """2^23 places: the lengths in use count, not the buffer's width."""
    tokens = torch.zeros((1, 1 << 23), dtype=torch.int32, device=DEV)
    z, s = torch.zeros((1, 8), device=DEV), H.Sampler(1, DEV)
    s.penalize(z, _i32([0, 1]), H.LogitRules(tokens, _i32([5]), presence=torch.ones(1, device=DEV)))
    s.check_status()
    assert z.tolist() == [[-1.0] + [0.0] * 7]
    s.penalize(z, _i32([0, 1]), H.LogitRules(tokens, _i32([1 << 23]), presence=torch.ones(1, device=DEV)))
    assert s.status[0].item() == B.E_INVALID


def test_rules_without_a_history():
    z, s = torch.zeros((1, 8), device=DEV), H.Sampler(1, DEV)
    s.penalize(z, _i32([0, 1]), H.LogitRules(bias_indptr=_i32([0, 1]), bias_token=_i32([2]), bias_value=torch.ones(1, device=DEV)))
    s.check_status()
    assert z.tolist() == [[0, 0, 1, 0, 0, 0, 0, 0]]
