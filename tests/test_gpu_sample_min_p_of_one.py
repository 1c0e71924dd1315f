"""A min-p of 1 or more keeps the largest logit and its equals, also where others come so close that their weights round to 1."""
import pytest
import torch

from paper_2609_31395_b200 import harness as H

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("vocab", [200, 5000])
@pytest.mark.parametrize("m", [1.0, float("inf")])
@pytest.mark.parametrize("t", [1.0, 1e10, 3e38])
@pytest.mark.parametrize("k,p", [(0, 1.0), (50, 1.0), (0, 0.9)])
@pytest.mark.parametrize("top", [10.0, -3.0, 1e-30])
def test_equals_alone_are_kept(top, k, p, t, m, vocab):
    """Float32 neighbours below the largest, one to forty of them apart, and three equals of it."""
    g = torch.Generator(device=DEV).manual_seed(vocab)
    z = torch.full((2, vocab), top, device=DEV)
    below = torch.randint(1, 41, z.shape, generator=g, device=DEV).to(torch.int32)
    bits = z.view(torch.int32)
    bits += below if top < 0 else -below         # (the larger the bits of a negative number, the smaller it is)
    at = [7, 100, vocab - 1]
    z[:, at] = top
    full = lambda x, d=torch.float32: torch.full((2,), x, dtype=d, device=DEV)
    s = H.Sampler(2, DEV)
    s.sample(z, torch.tensor([0.1, 0.9], device=DEV), full(t), full(k, torch.int32), full(p), full(m))
    s.check_status()
    # (in order the three equals come first: 9 tenths of the mass, or 50 tokens, reach over them)
    assert s.kept.tolist() == [3, 3] and s.token.tolist() == [7, vocab - 1]
    assert torch.allclose(s.logprob, torch.full((2,), 1 / 3, device=DEV).log(), rtol=2.0 ** -22, atol=0)
