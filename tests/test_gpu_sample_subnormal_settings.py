"""Settings of actkv_sample below the smallest normal float32, of both signs, and zeros with a sign."""
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
    return torch.from_numpy(np.array(x, dtype=np.float32)).to(DEV)


def _sampler(n):
    s = H.Sampler(n, DEV)
    s.token.fill_(-7), s.logprob.fill_(-7), s.kept.fill_(-7)
    return s


def _same(s, i, z, u, t, k, p, m):
    token, logprob, kept = O.sample_row(z[i].double().cpu().numpy(), u, t, k, p, m)
    assert (int(s.token[i]), int(s.kept[i])) == (token, kept)
    assert abs(float(s.logprob[i]) - logprob) <= 2.0 ** -23 * abs(logprob) + 2.0 ** -26


@pytest.mark.parametrize("kw", [dict(t=-1e-45), dict(t=-1e-39), dict(t=-1.1754942e-38), dict(u=-1e-45), dict(u=-1e-39)])
@pytest.mark.parametrize("k,p", [(0, 1.0), (20, 1.0), (0, 0.9), (500, 0.8)])
def test_negative_subnormal_settings_are_reported(kw, k, p):
    z = torch.randn((3, 4000), generator=torch.Generator(device=DEV).manual_seed(2), device=DEV) * 2
    t, u = [1.0] * 3, [0.25] * 3
    t[1], u[1] = kw.get("t", 1.0), kw.get("u", 0.25)
    s = _sampler(3)
    s.sample(z, _f32(u), _f32(t), torch.full((3,), k, dtype=torch.int32, device=DEV), _f32([p] * 3))
    assert s.status.tolist()[:2] == [B.E_INVALID, 1]
    assert (s.token[1].item(), s.logprob[1].item(), s.kept[1].item()) == (-1, -INF, 0)
    for i in (0, 2):
        _same(s, i, z, 0.25, 1.0, k, float(np.float32(p)), 0.0)


def test_zeros_with_a_sign_and_positive_subnormal_settings_are_settings():
    z = torch.randn((6, 3000), generator=torch.Generator(device=DEV).manual_seed(3), device=DEV) * 2
    t, u, p, m = [-0.0, 1e-45, 1.0, 1.0, 1.0, 1.0], [0.5, 0.5, -0.0, 1e-45, 0.5, 0.5], [0.9, 0.9, 0.9, 0.9, -1e-45, 1e-45], [-1e-45, -0.0, 0.0, 0.0, 0.0, 0.0]
    s = _sampler(6)
    s.sample(z, _f32(u), _f32(t), None, _f32(p), _f32(m))
    s.check_status()
    for i in range(6):
        f = lambda x: float(np.float32(x[i]))
        _same(s, i, z, f(u), f(t), 0, f(p), f(m))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("m", [1e-45, 1e-40, 1.1754942e-38, 1.17549435e-38, 2e-38])
@pytest.mark.parametrize("k,p,t", [(0, 1.0, 1.0), (0, 1.0, 0.5), (430, 1.0, 1.0), (100, 1.0, 0.25), (0, 0.9999, 1.0)])
def test_a_subnormal_min_p_cuts(m, k, p, t, dtype):
    """Gaps in steps of a quarter: between ln of the limits and the nearest step lie 0.003 at least, 2^-8 of a weight, which are right to 2^-45."""
    g = torch.arange(0, 480, device=DEV, dtype=torch.float32) * 0.25
    z = torch.stack([5.0 - g, (5.0 - g).flip(0)]).to(dtype)
    s = _sampler(2)
    full = lambda x: _f32([x] * 2)
    s.sample(z, full(0.7), full(t), torch.full((2,), k, dtype=torch.int32, device=DEV), full(p), full(m))
    s.check_status()
    mm = float(np.float32(m))
    near = np.abs(np.log(mm) * t / 0.25 - np.round(np.log(mm) * t / 0.25)) * 0.25
    assert near > 0.003
    for i in range(2):
        _same(s, i, z, float(np.float32(0.7)), t, k, float(np.float32(p)), mm)
    if k == 0 and p == 1.0 and dtype is torch.float32:
        assert int(s.kept[0]) == int(np.floor(-np.log(mm) * t / 0.25)) + 1
