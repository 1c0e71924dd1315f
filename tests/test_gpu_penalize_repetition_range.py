"""Repetition penalties at the ends of float32: from 2^-126 to 2^126, whose reciprocals are normal numbers too, they work; beyond they are reported."""
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
    return torch.from_numpy(np.array(x, dtype=np.float32)).to(DEV)


Z = [0.5, 3e38, INF, -INF, -2.0, -1e-3, 0.0, 1.0, -3e38, 1e30]


def _run(rep, dtype):
    z = torch.tensor([Z, Z], device=DEV).to(dtype)
    rules = H.LogitRules(_i32([range(len(Z))] * 2), _i32([len(Z)] * 2), None, _f32([rep, 2.0]))
    s, out = H.Sampler(1, DEV), torch.full_like(z, 7.0)
    s.penalize(z, _i32([0, 1, 2]), rules, 1, len(Z), out=out)
    back = z.clone()
    status = s.status.tolist()
    s.penalize(back, _i32([0, 1, 2]), rules, 1, len(Z))
    return z, out, back, status


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rep", [2.0 ** -126, 2.0 ** 126, 1e-37, 8e37, 1.0])
def test_the_ends_of_the_range(rep, dtype):
    z, out, back, status = _run(rep, dtype)
    assert status == [0] * 4 and torch.equal(out, back)
    for row, r in ((0, float(np.float32(rep))), (1, 2.0)):
        with np.errstate(over="ignore", invalid="ignore"):
            want = O.penalize_row(z[row].double().cpu().numpy(), range(len(Z)), 0, r, 0.0, 0.0, {}, None).astype(np.float64)
        got = out[row].double().cpu().numpy()
        limit = float(torch.finfo(dtype).max) * (1 + float(torch.finfo(dtype).eps) / 4)
        want[want > limit], want[want < -limit] = INF, -INF
        fin = np.isfinite(want)
        assert np.array_equal(got[~fin], want[~fin])
        # the reciprocal and the product, 2^-24 each, and half a step of bf16; results below 2^-126 come out as 0
        tol = np.abs(want[fin]) * (2 * 2.0 ** -24 + (2.0 ** -8 if dtype is torch.bfloat16 else 0)) + 2.0 ** -126
        assert (np.abs(got[fin] - want[fin]) <= tol).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rep", [1e-45, 1e-39, 1.0000001 * 2.0 ** 126, 3e38, -1e-39, -0.0])
def test_beyond_the_range_is_reported(rep, dtype):
    z, out, back, status = _run(rep, dtype)
    assert status[:2] == [B.E_INVALID, 0]
    assert torch.equal(back[0], z[0])            # in place: left as it is
    want = z[1].double().cpu().numpy()
    want = np.where(want > 0, want / 2, want * 2)
    want[want < -3.4e38] = -INF
    assert np.array_equal(out[1].double().cpu().numpy(), want) and torch.equal(back[1], out[1])
