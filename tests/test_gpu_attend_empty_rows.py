"""Rows of actkv_attend whose logits are all -inf: 0 and lse -inf, but for the dims in which a visible V entry is infinite or NaN; the same
in every way that the shares of a row are put together."""
import math

import pytest
import torch

from paper_2609_31395_b200 import harness as H

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


# one cluster per unit; pieces joined by a CTA per row; by a warp per row; the tensor-core kernel, with either join and in one piece
@pytest.mark.parametrize("R,L,W,max_tok", [(2, 100, 1, 100), (2, 9000, 1, 9000), (90, 5000, 1, 5000), (2, 9000, 3, 1 << 19),
                                           (40, 5000, 8, 1 << 19), (200, 60, 4, 1 << 19)])
@pytest.mark.parametrize("value", [0.0, math.inf, -math.inf, math.nan])
def test_rows_without_a_finite_logit(R, L, W, max_tok, value):
    P, hk, G, D = 32, 2, 4, 64
    need = -(-L // P)
    pool = torch.zeros((1, 2, need + 1, P, hk, D), dtype=torch.bfloat16, device=DEV)
    pool[:, 0, ..., 0] = -math.inf                     # q > 0: every logit is -inf
    pool[:, 1] = 1.0
    pool[:, 1, 1, 7, :, 5] = value                     # token 39, which all requests have and all rows see
    pool[:, :, need] = 3.0
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    table = torch.arange(need, device=DEV, dtype=torch.int32).repeat(R, 1)
    table[-1, 1] = need                                # the last request has an ordinary page instead
    q = torch.full((1, R * W, hk * G, D), 0.25, dtype=torch.bfloat16, device=DEV)
    dec = H.Decoder(pool, table, i32([L] * R), i32([0]), i32([0]), hk * G, R * W, W, max_tok)
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:3], 7.0, device=DEV)
    dec.attend(q, i32([W * r for r in range(R + 1)]), 0.125, True, out, lse)
    dec.check_status()
    empty = out[0, :(R - 1) * W].float()
    assert torch.isneginf(lse[0, :(R - 1) * W]).all()
    assert (empty[:, :, :5] == 0).all() and (empty[:, :, 6:] == 0).all()
    if value == 0.0:
        assert (empty == 0).all()
    else:
        assert not torch.isfinite(empty[:, :, 5]).any()
    assert (out[0, (R - 1) * W:] == 3.0).all() and torch.isfinite(lse[0, (R - 1) * W:]).all()
