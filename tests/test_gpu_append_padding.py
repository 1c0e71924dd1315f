"""Rows behind the last request of a padded batch (a captured graph's fixed number of rows): actkv_append leaves their q_out, and the pool;
actkv_attend their out and lse."""
import pytest
import torch

from paper_2609_31395_b200 import harness as H

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("shift", [0, 1])                 # (1: rows off a 16-byte boundary take the other kernel)
@pytest.mark.parametrize("turned", [True, False])
@pytest.mark.parametrize("wins", [[2, 1, 3], [0, 0, 0], [0, 5, 0]])
def test_rows_of_no_request(shift, turned, wins):
    rows, hq, hk, D, used = 9, 4, 2, 32, sum(wins)
    g = torch.Generator(device=DEV).manual_seed(1)
    pool = torch.randn((1, 2, 12, 16, hk, D), generator=g, device=DEV).to(torch.bfloat16)
    dec = H.Decoder(pool, _i32([[0, 1], [2, 3], [4, 5]]), _i32([20, 30, 17]), _i32([0] * 12), _i32([0]), hq, rows, rows, 32)
    x = torch.randn((1, rows, (hq + 2 * hk) * D + shift), generator=g, device=DEV).to(torch.bfloat16)[:, :, shift:].unflatten(2, (hq + 2 * hk, D))
    rope = H.Rope(torch.rand(D // 2, generator=g, device=DEV), [D // 2]) if turned else None
    pos = torch.randint(0, 1000, (1, rows), generator=g, device=DEV).to(torch.int32)
    wi = _i32([0, wins[0], wins[0] + wins[1], used])

    def call(n):
        out = torch.full((1, n, hq, D), 9.0, dtype=torch.bfloat16, device=DEV)
        dec.append(x[:, :n, hq:hq + hk], x[:, :n, hq + hk:], wi, q=x[:, :n, :hq], q_out=out, rope=rope, positions=pos[:, :n].contiguous())
        return out
    first = call(used) if used else None
    before = pool.clone()
    out = call(rows)
    dec.check_status()
    assert torch.equal(pool, before)                      # the same rows again, and nothing for the others
    assert used == 0 or torch.equal(out[:, :used], first)
    assert (out[:, used:] == 9.0).all()


@pytest.mark.parametrize("max_tok", [32, 1 << 19])        # (the bound decides between the warp-level and the tensor-core kernel)
@pytest.mark.parametrize("wins", [[2, 1, 3], [0, 0, 0], [0, 5, 0]])
def test_attention_leaves_rows_of_no_request(max_tok, wins):
    rows, hq, hk, D, used = 9, 16, 2, 64, sum(wins)
    g = torch.Generator(device=DEV).manual_seed(2)
    pool = torch.randn((1, 2, 12, 16, hk, D), generator=g, device=DEV).to(torch.bfloat16)
    dec = H.Decoder(pool, _i32([[0, 1], [2, 3], [4, 5]]), _i32([20, 30, 17]), _i32([0] * 12), _i32([0]), hq, rows, 5, max_tok)
    q = torch.randn((1, rows, hq, D), generator=g, device=DEV).to(torch.bfloat16)
    wi = _i32([0, wins[0], wins[0] + wins[1], used])

    def call(n):
        out, lse = torch.full((1, n, hq, D), 9.0, dtype=torch.bfloat16, device=DEV), torch.full((1, n, hq), 9.0, device=DEV)
        dec.attend(q[:, :n].contiguous(), wi, 0.125, True, out, lse)
        return out, lse
    out, lse = call(rows)
    dec.check_status()
    assert (out[:, used:] == 9.0).all() and (lse[:, used:] == 9.0).all()
    if used:
        first = call(used)
        assert torch.equal(out[:, :used], first[0]) and torch.equal(lse[:, :used], first[1]) and (lse[:, :used] != 9.0).all()
