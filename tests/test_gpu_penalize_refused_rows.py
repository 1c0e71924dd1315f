"""Rows whose rules actkv_penalize refused, out of place: every logit is -inf, so that no token is drawn from them, whatever the buffer held before."""
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
    return torch.tensor(x, dtype=torch.float32, device=DEV)


CAUSES = {"repetition": B.E_INVALID, "presence": B.E_INVALID, "history": B.E_INVALID, "window": B.E_INVALID, "order": B.E_BADINDEX, "token": B.E_BADINDEX,
          "bias range": B.E_INVALID, "mask": B.E_BADINDEX}


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("win,vocab,shift", [([2, 1, 3], 500, 0), ([1, 40, 2], 60000, 0), ([3, 5, 1], 3001, 1)])
@pytest.mark.parametrize("cause,masks", [(c, m) for c in CAUSES for m in (False, True) if m or c != "mask"])
def test_nothing_is_drawn_from_refused_rows(cause, win, vocab, shift, masks, dtype):
    """The second request is refused, or with "mask" one of its rows; shift: the output begins elsewhere in a vector than the logits."""
    g = torch.Generator(device=DEV).manual_seed(4)
    rows, first = sum(win) + 1, win[0]                          # (the last row is of no request)
    z = (torch.randn((rows, vocab), generator=g, device=DEV) * 3).to(dtype)
    tokens = torch.randint(0, vocab, (3, 60), generator=g, device=DEV).to(torch.int32)
    hist, rep, pres = [60, 50, 40], [1.5, 1.25, 0.75], [0.5, 0.25, 1.0]
    bias_indptr, bias_token, bias_value = [0, 2, 4, 4], [3, 90, 7, 400], [1.0, -2.0, 0.5, 4.0]
    max_win, max_hist = max(win), 60
    allow_row = [0 if i % 2 else -1 for i in range(rows)]
    refused = list(range(first, first + win[1]))
    if cause == "repetition":
        rep[1] = -1.0
    elif cause == "presence":
        pres[1] = INF
    elif cause == "history":
        hist[1] = 61
    elif cause == "window":
        win = win[:1] + [max_win + 1] + win[2:]
        rows += max_win + 1 - len(refused)
        z = torch.cat([z, z[:rows - z.shape[0]]]) if rows <= 2 * z.shape[0] else z.repeat(3, 1)[:rows]
        allow_row = [0 if i % 2 else -1 for i in range(rows)]
        refused = list(range(first, first + win[1]))
    elif cause == "order":
        bias_token[2:] = [400, 7]
    elif cause == "token":
        bias_token[3] = vocab
    elif cause == "bias range":
        bias_indptr[2:] = [5, 4]
    elif cause == "mask":
        refused = [first + win[1] // 2]
        allow_row[refused[0]] = 3
    words = torch.randint(-2 ** 31, 2 ** 31 - 1, (3, (vocab + 31) // 32), generator=g, device=DEV).to(torch.int32)
    rules = H.LogitRules(tokens, _i32(hist), None, _f32(rep), None, _f32(pres), _i32(bias_indptr), _i32(bias_token), _f32(bias_value),
                         words if masks else None, _i32(allow_row) if masks else None)
    whole = torch.full((rows, vocab + 8), 7.0, dtype=dtype, device=DEV)
    out = whole[:, shift:shift + vocab]
    before, s = z.clone(), H.Sampler(rows, DEV)
    s.penalize(z, _i32([0] + np.cumsum(win).tolist()), rules, max_win, max_hist, out=out)
    st = s.status.tolist()
    assert st[0] == CAUSES[cause] and st[1] in (1, 2) and torch.equal(z, before)
    assert (out[refused] == -INF).all()
    s.sample(out, torch.full((rows,), 0.5, device=DEV))
    s.token, t = s.token.cpu(), s.token.tolist()
    at = dict(zip(range(rows), t))
    assert all(at[i] == -1 for i in refused)
    allowed = np.unpackbits(words[0].cpu().numpy().view(np.uint8), bitorder="little")[:vocab].astype(bool)
    size = 2.0 ** -8 if dtype is torch.bfloat16 else 0.0
    starts = [0] + np.cumsum(win).tolist()
    for r in (0, 2):
        if r == 2 and cause == "bias range":
            continue                                            # (whose biases begin behind the end)
        for w in range(win[r]):
            i = starts[r] + w
            bias = {bias_token[b]: bias_value[b] for b in range(bias_indptr[r], bias_indptr[r + 1])}
            past = tokens[r, :hist[r] - (win[r] - 1 - w)].cpu().numpy()
            raw = z[i].double().cpu().numpy()
            want = O.penalize_row(raw, past, 0, rep[r], 0.0, pres[r], bias, allowed if masks and allow_row[i] == 0 else None)
            got, fin = out[i].double().cpu().numpy(), np.isfinite(want)
            assert np.array_equal(np.isfinite(got), fin)
            # five float32 roundings of at most what a logit meets on its way, and half a step of bf16
            tol = size * np.abs(want[fin]) + 5 * 2.0 ** -24 * ((np.abs(raw[fin]) + 4) * 1.5 + 1)
            assert (np.abs(got[fin] - want[fin]) <= tol).all() and at[i] >= 0
    assert (whole[:, :shift] == 7.0).all() and (whole[:, shift + vocab:] == 7.0).all()
    free = set(range(rows)) - set(range(starts[3]))
    assert all((out[i] == 7.0).all() for i in free)


def test_windows_that_cannot_be_told_leave_rows_outside_the_logits_alone():
    """A window that ends behind the logits, and one that ends before it begins."""
    z = torch.randn((4, 100), device=DEV)
    for ind, refused in (([0, 1, 9], [1, 2, 3]), ([0, 3, 1], []), ([-2, 2, 4], [0, 1])):
        whole, s = torch.full((6, 100), 7.0, device=DEV), H.Sampler(1, DEV)
        s.penalize(z, _i32(ind), H.LogitRules(presence=_f32([0.0, 0.0])), 4, 0, out=whole[1:5])
        assert s.status[0].item() == B.E_INVALID
        assert (whole[[0, 5]] == 7.0).all() and (whole[1:5][refused] == -INF).all()
        for r, (a, b) in enumerate(zip(ind, ind[1:])):
            if 0 <= a <= b <= 4:
                assert torch.equal(whole[1 + a:1 + b], z[a:b])
