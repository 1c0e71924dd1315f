"""Sliding windows longer than any cache see what causal attention sees, also for rows that stand before the first token."""
import pytest
import torch

from paper_2609_31395_b200 import harness as H
from paper_2609_31395_b200 import synth

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("S", [2 ** 31 - 1, 2 ** 31 - 5, 1 << 30, 5000])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("max_tok", [700, 1 << 19])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens,wins", [([5, 700, 0, 1, 129], [10, 3, 4, 9, 1]), ([5], [2])])
def test_a_window_beyond_everything(S, causal, max_tok, D, lens, wins):
    wl = synth.Workload("attend", 1, 2, 4, lens, wins, [0] * len(lens), head_dim=D, page_size=16, causal=causal, table_style="fragmented",
                        plant_frac=0.0, seed=D, poison_tail=True)
    inst = synth.generate(wl, DEV)

    def attend(window_left):
        dec = H.Decoder(inst.pool, inst.page_table, inst.seq_len, inst.free_list, inst.free_count, 8, sum(wins), max(wins), max_tok)
        out, lse = torch.full_like(inst.q, 7.0), torch.full(inst.q.shape[:3], 7.0, device=DEV)
        dec.attend(inst.q, inst.win_indptr, wl.sm_scale, causal, out, lse, window_left)
        dec.check_status()
        return out, lse
    want, got = attend(0), attend(S)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
