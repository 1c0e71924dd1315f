"""actkv_logprob into buffers made for more rows than a call has (`LogprobBuffers` holds "up to" its rows)."""
import pytest
import torch

from paper_2609_31395_b200 import binding as B
from paper_2609_31395_b200 import harness as H

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _call(z, given, o):
    B.actkv_logprob(z, given, o.logprob, o.entropy, o.lse, o.top_logprob, o.top_index, o.status)


@pytest.mark.parametrize("rows", [16, 8, 12, 5, 4, 1])
@pytest.mark.parametrize("n_given", [0, 1, 3])
def test_fewer_rows_than_the_buffers_hold(rows, n_given):
    g = torch.Generator(device=DEV).manual_seed(rows)
    z = torch.randn((16, 2003), generator=g, device=DEV)
    given = torch.randint(2003, (16, n_given), generator=g, device=DEV).to(torch.int32) if n_given else None
    want, o = H.LogprobBuffers(16, n_given, 20, DEV), H.LogprobBuffers(16, n_given, 20, DEV)
    _call(z, given, want)
    o.top_index.fill_(-7)
    for t in (o.logprob, o.entropy, o.lse, o.top_logprob):
        t.fill_(77.0)
    _call(z[:rows], None if given is None else given[:rows], o)
    for name in ("logprob", "entropy", "lse", "top_logprob", "top_index"):
        got = getattr(o, name)
        assert torch.equal(got[:rows], getattr(want, name)[:rows]), name
        assert (got[rows:] == (-7 if name == "top_index" else 77.0)).all(), name
    assert int(o.status[0]) == 0


def test_no_rows():
    o = H.LogprobBuffers(4, 1, 5, DEV)
    _call(torch.empty((0, 100), device=DEV), torch.empty((0, 1), dtype=torch.int32, device=DEV), o)
    torch.cuda.synchronize()


@pytest.mark.parametrize("change", [
    dict(given=(3, 1)), dict(given=(5, 1)), dict(given=(8,)), dict(given=(2, 2)), dict(logprob=(3, 1)), dict(logprob=(4, 2)), dict(top_index=(3, 5)),
    dict(top_index=(20,)), dict(top_logprob=(4, 6)), dict(top_logprob=(3, 5)), dict(top_index=None), dict(top_logprob=None),
    dict(logprob=None), dict(lse=(3,)), dict(entropy=(3,))])
def test_buffers_of_other_shapes_are_refused(change):
    shape = dict(given=(4, 1), logprob=(4, 1), entropy=(4,), lse=(4,), top_logprob=(4, 5), top_index=(4, 5))
    shape.update(change)
    ints = ("given", "top_index")
    t = {n: None if s is None else torch.zeros(s, dtype=torch.int32 if n in ints else torch.float32, device=DEV) for n, s in shape.items()}
    with pytest.raises(ValueError):
        B.actkv_logprob(torch.zeros((4, 100), device=DEV), t["given"], t["logprob"], t["entropy"], t["lse"], t["top_logprob"], t["top_index"], None)
