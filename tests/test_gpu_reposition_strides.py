"""actkv_reposition on pools whose base, heads, slots, pages or layers begin off a vector: every width of its loads, down to one element."""
import pytest
import torch

from paper_2609_31395_b200 import harness as H

from test_gpu_reposition import _case, _check, _run

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _spread(c, offset, pads):
    """The case's pool with `pads` elements more from one head, slot, page, K or V, layer to the next; returns the memory and what of it is no pool."""
    pool, strides, n = c["pool"], [1], 1
    for size, pad in zip(reversed(pool.shape[1:]), pads):
        n = n * size + pad
        strides.append(n)
    flat = torch.full((offset + strides[-1] * pool.shape[0] + 5,), 3.0, dtype=torch.bfloat16, device=DEV)
    view = flat.as_strided(pool.shape, tuple(reversed(strides)), offset)
    view.copy_(pool)
    d = c["dec"]
    c["pool"], c["dec"] = view, H.Decoder(view, d.page_table, d.seq_len, d.free_list, d.free_count, c["hk"], layers_per_call=c["layers"])
    other = torch.ones(flat.shape, dtype=torch.bool, device=DEV)
    other.as_strided(view.shape, view.stride(), offset).fill_(False)
    return flat, other


# the base's offset, and elements added to a head, a slot, a page, the K half, a layer
PLACES = [(1, (0, 0, 0, 0, 0)), (0, (1, 0, 0, 0, 0)), (0, (0, 1, 0, 0, 0)), (0, (0, 0, 3, 0, 0)), (0, (0, 0, 0, 0, 5)), (3, (1, 1, 1, 1, 1)), (2, (2, 2, 2, 2, 2)),
          (2, (0, 0, 0, 0, 0)), (4, (4, 0, 4, 0, 4)), (0, (0, 4, 0, 0, 0)), (8, (8, 8, 0, 8, 8)), (0, (0, 0, 0, 1, 0))]


@pytest.mark.parametrize("offset,pads", PLACES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("kw", [dict(D=64), dict(D=128, hk=3, to=True, rescale=True), dict(D=64, sections=[8, 12, 12], frm=False, to=True), dict(D=80, rotary=40, rescale=True),
                                dict(D=24, rotary=10, per_unit=False), dict(D=256, hk=1, sections=[100, 28])])
def test_parity(kw, interleaved, offset, pads):
    c = _case([70, 0, 33], layers=2, l0=1, interleaved=interleaved, seed=2, **kw)
    flat, other = _spread(c, offset, pads)
    before, around = c["pool"].clone(), flat[other]
    _run(c)
    _check(c, before)
    assert torch.equal(flat[other], around)
