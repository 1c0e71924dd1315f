"""The angle of actkv_reposition is rounded to its steps of 2^-23 turns, not cut."""
import numpy as np
import pytest
import torch

from paper_2609_31395_b200 import harness as H

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _sines(interleaved, rescale, sign):
    """Sine of 64 x 300 small angles that lie anywhere within a step, as the second dim of a pair (1, 0) that turned by them, and the angles."""
    n, pairs, page = 300, 64, 16
    pool = torch.zeros((1, 2, 19, page, 1, 2 * pairs), dtype=torch.bfloat16, device=DEV)
    first = (slice(0, None, 2) if interleaved else slice(0, pairs))
    second = (slice(1, None, 2) if interleaved else slice(pairs, None))
    pool[..., first] = 1.0
    freq = torch.from_numpy((1.37e-7 * (1 + np.arange(pairs) / 97)).astype(np.float32)).to(DEV)
    dec = H.Decoder(pool, _i32([list(range(19))]), _i32([n]), _i32([0] * 19), _i32([0]), 1)
    to = sign * torch.arange(1, n + 1, dtype=torch.int32, device=DEV)
    if rescale:
        dec.reposition(H.Rope(freq * 0, [pairs], interleaved), _i32([0, n]), n, torch.zeros_like(to), to, to_inv_freq=freq)
    else:
        dec.reposition(H.Rope(freq, [pairs], interleaved), _i32([0, n]), n, torch.zeros_like(to), to)
    dec.check_status()
    got = pool[0, 0, :, :, 0].reshape(19 * page, 2 * pairs)[:n, second].double().cpu().numpy()
    return got, np.sin(to.double().cpu().numpy()[:, None] * freq.double().cpu().numpy())


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rescale", [False, True])
def test_small_angles_are_off_to_both_sides_alike(interleaved, rescale):
    """A step is 2 pi 2^-23 = 7.5e-7.  Rounded, an angle is off by at most half of it, as often to either side; cut, by up to a whole one, by
    half a step on average.  The sines here lie below 7e-5, so that their own rounding to bf16 (2^-8 relative, 2.8e-7 at most) and the sine's
    error, which has the sign of the angle, go to both sides over both signs of the angle: the mean over 38400 angles of both signs stays below a
    twentieth of a step, 3.7e-8; cut it would be 3.7e-7."""
    step = 2 * np.pi * 2.0 ** -23
    off = []
    for sign in (1, -1):
        got, want = _sines(interleaved, rescale, sign)
        assert (np.abs(got - want) <= step / 2 + 2.0 ** -8 * (np.abs(want) + step) + 2.0 ** -32 * 2 * np.pi + 2.0 ** -21.4).all()
        off.append(got - want)
    assert abs(np.mean(off)) <= step / 20
