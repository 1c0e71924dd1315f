"""GPU parity of actkv_attend against the float64 oracle.

Tolerances.  With u = 2^-24 and A the largest scale * sum |q_i k_i| of the case:
  a logit: D products summed in float32, the sum scaled and shifted: |dt| <= (D + 4) 2u A (tensor-core sums may truncate: 2u a step);
  a probability: relative error |dt| + 2^-21 (exp2 of 2 ulp, its argument rounded at magnitudes below 64);
  the summand pair of P in the product with V: 2^-16 relative;
  sums over n keys in float32: n / 16 + 64 steps of at most 2^-22 relative to sum p |v|;
  the divisor carries the errors of the probabilities again.
So |out - want| <= 2^-8 |want| + (2 dp + 2^-16 + (n / 16 + 64) 2^-22) sum p |v|, the first term bf16's half step, and
|lse - want| <= dp + n 2^-24 + |want| 2^-22.
"""
import numpy as np
import pytest
import torch

from oracle import actkv_oracle as O
from paper_2609_31395_b200 import binding as B
from paper_2609_31395_b200 import harness as H
from paper_2609_31395_b200 import synth

import parity_util as U

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
MANY = 1 << 19            # a bound on the lengths by which any number of rows above 8 is work for the tensor-core kernel


def _make(lens, wins, hkv=2, G=4, D=64, page=16, layers=1, causal=True, seed=0, head_major=False):
    wl = synth.Workload("attend", layers, hkv, G, list(lens), list(wins), [0] * len(lens), head_dim=D, page_size=page, causal=causal,
                        table_style="fragmented", plant_frac=0.0, seed=seed, poison_tail=True)
    inst = synth.generate(wl, DEV)
    inst.q.mul_(2.0)
    if head_major:
        inst.pool = inst.pool.permute(0, 1, 2, 4, 3, 5).contiguous().permute(0, 1, 2, 4, 3, 5)
    return inst


def _attend(inst, window_left=0, l0=0, l1=None, max_tok=None, stream=None, dec=None, causal=None):
    wl = inst.wl
    l1 = wl.n_layers if l1 is None else l1
    if dec is None:
        dec = H.Decoder(inst.pool, inst.page_table, inst.seq_len, inst.free_list, inst.free_count, wl.n_q_heads, sum(wl.windows),
                        max(wl.windows), max(wl.seq_lens) if max_tok is None else max_tok, wl.n_layers)
    out = torch.full_like(inst.q[l0:l1], 7.0)
    lse = torch.full(inst.q[l0:l1].shape[:3], 7.0, device=DEV)
    dec.attend(inst.q[l0:l1], inst.win_indptr, wl.sm_scale, wl.causal if causal is None else causal, out, lse, window_left, l0, l1, stream)
    return out, lse, dec


def _check(inst, out, lse, window_left=0, layers=None):
    wl = inst.wl
    layers = list(range(wl.n_layers)) if layers is None else layers
    pb, qb = U.bits(inst.pool), U.bits(inst.q[layers])
    pt, sl, wi = inst.page_table.cpu().numpy(), inst.seq_len.cpu().numpy(), inst.win_indptr.cpu().numpy()
    want, wlse = O.attend(pb, pt, sl, qb, wi, wl.n_q_heads, wl.sm_scale, wl.causal, window_left, layers)
    # sum p |v| and A by the same definition on absolute values
    kv_abs = pb.copy()
    kv_abs[:, 1] &= 0x7fff
    mass, _ = O.attend(kv_abs, pt, sl, qb, wi, wl.n_q_heads, wl.sm_scale, wl.causal, window_left, layers)
    A = 0.0
    for a, l in enumerate(layers):
        for r in range(wl.n_req):
            slots = O.slot_map(pt[r], int(sl[r]), wl.page_size)
            for h in range(wl.n_kv_heads):
                k = np.abs(O.bf16_bits_to_f64(O.gather_rows(pb, l, 0, h, slots)))
                q = np.abs(O.bf16_bits_to_f64(qb[a, wi[r]:wi[r + 1], h * wl.group:(h + 1) * wl.group])).reshape(-1, wl.head_dim)
                if k.size and q.size:
                    x = q @ k.T * wl.sm_scale
                    A = max(A, float(x[np.isfinite(x)].max(initial=0.0)))
    n = max(list(sl) + [1])
    dp = (wl.head_dim + 4) * 2.0 ** -23 * A + 2.0 ** -21
    tol = 2.0 ** -8 * np.abs(want) + (2 * dp + 2.0 ** -16 + (n / 16 + 64) * 2.0 ** -22) * mass + 1e-37
    got, glse = out.float().cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)
    empty = np.isneginf(wlse)
    assert np.array_equal(np.isneginf(glse), empty) and np.all(got[empty] == 0)
    assert np.isfinite(got).all()
    over = np.abs(got - want) - tol
    assert over.max(initial=-1.0) <= 0, f"out beyond tolerance by {over.max()} at {np.unravel_index(over.argmax(), over.shape)}"
    d = np.abs(glse[~empty] - wlse[~empty]) - (dp + n * 2.0 ** -24 + np.abs(wlse[~empty]) * 2.0 ** -22)
    assert d.max(initial=-1.0) <= 0, f"lse beyond tolerance by {d.max()}"
    # and all of it together is a float32 computation rounded once: half a bf16 step is uniform, 2^-9 / sqrt(3) of the value
    if want.size > 4000:
        assert np.linalg.norm(got - want) <= 1.2 * 2.0 ** -8 / np.sqrt(3) * np.linalg.norm(want)


def test_one_token_of_one_request():
    inst = _make([333], [1])
    out, lse, dec = _attend(inst)
    dec.check_status()
    _check(inst, out, lse)


@pytest.mark.parametrize("lens,wins", [
    ([1], [1]), ([16, 17, 15, 1, 0, 2], [1, 1, 1, 1, 0, 1]), ([0, 5, 0], [2, 3, 0]), ([2, 700], [5, 3]),
    ([4096, 33, 1025, 7], [1, 4, 2, 7]), ([130, 1500], [16, 33])])
@pytest.mark.parametrize("causal", [True, False])
def test_lengths_windows_and_rows_that_see_nothing(lens, wins, causal):
    inst = _make(lens, wins, causal=causal, seed=len(lens))
    out, lse, dec = _attend(inst)
    dec.check_status()
    _check(inst, out, lse)


@pytest.mark.parametrize("D", [8, 40, 64, 80, 128, 136, 192, 256])
@pytest.mark.parametrize("G,wins", [(1, (1, 1)), (4, (2, 3)), (7, (4, 1)), (8, (8, 5)), (32, (4, 3))])
def test_head_dims_and_groups(D, G, wins):
    inst = _make([300, 77], wins, hkv=2, G=G, D=D, seed=D + G)
    out, lse, dec = _attend(inst)
    dec.check_status()
    _check(inst, out, lse)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("max_tok", [400, MANY])
def test_more_rows_than_a_block(D, max_tok):
    inst = _make([400, 90], [37, 21], hkv=1, G=8, D=D, seed=3)
    out, lse, dec = _attend(inst, max_tok=max_tok)
    dec.check_status()
    _check(inst, out, lse)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G,wins", [(4, (3, 4)), (7, (4, 1)), (8, (8, 5)), (8, (9, 16)), (32, (4, 3)), (12, (0, 2)), (1, (60, 9))])
@pytest.mark.parametrize("lens", [(300, 77), (1, 5000), (0, 129)])
@pytest.mark.parametrize("S", [0, 40])
def test_the_tensor_core_kernel(D, G, wins, lens, S):
    # a large bound on the lengths takes the call there, as in a captured graph
    inst = _make(lens, wins, hkv=2, G=G, D=D, seed=D + G)
    out, lse, dec = _attend(inst, S, max_tok=MANY)
    dec.check_status()
    _check(inst, out, lse, S)


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("head_major", [False, True])
@pytest.mark.parametrize("causal", [True, False])
def test_pages_and_strides_of_the_tensor_core_kernel(page, head_major, causal):
    inst = _make([500, 129, 0, 16], [5, 3, 2, 4], D=128, page=page, layers=2, seed=page, head_major=head_major, causal=causal)
    out, lse, dec = _attend(inst, max_tok=MANY)
    dec.check_status()
    _check(inst, out, lse)


@pytest.mark.parametrize("page", [1, 5, 16, 32, 48, 128])
@pytest.mark.parametrize("head_major", [False, True])
def test_pages_and_strides(page, head_major):
    inst = _make([500, 129], [1, 3], D=128, page=page, layers=2, seed=page, head_major=head_major)
    out, lse, dec = _attend(inst)
    dec.check_status()
    _check(inst, out, lse)


@pytest.mark.parametrize("S", [1, 5, 16, 100, 10000])
@pytest.mark.parametrize("causal", [True, False])
def test_sliding_window(S, causal):
    inst = _make([700, 33, 128], [1, 9, 4], causal=causal, seed=S)
    out, lse, dec = _attend(inst, S)
    dec.check_status()
    _check(inst, out, lse, S)


def test_many_requests_and_layer_ranges():
    g = np.random.default_rng(5)
    lens = g.integers(0, 60, 300).tolist()
    inst = _make(lens, g.integers(0, 3, 300).tolist(), hkv=1, G=2, layers=3, seed=9)
    out, lse, dec = _attend(inst, l0=1, l1=3)
    dec.check_status()
    _check(inst, out, lse, layers=[1, 2])


def test_long_cache_in_many_pieces():
    inst = _make([30000, 11], [2, 1], hkv=1, G=8, D=128, seed=4)
    out, lse, dec = _attend(inst)
    dec.check_status()
    _check(inst, out, lse)


def test_offsets_beyond_32_bits():
    # pages at the end of a pool whose K half alone has 40000 * 56 * 1024 > 2^31 elements
    P, Hk, D, n_pages = 16, 1, 64, 40000
    pool = torch.zeros((1, 2, n_pages * 56, P, Hk, D), dtype=torch.bfloat16, device=DEV)
    assert pool.stride(1) > 2 ** 31
    pt = torch.tensor([[n_pages * 56 - 1, 0, n_pages * 56 - 2]], dtype=torch.int32, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(1)
    small = torch.randn((2, 3, P, Hk, D), generator=g, device=DEV, dtype=torch.bfloat16)
    for i, p in enumerate(pt[0].tolist()):
        pool[0, :, p] = small[:, i]
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)
    q = torch.randn((1, 1, 4, D), generator=g, device=DEV, dtype=torch.bfloat16)
    out, lse = torch.empty_like(q), torch.empty((1, 1, 4), device=DEV)
    dec = H.Decoder(pool, pt, i32(41), i32(0), i32(0), 4, 1, 1, 48)
    dec.attend(q, i32(0, 1), 0.125, True, out, lse)
    dec.check_status()
    want, wl = O.attend(U.bits(small[None]), np.array([[0, 1, 2]]), [41], U.bits(q), [0, 1], 4, 0.125, True)
    assert np.abs(out.float().cpu().numpy() - want).max() <= 2.0 ** -8 * np.abs(want).max() + 1e-4
    assert np.abs(lse.cpu().numpy() - wl).max() < 1e-5


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("max_tok", [220, MANY])
def test_masked_slots_do_not_reach_a_row(value, max_tok):
    # window rows 0 and 1 must not see the last two keys; with a sliding window of 50 nor the first ones
    inst = _make([220], [3], hkv=1, G=4, D=128)
    P = inst.wl.page_size
    clean = inst.pool.clone()

    def plant(j):
        inst.pool[:, :, inst.page_table[0, j // P].item(), j % P] = value
    plant(219)
    plant(218)
    for j in (0, 100, 160, 166):
        plant(j)
    out, lse, dec = _attend(inst, 50, max_tok=max_tok)
    inst.pool = clean
    wl = inst.wl
    want, wlse = O.attend(U.bits(clean), inst.page_table.cpu().numpy(), [220], U.bits(inst.q), [0, 3], 4, wl.sm_scale, True, 50)
    got = out.float().cpu().numpy()
    # row 0 stands at 217 and sees 168 .. 217
    np.testing.assert_allclose(got[0, 0], want[0, 0], rtol=2.0 ** -8, atol=1e-3)
    np.testing.assert_allclose(lse.cpu().numpy()[0, 0], wlse[0, 0], rtol=1e-5)
    assert not np.isfinite(got[0, 2]).all()                  # row 2 sees both
    dec.check_status()


def test_nan_and_infinite_logits_make_their_rows_nan():
    inst = _make([100, 100], [1, 1], hkv=1, G=2, D=64)
    P = inst.wl.page_size
    inst.pool[:, 0, inst.page_table[0, 1].item(), 3] = float("nan")
    out, lse, _ = _attend(inst)
    assert torch.isnan(out[0, 0].float()).all() and torch.isnan(lse[0, 0]).all()
    assert torch.isfinite(out[0, 1].float()).all() and torch.isfinite(lse[0, 1]).all()


def test_upper_bounds_and_determinism():
    inst = _make([900, 40, 333], [1, 2, 1], hkv=2, G=4, D=128, seed=8)
    a, la, dec = _attend(inst, max_tok=5000)
    b, lb, _ = _attend(inst, max_tok=5000, dec=dec)
    assert torch.equal(a, b) and torch.equal(la, lb)
    dec.check_status()
    _check(inst, a, la)


def test_bad_tables_are_reported():
    inst = _make([100, 200], [1, 1])
    inst.page_table[1, 3] = 1 << 20
    out, lse, dec = _attend(inst)
    assert dec.status.cpu().tolist()[:3] == [B.E_BADPAGE, 1, 1 << 20]
    assert torch.isfinite(out[0, 0].float()).all()
    # a length beyond the host's bound: that request is left alone
    inst = _make([100, 200], [1, 1], seed=2)
    out, lse, dec = _attend(inst, max_tok=150)
    assert dec.status.cpu().tolist()[:3] == [B.E_INVALID, 1, 200]
    assert (out[0, 1] == 7).all() and (lse[0, 1] == 7).all()
    inst.seq_len[1] = 0
    want, _, _ = _attend(inst)
    assert torch.equal(out[0, 0], want[0, 0])


def test_another_stream_and_a_captured_graph_with_growing_lengths():
    inst = _make([300, 200], [1, 1], hkv=2, G=4, D=128, seed=11)
    wl = inst.wl
    want, wl_lse, _ = _attend(inst, max_tok=400)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out, lse, dec = _attend(inst, stream=s, max_tok=400)
    s.synchronize()
    assert torch.equal(out, want)
    g = torch.cuda.CUDAGraph()
    out, lse = torch.empty_like(inst.q), torch.empty(inst.q.shape[:3], device=DEV)
    with torch.cuda.graph(g):
        dec.attend(inst.q, inst.win_indptr, wl.sm_scale, True, out, lse, l1=1)
    full = inst.seq_len.clone()
    for lens in ([300, 200], [17, 200], [260, 1]):
        inst.seq_len.copy_(torch.tensor(lens, dtype=torch.int32))
        g.replay()
        torch.cuda.synchronize()
        _check(inst, out, lse)
    inst.seq_len.copy_(full)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(lse, wl_lse)
    dec.check_status()


def test_two_calls_at_once_with_a_workspace_each():
    a, b = _make([5000, 70], [1, 1], D=128, seed=1), _make([90, 4000], [1, 1], D=128, seed=2)
    want = [_attend(x)[0] for x in (a, b)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(20):
        got = []
        for x, s in zip((a, b), streams):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                got.append(_attend(x)[0])
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("D,lens,after", [(64, [900, 1500], 0), (128, [900, 1500], 0), (64, [50000, 1500], 1), (128, [50000, 1500], 3)])
def test_a_wait_that_runs_out_is_reported(D, lens, after):
    # the hook lets the first `after` tiles of every stretch arrive and no other (short requests: a stretch is one tile); the waits
    # give up after 5 ms and every role leaves
    inst = _make(lens, [4, 3], hkv=2, G=8, D=D, seed=D)
    want, wlse, dec = _attend(inst, max_tok=MANY)
    dec.check_status()
    B.actkv_debug_inject_stall(after, 5000)
    try:
        _attend(inst, dec=dec)
        torch.cuda.synchronize()
    finally:
        B.actkv_debug_inject_stall(-1, 0)
    assert dec.status.cpu().tolist()[0] == B.E_TIMEOUT
    dec.status.zero_()
    out, lse, _ = _attend(inst, dec=dec)
    dec.check_status()
    assert torch.equal(out, want) and torch.equal(lse, wlse)
