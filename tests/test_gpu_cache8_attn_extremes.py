"""Attention over the 8-bit cache at the ends of what its inputs can hold: values of V so small or so far
apart that their scales leave a float's normal range, or so large that sums over them do; scores of any size.
Sums of probabilities, and the weights that come of them, do not depend on V."""
import sys

import numpy as np
import pytest
import torch

from cache8_check import Cache, attend, check_attention
from oracle import decode as od

pytestmark = pytest.mark.gpu

CODES = pytest.mark.parametrize("code", [od.I8, od.E4M3], ids=["i8", "e4m3"])
# queries and max_len: the kernel of few rows (in one piece, and split), and that of tiles of 256 rows
KINDS = pytest.mark.parametrize("nq,claim", [(1, 700), (1, 20000), (40, 2 ** 30), (40, 60000)],
                                ids=["few", "split", "tile", "tile_split"])


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _say(*a):
    print("[extremes]", *a, file=sys.stderr, flush=True)


def _normal(seed, *shape):
    return od.bf16(np.random.default_rng(seed).standard_normal(shape))


def _attend(c, q, nq, claim, scale=None):
    from paper_2608_21362_amd import kvb

    win = torch.rand((c.n, c.H, c.M), device="cuda")
    out, lse, w = attend(kvb, c, c.device(), q, [nq], win, True, max_len=claim, scale=scale)
    torch.cuda.synchronize()
    return out, lse, w, win


@CODES
@KINDS
@pytest.mark.parametrize("B,d,T", [(16, 64, 2300), (64, 128, 700)])
@pytest.mark.parametrize("big,small", [(1.0, 2.0 ** -126), (1.0, 2.0 ** -133), (100.0, 2.0 ** -126), (100.0, 2.0 ** -128),
                                       (1e4, 2.0 ** -120), (1e4, 2.0 ** -123), (1e4, 2.0 ** -133)])
def test_sums_do_not_depend_on_the_size_of_the_values(big, small, B, d, T, nq, claim, code):
    """Blocks of V at a float's lower end among ordinary ones (and 64 of them before the first ordinary one)."""
    _say(f"V {big} and {small} B {B} d {d} queries {nq} max_len {claim} code {code}")
    c = Cache([T], 1, d, B, code, seed=1)
    k, v = _normal(1, T, d), od.bf16(_normal(2, T, d) * big)
    rng = np.random.default_rng(3)
    for j in range(T // B):
        if j % 3 == 1 or (B == 16 and j < 64):
            v[j * B:(j + 1) * B] = np.float32(small) * rng.integers(-2, 3, (B, d))
    c.put(0, 0, 0, k, v)
    q = torch.from_numpy(_normal(4, nq, 4, d)).bfloat16().cuda()
    out, lse, w, win = _attend(c, q, nq, claim)
    check_attention(c, q, [nq], out, lse, w, win, sharp=True)


def _one_key(c, q, nq, claim, scale, at):
    """All of the weight is on key `at`."""
    out, lse, w, win = _attend(c, q, nq, claim, scale)
    check_attention(c, q, [nq], out, lse, w, win, scale=scale)
    want = torch.from_numpy(c.v[0, 0, 0][at]).cuda()
    # the sum's term is its own divisor but for the rounding of the probability to fp16; one rounding of the output
    assert ((out.double() - want).abs() <= (2.0 ** -8 + 2.0 ** -10) * want.abs()).all()
    share = (w - win).double()[0, 0]
    rows = q.shape[0] * q.shape[1]
    assert abs(share[at // c.B].item() - rows) <= 2.0 ** -16 * rows
    share[at // c.B] = 0
    assert share.abs().max() <= 2.0 ** -20


@CODES
@KINDS
@pytest.mark.parametrize("at", [5, 333, 650])
@pytest.mark.parametrize("B", [16, 64])
@pytest.mark.parametrize("scale", [1e5, 1e7, 1e9, 1e30])
def test_large_scores(scale, B, at, nq, claim, code):
    """Scores whose last bit is worth more than a probability's whole range.  q . k of one key is about
    4 |q|^2, over 350; of the others |q| times a normal number, below 80: further apart than any rounding."""
    _say(f"scale {scale} key {at} B {B} queries {nq} max_len {claim} code {code}")
    T, d = 700, 128
    c = Cache([T], 1, d, B, code, seed=3)
    k, v, u = _normal(8, T, d), _normal(9, T, d), _normal(10, d)
    k[at] = od.bf16(u * 4)
    c.put(0, 0, 0, k, v)
    q = u * np.random.default_rng(11).uniform(0.9, 1.1, (nq, 16, d))  # rows whose scores round up and down
    _one_key(c, torch.from_numpy(q).bfloat16().cuda(), nq, claim, scale, at)


@CODES
@KINDS
@pytest.mark.parametrize("at", [5, 333, 650])
def test_scores_far_below_zero(at, nq, claim, code):
    """Every score of a row is below -1e33: the largest of them still has all of the weight."""
    _say(f"key {at} queries {nq} max_len {claim} code {code}")
    T, d, B = 700, 128, 64
    c = Cache([T], 1, d, B, code, seed=4)
    v, u = _normal(11, T, d), _normal(12, d)
    k = od.bf16(u * np.random.default_rng(13).uniform(1, 2, (T, 1)))
    k[at] = od.bf16(u * 0.5)
    c.put(0, 0, 0, k, v)
    q = torch.from_numpy(np.broadcast_to(u, (nq, 4, d)).copy()).bfloat16().cuda()
    _one_key(c, q, nq, claim, -1e32, at)


@CODES
@KINDS
@pytest.mark.parametrize("coded,tail", [(2.0 ** 124, 2.0 ** 124), (1.0, 2.0 ** 124), (2.0 ** 124, 1.0), (2.0 ** -80, 2.0 ** 124), (2.0 ** -80, 2.0 ** -80)])
def test_values_near_the_end_of_the_range(coded, tail, nq, claim, code):
    """Sums of probabilities times V leave a float where their quotient does not."""
    _say(f"V {coded} tail {tail} queries {nq} max_len {claim} code {code}")
    T, d, B = 700, 128, 64
    c = Cache([T], 1, d, B, code, seed=5)
    k, v = _normal(14, T, d), _normal(15, T, d).astype(np.float64)
    v[:T // B * B] *= coded
    v[T // B * B:] *= tail
    assert np.abs(v).max() < 3.3e38
    c.put(0, 0, 0, k, od.bf16(v))
    q = torch.from_numpy(_normal(16, nq, 4, d)).bfloat16().cuda()
    out, lse, w, win = _attend(c, q, nq, claim)
    check_attention(c, q, [nq], out, lse, w, win, sharp=coded != tail)


@CODES
@KINDS
@pytest.mark.parametrize("before", [True, False], ids=["large_first", "small_first"])
@pytest.mark.parametrize("down", [20, 24, 28, 32])
def test_weight_on_a_block_of_small_values(down, before, nq, claim, code):
    """Nearly all of the weight on a block 2^-down of the others: within what a key may add, 2^-29 of the largest value."""
    _say(f"V down by 2^{down} large first {before} queries {nq} max_len {claim} code {code}")
    T, d, B, at = 700, 128, 64, 448 if before else 64
    c = Cache([T], 1, d, B, code, seed=2)
    k, v = _normal(5, T, d), _normal(6, T, d)
    v[at:at + B] *= np.float32(2.0 ** -down)
    u = _normal(7, d)
    k[at + 7] = od.bf16(u * 2)
    c.put(0, 0, 0, k, v)
    q = torch.from_numpy(np.broadcast_to(u, (nq, 4, d)).copy()).bfloat16().cuda()
    out, lse, w, win = _attend(c, q, nq, claim)
    check_attention(c, q, [nq], out, lse, w, win, sharp=True)


@CODES
@KINDS
@pytest.mark.parametrize("coded,tail", [(1.0, 1.0), (0.0, 1.0), (1.0, 0.0)], ids=["both", "tail", "coded"])
def test_small_values_keep_their_bits(coded, tail, nq, claim, code):
    """V of the size 2^-100.  Beside the bounds of check_attention a key of a full block adds what fp16 drops:
    2^-25 in units of 2^-106, times a code of up to 448."""
    _say(f"V 2^-100 coded {coded} tail {tail} queries {nq} max_len {claim} code {code}")
    T, d, B = 700, 128, 64
    c = Cache([T], 1, d, B, code, seed=6)
    k, v = _normal(17, T, d), _normal(18, T, d).astype(np.float64) * 2.0 ** -100
    v[:T // B * B] *= coded
    v[T // B * B:] *= tail
    c.put(0, 0, 0, k, od.bf16(v))
    q = torch.from_numpy(_normal(19, nq, 4, d)).bfloat16().cuda()
    out, lse, w, win = _attend(c, q, nq, claim)
    got, q = out.double().cpu().numpy(), q.double().cpu().numpy()
    for h in range(4):
        o, _, p = od.attention(q[:, h], c.k[0, 0, 0], c.v[0, 0, 0], d ** -0.5)
        off = 2.0 ** -24 * (d + 8) * d ** -0.5 * (np.abs(q[:, h]) @ np.abs(c.k[0, 0, 0]).T).max(1)
        off = off + 2.0 ** -25 * d ** -0.5 * np.abs(q[:, h]).max(1) * np.abs(c.k[0, 0, 0]).sum(1).max()
        near = p @ np.abs(c.v[0, 0, 0]) * (2.0 ** -11 + 2 * off + 2.0 ** -20)[:, None] + 2.0 ** -8 * np.abs(o)
        near = near + coded * T * 448 * 2.0 ** -131
        assert np.all(np.abs(got[:, h] - o) <= near), (h, float((np.abs(got[:, h] - o) / near).max()))
