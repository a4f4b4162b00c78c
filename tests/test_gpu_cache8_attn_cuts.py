"""Attention over the 8-bit cache, cut in every way: max_len only bounds the lengths, and with the number
of rows it decides tiles, waves and splits, so claims far above the lengths reach each kind of cut with
small caches.  Against the float64 oracle, as in the tests of its values."""
import sys

import numpy as np
import pytest
import torch

from cache8_check import Cache, attend, check_attention
from oracle import decode as od

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _run(lens, nq, Hq, H, d, B, code, claims, weights=True, seed=0, scale=None, sharp=False):
    from paper_2608_21362_amd import kvb

    c = Cache(lens, H, d, B, code, seed=seed)
    g = torch.Generator().manual_seed(seed)
    q = (torch.randn((sum(nq), Hq, d), generator=g) * 1.3).bfloat16().cuda()
    dev = c.device()
    win = torch.rand((c.n, H, c.M), device="cuda") if weights else None
    for claim in claims:
        print(f"[cuts] lens {lens[:4]} queries {nq[:4]} heads {Hq}/{H} d {d} B {B} code {code} max_len {claim}",
              file=sys.stderr, flush=True)
        out, lse, w = attend(kvb, c, dev, q, nq, win, weights, max_len=claim, scale=scale)
        torch.cuda.synchronize()
        check_attention(c, q, nq, out, lse, w, win, scale=scale, sharp=sharp)


# 8 rows a query and 2 heads: tiles of 256 rows from 2^25 / (16 * queries) tokens on
@pytest.mark.parametrize("B,code,lens", [
    (16, od.I8, [3000]), (16, od.E4M3, [2048, 1040]), (32, od.E4M3, [4200]), (64, od.I8, [4160]),
    (64, od.E4M3, [8300, 64]), (128, od.I8, [8200]), (128, od.E4M3, [4223, 70]),
])
@pytest.mark.parametrize("weights", [True, False])
def test_tiles_of_256_rows_over_several_chunks(B, code, lens, weights):
    """Blocks' ids and scales come 64 at a time; odd and even numbers of steps; one split, 2 to 9, and
    many; a sequence that ends inside the first split."""
    nq = [40, 17][:len(lens)]
    _run(lens, nq, 16, 2, 128, B, code, [2 ** 30, 500000, 130000, 60000], weights, seed=B)


@pytest.mark.parametrize("B", [16, 32, 64, 128])
@pytest.mark.parametrize("code", [od.I8, od.E4M3], ids=["i8", "e4m3"])
def test_tiles_of_256_rows_short(B, code):
    """No block, one block, few steps; rows that end inside a tile and a wave; head size 64."""
    lens = [1, B - 1, B, B + 1, 64, 65, 129, 300, 0]
    nq = [1, 9, 33, 2, 64, 40, 129, 36, 3]
    _run(lens, nq, 4, 1, 64, B, code, [2 ** 30], seed=1)
    _run(lens, nq, 8, 2, 128, B, code, [2 ** 30], seed=2)


def test_tiles_of_256_rows_over_longer_sequences_than_claimed():
    _run([9000], [700], 8, 1, 64, 64, od.I8, [6000], seed=3)


@pytest.mark.parametrize("B,code", [(16, od.I8), (32, od.E4M3), (64, od.E4M3), (128, od.I8)])
@pytest.mark.parametrize("claim", [1200, 4000, 40000])
def test_weights_of_thousands_of_rows(B, code, claim):
    """8800 rows and 200: tiles of 32 and of 256 rows, one split, 7 and many."""
    _run([1200, 25], [1100, 25], 8, 1, 64, B, code, [claim], seed=12)


@pytest.mark.parametrize("B,code", [(16, od.I8), (32, od.E4M3), (128, od.I8)])
def test_four_waves(B, code):
    """More than 256 heads of up to 2048 tokens."""
    rng = np.random.default_rng(0)
    lens = [int(x) for x in rng.integers(0, 260, 140)]
    _run(lens, [1] * 140, 4, 2, 64, B, code, [260], seed=4)
    _run(lens[:90], [3] * 90, 24, 3, 128, B, code, [2048], seed=5)


@pytest.mark.parametrize("claim", [1000, 2049, 5000, 40000, 2 ** 30])
@pytest.mark.parametrize("nq", [1, 6, 16])
def test_few_rows_in_every_number_of_splits(claim, nq):
    _run([2500, 900], [nq, nq], 16, 2, 128, 32, od.I8, [claim], seed=6)
    _run([2500, 900], [nq, nq], 8, 1, 64, 64, od.E4M3, [claim], seed=7)


@pytest.mark.parametrize("nq,claim", [(1, 700), (20, 700), (20, 2 ** 30)])
@pytest.mark.parametrize("scale", [-0.09, 0.0, 1e-6, 0.7])
def test_scales_of_the_scores(nq, claim, scale):
    _run([700, 33], [nq, nq], 16, 2, 128, 32, od.I8, [claim], seed=8, scale=scale, sharp=scale > 0.5)


@pytest.mark.parametrize("nq,claim", [(1, 3000), (3, 90000), (40, 3000), (40, 2 ** 30), (40, 60000)])
@pytest.mark.parametrize("gone", [(0, 64), (64, 128), (10, 150), (100, 180)])
def test_runs_of_entries_that_are_no_blocks(nq, claim, gone):
    """Whole chunks of a row without a block: as if their tokens were not in the sequence."""
    from paper_2608_21362_amd import kvb

    B, H, d, T = 16, 2, 128, 2990
    c = Cache([T], H, d, B, od.I8, seed=9)
    dev = c.device()
    t = c.table.copy()
    t[:, :, :, gone[0]:gone[1]] = -1
    dev["table"] = torch.from_numpy(t).cuda()
    g = torch.Generator().manual_seed(9)
    q = torch.randn((nq, 16, d), generator=g).bfloat16().cuda()
    out, lse, w = attend(kvb, c, dev, q, [nq], None, True, max_len=claim)
    torch.cuda.synchronize()
    keep = np.ones(T, bool)
    keep[gone[0] * B:gone[1] * B] = False
    for h in range(H):
        c.k[0, 0, h], c.v[0, 0, h] = c.k[0, 0, h][keep], c.v[0, 0, h][keep]
    left = torch.from_numpy(np.delete(w.cpu().numpy(), np.s_[gone[0]:gone[1]], 2))
    assert (w[:, :, gone[0]:gone[1]] == 0).all()
    full = torch.zeros_like(w)
    full[:, :, :left.shape[2]] = left.cuda()
    check_attention(c, q, [nq], out, lse, full)


@pytest.mark.parametrize("nq,at", [(80, 1160), (140, 1100)], ids=["tail", "block"])
def test_values_that_are_not_numbers_in_tiles_of_256_rows(nq, at):
    """An infinite value of V.  In the tail (tokens from 1152 on) it reaches its channel of the rows that see
    it; in a full block every channel of the rows that see of the block.  The others stay clean."""
    from paper_2608_21362_amd import kvb

    T = 1200
    c = Cache([T], 1, 128, 64, od.I8, seed=10)
    k, v = (od.bf16(np.random.default_rng(s).standard_normal((T, 128))) for s in (1, 2))
    c.put(0, 0, 0, k, v)
    g = torch.Generator().manual_seed(10)
    q = torch.randn((nq, 4, 128), generator=g).bfloat16().cuda()  # the last nq tokens
    bad = v.copy()
    bad[at, 7] = np.inf
    clean = dict(c.k), dict(c.v)
    c.put(0, 0, 0, k, bad)
    out, lse, _ = attend(kvb, c, c.device(), q, [nq], max_len=2 ** 30)
    torch.cuda.synchronize()
    assert torch.isfinite(lse).all()
    if at >= 1152:
        sees = at - (T - nq)
        assert (out[sees:, :, 7] == np.inf).all()
        other = torch.arange(128, device="cuda") != 7
        assert torch.isfinite(out[sees:, :, other].float()).all()
    else:
        sees = at // 64 * 64 - (T - nq)
        assert torch.isnan(out[sees:].float()).all()
    c.k, c.v = ({key: x[:T - nq + sees] for key, x in y.items()} for y in clean)
    check_attention(c, q[:sees], [sees], out[:sees], lse[:sees])


def test_captured_calls_of_both_kernels():
    """A graph of calls of each kind, replayed with new queries and eager calls between: equal bits."""
    from paper_2608_21362_amd import kvb

    c = Cache([3000, 500], 2, 128, 64, od.E4M3, seed=11)
    dev = c.device()
    kinds = [([1, 1], 3000), ([5, 9], 3000), ([40, 30], 60000), ([40, 30], 3000)]
    qs = [torch.randn((sum(nq), 16, 128), device="cuda").bfloat16() for nq, _ in kinds]

    def calls(workspaces):
        return [attend(kvb, c, dev, q, nq, None, True, max_len=claim, ws=ws)
                for q, (nq, claim), ws in zip(qs, kinds, workspaces)]

    spaces = [[torch.full((64 << 20,), 0xFF, dtype=torch.uint8, device="cuda") for _ in kinds] for _ in range(2)]
    from cache8_check import cu
    fixed = {tuple(nq): cu(nq) for nq, _ in kinds}  # a copy from the host does not belong in a graph
    import cache8_check
    real, cache8_check.cu = cache8_check.cu, lambda nq: fixed[tuple(nq)]
    try:
        calls(spaces[0])
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = calls(spaces[0])
        for _ in range(4):
            for q in qs:
                q.copy_(torch.randn(q.shape, device="cuda").bfloat16())
            torch.cuda.synchronize()
            graph.replay()
            ref = calls(spaces[1])
            torch.cuda.synchronize()
            for a, b in zip(got, ref):
                assert all(torch.equal(x, y) for x, y in zip(a, b))
    finally:
        cache8_check.cu = real
