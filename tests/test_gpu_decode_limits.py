"""The largest calls that the decode entry points take: where a launch of one workgroup a row, or a block,
would hold more work items than a grid dimension does."""
import sys

import pytest
import torch

from cache8_check import Cache, attend, check_attention
from oracle import decode as od

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _say(*a):
    print("[limits]", *a, file=sys.stderr, flush=True)


def _need(gib):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gib << 30:
        pytest.skip(f"needs {gib} GiB of device memory")


@pytest.fixture(autouse=True)
def _give_back(_gpu):
    yield
    torch.cuda.empty_cache()


def test_weights_of_the_longest_table():
    """2^26 blocks of 16 tokens, 72 rows: four blocks a workgroup of the launch that adds weights."""
    from paper_2608_21362_amd import kvb

    _need(24)
    c = Cache([700], 1, 64, 16, od.I8, seed=1)
    dev, held = c.device(), c.M
    c.M = 1 << 26
    table = torch.full((1, 1, 1, c.M), -1, dtype=torch.int32, device="cuda")
    table[..., :held] = dev["table"]
    dev["table"] = table
    q = torch.randn((9, 8, 64), generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    win = torch.ones((1, 1, c.M), device="cuda")
    _say("2^26 blocks, 72 rows")
    out, lse, w = attend(kvb, c, dev, q, [9], win, True)
    torch.cuda.synchronize()
    assert (w[..., held:] == 1).all()
    c.M = held
    check_attention(c, q, [9], out, lse, w[..., :held], win[..., :held])


def test_eviction_of_more_long_rows_than_one_grid_dimension_takes():
    """2^22 rows of 2049 entries: a workgroup of 1024 threads a row.  Three sequences are over their budget."""
    from paper_2608_21362_amd import kvb

    _need(110)
    L, n, M, B, budget = 4, 1 << 20, 2049, 16, 2000
    table = torch.empty((L, n, M), dtype=torch.int32, device="cuda")
    for l in range(L):  # numbers that are finite floats too: the weights are the same bits
        torch.randint(0x3F800000, 0x41000000, (n, M), dtype=torch.int32, device="cuda", out=table[l])
    weights = table.view(torch.float32)
    lens = torch.zeros(n, dtype=torch.int32, device="cuda")
    over = [0, n // 2 + 1, n - 1]
    lens[over] = M * B + 3
    table_out, weights_out = torch.empty_like(table), torch.empty_like(weights)
    lens_out = torch.empty_like(lens)
    lay = kvb.cache8_layout(1, 1, 64, B, kvb.KVB_I8, M)
    _say("2^22 rows of 2049 entries")
    kvb.kvb_cache8_evict(lay, L, n, budget, 1, 16, table, lens, weights, table_out, lens_out, weights_out)
    torch.cuda.synchronize()
    want = lens.clone()
    want[over] -= (M - budget) * B
    assert torch.equal(lens_out, want)
    for l in range(L):
        for b in over:
            t, w = od.evict(table[l, b].cpu().numpy(), weights[l, b].cpu().numpy(), M, budget, 1, 16)
            assert torch.equal(table_out[l, b].cpu(), torch.from_numpy(t))
            assert torch.equal(weights_out[l, b].cpu(), torch.from_numpy(w))
            table_out[l, b], weights_out[l, b] = table[l, b], weights[l, b]
        for x, y in ((table_out, table), (weights_out.view(torch.int32), table)):
            for part in range(0, n, n // 8):
                assert torch.equal(x[l, part:part + n // 8], y[l, part:part + n // 8]), (l, part)


def test_norm_of_the_most_heads():
    """2^26 - 4 heads of 8: the most that a call takes."""
    from paper_2608_21362_amd import kvb

    _need(8)
    n = (1 << 26) - 4
    x = torch.randn((n, 1, 8), dtype=torch.bfloat16, device="cuda")
    out, one = torch.full_like(x, 5.0), torch.ones(8, device="cuda")
    _say(f"{n} tokens of one head")
    kvb.kvb_qk_norm_rope(n, 1, 0, 8, kvb.KVB_BF16, x, 8, 8, None, 0, 0, one, None, 1e-6, None, None, None, 0, 0,
                         kvb.KVB_PAIR_HALF, out, 8, 8, None, 0, 0)
    torch.cuda.synchronize()
    for first in range(0, n, 1 << 23):
        y = x[first:first + (1 << 23)].float()
        ref = y / (y.square().mean(-1, keepdim=True) + 1e-6).sqrt()
        # one rounding to bfloat16, 2^-8, after float arithmetic
        assert ((out[first:first + (1 << 23)].float() - ref).abs() <= (2.0 ** -8 + 2.0 ** -18) * ref.abs()).all(), first
    with pytest.raises(kvb.KvbError) as e:
        kvb.kvb_qk_norm_rope(n + 1, 1, 0, 8, kvb.KVB_BF16, x, 8, 8, None, 0, 0, one, None, 1e-6, None, None, None, 0, 0,
                             kvb.KVB_PAIR_HALF, out, 8, 8, None, 0, 0)
    assert e.value.status == kvb.KVB_EINVAL
