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
