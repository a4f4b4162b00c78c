


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
