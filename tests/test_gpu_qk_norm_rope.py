"""Norms of queries and keys with their rotation, against the float64 oracle."""
import sys

import numpy as np
import pytest
import torch

from oracle import decode as od

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _kvb():
    from paper_2608_21362_amd import kvb
    return kvb


def _check(got, x, w, eps, cos, sin, rot, pairing, dtype):
    """u = 2^-24: a sum of d squares (16 in a row, 5 levels), its root and quotient, and the products are
    off by at most 16 u of the output's terms, so 2^-19 of them with the table's rounding; then one
    rounding to the type, 2^-8 or 2^-24."""
    ref, size = od.norm_rope(x, w, eps, cos, sin, rot, pairing)
    last = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    d = np.abs(got.double().cpu().numpy() - ref)
    assert np.all(d <= last * np.abs(ref) + 2.0 ** -19 * size), float((d - last * np.abs(ref)).max())


def _call(kvb, T, Hq, H, d, dtype, q, k, wq, wk, eps, pos, cos, sin, rot, pairing, qo, ko, **kw):
    s = lambda t: (0, 0) if t is None else (t.stride(0), t.stride(1))  # noqa: E731
    kvb.kvb_qk_norm_rope(T, Hq, H, d, kvb.KVB_BF16 if dtype == torch.bfloat16 else kvb.KVB_F32, q, *s(q), k, *s(k), wq,
                         wk, eps, pos, cos, sin, 0 if cos is None else cos.shape[0], rot, pairing, qo, *s(qo), ko, *s(ko),
                         **kw)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("pairing", [od.HALF, od.INTERLEAVED], ids=["half", "interleaved"])
@pytest.mark.parametrize("T,Hq,H,d,rot,norm", [
    (1, 16, 2, 128, 128, True), (1, 1, 1, 8, 8, True), (7, 4, 2, 64, 32, True), (33, 5, 1, 80, 80, True),
    (3, 20, 4, 128, 40, False), (65, 8, 8, 256, 64, True), (2, 33, 1, 128, 0, True), (5, 3, 0, 24, 16, False),
    (9, 0, 3, 136, 136, True), (300, 16, 2, 128, 128, True), (4, 70, 10, 64, 64, False)])
def test_against_the_oracle(T, Hq, H, d, rot, norm, pairing, dtype):
    kvb = _kvb()
    print(f"[norm_rope] T {T} heads {Hq}/{H} d {d} rot {rot} norm {norm} {pairing} {dtype}", file=sys.stderr, flush=True)
    rng = np.random.default_rng(T * d + rot)
    x = torch.from_numpy(rng.standard_normal((T, Hq + 2 * H, d)) * np.exp(rng.standard_normal((T, Hq + 2 * H, 1)) * 3)).to(dtype)
    dev = x.cuda()  # one projection's output: queries, keys, values
    n = 4000
    tc, ts = od.table(od.frequencies(1e4, max(rot, 2)), np.arange(n))
    pos = rng.integers(0, n, T).astype(np.int32)
    wq, wk = (rng.standard_normal(d).astype(np.float32) for _ in range(2))
    cuda = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    qo = torch.full((T, max(Hq, 1), d), 5.0, dtype=dtype, device="cuda")
    cache = torch.full((max(H, 1), T + 2, d), 5.0, dtype=dtype, device="cuda")  # [Hkv][T][d]
    ko = cache.transpose(0, 1)
    on = rot > 0
    _call(kvb, T, Hq, H, d, dtype, dev[:, :Hq] if Hq else None, dev[:, Hq:Hq + H] if H else None,
          cuda(wq) if norm else None, cuda(wk) if norm else None, 1e-5, cuda(pos) if on else None,
          cuda(tc) if on else None, cuda(ts) if on else None, rot, pairing, qo if Hq else None, ko if H else None)
    torch.cuda.synchronize()
    xs = x.double().numpy()
    cos, sin = tc[pos][:, :rot // 2], ts[pos][:, :rot // 2]
    if Hq:
        _check(qo, xs[:, :Hq], wq if norm else None, 1e-5, cos, sin, rot, pairing, dtype)
    if H:
        _check(ko[:T], xs[:, Hq:Hq + H], wk if norm else None, 1e-5, cos, sin, rot, pairing, dtype)
    assert (cache[:, T:] == 5).all()


@pytest.mark.parametrize("T,Hq,H,d,rot,norm,pairing,dtype", [
    (17001, 5, 1, 128, 128, True, od.HALF, torch.bfloat16), (9001, 20, 4, 128, 64, True, od.INTERLEAVED, torch.float32),
    (17003, 9, 7, 64, 32, True, od.HALF, torch.float32), (10001, 3, 5, 256, 256, True, od.INTERLEAVED, torch.bfloat16),
    (10001, 3, 5, 200, 80, False, od.HALF, torch.bfloat16), (50001, 0, 5, 40, 40, True, od.HALF, torch.bfloat16)])
def test_many_tokens(T, Hq, H, d, rot, norm, pairing, dtype):
    """A wave takes several groups of heads; groups and heads that end inside one."""
    test_against_the_oracle(T, Hq, H, d, rot, norm, pairing, dtype)


def test_one_norm_without_the_other_and_in_place():
    kvb = _kvb()
    T, d = 50, 128
    g = torch.Generator().manual_seed(0)
    q, k = torch.randn((T, 4, d), generator=g), torch.randn((T, 2, d), generator=g)
    w = torch.randn(d, generator=g)
    tc, ts = (torch.from_numpy(t).cuda() for t in od.table(od.frequencies(1e6, d), np.arange(T)))
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    for wq, wk in ((w, None), (None, w)):
        qd, kd = q.cuda(), k.cuda()
        c = lambda t: None if t is None else t.cuda()  # noqa: E731
        _call(kvb, T, 4, 2, d, torch.float32, qd, kd, c(wq), c(wk), 0.0, pos, tc, ts, d, od.HALF, qd, kd)
        n = lambda t: None if t is None else t.numpy()  # noqa: E731
        _check(qd, q.numpy(), n(wq), 0.0, tc.cpu().numpy(), ts.cpu().numpy(), d, od.HALF, torch.float32)
        _check(kd, k.numpy(), n(wk), 0.0, tc.cpu().numpy(), ts.cpu().numpy(), d, od.HALF, torch.float32)


def test_positions_outside_the_table_and_zero_heads():
    kvb = _kvb()
    T, d = 6, 64
    q = torch.randn((T, 2, d)).cuda()
    q[5, 1] = 0
    out = torch.zeros_like(q)
    tc, ts = (torch.from_numpy(t).cuda() for t in od.table(od.frequencies(1e4, 32), np.arange(10)))
    pos = torch.tensor([0, -1, 9, 10, 2 ** 31 - 1, 3], dtype=torch.int32, device="cuda")
    _call(kvb, T, 2, 0, d, torch.float32, q, None, torch.ones(d, device="cuda"), None, 1e-6, pos, tc, ts, 32,
          od.INTERLEAVED, out, None)
    bad = torch.isnan(out).flatten(1)
    assert bad[[1, 3, 4]].all() and not bad[[0, 2, 5]].any() and (out[5, 1] == 0).all()


def test_more_than_two_gib_of_rows():
    """Offsets past 2^31 elements: the last tokens of a long strided input."""
    kvb = _kvb()
    T, d, ts_ = 270000, 64, 8192  # a token every 8192 elements
    x = torch.zeros(T * ts_, dtype=torch.bfloat16, device="cuda")
    x.view(T, ts_)[:, :d] = torch.randn((T, d), device="cuda").bfloat16()
    out = torch.zeros((T, 1, d), dtype=torch.bfloat16, device="cuda")
    kvb.kvb_qk_norm_rope(T, 1, 0, d, kvb.KVB_BF16, x, ts_, d, None, 0, 0, torch.ones(d, device="cuda"), None, 1e-6,
                         None, None, None, 0, 0, kvb.KVB_PAIR_HALF, out, d, d, None, 0, 0)
    y = x.view(T, ts_)[:, :d].float()
    ref = y / (y.square().mean(1, keepdim=True) + 1e-6).sqrt()
    # one rounding to bfloat16, 2^-8, after float arithmetic
    assert ((out[:, 0].float() - ref).abs() <= 2.0 ** -8 * ref.abs() + 2.0 ** -18 * ref.abs()).all()
