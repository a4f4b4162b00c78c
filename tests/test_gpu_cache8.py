"""Rows into the 8-bit cache and back, and the eviction of blocks, against the float64
oracle: codes, scales and tables are equal, bit for bit."""
import sys

import numpy as np
import pytest
import torch

from cache8_check import Cache, cu
from oracle import decode as od

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _say(*a):
    print(*a, file=sys.stderr, flush=True)


def _kvb():
    from paper_2608_21362_amd import kvb
    return kvb


ARRAYS = ("k_codes", "k_scale", "v_codes", "v_scale", "k_tail", "v_tail")


def _empty(c):
    dev = c.device()
    for k in ("k_codes", "v_codes"):
        dev[k].fill_(0x55)
    for k in ("k_scale", "v_scale"):
        dev[k].fill_(-1.0)
    for k in ("k_tail", "v_tail"):
        dev[k].fill_(3.0)
    return dev


def _append(kvb, c, dev, k, v, new, lens, layout="htd", max_new=None):
    """Rows [L][n rows][H][d] of numpy, handed over in one of three layouts."""
    rows = [torch.from_numpy(x).bfloat16().cuda() for x in (k, v)]
    L, T, H, d = rows[0].shape
    if layout == "htd":  # the stitched cache
        rows = [x.transpose(1, 2).contiguous() for x in rows]
        strides = (H * T * d, d, T * d)
    elif layout == "thd":
        strides = (T * H * d, H * d, d)
    else:  # queries, keys and values of a projection side by side, k and v apart by strides only
        both = torch.zeros((L, T, 4 * H, d), dtype=torch.bfloat16, device="cuda")
        both[:, :, 2 * H:3 * H], both[:, :, 3 * H:] = rows[0], rows[1]
        rows = [both[:, :, 2 * H:3 * H], both[:, :, 3 * H:]]
        strides = (T * 4 * H * d, 4 * H * d, d)
    dev["lens"] = torch.from_numpy(np.array(lens, np.int32)).cuda()
    kvb.kvb_cache8_append(c.layout(kvb), L, c.n, cu(new), max_new or max(1, max(new)), rows[0], rows[1], *strides,
                          dev["table"], dev["lens"], *(dev[a] for a in ARRAYS))
    torch.cuda.synchronize()


def _feed(c, dev, steps, layout, seed, draw):
    """Appends the rows of each step (new rows per sequence); returns all rows per (layer, sequence)."""
    kvb, rng = _kvb(), np.random.default_rng(seed)
    held = [[[np.zeros((0, c.H, c.d), np.float32)] * 2 for _ in range(c.n)] for _ in range(c.L)]
    lens = np.zeros(c.n, int)
    for new in steps:
        k, v = (od.bf16(draw(rng, (c.L, sum(new), c.H, c.d))) for _ in range(2))
        lens = lens + np.array(new)
        _append(kvb, c, dev, k, v, new, lens, layout)
        first = 0
        for b, m in enumerate(new):
            for l in range(c.L):
                held[l][b] = [np.concatenate([held[l][b][0], k[l, first:first + m]]),
                              np.concatenate([held[l][b][1], v[l, first:first + m]])]
            first += m
    return held, lens


def _check_blocks(c, dev, held, lens):
    got = {k: dev[k].float().cpu().numpy() if "tail" in k else dev[k].cpu().numpy() for k in ARRAYS}
    used = set()
    for l in range(c.L):
        for b in range(c.n):
            for h in range(c.H):
                k, v = held[l][b][0][:, h], held[l][b][1][:, h]
                for j in range(lens[b] // c.B):
                    i, at = c.table[l, b, h, j], slice(j * c.B, (j + 1) * c.B)
                    used.add(int(i))
                    for x, name in ((k[at], "k"), (v[at], "v")):
                        scale, codes = od.quantise(x, c.code)
                        assert np.array_equal(got[name + "_scale"][i], scale, equal_nan=True), (name, l, b, h, j)
                        assert np.array_equal(got[name + "_codes"][i], codes if name == "k" else codes.T), (name, l, b, h, j)
                rest = lens[b] % c.B
                assert np.array_equal(got["k_tail"][l, b, h, :rest], k[lens[b] - rest:], equal_nan=True)
                assert np.array_equal(got["v_tail"][l, b, h, :, :rest], v[lens[b] - rest:].T, equal_nan=True)
    free = np.setdiff1d(np.arange(c.N), list(used))
    assert (got["k_codes"][free] == 0x55).all() and (got["v_codes"][free] == 0x55).all()
    assert (got["k_scale"][free] == -1).all() and (got["v_scale"][free] == -1).all()
    return got


NORMAL = lambda rng, s: rng.standard_normal(s)  # noqa: E731
WILD = lambda rng, s: rng.standard_normal(s) * np.exp(rng.standard_normal(s) * 8)  # noqa: E731
TINY = lambda rng, s: rng.standard_normal(s) * 2.0 ** -130  # noqa: E731  subnormal scales
HUGE = lambda rng, s: rng.standard_normal(s) * 2.0 ** 124  # noqa: E731
GRID = lambda rng, s: rng.integers(-127, 128, s) / 2.0  # noqa: E731  quotients on the borders


@pytest.mark.parametrize("code", [od.I8, od.E4M3], ids=["i8", "e4m3"])
@pytest.mark.parametrize("B", [16, 32, 64, 128])
@pytest.mark.parametrize("d", [64, 128])
def test_rows_one_by_one_and_in_runs(d, B, code):
    """Prompts of every kind of length, then single tokens across a border, then runs that
    start in a tail and end in another one, one and several blocks later."""
    c = Cache([6 * B + 40] * 5, 2, d, B, code, L=2, seed=B)
    dev = _empty(c)
    steps = [[0, 1, B - 1, B, 2 * B + 3], [1, 1, 1, 1, 1], [1, 0, 1, 0, 1], [B - 1, B, B + 1, 2 * B - 1, 3],
             [3 * B + 1, 2 * B + 7, 5, 1, B]]
    _say(f"[cache8] d {d} B {B} code {code}")
    held, lens = _feed(c, dev, steps, "htd", B + d, NORMAL)
    got = _check_blocks(c, dev, held, lens)
    assert (got["k_tail"][:, 0, :, max(x % B for x in (1, 2, B + 1, 4 * B + 2)):] == 3).all()


@pytest.mark.parametrize("layout", ["thd", "fused"])
def test_layouts_of_the_rows(layout):
    c = Cache([200] * 3, 4, 64, 32, od.I8, L=3)
    dev = _empty(c)
    held, lens = _feed(c, dev, [[33, 64, 0], [1, 1, 100]], layout, 1, NORMAL)
    _check_blocks(c, dev, held, lens)


@pytest.mark.parametrize("code", [od.I8, od.E4M3], ids=["i8", "e4m3"])
@pytest.mark.parametrize("draw", [WILD, TINY, HUGE, GRID], ids=["wild", "tiny", "huge", "grid"])
def test_values_of_every_size(draw, code):
    c = Cache([256] * 2, 2, 128, 32, code)
    dev = _empty(c)
    held, lens = _feed(c, dev, [[256, 130]], "htd", 3, draw)
    _check_blocks(c, dev, held, lens)


@pytest.mark.parametrize("code", [od.I8, od.E4M3], ids=["i8", "e4m3"])
def test_zeros_infinities_and_nan(code):
    def draw(rng, s):
        x = rng.standard_normal(s)
        x[:, :32] = 0
        x[:, 40, 0, 5], x[:, 70, 1, 7], x[:, 100, 0, 0] = np.inf, np.nan, -np.inf
        x[:, 130, 1, 1] = -0.0
        return x
    c = Cache([160], 2, 64, 32, code)
    dev = _empty(c)
    held, lens = _feed(c, dev, [[135]], "htd", 4, draw)
    got = _check_blocks(c, dev, held, lens)
    assert np.isnan(got["k_scale"][c.table[0, 0, 0, 1]]) and got["k_scale"][c.table[0, 0, 0, 0]] == 0


def test_calls_that_write_nothing():
    """No new rows, a length below the new rows, ids outside the pool, tokens past the table."""
    kvb = _kvb()
    c = Cache([64] * 4, 1, 64, 32, od.I8, extra=0)
    t = c.table.copy()
    t[0, 1, 0, 0], t[0, 2, 0, 1] = -1, c.N
    c.table = t
    dev = _empty(c)
    before = {k: dev[k].clone() for k in ARRAYS}
    k = v = od.bf16(np.random.default_rng(0).standard_normal((1, 32 + 64 + 5 + 40, 1, 64)))
    # sequence 0: none; 1: its only full block has no place; 2: length below the rows; 3: past the table
    _append(kvb, c, dev, k, v, [0, 32, 64, 45], [50, 32, 63, 2 * 32 + 32 + 45])
    for name in ARRAYS:
        assert torch.equal(before[name], dev[name]), name


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,B,code", [(64, 16, od.E4M3), (128, 128, od.I8), (128, 32, od.E4M3), (64, 64, od.I8)])
def test_read_back(d, B, code, dtype):
    kvb = _kvb()
    lens = [3 * B + 5, B, 7, 0, 2 * B - 1]
    c = Cache(lens, 2, d, B, code, L=2)
    dev = c.device()
    for back in (lens, [1, 1, 1, 0, 1], [B + 6, 3, 0, 0, B + 1]):
        T = sum(back)
        tt = torch.bfloat16 if dtype == "bf16" else torch.float32
        k, v = (torch.full((2, 2, T + 3, d), 9.0, dtype=tt, device="cuda") for _ in range(2))
        kvb.kvb_cache8_read(c.layout(kvb), 2, c.n, cu(back), max(back), dev["table"], dev["lens"],
                            *(dev[a] for a in ARRAYS), kvb.KVB_BF16 if dtype == "bf16" else kvb.KVB_F32, k, v,
                            k.stride(0), k.stride(2), k.stride(1))
        torch.cuda.synchronize()
        for got, ref in ((k.float().cpu().numpy(), c.k), (v.float().cpu().numpy(), c.v)):
            first = 0
            for b, m in enumerate(back):
                for l in range(2):
                    for h in range(2):
                        want = ref[l, b, h][lens[b] - m:].astype(np.float32)
                        assert np.array_equal(got[l, h, first:first + m], od.bf16(want) if dtype == "bf16" else want)
                first += m
            assert (got[:, :, T:] == 9).all()


def test_more_rows_than_one_grid_dimension_takes():
    """18000 rows of the table, K and V: the same new rows for every layer and head (strides 0)."""
    kvb = _kvb()
    L, n, H, d, B, T = 20, 300, 3, 64, 16, 17
    rng = np.random.default_rng(0)
    k, v = (od.bf16(rng.standard_normal((n, T, d))) for _ in range(2))
    lay = kvb.cache8_layout(L * n * H, H, d, B, kvb.KVB_I8, 1)
    table = torch.randperm(L * n * H, device="cuda").int().view(L, n, H, 1)
    new = lambda *s, dtype: torch.full(s, 7, dtype=dtype, device="cuda")  # noqa: E731
    arrays = (new(L * n * H, B, d, dtype=torch.uint8), new(L * n * H, dtype=torch.float32),
              new(L * n * H, d, B, dtype=torch.uint8), new(L * n * H, dtype=torch.float32),
              new(L, n, H, B, d, dtype=torch.bfloat16), new(L, n, H, d, B, dtype=torch.bfloat16))
    kd, vd = (torch.from_numpy(x).bfloat16().cuda() for x in (k, v))
    lens = new(n, dtype=torch.int32).fill_(T)
    _say(f"[append] {2 * L * n * H} rows of K and V")
    kvb.kvb_cache8_append(lay, L, n, cu([T] * n), T, kd, vd, 0, d, 0, table, lens, *arrays)
    out = [new(L, H, n * T, d, dtype=torch.float32) for _ in range(2)]
    kvb.kvb_cache8_read(lay, L, n, cu([T] * n), T, table, lens, *arrays, kvb.KVB_F32, *out, H * n * T * d, d, n * T * d)
    torch.cuda.synchronize()
    at = table[:, :, :, 0].long()
    for x, codes, scale, got in ((k, arrays[0], arrays[1], out[0]), (v, arrays[2].transpose(1, 2), arrays[3], out[1])):
        q = [od.quantise(x[b, :B], od.I8) for b in range(n)]
        want = torch.from_numpy(np.stack([c for _, c in q]).view(np.uint8)).cuda()
        assert torch.equal(codes[at], want[None, :, None].expand(L, n, H, B, d))
        assert torch.equal(scale[at], torch.tensor([float(s) for s, _ in q], device="cuda")[None, :, None].expand(L, n, H))
        back = np.stack([np.concatenate([od.values(c, s, od.I8).astype(np.float32), x[b, B:]]) for b, (s, c) in enumerate(q)])
        assert torch.equal(got, torch.from_numpy(back.reshape(n * T, d)).cuda().expand(L, H, n * T, d))
    assert torch.equal(arrays[4][:, :, :, 0], kd[None, :, None, B].expand(L, n, H, d))
    assert (arrays[4][:, :, :, 1:] == 7).all() and (arrays[5][..., 1:] == 7).all()


def test_read_leaves_what_it_cannot_find():
    kvb = _kvb()
    c = Cache([64, 40], 1, 64, 32, od.I8, extra=0)
    c.table[0, 0, 0, 0] = -7
    dev = c.device()
    k, v = (torch.full((1, 1, 64 + 41, 64), 9.0, device="cuda") for _ in range(2))
    kvb.kvb_cache8_read(c.layout(kvb), 1, 2, cu([64, 41]), 64, dev["table"], dev["lens"], *(dev[a] for a in ARRAYS),
                        kvb.KVB_F32, k, v, k.stride(0), k.stride(2), k.stride(1))
    for x in (k, v):
        assert (x[0, 0, :32] == 9).all() and (x[0, 0, 32:64] != 9).any() and (x[0, 0, 64:] == 9).all()


def _evict(kvb, table, lens, w, B, budget, first, recent):
    L, n, H, M = table.shape
    f = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    out = [torch.full((L, n, H, M), -9, dtype=torch.int32, device="cuda"),
           torch.full((n,), -9, dtype=torch.int32, device="cuda"), torch.full((L, n, H, M), -9.0, device="cuda")]
    lay = kvb.cache8_layout(1, H, 64, B, kvb.KVB_I8, M)
    kvb.kvb_cache8_evict(lay, L, n, budget, first, recent, f(table), f(lens), f(w), *out)
    torch.cuda.synchronize()
    return [x.cpu().numpy() for x in out]


@pytest.mark.parametrize("M,budget,first,recent", [
    (1, 0, 0, 0), (3, 1, 0, 1), (7, 3, 1, 1), (64, 20, 2, 5), (65, 64, 0, 0), (300, 100, 1, 16), (300, 17, 1, 16),
    (1025, 500, 4, 32), (3000, 1, 0, 0), (2049, 2000, 0, 1)])
def test_evict(M, budget, first, recent):
    kvb, rng = _kvb(), np.random.default_rng(M)
    L, n, H, B = 2, 6, 3, 16
    table = rng.permutation(L * n * H * M).astype(np.int32).reshape(L, n, H, M)
    nb = np.array([M, M - 1, max(0, budget), min(M, budget + 1), 0, max(1, M // 2)])
    lens = (nb * B + np.array([0, 15, 3, 0, 9, 7])).astype(np.int32)
    w = np.exp(rng.standard_normal((L, n, H, M)) * 4).astype(np.float32)
    w[:, 1] = rng.integers(0, 3, (L, H, M))            # many ties
    w[:, 5][rng.random((L, H, M)) < 0.4] = np.nan      # ranks last
    w[0, 0, 0, ::3], w[0, 0, 1, ::2], w[0, 0, 2, ::4] = 0.0, -0.0, np.inf
    w[1, 0, 0, ::3], w[1, 0, 1, ::5] = -np.inf, -1.0
    _say(f"[evict] M {M} budget {budget} first {first} recent {recent}")
    t, ln, wo = _evict(kvb, table, lens, w, B, budget, first, recent)
    assert np.array_equal(ln, lens - np.maximum(nb - budget, 0) * B)
    for l in range(L):
        for b in range(n):
            for h in range(H):
                rt, rw = od.evict(table[l, b, h], w[l, b, h], nb[b], budget, first, recent)
                assert np.array_equal(t[l, b, h], rt), (l, b, h)
                assert np.array_equal(wo[l, b, h], rw, equal_nan=True), (l, b, h)


@pytest.mark.parametrize("M,budget,first,recent", [
    (257, 100, 1, 16), (512, 511, 0, 0), (513, 64, 4, 32), (1024, 1000, 2, 1), (1025, 0, 0, 0), (2047, 700, 0, 33),
    (2048, 1, 0, 1), (2049, 300, 7, 7),
])
def test_evict_long_rows_of_many_heads(M, budget, first, recent):
    """More than 256 rows: a wave a row up to 2048 entries."""
    kvb, rng = _kvb(), np.random.default_rng(M)
    L, n, H, B = 33, 4, 2, 16
    table = rng.integers(-5, 1 << 20, (L, n, H, M)).astype(np.int32)
    nb = np.array([M, M - 1, min(M, budget + 1), M // 2])
    lens = (nb * B + np.array([0, 15, 9, 7])).astype(np.int32)
    w = np.exp(rng.standard_normal((L, n, H, M)) * 4).astype(np.float32)
    w[:, 1] = rng.integers(0, 3, (L, H, M))
    w[:, 3][rng.random((L, H, M)) < 0.3] = np.nan
    w[::2, 0, 0, ::3], w[1::2, 0, 0, ::2] = 0.0, -np.inf
    _say(f"[evict] M {M} budget {budget} rows {L * n * H}")
    t, ln, wo = _evict(kvb, table, lens, w, B, budget, first, recent)
    assert np.array_equal(ln, lens - np.maximum(nb - budget, 0) * B)
    for l in range(L):
        for b in range(n):
            for h in range(H):
                rt, rw = od.evict(table[l, b, h], w[l, b, h], nb[b], budget, first, recent)
                assert np.array_equal(t[l, b, h], rt), (l, b, h)
                assert np.array_equal(wo[l, b, h], rw, equal_nan=True), (l, b, h)


def test_evict_lengths_outside_the_table():
    kvb = _kvb()
    table = np.arange(8, dtype=np.int32).reshape(1, 2, 1, 4)
    w = np.array([3, 1, 2, 0, 5, 5, 5, 5], np.float32).reshape(1, 2, 1, 4)
    t, ln, wo = _evict(kvb, table, np.array([6 * 16 + 2, -40], np.int32), w, 16, 2, 0, 0)
    assert t[0, 0, 0].tolist() == [0, 2, 1, 3] and ln.tolist() == [6 * 16 + 2 - 32, -40]
    assert t[0, 1, 0].tolist() == [4, 5, 6, 7] and wo[0, 0, 0].tolist() == [3, 2, 0, 0]
