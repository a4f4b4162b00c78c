"""The decode operators together, as a serving program runs them: a stitched prompt is
packed into the 8-bit cache, then steps of norm + rotation, append and attention with
accumulated weights, then an eviction and further steps; and the same steps captured in
HIP graphs, replayed in turn with eager work between them."""
import sys

import numpy as np
import pytest
import torch

import kvb_workload as kw
from cache8_check import cu
from oracle import decode as od

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _say(*a):
    print(*a, file=sys.stderr, flush=True)


class Decoder:
    """The buffers a program keeps for `n` sequences of one layer."""

    def __init__(self, kvb, lens, Hq, H, d, B, code, room, seed=0):
        g = torch.Generator("cuda").manual_seed(seed)
        self.kvb, self.n, self.Hq, self.H, self.d, self.B, self.code = kvb, len(lens), Hq, H, d, B, code
        self.M = (max(lens) + room) // B + 1
        self.N = self.n * H * self.M
        self.layout = kvb.cache8_layout(self.N, H, d, B, code, self.M)
        new = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype, device="cuda")  # noqa: E731
        self.table = torch.randperm(self.N, generator=g, device="cuda").int().view(1, self.n, H, self.M)
        self.lens = torch.zeros(self.n, dtype=torch.int32, device="cuda")
        self.pos = torch.zeros(self.n, dtype=torch.int32, device="cuda")
        self.codes = [new(self.N, B * d, dtype=torch.uint8) for _ in range(2)]
        self.scales = [new(self.N) for _ in range(2)]
        self.tails = [torch.full((1, self.n, H, B * d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        self.weights = new(1, self.n, H, self.M)
        self.max_len = max(lens) + room
        self.bytes = kvb.kvb_cache8_attn_workspace_bytes(self.layout, Hq, self.n, self.n, 1, self.max_len, 1)
        self.ws = torch.full((max(16, self.bytes),), 0xFF, dtype=torch.uint8, device="cuda")
        self.q, self.out = (new(self.n, Hq, d, dtype=torch.bfloat16) for _ in range(2))
        self.k = new(self.n, H, d, dtype=torch.bfloat16)
        self.lse = new(self.n, Hq)
        self.qw, self.kw = (1 + 0.2 * torch.randn(d, generator=g, device="cuda") for _ in range(2))
        c, s = kvb.kvb_rope_scaled_table(1e6, d, kvb.rope_scaling(kvb.KVB_ROPE_INDEX, factor=4.0, original_len=32768),
                                         np.arange(8192))
        self.cos, self.sin = torch.from_numpy(c).cuda(), torch.from_numpy(s).cuda()
        self.ones = cu([1] * self.n)

    def arrays(self):
        return (self.codes[0], self.scales[0], self.codes[1], self.scales[1], self.tails[0], self.tails[1])

    def pack(self, k, v, lens):
        """The prompts' rows of the stitched cache [1][Hkv][T][d]."""
        T, d = k.shape[2], self.d
        self.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        self.pos.copy_(self.lens)
        self.kvb.kvb_cache8_append(self.layout, 1, self.n, cu(lens), max(lens), k, v, k.stride(0), d, T * d, self.table,
                                   self.lens, *self.arrays())

    def step(self, qkv):
        """One token of each sequence; qkv [n][Hq + 2 Hkv][d] of the layer's projection."""
        kvb, Hq, H, d = self.kvb, self.Hq, self.H, self.d
        row = qkv.stride(0)
        kvb.kvb_qk_norm_rope(self.n, Hq, H, d, kvb.KVB_BF16, qkv, row, d, qkv[:, Hq:], row, d, self.qw, self.kw, 1e-6,
                             self.pos, self.cos, self.sin, self.cos.shape[0], d, kvb.KVB_PAIR_HALF, self.q, Hq * d, d,
                             self.k, H * d, d)
        self.pos.add_(1)
        self.lens.add_(1)
        # K and V of one call have the same strides: the rotated keys go back beside the values
        qkv[:, Hq:Hq + H].copy_(self.k)
        kvb.kvb_cache8_append(self.layout, 1, self.n, self.ones, 1, qkv[:, Hq:], qkv[:, Hq + H:], 0, row, d, self.table,
                              self.lens, *self.arrays())
        kvb.kvb_cache8_attn(self.layout, Hq, self.n, self.ones, self.n, 1, self.max_len, self.q, self.table, self.lens,
                            *self.arrays(), d ** -0.5, self.out, self.lse, self.weights, self.weights, self.ws, self.bytes)

    def evict(self, budget, first, recent):
        out = [torch.empty_like(t) for t in (self.table, self.lens, self.weights)]
        self.kvb.kvb_cache8_evict(self.layout, 1, self.n, budget, first, recent, self.table, self.lens, self.weights, *out)
        self.table, self.lens, self.weights = out


class Model:
    """The same in the oracle: rows of each (sequence, head), full blocks as their values."""

    def __init__(self, dec, k, v, lens):
        self.d = dec
        self.k, self.v, self.w = {}, {}, {}
        start = np.concatenate([[0], np.cumsum(lens)])
        for b in range(dec.n):
            for h in range(dec.H):
                self.k[b, h], self.v[b, h] = (x[0, h, start[b]:start[b + 1]].astype(np.float64) for x in (k, v))
                self.w[b, h] = np.zeros(dec.M)
                for j in range(lens[b] // dec.B):
                    self._round(b, h, j)
        self.pos = list(lens)

    def _round(self, b, h, j):
        for x in (self.k, self.v):
            at = slice(j * self.d.B, (j + 1) * self.d.B)
            s, c = od.quantise(x[b, h][at], self.d.code)
            x[b, h][at] = od.values(c, s, self.d.code)

    def step(self, qkv):
        """Returns out and lse; the appended keys are the program's own (their rounding is tested apart)."""
        d, Hq, H, B = self.d, self.d.Hq, self.d.H, self.d.B
        G = Hq // H
        f = lambda t: t.float().cpu().numpy().astype(np.float64)  # noqa: E731
        x, q, k = f(qkv), f(d.q), f(d.k)
        out, lse, near = np.zeros((d.n, Hq, d.d)), np.zeros((d.n, Hq)), np.zeros((d.n, Hq, 1))
        for b in range(d.n):
            self.pos[b] += 1
            for h in range(H):
                self.k[b, h] = np.concatenate([self.k[b, h], k[b, h][None]])
                self.v[b, h] = np.concatenate([self.v[b, h], x[b, Hq + H + h][None]])
                T = len(self.k[b, h])
                if T % B == 0:
                    self._round(b, h, T // B - 1)
                for g in range(G):
                    hq = h * G + g
                    o, e, p = od.attention(q[b, hq][None], self.k[b, h], self.v[b, h], d.d ** -0.5)
                    out[b, hq], lse[b, hq] = o[0], e[0]
                    near[b, hq] = (p[0] @ np.abs(self.v[b, h])).max()
                    for j in range(min(d.M, T // B + 1)):
                        self.w[b, h][j] += p[0][j * B:(j + 1) * B].sum()
        return out, lse, near

    def evict(self, budget, first, recent):
        B = self.d.B
        for key in self.k:
            nb = len(self.k[key]) // B
            order = np.arange(self.d.M)
            # float weights decide, as they do in the library
            order, _ = od.evict(order.astype(np.int32), self.d.weights[0][key].cpu().numpy(), nb, budget, first, recent)
            _, self.w[key] = od.evict(order, self.w[key], 0, 0, 0, 0)[0], self.w[key][order]
            if nb > budget:
                self.w[key][self.d.M - (nb - budget):] = 0
                keep = np.concatenate([np.arange(j * B, (j + 1) * B) for j in order[:budget]] + [np.arange(nb * B, len(self.k[key]))])
                self.k[key], self.v[key] = self.k[key][keep.astype(int)], self.v[key][keep.astype(int)]


def _prompt(n, H, d, lens, seed):
    rng = np.random.default_rng(seed)
    k, v = (od.bf16(rng.standard_normal((1, H, sum(lens), d))) for _ in range(2))
    return k, v


@pytest.mark.parametrize("code", [od.I8, od.E4M3], ids=["i8", "e4m3"])
def test_pack_steps_eviction_steps(code):
    from paper_2608_21362_amd import kvb

    lens, Hq, H, d, B = [310, 64, 5, 1000], 8, 2, 128, 32
    dec = Decoder(kvb, lens, Hq, H, d, B, code, room=100)
    k, v = _prompt(4, H, d, lens, 3)
    dec.pack(*(torch.from_numpy(x).bfloat16().cuda() for x in (k, v)), lens)
    model = Model(dec, k, v, lens)
    g = torch.Generator("cuda").manual_seed(9)
    for t in range(40):
        qkv = torch.randn((4, Hq + 2 * H, d), generator=g, device="cuda").bfloat16()
        raw, pos = qkv.clone(), dec.pos.cpu().numpy()
        dec.step(qkv)
        torch.cuda.synchronize()
        # the step's queries and keys against their formula: one rounding, 2^-8, after float arithmetic
        x = raw.double().cpu().numpy()
        c, s = dec.cos.cpu().numpy()[pos], dec.sin.cpu().numpy()[pos]
        for got, part, w in ((dec.q, x[:, :Hq], dec.qw), (dec.k, x[:, Hq:Hq + H], dec.kw)):
            ref, size = od.norm_rope(part, w.cpu().numpy(), 1e-6, c, s, d, od.HALF)
            assert np.all(np.abs(got.double().cpu().numpy() - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -19 * size)
        out, lse, near = model.step(qkv)
        # the bounds of the attention's own tests: fp16 probabilities 2^-11, scores 2^-12, output 2^-8
        err = np.abs(dec.out.float().cpu().numpy() - out)
        assert np.all(err <= 2.0 ** -8 * np.abs(out) + 2.0 ** -10 * near), t
        assert np.abs(dec.lse.cpu().numpy() - lse).max() < 2.0 ** -12, t
        for b in range(4):
            for h in range(H):
                # a weight is a sum of probabilities, each within 2^-12 of itself
                w = model.w[b, h]
                assert np.all(np.abs(dec.weights[0, b, h].cpu().numpy() - w) <= 2.0 ** -11 * w + 1e-6), (t, b, h)
        if t in (17, 30):
            _say(f"[decode] step {t}: eviction, lengths {dec.lens.tolist()}")
            model.evict(8, 1, 2)
            dec.evict(8, 1, 2)
            assert dec.lens.tolist() == [len(model.k[b, 0]) for b in range(4)]


def test_a_stitched_prompt_is_packed_and_decoded():
    """The path's own cache: stitch, selection, patch, then the pack of all its layers in one call and a step
    on each layer, against the oracle over the values the pack stored."""
    from paper_2608_21362_amd import kvb, pipeline

    w = kw.WORKLOADS["tiny"]
    s = kw.structure(w)
    di = pipeline.populate(w, s)
    pb = pipeline.buffers(di)
    pipeline.run_path(di, pb)
    L, H, T, d = pb.k_cache.shape
    B = 64
    M = T // B + 1
    lay = kvb.cache8_layout(L * H * M, H, d, B, kvb.KVB_I8, M)
    table = torch.arange(L * H * M, dtype=torch.int32, device="cuda").view(L, 1, H, M)
    lens = torch.tensor([T], dtype=torch.int32, device="cuda")
    new = lambda *x, dtype=torch.uint8: torch.zeros(x, dtype=dtype, device="cuda")  # noqa: E731
    arrays = (new(lay.n_blocks, B, d), new(lay.n_blocks, dtype=torch.float32), new(lay.n_blocks, d, B),
              new(lay.n_blocks, dtype=torch.float32), new(L, 1, H, B, d, dtype=torch.bfloat16),
              new(L, 1, H, d, B, dtype=torch.bfloat16))
    kvb.kvb_cache8_append(lay, L, 1, cu([T]), T, pb.k_cache, pb.v_cache, H * T * d, d, T * d, table, lens, *arrays)
    back = [new(L, H, T, d, dtype=torch.float32) for _ in range(2)]
    kvb.kvb_cache8_read(lay, L, 1, cu([T]), T, table, lens, *arrays, kvb.KVB_F32, *back, H * T * d, d, T * d)
    torch.cuda.synchronize()
    for cache, got in ((pb.k_cache, back[0]), (pb.v_cache, back[1])):
        x = cache.view(torch.bfloat16).float().cpu().numpy() if cache.dtype != torch.bfloat16 else cache.float().cpu().numpy()
        for l in range(L):
            for h in range(H):
                for j in range(T // B):
                    sc, c = od.quantise(x[l, h, j * B:(j + 1) * B], od.I8)
                    assert np.array_equal(got[l, h, j * B:(j + 1) * B].cpu().numpy(), od.values(c, sc, od.I8).astype(np.float32))
                assert np.array_equal(got[l, h, T // B * B:].cpu().numpy(), x[l, h, T // B * B:])
    Hq = w.n_q_heads
    q = torch.randn((1, Hq, d), device="cuda").bfloat16()
    out, lse = torch.zeros_like(q), new(1, Hq, dtype=torch.float32)
    need = kvb.kvb_cache8_attn_workspace_bytes(lay, Hq, 1, 1, 1, T, 0)
    ws = new(max(16, need))
    for l in range(L):
        kvb.kvb_cache8_attn(lay, Hq, 1, cu([1]), 1, 1, T, q, table[l], lens, *arrays[:4], arrays[4][l], arrays[5][l],
                            d ** -0.5, out, lse, None, None, ws, need)
        for hq in range(Hq):
            kk, vv = (x[l, hq * H // Hq].cpu().numpy().astype(np.float64) for x in back)
            o, e, p = od.attention(q[0, hq].float().cpu().numpy()[None], kk, vv, d ** -0.5)
            near = 2.0 ** -8 * np.abs(o[0]) + 2.0 ** -10 * (p[0] @ np.abs(vv))
            assert np.all(np.abs(out[0, hq].float().cpu().numpy() - o[0]) <= near)
            assert abs(lse[0, hq].item() - e[0]) <= 2.0 ** -12 * max(1, abs(e[0]))


@pytest.mark.parametrize("code", [od.I8, od.E4M3], ids=["i8", "e4m3"])
def test_drafted_rows_are_taken_back(code):
    """Five drafted tokens, two of which are accepted: over a block's border the tails' copy comes back and the
    accepted rows are appended again; inside a block a smaller length is enough.  The same bits as without a draft."""
    from paper_2608_21362_amd import kvb

    H, d, B, lens = 2, 64, 32, [62, 94, 65, 60]  # the border is passed by all five, by the accepted two, or by none
    k, v = (torch.from_numpy(x).bfloat16().cuda() for x in _prompt(4, H, d, lens, 5))
    g = torch.Generator("cuda").manual_seed(5)
    drafted = [torch.randn((4, 5, H, d), generator=g, device="cuda").bfloat16() for _ in range(2)]

    def append(dec, n, lens):
        rows = [x[:, :n].reshape(4 * n, H, d).contiguous() for x in drafted]
        dec.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        kvb.kvb_cache8_append(dec.layout, 1, 4, cu([n] * 4), n, *rows, 0, H * d, d, dec.table, dec.lens, *dec.arrays())

    pair = [Decoder(kvb, lens, 4, H, d, B, code, room=40, seed=1) for _ in range(2)]
    for dec in pair:
        dec.pack(k, v, lens)
    held = [t.clone() for t in pair[0].tails]
    append(pair[0], 5, [n + 5 for n in lens])
    for t, was in zip(pair[0].tails, held):
        t.copy_(was)
    for dec in pair:
        append(dec, 2, [n + 2 for n in lens])
    back = []
    for dec in pair:
        T = sum(lens) + 8
        out = [torch.zeros((1, H, T, d), device="cuda") for _ in range(2)]
        kvb.kvb_cache8_read(dec.layout, 1, 4, cu([n + 2 for n in lens]), max(lens) + 2, dec.table, dec.lens, *dec.arrays(),
                            kvb.KVB_F32, *out, H * T * d, d, T * d)
        back.append(out)
    assert all(torch.equal(a, b) for a, b in zip(*back))
    # the third and the fourth sequence passed no border with the draft or with its first rows: the length is enough
    dec = Decoder(kvb, lens, 4, H, d, B, code, room=40, seed=1)
    dec.pack(k, v, lens)
    append(dec, 3, [n + 3 for n in lens])
    dec.lens.copy_(torch.tensor([n + 2 for n in lens], dtype=torch.int32))
    T = sum(lens) + 8
    out = [torch.zeros((1, H, T, d), device="cuda") for _ in range(2)]
    kvb.kvb_cache8_read(dec.layout, 1, 4, cu([n + 2 for n in lens]), max(lens) + 2, dec.table, dec.lens, *dec.arrays(),
                        kvb.KVB_F32, *out, H * T * d, d, T * d)
    inside = slice(sum(lens[:2]) + 4, T)
    assert all(torch.equal(a[:, :, inside], b[:, :, inside]) for a, b in zip(out, back[1]))


def test_captured_steps_replayed_in_turn():
    """Two captured decoders with buffers of their own, replayed in turn, each replay after eager work and a
    synchronisation, against an eager decoder fed with the same tokens: equal bits throughout."""
    from paper_2608_21362_amd import kvb

    cases = [([700, 33], 16, 2, 128, 64, od.I8), ([64, 200, 3], 4, 2, 64, 16, od.E4M3)]
    graphs = []
    for i, (lens, Hq, H, d, B, code) in enumerate(cases):
        k, v = (torch.from_numpy(x).bfloat16().cuda() for x in _prompt(len(lens), H, d, lens, i))
        pair = [Decoder(kvb, lens, Hq, H, d, B, code, room=64, seed=i) for _ in range(2)]
        for dec in pair:
            dec.pack(k, v, lens)
        qkv = torch.zeros((len(lens), Hq + 2 * H, d), dtype=torch.bfloat16, device="cuda")
        state = [t.clone() for t in (pair[0].lens, pair[0].pos, pair[0].weights, *pair[0].arrays())]
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            pair[0].step(qkv)
        for t, was in zip((pair[0].lens, pair[0].pos, pair[0].weights, *pair[0].arrays()), state):
            t.copy_(was)
        graphs.append((graph, qkv, *pair))
    g = torch.Generator("cuda").manual_seed(1)
    for t in range(20):
        for i, (graph, qkv, captured, eager) in enumerate(graphs):
            x = torch.randn(qkv.shape, generator=g, device="cuda").bfloat16()
            qkv.copy_(x)
            torch.cuda.synchronize()
            graph.replay()
            eager.step(x)
            torch.cuda.synchronize()
            for name in ("q", "k", "out", "lse", "lens", "weights"):
                assert torch.equal(getattr(captured, name), getattr(eager, name)), (i, t, name)
            for a, b in zip(captured.arrays(), eager.arrays()):
                assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), (i, t)
    del graphs
