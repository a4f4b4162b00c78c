"""Timed cases of the operators that decode from a stitched prompt: what a serving
program calls once the prompt's cache is complete.

* ``rope``    norms of the queries and keys of each head and their rotation, in one
              pass from the projection's output to the queries and the key cache;
* ``append``  rows of K and V into the 8-bit cache (blocks of tokens with one scale
              for each block and head, the last block's rows in bfloat16 until it is
              full), and the same rows read back as values;
* ``attend``  attention of the last tokens of each sequence over that cache, with the
              accumulated attention weight of every block where ``weights`` is set;
* ``evict``   the blocks of least accumulated weight leave each head's table.

With ``own`` false a pass computes the operators from their formulas with elementary
torch operations in 32 bits (quotients next to a rounding border in 64); with ``own``
true it makes the calls of the library.
"""
import math

import numpy as np
import torch

own = False

THETA = 1e6
# attention shape of the 36-layer model that the benchmark uses
HEADS = dict(q_heads=16, kv_heads=2, dim=128)


def listed():
    return [
        # a decode step of 8 sequences: every layer calls this between its projection and its attention
        dict(HEADS, name="rope_step", op="rope", type="bf16", tokens=8, rot=128, pairing="half", norm=True, factor=1,
             fused=True),
        # the longest prompt's probe pass, keys into the cache layout
        dict(HEADS, name="rope_prompt", op="rope", type="bf16", tokens=32772, rot=128, pairing="half", norm=True,
             factor=1, fused=True),
        # half of each head rotated, interleaved pairs, a context stretched four times, no norms, floats
        dict(name="rope_partial", op="rope", type="f32", q_heads=8, kv_heads=8, dim=64, tokens=2047, rot=32,
             pairing="interleaved", norm=False, factor=4, fused=False),
        # one token for each sequence of a batch: most go to the tails, a few fill their block
        dict(HEADS, name="append_step", op="append", code="e4m3", block=32, layers=1, seqs=64, new=1, max_len=4096,
             ragged=70),
        # the caches of four prompts packed after their prefill, every layer
        dict(HEADS, name="append_prompts", op="append", code="i8", block=128, layers=36, seqs=4, new=0, max_len=2403,
             ragged=50),
        # one request's decode step at a common context length
        dict(HEADS, name="attend_one", op="attend", code="i8", block=64, seqs=1, queries=1, max_len=2000, ragged=0,
             weights=False),
        # a full batch of decoding sequences, uneven, with the weights that a later eviction goes by
        dict(HEADS, name="attend_batch", op="attend", code="i8", block=64, seqs=64, queries=1, max_len=8192, ragged=60,
             weights=True),
        # two very long contexts: the keys have to be split to fill the card
        dict(HEADS, name="attend_long", op="attend", code="e4m3", block=128, seqs=2, queries=1, max_len=131000,
             ragged=10, weights=False),
        # five drafted tokens of each sequence checked at once, small blocks, a small model's heads
        dict(name="attend_draft", op="attend", code="e4m3", block=16, seqs=16, queries=5, max_len=4096, ragged=50,
             weights=True, q_heads=4, kv_heads=2, dim=64),
        # the next turn of a conversation: 2048 new tokens over a 32K cache
        dict(HEADS, name="attend_turn", op="attend", code="i8", block=128, seqs=1, queries=2048, max_len=32772,
             ragged=0, weights=False),
        # one long sequence, every layer, brought back to a quarter of its blocks
        dict(name="evict_long", op="evict", layers=36, seqs=1, kv_heads=2, block=64, blocks=512, ragged=0, budget=128,
             first=1, recent=16),
        # a batch of sequences, every layer; those within the budget keep all
        dict(name="evict_batch", op="evict", layers=36, seqs=64, kv_heads=8, block=16, blocks=900, ragged=80,
             budget=300, first=2, recent=32),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "append", "attend", "attend", "attend", "evict"])
    heads = rng.choice([HEADS, HEADS, dict(q_heads=4, kv_heads=2, dim=64), dict(q_heads=32, kv_heads=4, dim=128),
                        dict(q_heads=8, kv_heads=8, dim=64), dict(q_heads=20, kv_heads=4, dim=128),
                        dict(q_heads=32, kv_heads=1, dim=128)])
    cache = dict(code=rng.choice(["i8", "e4m3"]), block=rng.choice([16, 32, 64, 128]), ragged=rng.randint(0, 90))
    if op == "rope":
        c = dict(heads, op=op, type=rng.choice(["bf16", "bf16", "f32"]), tokens=_log(rng, 1, 32772),
                 pairing=rng.choice(["half", "interleaved"]), norm=rng.random() < 0.7, factor=rng.choice([1, 2, 8]),
                 fused=rng.random() < 0.6)
        if rng.random() < 0.3:
            c["dim"] = rng.choice([80, 256])
        c["rot"] = rng.choice([c["dim"], c["dim"], 16 * rng.randint(1, c["dim"] // 16)])
    elif op == "append":
        if rng.random() < 0.5:
            c = dict(heads, **cache, op=op, layers=1, seqs=_log(rng, 1, 256), new=1, max_len=_log(rng, 1, 9000))
        else:
            c = dict(heads, **cache, op=op, layers=rng.choice([1, 12, 36]), seqs=rng.randint(1, 8), new=0,
                     max_len=_log(rng, 1, 9000))
    elif op == "attend":
        queries = rng.choice([1, 1, 1, rng.randint(2, 16), _log(rng, 17, 2048)])
        c = dict(heads, **cache, op=op, queries=queries, weights=rng.random() < 0.5,
                 seqs=_log(rng, 1, 128 if queries == 1 else 16), max_len=max(queries, _log(rng, 1, 131000)))
    else:
        blocks = _log(rng, 4, 2048)
        first, recent = rng.randint(0, 4), rng.choice([1, 8, 32])
        c = dict(op=op, layers=rng.choice([1, 12, 36]), seqs=_log(rng, 1, 64), kv_heads=heads["kv_heads"],
                 block=cache["block"], blocks=blocks, ragged=cache["ragged"], first=first, recent=recent,
                 budget=first + recent + _log(rng, 1, blocks))
    while work(c)["flops"] > 5e11 or work(c)["bytes"] > 6e8 or _spread(c) > 1.6e8:
        size = "seqs" if c.get("seqs", 1) > 1 else "tokens" if op == "rope" else "blocks" if op == "evict" else "max_len"
        c[size] = c[size] * 3 // 4
        if op == "attend":
            c["queries"] = min(c["queries"], c["max_len"])
    return c


def _spread(c):
    """Values of the cache, and scores, when every sequence is as long as the longest."""
    if "max_len" not in c:
        return 0
    n = c["seqs"] * c["max_len"]
    return max(2 * n * c["kv_heads"] * c["dim"] * c.get("layers", 1), n * c["q_heads"] * c.get("queries", 1) / 14)


def _lens(c, key="max_len"):
    """Tokens (or blocks) of each sequence: the first is the longest, the last up to `ragged` percent shorter."""
    n = c["seqs"]
    least = c.get("queries", 1)
    return [max(least, round(c[key] * (1 - c["ragged"] / 100 * b / max(1, n - 1))) - (7 * b) % 5) for b in range(n)]


def work(c):
    if c["op"] == "rope":
        size = 2 if c["type"] == "bf16" else 4
        n = c["tokens"] * (c["q_heads"] + c["kv_heads"]) * c["dim"]
        return {"bytes": 2 * n * size + c["tokens"] * c["rot"] * 4, "flops": 8 * n}
    if c["op"] == "evict":
        n = c["layers"] * c["kv_heads"] * c["seqs"] * (c["blocks"] + 2)
        return {"bytes": 16 * n, "flops": 2 * n}
    lens, H, d, B = _lens(c), c["kv_heads"], c["dim"], c["block"]
    row = 2 * H * d * c.get("layers", 1)  # values of K and V of one token
    scales = sum(n // B for n in lens) * 8 * H * c.get("layers", 1)
    if c["op"] == "append":
        if c["new"]:  # the row in and out; a block that fills is read from its tail and written as codes
            full = sum(n % B == 0 for n in lens)
            reread = sum((n - 1) % B + 1 for n in lens)
            return {"bytes": row * (len(lens) * 4 + full * B * 3 + reread * 6) + full * 8 * H, "flops": row * reread}
        n = sum(lens)
        tails = sum(n % B for n in lens)
        # in as bfloat16, out as codes or tails, back in, out as bfloat16
        return {"bytes": row * (2 * n + 2 * (n - tails) + 4 * tails + 2 * n) + 2 * scales, "flops": 4 * row * n}
    q = c["queries"]
    tails = sum(n % B for n in lens)
    seen = sum(q * n - q * (q - 1) // 2 for n in lens)
    rows = len(lens) * q * c["q_heads"]
    size = row * (sum(lens) + tails) + scales + rows * (4 * d + 4)
    if c["weights"]:
        size += 8 * H * sum(n // B + 1 for n in lens)
    return {"bytes": size, "flops": 4 * d * c["q_heads"] * seen}


# ---- inputs -----------------------------------------------------------------


def _dev(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=dtype)).cuda()


def _cu(n):
    return np.concatenate([[0], np.cumsum(n)])


def _scales(amax, code):
    """Scale of a block from its largest magnitude."""
    if code == "i8":
        return amax / 127.0
    m, e = torch.frexp(amax)  # the power of two from which on 448 steps hold amax
    e = e.long() - torch.where(m <= 0.875, 9, 8)
    s = ((e + 1023) << 52).view(torch.float64).float()  # 2^e from its bits: a power function may be an ulp off
    return torch.where(amax > 0, s, torch.zeros_like(s))


def _codes(x, scale, code):
    """Codes of x [..., n, m] with one scale for the last two dimensions; the quotient in 64 bits."""
    s = scale[..., None, None].double()
    t = torch.where(s > 0, x.double() / torch.where(s > 0, s, torch.ones_like(s)), torch.zeros_like(s))
    if code == "i8":
        return torch.round(t).clamp(-127, 127).to(torch.int8)
    return t.float().to(torch.float8_e4m3fn)


def _bytes(codes):
    return codes.view(torch.uint8)


def _numbers(codes, code):
    return codes.view(torch.int8 if code == "i8" else torch.float8_e4m3fn).float()


def prepare(case, seed):
    c = case
    g = torch.Generator("cuda").manual_seed(int(seed) & 0x7FFFFFFF)
    rng = np.random.default_rng([int(seed) & 0x7FFFFFFF, 2])
    normal = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    uniform = lambda *s: torch.rand(s, generator=g, device="cuda")  # noqa: E731
    empty = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype, device="cuda")  # noqa: E731
    s = {"case": c}
    if c["op"] == "rope":
        T, Hq, H, d, rot = c["tokens"], c["q_heads"], c["kv_heads"], c["dim"], c["rot"]
        dtype = torch.bfloat16 if c["type"] == "bf16" else torch.float32
        if c["fused"]:  # the queries, keys and values of a token side by side, as one projection leaves them
            x = normal(T, Hq + 2 * H, d).to(dtype)
            s["q"], s["k"] = x[:, :Hq], x[:, Hq:Hq + H]
        else:
            s["q"], s["k"] = normal(T, Hq, d).to(dtype), normal(T, H, d).to(dtype)
        s["q_weight"], s["k_weight"] = (1 + 0.3 * normal(d), 1 + 0.3 * normal(d)) if c["norm"] else (None, None)
        n = max(T, 32768)
        w = THETA ** (-2.0 * np.arange(rot // 2) / rot) / c["factor"]
        a = np.arange(n, dtype=np.float64)[:, None] * w
        s["cos"], s["sin"], s["table_len"] = _dev(np.cos(a), np.float32), _dev(np.sin(a), np.float32), n
        s["pos"] = _dev(np.arange(T) if T > 256 else rng.integers(0, n, T), np.int32)
        s["q_out"], s["k_out"] = empty(T, Hq, d, dtype=dtype), empty(H, T, d, dtype=dtype)
        return s
    H, B, n = c["kv_heads"], c["block"], c["seqs"]
    L = c.get("layers", 1)
    if c["op"] == "evict":
        nb = np.array(_lens(c, "blocks"))
        M = c["blocks"] + 2  # the tail's block and one more are assigned
        s["M"] = M
        s["table"] = torch.randperm(L * n * H * M, generator=g, device="cuda").int().view(L, n, H, M)
        s["lens"] = _dev(nb * B + rng.integers(0, B, n), np.int32)
        # a few blocks have most of the weight; a part was never looked at
        w = torch.exp(4 * normal(L, n, H, M)) * (uniform(L, n, H, M) < 0.8)
        s["weights"] = w * (torch.arange(M, device="cuda") <= _dev(nb, np.int64)[:, None, None])
        s["table_out"], s["lens_out"], s["weights_out"] = (torch.zeros_like(s[k]) for k in ("table", "lens", "weights"))
        return s
    d, code = c["dim"], c["code"]
    lens = np.array(_lens(c))
    M = -(-int(lens.max()) // B)
    N = L * n * H * M
    s["lens"], s["M"], s["N"], s["max_len"] = _dev(lens, np.int32), M, N, int(lens.max())
    table = torch.randperm(N, generator=g, device="cuda").int()
    s["table"] = table.view(L, n, H, M)
    ch = torch.exp(uniform(2, d) * 1.4 - 0.7)  # some channels are larger than others
    s["k_tail"] = (normal(L, n, H, B, d) * ch[0]).bfloat16()
    s["v_tail"] = (normal(L, n, H, d, B) * ch[1][:, None]).bfloat16()
    if c["op"] == "append":
        new = np.full(n, c["new"]) if c["new"] else lens
        back = (lens - 1) % B + 1 if c["new"] else lens  # the rows that are read back
        T = int(new.sum())
        s["cu_new"], s["max_new"], s["T"] = _dev(_cu(new), np.int32), int(new.max()), T
        s["cu_back"], s["max_back"], s["R"] = _dev(_cu(back), np.int32), int(back.max()), int(back.sum())
        s["k"], s["v"] = ((normal(L, H, T, d) * ch[i]).bfloat16() for i in (0, 1))
        s["k_codes"], s["v_codes"] = empty(N, B, d, dtype=torch.uint8), empty(N, d, B, dtype=torch.uint8)
        s["k_scale"], s["v_scale"] = empty(N, dtype=torch.float32), empty(N, dtype=torch.float32)
        s["out_type"] = torch.float32 if c["new"] else torch.bfloat16
        s["k_out"], s["v_out"] = (empty(L, H, s["R"], d, dtype=s["out_type"]) for _ in range(2))
        return s
    for name, shape, scale in (("k", (N, B, d), ch[0]), ("v", (N, d, B), ch[1][:, None])):
        x = normal(*shape) * scale * torch.exp(0.3 * normal(N, 1, 1))  # blocks differ in size too
        s[name + "_scale"] = _scales(x.abs().amax((1, 2)), code)
        s[name + "_codes"] = _bytes(_codes(x, s[name + "_scale"], code))
        del x
    q = np.full(n, c["queries"])
    Q = int(q.sum())
    s["cu_q"], s["Q"] = _dev(_cu(q), np.int32), Q
    s["q"] = (1.3 * normal(Q, c["q_heads"], d)).bfloat16()
    s["out"], s["lse"] = empty(Q, c["q_heads"], d), empty(Q, c["q_heads"], dtype=torch.float32)
    if c["weights"]:
        s["weights"] = torch.exp(2 * normal(n, H, M))
        s["weights_out"] = torch.zeros_like(s["weights"])
    return s


# ---- the plain forms ----------------------------------------------------------


def _plain_rope(s):
    c = s["case"]
    h, dtype = c["rot"] // 2, s["q"].dtype
    cos, sin = (s[k][s["pos"].long()][:, None] for k in ("cos", "sin"))

    def turn(x, w):
        x = x.float()
        if w is not None:
            x = x * (1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6)) * w
        r, rest = x[..., :2 * h], x[..., 2 * h:]
        a, b = (r[..., :h], r[..., h:]) if c["pairing"] == "half" else (r[..., 0::2], r[..., 1::2])
        y = (a * cos - b * sin, b * cos + a * sin)
        y = torch.cat(y, -1) if c["pairing"] == "half" else torch.stack(y, -1).flatten(-2)
        return torch.cat([y, rest], -1).to(dtype)

    return {"q": turn(s["q"], s["q_weight"]), "k": turn(s["k"], s["k_weight"]).transpose(0, 1).contiguous()}


def _plain_append(s):
    c = s["case"]
    L, H, B, d, n = c["layers"], c["kv_heads"], c["block"], c["dim"], c["seqs"]
    lens, cu = s["lens"].long(), s["cu_new"].long()
    before = lens - (cu[1:] - cu[:-1])
    first = before // B  # the first block that changes
    X = s["M"] if not c["new"] else 1  # blocks that can change
    at = first[:, None] * B + torch.arange(X * B, device="cuda")  # [n, X * B] tokens
    is_new, is_old = (at >= before[:, None]) & (at < lens[:, None]), at < before[:, None]
    row = torch.where(is_new, cu[:-1, None] + at - before[:, None], torch.zeros_like(at))
    full = (first[:, None] + torch.arange(X, device="cuda") + 1) * B <= lens[:, None]  # [n, X]
    block = (first[:, None] + torch.arange(X, device="cuda")).clamp(max=s["M"] - 1)
    ids = s["table"].long().gather(3, block[None, :, None].expand(L, n, H, X))[full[None, :, None].expand(L, n, H, X)]
    # where each token of a partial block goes in the tails, and where the rows that are read back come from
    seq, col = torch.nonzero(is_new & ~full.repeat_interleave(B, 1), as_tuple=True)
    cb = s["cu_back"].long()
    of = torch.repeat_interleave(torch.arange(n, device="cuda"), cb[1:] - cb[:-1], output_size=s["R"])
    token = lens[of] - (cb[1:][of] - torch.arange(s["R"], device="cuda"))
    out = {}
    for name in ("k", "v"):
        x = s[name][:, :, row].permute(0, 2, 1, 3, 4).float()  # [L, n, H, X * B, d]
        tail = s[name + "_tail"] if name == "k" else s["v_tail"].transpose(3, 4)
        old = tail.float().gather(3, (at % B)[None, :, None, :, None].expand(L, n, H, X * B, d))
        x = torch.where(is_old[None, :, None, :, None], old, x)
        blocks = x.view(L, n, H, X, B, d)
        scale = _scales(blocks.abs().amax((4, 5)), c["code"])
        codes = _codes(blocks, scale, c["code"])
        values = codes.float() * scale[..., None, None]
        take = codes[full[None, :, None].expand(L, n, H, X)]
        s[name + "_codes"][ids] = _bytes(take if name == "k" else take.transpose(1, 2).contiguous())
        s[name + "_scale"][ids] = scale[full[None, :, None].expand(L, n, H, X)]
        tail[:, seq, :, at[seq, col] % B] = x[:, seq, :, col].bfloat16()
        values = torch.where(full[None, :, None, :, None, None], values, blocks).flatten(3, 4)
        out[name] = values[:, of, :, token - first[of] * B].permute(1, 2, 0, 3).contiguous().to(s["out_type"])
        out[name + "_scale"], out[name + "_tail"] = s[name + "_scale"], s[name + "_tail"]
    return out


def _plain_attend(s):
    c = s["case"]
    H, B, d, n, M, code = c["kv_heads"], c["block"], c["dim"], c["seqs"], s["M"], c["code"]
    G, nq = c["q_heads"] // H, c["queries"]
    table, lens, every = s["table"][0].long(), s["lens"].long(), torch.arange(n, device="cuda")
    last = (lens // B).clamp(max=M)

    def rows(name):
        x = torch.zeros((n, H, M + 1, B, d), device="cuda")
        v = _numbers(s[name + "_codes"][table], code) * s[name + "_scale"][table][..., None, None]
        x[:, :, :M] = v if name == "k" else v.transpose(3, 4)
        x[every, :, last] = (s["k_tail"][0] if name == "k" else s["v_tail"][0].transpose(2, 3)).float()
        return x.flatten(2, 3)

    q = s["q"].float().view(n, nq, H, G, d).transpose(1, 2).reshape(n, H, nq * G, d)
    score = torch.matmul(q, rows("k").transpose(2, 3)) * d ** -0.5
    ends = lens[:, None] - nq + 1 + torch.arange(nq, device="cuda")  # [n, nq]
    seen = torch.arange((M + 1) * B, device="cuda") < ends.repeat_interleave(G, 1)[:, None, :, None]
    score = torch.where(seen, score, torch.full_like(score[:1, :1, :1, :1], -math.inf))
    del seen
    top = score.amax(-1, keepdim=True)
    score = score.sub_(top).exp_()
    total = score.sum(-1, keepdim=True)
    back = lambda x: x.view(n, H, nq, G, -1).transpose(1, 2).reshape(n * nq, H * G, -1)  # noqa: E731
    out = {"out": back(torch.matmul(score, rows("v")) / total).bfloat16(), "lse": back(top + torch.log(total))[..., 0]}
    if c["weights"]:
        share = (score / total).sum(2).view(n, H, M + 1, B).sum(-1)
        out["weights"] = s["weights"] + share[:, :, :M]
    return out


def _plain_evict(s):
    c = s["case"]
    M, B, budget = s["M"], c["block"], c["budget"]
    nb = s["lens"].long() // B
    i, end = torch.arange(M, device="cuda"), nb[:, None, None]
    w = s["weights"]
    w = torch.where(i >= end, torch.full_like(w, -math.inf), w)
    w = torch.where(((i < c["first"]) | (i >= end - c["recent"])) & (i < end), torch.full_like(w, math.inf), w)
    order = torch.argsort(w, dim=-1, descending=True, stable=True)
    rank = torch.empty_like(order).scatter_(-1, order, i.expand_as(order).contiguous())
    dropped = (i < end) & (end > budget) & (rank >= budget)
    kind = torch.where(dropped, 2, torch.where(i < end, 0, 1))  # kept, not yet full, dropped
    order = torch.argsort(kind, dim=-1, stable=True)
    return {"table": s["table"].gather(-1, order), "lens": (s["lens"] - (nb - budget).clamp(min=0) * B).int(),
            "weights": torch.where(dropped, torch.zeros_like(w), s["weights"]).gather(-1, order)}


# ---- the library's calls --------------------------------------------------------


def _own(s):
    from paper_2608_21362_amd import kvb

    c = s["case"]
    op, H = c["op"], c["kv_heads"]
    if op == "rope":
        q, k, qo, ko = s["q"], s["k"], s["q_out"], s["k_out"]
        kvb.kvb_qk_norm_rope(
            c["tokens"], c["q_heads"], H, c["dim"], kvb.KVB_BF16 if c["type"] == "bf16" else kvb.KVB_F32, q, q.stride(0),
            q.stride(1), k, k.stride(0), k.stride(1), s["q_weight"], s["k_weight"], 1e-6, s["pos"], s["cos"], s["sin"],
            s["table_len"], c["rot"], kvb.KVB_PAIR_HALF if c["pairing"] == "half" else kvb.KVB_PAIR_INTERLEAVED, qo,
            qo.stride(0), qo.stride(1), ko, ko.stride(1), ko.stride(0))
        return {"q": qo, "k": ko}
    if "layout" not in s:  # a program describes its cache once
        code = kvb.KVB_E4M3 if c.get("code") == "e4m3" else kvb.KVB_I8
        N = s.get("N", s["table"].numel())
        s["layout"] = kvb.cache8_layout(N, H, c.get("dim", 128), c["block"], code, s["M"])
    lay, n = s["layout"], c["seqs"]
    if op == "evict":
        kvb.kvb_cache8_evict(lay, c["layers"], n, c["budget"], c["first"], c["recent"], s["table"], s["lens"],
                             s["weights"], s["table_out"], s["lens_out"], s["weights_out"])
        return {"table": s["table_out"], "lens": s["lens_out"], "weights": s["weights_out"]}
    cache = [s[k] for k in ("table", "lens", "k_codes", "k_scale", "v_codes", "v_scale", "k_tail", "v_tail")]
    if op == "append":
        k, ko = s["k"], s["k_out"]
        kvb.kvb_cache8_append(lay, c["layers"], n, s["cu_new"], s["max_new"], k, s["v"], k.stride(0), k.stride(2),
                              k.stride(1), *cache)
        kvb.kvb_cache8_read(lay, c["layers"], n, s["cu_back"], s["max_back"], *cache,
                            kvb.KVB_BF16 if s["out_type"] == torch.bfloat16 else kvb.KVB_F32, ko, s["v_out"],
                            ko.stride(0), ko.stride(2), ko.stride(1))
        return {"k": ko, "v": s["v_out"], **{k: s[k] for k in ("k_scale", "k_tail", "v_scale", "v_tail")}}
    if "workspace" not in s:
        s["bytes"] = kvb.kvb_cache8_attn_workspace_bytes(lay, c["q_heads"], n, s["Q"], c["queries"], s["max_len"],
                                                         c["weights"])
        s["workspace"] = torch.empty(max(16, s["bytes"]), dtype=torch.uint8, device="cuda")
    kvb.kvb_cache8_attn(lay, c["q_heads"], n, s["cu_q"], s["Q"], c["queries"], s["max_len"], s["q"], *cache,
                        c["dim"] ** -0.5, s["out"], s["lse"], s.get("weights"), s.get("weights_out"), s["workspace"],
                        s["bytes"])
    out = {"out": s["out"], "lse": s["lse"]}
    if c["weights"]:
        out["weights"] = s["weights_out"]
    return out


def run(s):
    if own:
        return _own(s)
    return {"rope": _plain_rope, "append": _plain_append, "attend": _plain_attend, "evict": _plain_evict}[
        s["case"]["op"]](s)


# ---- the definitions in 64 bits ---------------------------------------------------


def _exact_rope(s):
    c, out = s["case"], {}
    rot, pos = c["rot"], s["pos"].long()
    lo = torch.arange(rot // 2, device="cuda")
    a, b = (lo, lo + rot // 2) if c["pairing"] == "half" else (2 * lo, 2 * lo + 1)
    for name in ("q", "k"):
        x = s[name].double()
        if c["norm"]:
            x = x / (x.square().sum(-1, keepdim=True) / c["dim"] + 1e-6).sqrt() * s[name + "_weight"].double()
        z = torch.view_as_complex(torch.stack([x[..., a], x[..., b]], -1))
        z = z * torch.view_as_complex(torch.stack([s["cos"][pos].double(), s["sin"][pos].double()], -1))[:, None]
        x = x.clone()
        x[..., a], x[..., b] = z.real, z.imag
        out[name] = x if name == "q" else x.permute(1, 0, 2)
    return out


def _exact_quantise(x, code):
    """Scale and stored values of one block (or a stack of them, the first dimension) in 64 bits."""
    top = x.abs().flatten(1).amax(1)
    if code == "i8":
        scale = (top.float() / 127.0).double()  # the scale is held as a float
        safe = torch.where(scale > 0, scale, torch.ones_like(scale)).view(-1, 1, 1)
        t = x / safe
        whole = torch.floor(t)
        rest = t - whole
        whole = whole + ((rest > 0.5) | ((rest == 0.5) & (whole % 2 != 0)))
        return scale, whole.clamp(-127, 127) * scale.view(-1, 1, 1)
    ratio = torch.where(top > 0, top, torch.ones_like(top)) / 448.0
    m, _ = torch.frexp(ratio)
    scale = torch.where(m > 0.5, ratio / m, ratio)  # m in [0.5, 1): ratio / m is a power of two
    t = x / scale.view(-1, 1, 1)
    m, _ = torch.frexp(t)
    small = t.abs() < 2.0 ** -6
    step = torch.where(small, 2.0 ** -9, (t / torch.where(small, 1.0, m)).abs() / 16)
    return torch.where(top > 0, scale, 0.0), torch.round(t / step) * step * scale.view(-1, 1, 1)


def _exact_append(s):
    c = s["case"]
    L, H, B, d, n = c["layers"], c["kv_heads"], c["block"], c["dim"], c["seqs"]
    lens, cu, cb = s["lens"].tolist(), s["cu_new"].tolist(), s["cu_back"].tolist()
    table = s["table"].long()
    out = {"k_tail": s["k_tail"].double(), "v_tail": s["v_tail"].double()}
    for name in ("k", "v"):
        tail = out[name + "_tail"] if name == "k" else out["v_tail"].transpose(3, 4)
        scales = torch.zeros(s["N"], dtype=torch.float64, device="cuda")
        read = torch.zeros((L, H, s["R"], d), dtype=torch.float64, device="cuda")
        for b in range(n):
            before = lens[b] - (cu[b + 1] - cu[b])
            start = before // B * B
            x = torch.cat([tail[:, b, :, :before - start], s[name][:, :, cu[b]:cu[b + 1]].double()], 2)
            held = x.clone()
            done = x.shape[2] // B
            if done:
                q, v = _exact_quantise(x[:, :, :done * B].reshape(L * H * done, B, d), c["code"])
                held[:, :, :done * B] = v.view(L, H, done * B, d)
                scales[table[:, b, :, start // B:start // B + done].reshape(-1)] = q
            left = x.shape[2] - done * B
            if left:
                tail[:, b, :, :left] = x[:, :, done * B:]
            m = cb[b + 1] - cb[b]
            read[:, :, cb[b]:cb[b + 1]] = held[:, :, held.shape[2] - m:]
        out[name], out[name + "_scale"] = read, scales
    return out


def _exact_attend(s):
    c = s["case"]
    H, B, d, n, code, nq = c["kv_heads"], c["block"], c["dim"], c["seqs"], c["code"], c["queries"]
    G = c["q_heads"] // H
    out = torch.zeros((n, nq, H, G, d), dtype=torch.float64, device="cuda")
    lse = torch.zeros((n, nq, H, G), dtype=torch.float64, device="cuda")
    weights = s["weights"].double().clone() if c["weights"] else None
    number = lambda x: x.view(torch.int8 if code == "i8" else torch.float8_e4m3fn).double()  # noqa: E731
    q = s["q"].double().view(n, nq, H, G, d)
    for b, size in enumerate(s["lens"].tolist()):
        nb, rest = size // B, size % B
        for h in range(H):
            ids = s["table"][0, b, h, :nb].long()
            k = number(s["k_codes"][ids]) * s["k_scale"][ids].double().view(-1, 1, 1)
            v = number(s["v_codes"][ids]) * s["v_scale"][ids].double().view(-1, 1, 1)
            k = torch.cat([k.reshape(-1, d), s["k_tail"][0, b, h, :rest].double()])
            v = torch.cat([v.transpose(1, 2).reshape(-1, d), s["v_tail"][0, b, h, :, :rest].double().T])
            for g in range(G):
                z = q[b, :, h, g] @ k.T / math.sqrt(d)
                late = torch.arange(size, device="cuda") > torch.arange(size - nq, size, device="cuda")[:, None]
                z[late] = -math.inf
                total = torch.logsumexp(z, -1)
                p = torch.exp(z - total[:, None])
                out[b, :, h, g], lse[b, :, h, g] = p @ v, total
                if c["weights"]:
                    mass = torch.zeros((nb + 1) * B, dtype=torch.float64, device="cuda")
                    mass[:size] = p.sum(0)
                    weights[b, h, :nb + 1] += mass.view(-1, B).sum(1)[:s["M"]]
    got = {"out": out.view(n * nq, H * G, d), "lse": lse.view(n * nq, H * G)}
    if c["weights"]:
        got["weights"] = weights
    return got


def _exact_evict(s):
    c = s["case"]
    table, w, lens = s["table"].cpu().numpy(), s["weights"].cpu().numpy().astype(np.float64), s["lens"].cpu().numpy()
    to, wo, lo = table.copy(), w.copy(), lens.copy()
    budget, B = c["budget"], c["block"]
    for b in range(c["seqs"]):
        nb = int(lens[b]) // B
        if nb <= budget:
            continue
        lo[b] = lens[b] - (nb - budget) * B
        middle = np.arange(c["first"], nb - c["recent"])
        for l in range(c["layers"]):
            for h in range(c["kv_heads"]):
                best = middle[np.lexsort((middle, -w[l, b, h, middle]))][:budget - c["first"] - c["recent"]]
                keep = np.zeros(nb, bool)
                keep[:c["first"]] = keep[nb - c["recent"]:] = True
                keep[best] = True
                kept, gone = np.nonzero(keep)[0], np.nonzero(~keep)[0]
                order = np.concatenate([kept, np.arange(nb, s["M"]), gone])
                to[l, b, h], wo[l, b, h] = table[l, b, h, order], w[l, b, h, order]
                wo[l, b, h, s["M"] - len(gone):] = 0
    return {"table": torch.from_numpy(to), "lens": torch.from_numpy(lo), "weights": torch.from_numpy(wo)}


def exact(case, seed):
    s = prepare(case, seed)
    return {"rope": _exact_rope, "append": _exact_append, "attend": _exact_attend, "evict": _exact_evict}[
        case["op"]](s)
