"""An 8-bit cache built by the oracle, its device arrays, and the checks that the
tests of the cache share."""
import numpy as np
import torch

from oracle import decode as od


class Cache:
    """Layers x sequences x heads with their values; blocks get pool ids of a random permutation."""

    def __init__(self, lens, H, d, B, code, L=1, seed=0, extra=1, spread=0.0, n_blocks=None):
        rng = np.random.default_rng(seed)
        self.lens, self.H, self.d, self.B, self.code, self.L = np.array(lens), H, d, B, code, L
        n = self.n = len(lens)
        self.M = max(1, max(lens) // B + extra)
        self.N = n_blocks or L * n * H * self.M
        self.table = rng.permutation(self.N)[:L * n * H * self.M].astype(np.int32).reshape(L, n, H, self.M)
        self.k_codes = np.zeros((self.N, B, d), np.uint8)
        self.v_codes = np.zeros((self.N, d, B), np.uint8)
        self.k_scale = np.zeros(self.N, np.float32)
        self.v_scale = np.zeros(self.N, np.float32)
        # what no token wrote is not a number
        self.k_tail = np.full((L, n, H, B, d), np.nan, np.float32)
        self.v_tail = np.full((L, n, H, d, B), np.nan, np.float32)
        self.k, self.v = {}, {}  # values of each (layer, sequence, head)
        for l in range(L):
            for b, t in enumerate(lens):
                for h in range(H):
                    k, v = (od.bf16(rng.standard_normal((t, d))) for _ in range(2))
                    if spread:  # blocks of very different size
                        for j in range(t // B):
                            v[j * B:(j + 1) * B] *= np.float32(2.0 ** round(rng.uniform(-spread, spread)))
                    self.put(l, b, h, k, v)

    def put(self, l, b, h, k, v):
        """The rows of one (layer, sequence, head), into blocks and tails."""
        B, t = self.B, len(k)
        kk, vv = k.astype(np.float64), v.astype(np.float64)
        for j in range(t // B):
            at, i = slice(j * B, (j + 1) * B), self.table[l, b, h, j]
            if not 0 <= i < self.N:
                continue
            self.k_scale[i], self.k_codes[i] = od.quantise(k[at], self.code)
            self.v_scale[i], c = od.quantise(v[at], self.code)
            self.v_codes[i] = c.T
            kk[at] = od.values(self.k_codes[i], self.k_scale[i], self.code)
            vv[at] = od.values(c, self.v_scale[i], self.code)
        rest = t % B
        if rest:
            self.k_tail[l, b, h, :rest] = k[t - rest:]
            self.v_tail[l, b, h, :, :rest] = v[t - rest:].T
        self.k[l, b, h], self.v[l, b, h] = kk, vv

    def device(self):
        f = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
        return dict(table=f(self.table), lens=f(self.lens.astype(np.int32)), k_codes=f(self.k_codes),
                    k_scale=f(self.k_scale), v_codes=f(self.v_codes), v_scale=f(self.v_scale),
                    k_tail=f(self.k_tail).bfloat16(), v_tail=f(self.v_tail).bfloat16())

    def layout(self, kvb):
        return kvb.cache8_layout(self.N, self.H, self.d, self.B, self.code, self.M)


def cu(n):
    return torch.from_numpy(np.concatenate([[0], np.cumsum(n)]).astype(np.int32)).cuda()


def attend(kvb, c, dev, q, nq, weights_in=None, weights=False, max_len=None, max_q=None, scale=None, ws=None, lse=True,
           out=None):
    """One call; returns out (bfloat16 tensor), lse and weights."""
    Hq = q.shape[1]
    lay = c.layout(kvb)
    max_len = max_len or max(1, int(c.lens.max()))
    max_q = max_q or max(1, max(nq))
    out = torch.full_like(q, 7.0) if out is None else out
    lse = torch.full(q.shape[:2], 7.0, device="cuda") if lse else None
    wo = torch.full((c.n, c.H, c.M), 7.0, device="cuda") if weights else None
    need = kvb.kvb_cache8_attn_workspace_bytes(lay, Hq, c.n, q.shape[0], max_q, max_len, weights)
    if ws is None:
        ws = torch.full((max(16, need),), 0xFF, dtype=torch.uint8, device="cuda")  # NaN everywhere
    kvb.kvb_cache8_attn(lay, Hq, c.n, cu(nq), q.shape[0], max_q, max_len, q, dev["table"], dev["lens"], dev["k_codes"],
                        dev["k_scale"], dev["v_codes"], dev["v_scale"], dev["k_tail"], dev["v_tail"],
                        c.d ** -0.5 if scale is None else scale, out, lse, weights_in, wo, ws, need)
    return out, lse, wo


def check_attention(c, q, nq, out, lse, weights=None, weights_in=None, scale=None, sharp=False):
    """Against the oracle.  Bounds (u = 2^-24): a score is off by at most e = u (d + 8) sum |q k| scale, the
    product in float, and 2^-25 of the row's largest query value for each of d small query values held in fp16;
    its probability by 2 e + 2^-20 of itself, with the sums; the probability's rounding to fp16 2^-11; bfloat16
    output 2^-8.
    sharp: scores are so far apart that probabilities leave fp16's range.  A wave holds p 2^(5 .. 6) of its largest
    scale of V (S), and p S' / S as much of a block with scale S'; below 2^-14 such a number is off by up to 2^-25.
    It multiplies a code c in units of at most 2^-5 S, so a key adds at most 2^-30 |c| S, where |c| S is at most
    max |v| (int8: 127 S is the block's largest value) or 2 max |v| (e4m3: 448 S is less than twice that)."""
    scale = c.d ** -0.5 if scale is None else scale
    size = abs(scale)
    q = q.float().cpu().numpy().astype(np.float64)
    out, lse = out.float().cpu().numpy(), None if lse is None else lse.cpu().numpy()
    G = q.shape[1] // c.H
    first = 0
    share = np.zeros((c.n, c.H, c.M))
    slack = np.zeros_like(share)
    for b in range(c.n):
        rows = slice(first, first + nq[b])
        first += nq[b]
        for hq in range(q.shape[1]):
            h = hq // G
            k, v = c.k[0, b, h], c.v[0, b, h]
            o, e, p = od.attention(q[rows, hq], k, v, scale)
            qa, ka = np.abs(q[rows, hq]), np.abs(k)
            off = np.zeros(nq[b])
            if len(k) and nq[b]:
                off = 2.0 ** -24 * (c.d + 8) * size * (qa @ ka.T).max(1)
                off = off + 2.0 ** -25 * size * qa.max(1) * ka.sum(1).max()
            near = p @ np.abs(v) * (2.0 ** -11 + 2 * off + 2.0 ** -20)[:, None] + 2.0 ** -8 * np.abs(o) + 1e-30
            if sharp and len(k):
                near = near + 2.0 ** -29 * len(k) * np.abs(v).max()
            got = out[rows, hq]
            assert np.all(np.abs(got - o) <= near), (b, hq, float(np.max(np.abs(got - o) / near)))
            if lse is not None:
                seen = np.isfinite(e)
                assert np.array_equal(seen, np.isfinite(lse[rows, hq])), (b, hq)
                assert np.all(lse[rows, hq][~seen] == -np.inf)
                d = np.abs(lse[rows, hq][seen] - e[seen])
                assert np.all(d <= off[seen] + 2.0 ** -17 + 2.0 ** -21 * np.abs(e[seen])), (b, hq, d.max())
            if weights is not None:
                mass = np.zeros((len(k) // c.B + 1) * c.B)
                bound = np.zeros_like(mass)
                mass[:len(k)] = p.sum(0)
                bound[:len(k)] = (p * (2 * off + 2.0 ** -16)[:, None]).sum(0)
                m = min(c.M, len(mass) // c.B)
                share[b, h, :m] += mass.reshape(-1, c.B).sum(1)[:m]
                slack[b, h, :m] += bound.reshape(-1, c.B).sum(1)[:m]
    if weights is not None:
        base = 0 if weights_in is None else weights_in.cpu().numpy().astype(np.float64)
        d = np.abs(weights.cpu().numpy() - (base + share))
        assert np.all(d <= slack + 2.0 ** -23 * np.abs(base + share) + 1e-30), float(d.max())
    return first
