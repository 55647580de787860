"""The paged MXFP4 cache in plain 64-bit arithmetic on the CPU, and caches filled by hand for its tests.

Whatever no token lies in is filled with random codes under scale byte 255 (NaN), and table entries behind a sequence's
pages name pages that do not exist, so that a read past a sequence's end shows in the results."""
import numpy as np
import torch

import oracle
from paper_2503_13565_amd import synth

GRID = np.array([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6])


def values(q, s):
    """uint8 [..., dim/2], [..., dim/32] -> float64 [..., dim]."""
    q, s = np.asarray(q), np.asarray(s)
    x = np.stack([GRID[q & 15], GRID[q >> 4]], axis=-1).reshape(*q.shape[:-1], 2 * q.shape[-1])
    f = np.where(s == 255, np.nan, 2.0 ** (s.astype(np.float64) - 127))
    return x * np.repeat(f, 32, axis=-1)


def cast(x):
    """BF16 tensor [..., dim] -> (codes, scale bytes) by the oracle."""
    q, s = oracle.direct_cast(synth.to_bits(x.reshape(-1, x.shape[-1]).contiguous()))
    return q.reshape(*x.shape[:-1], -1), s.reshape(*x.shape[:-1], -1)


def tokens(gen, n, heads, dim, large=4.0):
    x = torch.randn((n, heads, dim), generator=gen)
    x[..., ::13] *= large
    return x.to(torch.bfloat16)


class Paged:
    """Sequences of `lens` tokens in pages dealt out in a random order, keys and values on the host beside them."""

    def __init__(self, lens, heads, page, dim, seed=0, spare=3, room=0):
        gen = torch.Generator().manual_seed(seed)
        rng = np.random.RandomState(seed)
        self.lens, self.heads, self.page, self.dim = list(lens), heads, page, dim
        need = [-(-(n + room) // page) for n in lens]
        self.width = max(max(need), 1) + 1
        self.pages = sum(need) + spare
        order = rng.permutation(self.pages)
        self.table = np.full((len(lens), self.width), 1 << 30, dtype=np.int32)
        self.kq, self.vq = (rng.randint(0, 256, (self.pages, heads, page, dim // 2)).astype(np.uint8) for _ in range(2))
        self.ks, self.vs = (np.full((self.pages, heads, page, dim // 32), 255, dtype=np.uint8) for _ in range(2))
        self.k, self.v, at = [], [], 0
        for b, n in enumerate(lens):
            self.table[b, : need[b]] = order[at: at + need[b]]
            at += need[b]
            k, v = tokens(gen, n, heads, dim), tokens(gen, n, heads, dim, 1.0)
            mine = []
            for x, code, scale in ((k, self.kq, self.ks), (v, self.vq, self.vs)):
                q, s = cast(x) if n else (np.zeros((0, heads, dim // 2), np.uint8), np.zeros((0, heads, dim // 32), np.uint8))
                p, o = self.table[b, np.arange(n) // page], np.arange(n) % page
                code[p, :, o], scale[p, :, o] = q, s
                mine.append(values(q, s))
            self.k.append(mine[0])
            self.v.append(mine[1])

    def cache(self, device):
        from paper_2503_13565_amd import binding
        return binding.KvCache(*(torch.from_numpy(x).to(device) for x in (self.kq, self.ks, self.vq, self.vs)))

    def batch(self, device):
        return torch.from_numpy(self.table).to(device), torch.tensor(self.lens, dtype=torch.int32, device=device)

    def sees(self, b, n, causal=True, window=0, tree=None):
        """[n, lens[b]]: what each of the last n tokens sees; tree: their words."""
        length = self.lens[b]
        j = np.arange(length)[None]
        p = (length - n + np.arange(n))[:, None]
        ok = (j <= p) if causal and tree is None else np.ones((n, length), bool)
        if window:
            ok &= j > p - window
        if tree is not None:
            node = j - (length - n)
            for i in range(n):
                bits = np.array([m < 0 or (m < 64 and (tree[i] >> m) & 1 == 1) for m in node[0].tolist()], dtype=bool)
                ok[i] &= bits
        return ok


def attention(q, k, v, sees, scale):
    """q float64 [n, hq, d], k, v [len, hkv, d], sees [n, len] -> (out, lse, sum of weight x |v|, the largest error
    of a score in FP32): the weights' own errors and the sums' are bounded by these."""
    n, hq, d = q.shape
    group = hq // k.shape[1] if k.shape[1] else 1
    out, room = np.zeros((n, hq, d)), np.zeros((n, hq, d))
    lse, off = np.full((n, hq), -np.inf), np.zeros((n, hq))
    for h in range(hq):
        kk, vv = k[:, h // group], v[:, h // group]
        z = scale * (q[:, h] @ kk.T)
        za = scale * (np.abs(q[:, h]) @ np.abs(kk).T)
        for i in range(n):
            s = sees[i]
            if not s.any():
                continue
            top = z[i, s].max()
            w = np.exp(z[i, s] - top)
            lse[i, h] = top + np.log(w.sum())
            w = w / w.sum()
            out[i, h], room[i, h] = w @ vv[s], w @ np.abs(vv[s])
            off[i, h] = (d + 2) * 2.0 ** -24 * za[i, s].max()
    return out, lse, room, off


def tolerance(out, room, off, length):
    """BF16 weights: half a step, 2^-8 of each, so 2^-8 of the sum of weight x |v|; scores off by `off` change a weight by that
    share, numerator and denominator; the exponential and its argument are good to 2^-21 for arguments up to 2^2 in
    FP32 rounding, so 2^-20 each covers arguments to 2^4 where weights count; FP32 sums of `length` terms; then the result's own
    rounding, half a step."""
    share = 2.0 ** -8 + 2 * off[..., None] + 4 * 2.0 ** -20 + 2 * length * 2.0 ** -24
    return room * share + (np.abs(out) + room * share) * 2.0 ** -8 + 2.0 ** -133
