"""A plain 64-bit model of the 8-bit paged cache and of attention over it, on
the CPU, token by token from the definition; and batches of sequences."""
import math
import random

import torch

LEAST, MOST = 2.0 ** -32, 2.0 ** 60


def quantise(x):
    """(integers, fp32 scale) of one block and head: x [tokens, dim] of unrounded values."""
    a = float(x.double().abs().max()) if not torch.isnan(x).any() else math.nan
    if not a <= MOST:
        return torch.zeros(x.shape, dtype=torch.float64), math.nan
    s = float(torch.tensor(max(a, LEAST), dtype=torch.float32) * torch.tensor(1 / 127, dtype=torch.float32))
    q = torch.round(x.double() / s)  # ties to even; a quotient of an 11-bit by a 24-bit number is exact enough in 53
    return q.clamp(-127, 127), s


class Model:
    """Unrounded keys and values of each slot; what the cache holds follows from them."""

    def __init__(self, n_slots, heads, block, dim):
        self.block, self.heads, self.dim = block, heads, dim
        self.k = [torch.zeros(0, heads, dim) for _ in range(n_slots)]
        self.v = [torch.zeros(0, heads, dim) for _ in range(n_slots)]

    def append(self, slot, k, v):
        self.k[slot] = torch.cat([self.k[slot], k.float().cpu()])
        self.v[slot] = torch.cat([self.v[slot], v.float().cpu()])

    def held(self, which, slot, length=None):
        """fp64 values [tokens, heads, dim] that the cache stands for."""
        x = (self.k if which == "k" else self.v)[slot][:length]
        out = torch.zeros(x.shape, dtype=torch.float64)
        for b in range(0, len(x), self.block):
            for h in range(self.heads):
                q, s = quantise(x[b:b + self.block, h])
                out[b:b + self.block, h] = q * s
        return out


def attend(k, v, q, pos, scale, window, sinks):
    """(out, sum p |v|) in fp64 for queries [c, heads, dim] at positions pos over held k, v [tokens, kv heads, dim]."""
    c, heads, dim = q.shape
    g = heads // k.shape[1]
    out = torch.zeros(c, heads, dim, dtype=torch.float64)
    mag = torch.zeros(c, heads, dim, dtype=torch.float64)
    for i in range(c):
        keys = [j for j in range(pos[i] + 1) if window == 0 or j > pos[i] - window or j < sinks]
        kk, vv = k[keys], v[keys]
        for h in range(heads):
            y = kk[:, h // g] @ q[i, h].double() * scale
            p = torch.softmax(y, 0)
            out[i, h] = p @ vv[:, h // g]
            mag[i, h] = p @ vv[:, h // g].abs()
    return out, mag


class Batch:
    """Sequences in shuffled slots with shuffled blocks of a pool, on the GPU."""

    def __init__(self, tsd, lens, heads, block, dim, dtype=torch.bfloat16, seed=0, spare_slots=1, spare_width=1):
        r = random.Random(seed)
        self.n, self.heads, self.block, self.dim, self.dtype = len(lens), heads, block, dim, dtype
        n_slots = self.n + spare_slots
        width = max(1, max(-(-x // block) for x in lens)) + spare_width
        total = sum(-(-x // block) for x in lens)
        ids = list(range(total + 3))
        r.shuffle(ids)
        self.slots = r.sample(range(n_slots), self.n)
        table = torch.full((n_slots, width), -1, dtype=torch.int32)
        for i, x in enumerate(lens):
            for b in range(-(-x // block)):
                table[self.slots[i], b] = ids.pop()
        self.table = table.cuda()
        self.cache = tsd.KV8Cache.empty(total + 3, n_slots, heads, dim, block=block, dtype=dtype)
        self.cache.k.random_(-128, 128)  # blocks hold whatever was there before
        self.cache.v.random_(-128, 128)
        self.model = Model(n_slots, heads, block, dim)
        self.len = [0] * self.n
        self.g = torch.Generator().manual_seed(seed)

    def rows(self, n, heads, spread=1.0):
        return (torch.randn(n, heads, self.dim, generator=self.g) * spread).to(self.dtype).cuda()

    def args(self, counts):
        """Device arrays of a call with counts[i] rows of sequence i (lens includes them)."""
        lens = torch.full((self.table.shape[0],), 12345678, dtype=torch.int32)
        for i, s in enumerate(self.slots):
            lens[s] = self.len[i]
        starts = torch.zeros(self.n + 1, dtype=torch.int32)
        starts[1:] = torch.cumsum(torch.tensor(counts), 0)
        return dict(table=self.table, lens=lens.cuda(), starts=starts.cuda(),
                    slots=torch.tensor(self.slots, dtype=torch.int32).cuda())

    def append(self, counts, spread=1.0, k=None, v=None, **kw):
        n = sum(counts)
        k = self.rows(max(n, 1), self.heads, spread) if k is None else k
        v = self.rows(max(n, 1), self.heads, spread) if v is None else v
        at = 0
        for i, c in enumerate(counts):
            self.len[i] += c
            self.model.append(self.slots[i], k[at:at + c], v[at:at + c])
            at += c
        self.cache.append(k, v, **self.args(counts), **kw)
        return k, v

    def check_held(self, tail=None):
        """Every sequence's values, bit for bit the model's (an fp32 product of the same integer and scale)."""
        counts = [n if tail is None else min(n, tail) for n in self.len]
        if not sum(counts):
            return
        k, v = self.cache.read(rows=sum(counts), **self.args(counts))
        at = 0
        for i, c in enumerate(counts):
            for name, got in (("k", k), ("v", v)):
                want = self.model.held(name, self.slots[i])[self.len[i] - c:].float()
                assert torch.equal(torch.nan_to_num(got[at:at + c].cpu(), nan=1e30), torch.nan_to_num(want, nan=1e30)), (name, i)
            at += c

    def check_attend(self, counts, heads, window=0, sinks=0, scale=None, q=None, **kw):
        """Attention of counts[i] last tokens of each sequence against fp64.

        Bounds: each probability is rounded to fp16 (half a step is 2^-11 of it)
        for the products, and not for the sum that divides them; in both it carries
        the error of its exponent and of 2^x, 2^-14 together for scores below 2^6.
        So a result is off by at most (2^-11 + 2 * 2^-14) sum p |v|; then half a
        step of the result's type."""
        q = self.rows(max(1, sum(counts)), heads) if q is None else q
        scale = self.dim ** -0.5 if scale is None else scale
        out = self.cache.attend(q, **self.args(counts), window=window, sinks=sinks, scale=scale, **kw)
        self.compare(out, q, counts, window, sinks, scale)
        return out

    def compare(self, out, q, counts, window, sinks, scale):
        got = out.double().cpu()
        at = 0
        for i, c in enumerate(counts):
            if c:
                L = self.len[i]
                k, v = self.model.held("k", self.slots[i]), self.model.held("v", self.slots[i])
                want, mag = attend(k, v, q[at:at + c].cpu(), list(range(L - c, L)), scale, window, sinks)
                tol = 2 ** -11 * 1.25 * mag + torch.finfo(self.dtype).eps / 2 * want.abs() + 2 ** -25
                off = (got[at:at + c] - want).abs()
                assert bool((off <= tol).all()), (i, L, c, float((off / tol).max()))
            at += c
