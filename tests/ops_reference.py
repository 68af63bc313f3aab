"""Plain statements, in 64 bits, of the operators on the device cache: loops over sequences and heads, no blocks of work,
no running maximum, no knowledge of the kernels.  TEST INFRASTRUCTURE."""
import math

import torch

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}       # largest relative error of one rounding to the type


class Cache:
    """A device pool with scattered blocks for the given numbers of slots; everything no sequence owns holds NaN."""

    def __init__(self, lens, heads, dim, bs, dtype="bf16", layout=0, layers=2, seed=0, width=None, spare=3, blocks=None):
        g = torch.Generator().manual_seed(seed)
        self.g, self.lens_list, self.heads, self.dim, self.bs, self.layers, self.layout = g, list(lens), heads, dim, bs, layers, layout
        self.dtype, self.tdtype = dtype, TYPES[dtype]
        n = len(lens)
        counts = [-(-x // bs) for x in lens]
        self.longest = max(list(lens) + [1])
        self.width = width or max(1, -(-self.longest // bs))
        used = sum(counts)
        self.nb = blocks or used + spare
        ids = (self.nb - 1 - torch.randperm(used + spare, generator=g))[:used] if blocks else torch.randperm(self.nb, generator=g)[:used]
        tables = torch.full((n, self.width), -7, dtype=torch.int32)     # ids of slots that do not exist are never looked at
        at = 0
        for i, c in enumerate(counts):
            tables[i, :c] = ids[at:at + c].to(torch.int32)
            at += c
        self.tables_cpu = tables
        self.tables = tables.cuda()
        self.lens = torch.tensor(list(lens), dtype=torch.int32).cuda()
        shape = (self.nb, layers, 2, bs, heads, dim) if layout else (layers, 2, self.nb, bs, heads, dim)
        self.pool = torch.empty(shape, dtype=self.tdtype, device="cuda")
        if not blocks:
            self.pool.fill_(float("nan"))
        for i, x in enumerate(lens):
            for kv in range(2):
                for layer in range(layers):
                    self.write(i, layer, kv, torch.randn(x, heads, dim, generator=g).to(self.tdtype))

    def where(self, i, slots):
        return self.tables_cpu[i].long()[slots // self.bs].cuda(), (slots % self.bs).cuda()

    def plane(self, layer, kv):
        return self.pool[:, layer, kv] if self.layout else self.pool[layer, kv]

    def read(self, i, layer, kv, n=None):
        """[slot][head][dim] of a sequence, as the cache holds it."""
        b, r = self.where(i, torch.arange(self.lens_list[i] if n is None else n))
        return self.plane(layer, kv)[b, r]

    def write(self, i, layer, kv, rows, first=0):
        b, r = self.where(i, torch.arange(first, first + len(rows)))
        self.plane(layer, kv)[b, r] = rows.cuda()

    def handle(self, B):
        return B.KVCache(self.pool.data_ptr(), self.layers, self.bs, self.heads, self.dim, self.nb, device_layout=self.layout, dtype=self.dtype)


def attend(cache, layer, q, window=0, scale=None):
    """Per sequence and query head: (out, lse, p over the slots, bounds).  The bounds follow from the arithmetic: scores are sums of
    dim exact products in float32 (each addition, fused or not, off by 2^-23 at most), so a score is off by
    `score` = (dim + 8) 2^-23 scale sum|q k|, its exponential by that relative error and a few units of float32, the
    output by the rounding of the weights to the cache's type, the output's own rounding, and twice the exponentials'
    error (numerator and denominator); float16 weights below 2^-14 of the largest are rounded to multiples of 2^-24."""
    n, heads, dim = q.shape[0], q.shape[1], cache.dim
    scale = scale if scale is not None else dim ** -0.5
    u = UNIT[cache.dtype]
    res = []
    for i in range(n):
        length = cache.lens_list[i]
        first = max(0, length - window) if window else 0
        k, v = (cache.read(i, layer, kv).double().cpu() for kv in range(2))
        row = []
        for g in range(heads):
            h = g // (heads // cache.heads)
            if length == 0:
                row.append((torch.zeros(dim, dtype=torch.float64), -math.inf, torch.zeros(0, dtype=torch.float64), 0.0, torch.zeros(dim, dtype=torch.float64), 0.0))
                continue
            x = q[i, g].double().cpu()
            s = (k[first:, h] * x).sum(-1) * scale
            top = s.max()
            if top == -math.inf:
                row.append((torch.zeros(dim, dtype=torch.float64), -math.inf, torch.zeros(length, dtype=torch.float64), 0.0,
                            torch.zeros(dim, dtype=torch.float64), 0.0))
                continue
            e = (s - top).exp()
            total = e.sum()
            p = torch.zeros(length, dtype=torch.float64)
            p[first:] = e / total
            out = (p[first:, None] * v[first:, h]).sum(0)
            size = (p[first:, None] * v[first:, h].abs()).sum(0)
            score = (dim + 8) * 2.0 ** -23 * scale * float((k[first:, h] * x).abs().sum(-1).max())
            tail = (length - first) * 2.0 ** -25 * float(v[first:, h].abs().max()) / float(total) if cache.dtype == "f16" else 0.0
            bound = (2 * u + 2 * score + 2.0 ** -18) * size + tail
            row.append((out, float(top + total.log()), p, score, bound, float(total)))
        res.append(row)
    return res


def rotate(x, angle, halves):
    """[..., dim] turned by angle [..., rotary/2], float64."""
    r = x.clone()
    half = angle.shape[-1]
    f = torch.arange(half)
    lo, hi = (f, f + half) if halves else (2 * f, 2 * f + 1)
    r[..., lo] = x[..., lo] * angle.cos() - x[..., hi] * angle.sin()
    r[..., hi] = x[..., lo] * angle.sin() + x[..., hi] * angle.cos()
    return r


def evict(weights, order, length, keep, recent, sink, seen):
    """One (layer, sequence, head): the (hole, source) pairs, by sorting (class, weight, slot) tuples."""
    def rank(s):
        age = int(order[s])
        w = float(weights[s])
        held = age >= seen - recent or age < sink
        return (2, 0.0, -s) if held else (0, 0.0, -s) if math.isnan(w) else (1, w, -s)
    if length <= keep:
        return []
    best = set(sorted(range(length), key=rank, reverse=True)[:keep])
    holes = [s for s in range(keep) if s not in best]
    return list(zip(holes, [s for s in range(keep, length) if s in best]))
