"""Plain statements, in 64 bits, of the cache in 4 bits and of the operators on it: element by element from the format's
definition.  TEST INFRASTRUCTURE."""
import math

import torch

import ops_reference as R

NAN_WORD = {"bf16": 0x7FC07FC0, "f16": 0x7FC07E00}


def groups_of(dim):
    return 2 if dim <= 64 else 4 if dim <= 128 else 8


def place(plane, groups, e):
    """(byte, shift) of element e's code in a row of 16 * groups bytes."""
    g, d = e // 32, e % 32
    if plane == 0:      # words of eight elements, [4][groups]
        return (d // 8 * groups + g) * 4 + d % 8 // 2, d % 2 * 4
    return (d // 4 * groups + g) * 2 + d % 4 // 2, d % 2 * 4


def quantise(x):
    """(lo, step, code) of rows [..., dim] of a 16-bit type, in float64; lo and step per element.  Groups that are not finite: NaN."""
    lo, step, code = (torch.zeros(x.shape, dtype=torch.float64) for _ in range(3))
    for a in range(0, x.shape[-1], 32):
        y = x[..., a:a + 32].float()
        low, high = y.amin(-1, keepdim=True), y.amax(-1, keepdim=True)      # NaN wherever one is
        s = torch.maximum((high - low) * torch.tensor(1 / 15), low.abs() * 2.0 ** -20).to(torch.bfloat16).double()
        bad = ~(torch.isfinite(y).all(-1, keepdim=True) & torch.isfinite(s))
        d = (y - low).double()
        c = torch.where(s > 0, torch.floor(d / s.masked_fill(s <= 0, 1.0) + 0.5), torch.zeros_like(d)).clamp(0, 15)
        lo[..., a:a + 32] = low.double().masked_fill(bad, math.nan)
        step[..., a:a + 32] = s.masked_fill(bad, math.nan)
        code[..., a:a + 32] = c.masked_fill(bad, 0.0)
    return lo, step, code


def pack(x, plane, name):
    """Rows [n, heads, dim] as bytes: codes [n, heads, 16 G], words [n, heads, 4 G]."""
    n, heads, dim = x.shape
    G = groups_of(dim)
    lo, step, code = quantise(x)
    codes = torch.zeros(n, heads, 16 * G, dtype=torch.uint8)
    words = torch.zeros(n, heads, G, 2, dtype=torch.int16)
    for e in range(dim):
        b, shift = place(plane, G, e)
        codes[..., b] |= (code[..., e].to(torch.uint8) << shift)
    for g in range(-(-dim // 32)):
        words[..., g, 0] = lo[..., 32 * g].to(R.TYPES[name]).view(torch.int16)
        words[..., g, 1] = step[..., 32 * g].to(torch.bfloat16).view(torch.int16)
        bad = torch.isnan(step[..., 32 * g])
        nan = NAN_WORD[name]
        words[..., g, 0][bad] = nan & 0xFFFF
        words[..., g, 1][bad] = nan >> 16
    return codes, words.flatten(-2).view(torch.uint8)


class Cache:
    """A device pool in 4 bits with scattered blocks for the given numbers of slots; what no sequence owns has codes of any kind and
    words of NaN.  rows[(sequence, layer, plane)] are the 16-bit rows that were packed."""

    def __init__(self, lens, heads, dim, bs, dtype="bf16", layout=0, layers=2, seed=0, width=None, spare=3, blocks=None, scale=(1.0, 1.0)):
        g = torch.Generator().manual_seed(seed)
        self.g, self.lens_list, self.heads, self.dim, self.bs, self.layers, self.layout = g, list(lens), heads, dim, bs, layers, layout
        self.dtype, self.tdtype, self.G = dtype, R.TYPES[dtype], groups_of(dim)
        n = len(lens)
        counts = [-(-x // bs) for x in lens]
        self.longest = max(list(lens) + [1])
        self.width = width or max(1, -(-self.longest // bs))
        used = sum(counts)
        self.nb = blocks or used + spare
        ids = (self.nb - 1 - torch.randperm(used + spare, generator=g))[:used] if blocks else torch.randperm(self.nb, generator=g)[:used]
        tables = torch.full((n, self.width), -7, dtype=torch.int32)
        at = 0
        for i, c in enumerate(counts):
            tables[i, :c] = ids[at:at + c].to(torch.int32)
            at += c
        self.tables_cpu = tables
        self.tables = tables.cuda()
        self.lens = torch.tensor(list(lens), dtype=torch.int32).cuda()
        per = bs * 20 * self.G
        shape = (self.nb, layers, 2, heads, per) if layout else (layers, 2, self.nb, heads, per)
        self.pool = torch.empty(shape, dtype=torch.uint8, device="cuda")
        if not blocks:
            self.pool.random_(generator=torch.Generator(device="cuda").manual_seed(seed))
            nan = torch.tensor([NAN_WORD[dtype]], dtype=torch.int64).to(torch.int32).cuda()
            self.pool[..., bs * 16 * self.G:].view(torch.int32).copy_(nan)
        self.rows = {}
        for i, x in enumerate(lens):
            for plane in range(2):
                for layer in range(layers):
                    self.write(i, layer, plane, (torch.randn(x, heads, dim, generator=g) * scale[plane]).to(self.tdtype))

    def where(self, i, slots):
        return self.tables_cpu[i].long()[slots // self.bs].cuda(), (slots % self.bs).cuda()

    def parts(self, layer, plane):
        p = self.pool[:, layer, plane] if self.layout else self.pool[layer, plane]
        cut = self.bs * 16 * self.G
        return p[..., :cut].unflatten(-1, (self.bs, -1)), p[..., cut:].unflatten(-1, (self.bs, -1))

    def write(self, i, layer, plane, rows, first=0):
        if len(rows) == 0:
            return
        b, r = self.where(i, torch.arange(first, first + len(rows)))
        codes, words = pack(rows, plane, self.dtype)
        c, w = self.parts(layer, plane)
        c[b, :, r] = codes.cuda()
        w[b, :, r] = words.cuda()
        old = self.rows.get((i, layer, plane))
        if first and old is not None:
            rows = torch.cat([old[:first], rows, old[first + len(rows):]])
        self.rows[(i, layer, plane)] = rows

    def held(self, i, layer, plane, n=None):
        """(lo, step, code) [slot][head][dim] in float64, read from the bytes of the pool."""
        n = self.lens_list[i] if n is None else n
        shape = (n, self.heads, self.dim)
        lo, step, code = (torch.zeros(shape, dtype=torch.float64) for _ in range(3))
        if n == 0:
            return lo, step, code
        b, r = self.where(i, torch.arange(n))
        c, w = (x[b, :, r].cpu() for x in self.parts(layer, plane))
        w = w.contiguous().view(torch.int16).unflatten(-1, (self.G, 2))
        for e in range(self.dim):
            at, shift = place(plane, self.G, e)
            code[..., e] = (c[..., at] >> shift & 15).double()
            lo[..., e] = w[..., e // 32, 0].contiguous().view(self.tdtype).double()
            step[..., e] = w[..., e // 32, 1].contiguous().view(torch.bfloat16).double()
        return lo, step, code

    def handle(self, B):
        return B.KVCache(self.pool.data_ptr(), self.layers, self.bs, self.heads, self.dim, self.nb, device_layout=self.layout, dtype=self.dtype + "_q4")


def attend(cache, layer, q, window=0, scale=None):
    """Per sequence and query head: (out, lse, p over the slots, error of a score, bound of out).  Where the bounds come from:
    a score is sum_g s (sum q code) + sum_g lo Q_g, products and sums in float32, so with |q| (|lo| + s code) in the place of the
    terms it is off by dim + 8 additions of 2^-23 each, and by 32 more in Q_g; q is scaled into float16, off by 2^-28 of its largest element
    at most.  The weights p s are rounded to float16: 2^-11 of them, or 2^-25 of the reference unit, which is at least 2^8 of the
    largest step's power of two (2^-33 of the step per slot, times a code of 15).  Exponentials and float32 sums: 2^-18, as for 16 bits;
    twice the scores' error for numerator and denominator; the output's own rounding."""
    n, heads, dim = q.shape[0], q.shape[1], cache.dim
    scale = scale if scale is not None else dim ** -0.5
    u = R.UNIT[cache.dtype]
    res = []
    for i in range(n):
        length = cache.lens_list[i]
        first = max(0, length - window) if window else 0
        (klo, ks, kc), (vlo, vs, vc) = (cache.held(i, layer, plane) for plane in range(2))
        k, v = klo + ks * kc, vlo + vs * vc
        ksize, vsize = klo.abs() + ks * kc, vlo.abs() + vs * vc
        row = []
        for g in range(heads):
            h = g // (heads // cache.heads)
            nothing = (torch.zeros(dim, dtype=torch.float64), -math.inf, torch.zeros(length, dtype=torch.float64), 0.0, torch.zeros(dim, dtype=torch.float64))
            if length == 0:
                row.append(nothing)
                continue
            x = q[i, g].double().cpu()
            s = (k[first:, h] * x).sum(-1) * scale
            top = s.max()
            if top == -math.inf:
                row.append(nothing)
                continue
            e = (s - top).exp()
            total = e.sum()
            p = torch.zeros(length, dtype=torch.float64)
            p[first:] = e / total
            out = (p[first:, None] * v[first:, h]).sum(0)
            size = (p[first:, None] * vsize[first:, h]).sum(0)
            score = (dim + 40) * 2.0 ** -23 * scale * float((ksize[first:, h] * x.abs()).sum(-1).max())
            score += 2.0 ** -28 * scale * float(x.abs().max()) * float((ks * kc)[first:, h].sum(-1).max())
            tail = (length - first) * 15 * 2.0 ** -33 * float(vs[first:, h].max()) / float(total)
            bound = u * out.abs() + (2.0 ** -11 + 2 * score + 2.0 ** -18) * size + tail
            row.append((out, float(top + total.log()), p, score, bound))
        res.append(row)
    return res


def normed(x, weight, eps):
    """Rows [..., dim] in float64."""
    return x if weight is None else x / (x.pow(2).mean(-1, keepdim=True) + eps).sqrt() * weight
