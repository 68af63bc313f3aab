"""Workloads of the operators on a paged KV cache held in 4 bits, and of norms in front of the rotation, each with its plain
form in elementary torch operations.

    attend   attention of one new token per sequence over a paged cache in 4 bits; every slot's weight joins a running sum on request
    norm     queries and keys are normed per head and rotated, k and v go into a paged cache in 16 bits
    pack     the same into a cache in 4 bits, and the new rows are read back, as the attention of a prompt needs them
    evict    a cache in 4 bits shrinks to its slots of largest weight, the newest and the first

``run`` computes a case in its plain form, or, where ``own`` is true, with the calls a user makes of the package.

The cache in 4 bits: groups of 32 elements of a head (heads padded to 64, 128 or 256: G groups) have a lowest value ``lo`` (an element
of the 16-bit type) and a step ``s`` (bf16); element = lo + s * code.  A block's plane is [head][codes | words]: 16 G bytes of codes
per row, then G words per row, lo in the lower half and s in the upper.  K's code words of 8 elements lie as [4][G], V's half words of 4 as [8][G].
"""
import math
import statistics

import torch

own = False
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-6
_handles = {}


def listed():
    return [
        # one user's first steps on the 8B shape (32 query heads, 8 KV heads of 128): launch latency is all there is
        attend("attend one short", seqs=1, q_heads=32, kv_heads=8, dim=128, block=16, median=37, most=37),
        # the 8B shape under load, with the weights that an eviction goes by: 64 requests around 1k up to 8k, two idle places
        attend("attend 64 requests", seqs=64, q_heads=32, kv_heads=8, dim=128, block=16, median=1024, most=8192, idle=2, weights=True),
        # the 70B shape: 32 requests around 2k up to 16k, eight query heads to a KV head
        attend("attend 70B shape", seqs=32, q_heads=64, kv_heads=8, dim=128, block=16, median=2048, most=16384),
        # one rank's shard of a model split eight ways, one long document in blocks of 64: the length has to be split
        attend("attend one long shard", seqs=1, q_heads=8, kv_heads=1, dim=128, block=64, median=131072, most=131072, dtype="f16"),
        # odd sizes: heads of 80, five query heads to a KV head, blocks of 24, a sliding window, block-first pool
        attend("attend odd window", seqs=7, q_heads=15, kv_heads=3, dim=80, block=24, median=700, most=5000, window=333, layout=1),
        # one decode step of 64 requests on the 70B shape, 16-bit cache
        append("norm decode step", "norm", seqs=64, each=1, before=2048, q_heads=64, kv_heads=8, dim=128, block=16),
        # the prompts of four requests on the 8B shape, 14k tokens in all, 16-bit cache
        append("norm prompts", "norm", seqs=4, each=4096, before=0, q_heads=32, kv_heads=8, dim=128, block=16),
        # one new token for one request into the 4-bit cache: nothing but latency
        append("pack one token", "pack", seqs=1, each=1, before=99, q_heads=32, kv_heads=8, dim=128, block=16),
        # pieces of 300 tokens behind a long context, heads of 64 rotated by half, pairs side by side, no norms
        append("pack pieces", "pack", seqs=5, each=300, before=5000, q_heads=14, kv_heads=2, dim=64, block=24, rotary=32, halves=False, norms=False, dtype="f16"),
        # the prompts of four requests on the 8B shape into the 4-bit cache
        append("pack prompts", "pack", seqs=4, each=4096, before=0, q_heads=32, kv_heads=8, dim=128, block=16),
        # two layers, one request of 100 slots that shrinks to 64
        evict("evict one small", layers=2, seqs=1, kv_heads=8, dim=128, block=16, length=100, keep=64, recent=16, sink=4),
        # all 32 layers of the 8B shape in a steady state: every 256 tokens eight requests go back to 2048 slots
        evict("evict steady state", layers=32, seqs=8, kv_heads=8, dim=128, block=16, length=2304, keep=2048, recent=256, sink=4),
    ]


def attend(name, **case):
    return {"name": name, "op": "attend", "idle": 0, "window": 0, "weights": False, "dtype": "bf16", "layout": 0, **case}


def append(name, op, **case):
    return {"name": name, "op": op, "rotary": case["dim"], "halves": True, "norms": True, "dtype": "bf16", "layout": 0, **case}


def evict(name, **case):
    return {"name": name, "op": "evict", "dtype": "bf16", "layout": 0, **case}


def draw(rng):
    def log(a, b):
        return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))

    op = rng.choice(["attend", "attend", "attend", "norm", "pack", "pack", "evict"])
    kv_heads, dim = rng.choice([1, 2, 3, 5, 8]), rng.choice([64, 80, 96, 128, 128, 256])
    common = {"kv_heads": kv_heads, "dim": dim, "block": rng.choice([8, 16, 16, 24, 32, 64]), "dtype": rng.choice(["bf16", "bf16", "f16"]),
              "layout": rng.choice([0, 0, 1])}
    row = kv_heads * padded(dim)  # values of one plane's row
    if op == "attend":
        seqs = log(1, 128)
        median = max(1, min(log(1, 65536), (1 << 27) // (seqs * row)))
        c = attend("", **common, q_heads=kv_heads * rng.choice([1, 2, 4, 5, 7, 8, 16]), seqs=seqs, median=median, most=median * rng.choice([1, 3, 8]),
                   idle=rng.choice([0, 0, 1]) if seqs > 1 else 0, window=rng.choice([0, 0, 0, log(1, 4096)]), weights=rng.random() < 0.4)
        if seqs * c["most"] * row > 1 << 29:
            c["most"] = median
    elif op in ("norm", "pack"):
        seqs, each = log(1, 64), rng.choice([1, 1, log(2, 4096)])
        each = max(1, min(each, (1 << 24) // (seqs * row)))
        c = append("", op, **common, q_heads=kv_heads * rng.choice([1, 2, 4, 5, 7, 8]), seqs=seqs, each=each, before=rng.choice([0, log(1, 8192)]),
                   rotary=rng.choice([dim, dim // 2]), halves=rng.random() < 0.7, norms=op == "norm" or rng.random() < 0.6)
        c["before"] = min(c["before"], (1 << 27) // (seqs * row))
    else:
        layers, seqs = log(1, 32), log(1, 16)
        length = max(20, min(log(20, 65536), (1 << 28) // (layers * seqs * row)))
        keep = rng.randint(8, length - 1)
        c = evict("", **common, layers=layers, seqs=seqs, length=length, keep=keep, recent=rng.randint(0, keep // 2), sink=rng.choice([0, 1, 4]))
    del c["name"]
    size = {"attend": "median", "norm": "each", "pack": "each", "evict": "length"}[op]
    while work(c)["bytes"] > 3e8 and c[size] > 40:  # no more than the largest listed ones
        c[size] = c[size] * 3 // 4
        if op == "evict":
            c["keep"], c["recent"] = max(8, c["keep"] * 3 // 4), c["recent"] // 3
    return c


# ---- lengths of a case's sequences: fixed by the case, dealt out by the seed ----------------------------------------


def padded(dim):
    return 64 if dim <= 64 else 128 if dim <= 128 else 256


def lengths(case):
    n = case["seqs"]
    if case["op"] == "attend":
        live = n - case["idle"]  # lognormal quantiles, sigma 1; idle places of the batch hold no tokens
        z = [statistics.NormalDist().inv_cdf((i + 0.5) / live) for i in range(live)]
        return [min(case["most"], max(1, round(case["median"] * math.exp(x)))) for x in z] + [0] * case["idle"]
    if case["op"] != "evict":  # prompts of unequal length: the last ones are shorter
        return [case["before"] + new for new in news(case)]
    span = case["length"] - case["keep"]  # evict: from the full length down; with four or more, one is short enough to stay whole
    lens = [case["length"] - (span * i) // (2 * n) for i in range(n)]
    return lens[:-1] + [max(1, case["keep"] - 3)] if n >= 4 else lens


def news(case):
    return [max(1, case["each"] - (case["each"] * i) // (3 * case["seqs"])) for i in range(case["seqs"])]


# ---- the cache in 4 bits, in elementary operations ------------------------------------------------------------------


def encode(x, plane):
    """[..., dim] of the 16-bit type -> (codes uint8 [..., 16 G], words uint8 [..., 4 G]); plane 0: K's order, 1: V's."""
    dim, wide = x.shape[-1], padded(x.shape[-1])
    lo, hi = x, x
    if wide > dim:  # what pads a head is no element of its group
        lo = torch.nn.functional.pad(x, (0, wide - dim), value=math.inf)
        hi = torch.nn.functional.pad(x, (0, wide - dim), value=-math.inf)
    lo = lo.unflatten(-1, (-1, 32)).amin(-1).float()
    hi = hi.unflatten(-1, (-1, 32)).amax(-1).float()
    none = lo == math.inf
    lo, hi = lo.masked_fill(none, 0.0), hi.masked_fill(none, 0.0)
    step = torch.maximum((hi - lo) / 15, lo.abs() * 2.0 ** -20).bfloat16()
    d = torch.nn.functional.pad(x, (0, wide - dim)).float().unflatten(-1, (-1, 32)) - lo[..., None]
    s = step.double()[..., None]
    u = (d.double() / s.masked_fill(s == 0, 1.0) + 0.5).floor().clamp(0, 15).to(torch.int32)
    if wide > dim:
        u.flatten(-2)[..., dim:] = 0
    each, place = (8, 4) if plane == 0 else (4, 8)
    u = u.unflatten(-1, (place, each)) << (4 * torch.arange(each, device=x.device, dtype=torch.int32))
    codes = u.sum(-1).to(torch.int32 if plane == 0 else torch.int16).transpose(-1, -2).contiguous()
    words = torch.stack([lo.to(x.dtype).view(torch.int16), step.view(torch.int16)], -1)
    return codes.view(torch.uint8).flatten(-2), words.flatten(-2).view(torch.uint8)


def decode(codes, words, plane, dtype, dim):
    """The values in 32 bits."""
    groups = words.shape[-1] // 4
    words = words.contiguous().view(torch.int16).unflatten(-1, (groups, 2))
    lo, step = words[..., 0].view(dtype).float(), words[..., 1].view(torch.bfloat16).float()
    each, place, kind = (8, 4, torch.int32) if plane == 0 else (4, 8, torch.int16)
    w = codes.contiguous().view(kind).unflatten(-1, (place, groups)).transpose(-1, -2)
    u = (w[..., None] >> (4 * torch.arange(each, device=w.device, dtype=kind))) & 15
    x = lo[..., None] + step[..., None] * u.flatten(-2).float()
    return x.flatten(-2)[..., :dim]


def planes(s, layer, plane):
    """A plane of the 4-bit pool: (codes [block][head][row][16 G], words [block][head][row][4 G])."""
    c, p = s["case"], s["pool"]
    p = p[:, layer, plane] if c["layout"] else p[layer, plane]
    cut = c["block"] * padded(c["dim"]) // 2
    return p[..., :cut].unflatten(-1, (c["block"], -1)), p[..., cut:].unflatten(-1, (c["block"], -1))


# ---- inputs ---------------------------------------------------------------------------------------------------------


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    dt, bs, heads, dim, n = TYPES[case["dtype"]], case["block"], case["kv_heads"], case["dim"], case["seqs"]
    layers = case.get("layers", 2)
    s = {"case": case, "layer": layers - 1}

    def normal(*shape, scale=1.0):
        return (torch.randn(*shape, generator=g, device=DEV) * scale).to(dt)

    lens = torch.tensor(lengths(case), device=DEV)
    if case["op"] in ("attend", "evict"):
        lens = lens[torch.randperm(n, generator=g, device=DEV)]
    counts = -(-lens // bs)
    longest = int(lens.max())
    width = max(1, -(-longest // bs))
    total = int(counts.sum())
    blocks = total + total // 8 + 1
    ids = torch.randperm(blocks, generator=g, device=DEV)[:total].to(torch.int32)  # scattered, as a pool hands them out
    used = torch.arange(width, device=DEV)[None] < counts[:, None]
    s["tables"] = torch.full((n, width), -1, dtype=torch.int32, device=DEV)
    s["tables"][used] = ids
    s["lens"], s["longest"] = lens.to(torch.int32), longest
    if case["op"] == "norm":
        shape = (blocks, layers, 2, bs, heads, dim) if case["layout"] else (layers, 2, blocks, bs, heads, dim)
        s["pool"] = torch.empty(shape, dtype=dt, device=DEV).normal_(generator=g)
    else:
        plane = (heads, bs * padded(dim) * 5 // 8)
        s["pool"] = torch.randint(0, 256, (blocks, layers, 2, *plane) if case["layout"] else (layers, 2, blocks, *plane), generator=g, dtype=torch.uint8,
                                  device=DEV)
    if case["op"] == "attend":
        # keys have some channels that are larger than the others
        wide = torch.ones(heads, 1, dim, device=DEV)
        wide[..., torch.randint(0, dim, (max(1, dim // 32),), generator=g, device=DEV)] = 4.0
        for kv in range(2):
            x = torch.randn(blocks, heads, bs, dim, generator=g, device=DEV)
            for to, new in zip(planes(s, s["layer"], kv), encode((x * wide if kv == 0 else x).to(dt), kv)):
                to.copy_(new)
        s["q"] = normal(n, case["q_heads"], dim)
        s["out"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros(n, case["q_heads"], device=DEV)
        s["had"] = s["weights"] = None
        if case["weights"]:  # what earlier steps added up
            s["had"] = torch.rand(n, heads, max(1, longest), generator=g, device=DEV).square_()
            s["weights"] = torch.zeros_like(s["had"])
    elif case["op"] != "evict":
        new = torch.tensor(news(case), device=DEV)
        t, half = int(new.sum()), case["rotary"] // 2
        # as a projection leaves them: one buffer of q, k and v side by side
        s["qkv"] = normal(t, case["q_heads"] + 2 * heads, dim)
        s["q_out"] = torch.zeros(t, case["q_heads"], dim, dtype=dt, device=DEV)
        s["inv_freq"] = (10000.0 ** (-torch.arange(half, device=DEV, dtype=torch.float64) / half)).float()
        s["starts"] = torch.cat([new.new_zeros(1), new.cumsum(0)]).to(torch.int32)
        at = torch.arange(t, device=DEV) - torch.repeat_interleave(s["starts"][:-1].long(), new) + case["before"]
        s["positions"] = (torch.randint(0, 4096, (1,), generator=g, device=DEV) + at)[None].to(torch.int32)
        s["q_norm"] = s["k_norm"] = None
        if case["norms"]:  # learned weights around one
            s["q_norm"], s["k_norm"] = ((1 + 0.25 * torch.randn(dim, generator=g, device=DEV)).to(dt) for _ in range(2))
        if case["op"] == "pack":
            s["k_read"], s["v_read"] = (torch.zeros(t, heads, dim, dtype=dt, device=DEV) for _ in range(2))
    else:
        # heavy-tailed sums with a share of slots that nothing ever looked at (equal weights: the lowest slot stays)
        w = torch.randn(layers, n, heads, longest, generator=g, device=DEV).mul_(1.5).exp_()
        s["had"] = torch.where(torch.rand(w.shape, generator=g, device=DEV) < 0.1, torch.zeros_like(w), w)
        # earlier evictions left the first `keep` slots in any order of age; behind them are the newest, as they came
        keep = min(case["keep"], longest)
        age = torch.rand(layers, n, heads, keep, generator=g, device=DEV).argsort(-1) * 2
        s["ages"] = torch.cat([age, (torch.arange(keep, longest, device=DEV) + keep).expand(layers, n, heads, -1)], -1).to(torch.int32)
        s["seen"] = torch.where(lens > keep, lens + keep, 2 * lens).to(torch.int32)
        s["weights"] = torch.zeros(layers, n, heads, case["keep"], device=DEV)
        s["order"] = torch.zeros(layers, n, heads, case["keep"], dtype=torch.int32, device=DEV)
        s["new_lens"] = torch.zeros_like(s["lens"])
    if own:
        from paper_2601_20309_b200 import binding

        # the handles a serving program keeps: the operator context of its stream, and the cache's geometry
        if "ops" not in _handles:
            _handles["ops"] = binding.KVOps(device_id=0, stream=torch.cuda.current_stream().cuda_stream)
        s["ops"] = _handles["ops"]
        s["cache"] = binding.KVCache(s["pool"].data_ptr(), layers, bs, heads, dim, blocks, device_layout=case["layout"],
                                     dtype=case["dtype"] + ("" if case["op"] == "norm" else "_q4"))
    return s


# ---- one pass -------------------------------------------------------------------------------------------------------


def run(s):
    return globals()[("own_" if own else "plain_") + s["case"]["op"]](s)


def own_attend(s):
    s["ops"].kv_attend(s["cache"], s["layer"], s["q"], s["tables"], s["lens"], s["longest"], out=s["out"], lse=s["lse"], window=s["case"]["window"],
                       weights_in=s["had"], weights_out=s["weights"])
    return outputs(s, "out", "lse", "weights")


def own_norm(s):
    h, k = s["case"]["q_heads"], s["case"]["kv_heads"]
    qkv = s["qkv"]
    s["ops"].kv_append(s["cache"], s["layer"], qkv[:, :h], qkv[:, h:h + k], qkv[:, h + k:], s["tables"], s["lens"], positions=s["positions"],
                       inv_freq=s["inv_freq"], halves=s["case"]["halves"], q_out=s["q_out"], seq_starts=s["starts"], q_norm=s["q_norm"],
                       k_norm=s["k_norm"], norm_eps=EPS)
    return outputs(s, "q_out", "pool") if s["case"]["op"] == "norm" else None


def own_pack(s):
    own_norm(s)
    s["ops"].kv_read(s["cache"], s["layer"], s["tables"], s["lens"], k_out=s["k_read"], v_out=s["v_read"], seq_starts=s["starts"])
    return outputs(s, "q_out", "k_read", "v_read")


def own_evict(s):
    c = s["case"]
    s["ops"].kv_evict(s["cache"], s["tables"], s["lens"], s["longest"], keep=c["keep"], recent=c["recent"], sink=c["sink"], weights=s["had"], order=s["ages"],
                      seen=s["seen"], weights_out=s["weights"], order_out=s["order"], lens_out=s["new_lens"])
    return outputs(s, "pool", "weights", "order", "new_lens")


def outputs(s, *names):
    return {k: s[k] for k in names if s[k] is not None}


def plain_attend(s):
    c, n = s["case"], max(1, s["longest"])
    bs, heads, group, dim = c["block"], c["kv_heads"], c["q_heads"] // c["kv_heads"], c["dim"]
    slot = torch.arange(n, device=DEV)
    lens = s["lens"].long()[:, None]
    live = slot < lens
    seen = live & (slot >= lens - c["window"]) if c["window"] else live
    block = s["tables"].long()[:, slot // bs].clamp(min=0)

    def values(plane):  # [seq][slot][head][dim]
        codes, words = (x[block, :, slot % bs] for x in planes(s, s["layer"], plane))
        return decode(codes, words, plane, s["q"].dtype, dim).masked_fill_(~seen[..., None, None], 0.0)

    q = s["q"].float().reshape(-1, heads, group, dim)
    x = torch.einsum("bhgd,bnhd->bhgn", q, values(0)) * dim ** -0.5
    x = x.masked_fill(~seen[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    e = (x - top.masked_fill(top == -math.inf, 0.0)).exp()
    total = e.sum(-1, keepdim=True)
    p = torch.where(total > 0, e / total, 0.0)
    out = torch.einsum("bhgn,bnhd->bhgd", p, values(1)).reshape(s["q"].shape).to(s["q"].dtype)
    r = {"out": out, "lse": (top + total.log()).reshape(s["lse"].shape)}
    if c["weights"]:
        r["weights"] = torch.where(live[:, None], s["had"] + p.sum(2), s["weights"])
    return r


def normed_and_turned(s, x, weight):
    """Heads [token][head][dim] in the given precision: normed if there is a weight, then rotated."""
    c = s["case"]
    if weight is not None:
        x = x / (x.square().mean(-1, keepdim=True) + EPS).sqrt() * weight.to(x.dtype)
    angle = s["positions"][0].double()[:, None] * s["inv_freq"].double()  # far positions need 64 bits
    cos, sin = angle.cos()[:, None].to(x.dtype), angle.sin()[:, None].to(x.dtype)
    rot, rest = x[..., :c["rotary"]], x[..., c["rotary"]:]
    if c["halves"]:
        a, b = rot.chunk(2, -1)
        rot = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    else:
        a, b = rot[..., 0::2], rot[..., 1::2]
        rot = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    return torch.cat([rot, rest], -1)


def slots_of(s):
    """(block, row) of every new token."""
    t = len(s["qkv"])
    token, starts = torch.arange(t, device=DEV), s["starts"].long()
    seq = torch.searchsorted(starts[1:], token, right=True)
    slot = s["lens"].long()[seq] - (starts[seq + 1] - token)
    return s["tables"].long()[seq, slot // s["case"]["block"]], slot % s["case"]["block"]


def plain_norm(s):
    c = s["case"]
    h, kh = c["q_heads"], c["kv_heads"]
    q = normed_and_turned(s, s["qkv"][:, :h].float(), s["q_norm"]).to(s["qkv"].dtype)
    k = normed_and_turned(s, s["qkv"][:, h:h + kh].float(), s["k_norm"]).to(s["qkv"].dtype)
    p, (block, row) = s["pool"], slots_of(s)
    kp, vp = (p[:, s["layer"], kv] if c["layout"] else p[s["layer"], kv] for kv in range(2))
    kp[block, row] = k
    vp[block, row] = s["qkv"][:, h + kh:]
    return {"q_out": q, "pool": p}


def plain_pack(s):
    c, dt = s["case"], s["qkv"].dtype
    h, kh = c["q_heads"], c["kv_heads"]
    r = {"q_out": normed_and_turned(s, s["qkv"][:, :h].float(), s["q_norm"]).to(dt)}
    # a key next to the border of two codes must fall on the same side for everybody: 64 bits up to the 16-bit key
    k = normed_and_turned(s, s["qkv"][:, h:h + kh].double(), s["k_norm"]).float().to(dt)
    block, row = slots_of(s)
    for plane, x in enumerate((k, s["qkv"][:, h + kh:])):
        held = planes(s, s["layer"], plane)
        for to, new in zip(held, encode(x, plane)):
            to[block, :, row] = new
        codes, words = (y[block, :, row] for y in held)
        r[("k_read", "v_read")[plane]] = decode(codes, words, plane, dt, c["dim"]).to(dt)
    return r


def plain_evict(s):
    c, n, keep, bs = s["case"], s["longest"], s["case"]["keep"], s["case"]["block"]
    lens = s["lens"].long()[:, None, None]  # [seq][head][slot] under the layers
    seen = s["seen"].long()[:, None, None]
    slot = torch.arange(n, device=DEV)
    live = slot < lens
    held = (s["ages"] >= seen - c["recent"]) | (s["ages"] < c["sink"])
    score = torch.where(held, math.inf, s["had"]).masked_fill(~live, -math.inf)
    best = score.sort(dim=-1, descending=True, stable=True).indices[..., :keep]
    stays = torch.zeros_like(score, dtype=torch.bool).scatter_(-1, best, True) & live
    stays = stays | (live & (lens <= keep))
    hole = ~stays & live & (slot < keep)
    comes = stays & (slot >= keep)
    # the holes and the slots that move, both in ascending order, meet pairwise
    l, b, h, to = hole.nonzero(as_tuple=True)
    src = comes.nonzero(as_tuple=True)[3]
    take = slot.expand(score.shape).clone()
    take[l, b, h, to] = src
    take = take[..., :keep]
    tables = s["tables"].long()
    p = s["pool"] if c["layout"] else s["pool"].permute(2, 0, 1, 3, 4)  # [block][layer][K|V][head][bytes]
    cut = bs * padded(c["dim"]) // 2
    for part in (p[..., :cut].unflatten(-1, (bs, -1)), p[..., cut:].unflatten(-1, (bs, -1))):
        part[tables[b, to // bs], l, :, h, to % bs] = part[tables[b, src // bs], l, :, h, src % bs]
    kept = slot[:keep] < lens
    r = {"pool": s["pool"], "new_lens": s["lens"].clamp(max=keep)}
    width = min(n, keep)
    for name, old in (("weights", s["had"]), ("order", s["ages"])):
        new = s[name].clone()
        new[..., :width] = torch.where(kept[..., :width], old.gather(-1, take), new[..., :width])
        r[name] = new
    return r


# ---- what a pass cannot do without ----------------------------------------------------------------------------------


def work(case):
    heads, dim, lens = case["kv_heads"], case["dim"], lengths(case)
    packed = padded(dim) * 5 // 8  # bytes of a row in 4 bits
    if case["op"] == "attend":
        slots = sum(min(n, case["window"]) if case["window"] else n for n in lens)
        ends = case["seqs"] * case["q_heads"]
        weights = 8 * sum(lens) * heads if case["weights"] else 0
        return {"bytes": 2 * packed * slots * heads + weights + ends * (4 * dim + 4) + 4 * sum(-(-n // case["block"]) for n in lens),
                "flops": 4 * slots * case["q_heads"] * dim}
    if case["op"] == "norm":
        t = sum(news(case))
        return {"bytes": t * (4 * (case["q_heads"] + 2 * heads) * dim + 8), "flops": t * (3 * case["rotary"] + 4 * dim) * (case["q_heads"] + heads)}
    if case["op"] == "pack":  # q, k and v in, q out, the packed rows out and in again, their values out
        t = sum(news(case))
        return {"bytes": t * ((4 * case["q_heads"] + 8 * heads) * dim + 4 * packed * heads + 8),
                "flops": t * ((3 * case["rotary"] + 4 * dim) * (case["q_heads"] + heads) + 12 * heads * dim)}
    total = 0.0
    for n in lens:
        total += 8 * n + 8 * min(n, case["keep"])  # weight and age of each slot, and of each that stays
        if n > case["keep"]:  # rows that move: the protected new ones, and their share of the others
            tail = n - case["keep"]
            newest = min(case["recent"], tail)
            moved = newest + (tail - newest) * max(0, case["keep"] - case["recent"] - case["sink"]) / max(1, n - case["recent"] - case["sink"])
            total += 4 * packed * moved
    return {"bytes": total * heads * case["layers"], "flops": 0}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "attend":
        return exact_attend(s)
    if case["op"] in ("norm", "pack"):
        return exact_append(s)
    return None  # rows, weights and ages are moved, none is computed


def element(codes, words, d, plane, dtype):
    """Element d of every row, by the format's definition."""
    groups, g, e = words.shape[-1] // 4, d // 32, d % 32
    byte = (e // 8 * groups + g) * 4 + e % 8 // 2 if plane == 0 else (e // 4 * groups + g) * 2 + e % 4 // 2
    code = codes[..., byte].int() // (16 if e % 2 else 1) % 16
    word = words[..., 4 * g:4 * g + 4].contiguous()
    return word[..., :2].contiguous().view(dtype)[..., 0].double() + word[..., 2:].contiguous().view(torch.bfloat16)[..., 0].double() * code


def exact_attend(s):
    c = s["case"]
    heads, group, dim, bs = c["kv_heads"], c["q_heads"] // c["kv_heads"], c["dim"], c["block"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device=DEV)
    weights = s["weights"].double() if c["weights"] else None
    for i, n in enumerate(s["lens"].tolist()):
        if n == 0:
            continue
        first = max(0, n - c["window"]) if c["window"] else 0
        ids = s["tables"][i, : -(-n // bs)].long()
        kv = []
        for plane in range(2):
            codes, words = (x[ids].transpose(1, 2).flatten(0, 1)[first:n] for x in planes(s, s["layer"], plane))  # [slot][head][bytes]
            kv.append(torch.stack([element(codes, words, d, plane, s["q"].dtype) for d in range(dim)], -1))
        if weights is not None:
            weights[i, :, :n] = s["had"][i, :, :n].double()
        for h in range(heads):
            q = s["q"][i, h * group:(h + 1) * group].double()
            x = q @ kv[0][:, h].T / math.sqrt(dim)
            total = torch.logsumexp(x, 1)
            p = torch.exp(x - total[:, None])
            out[i, h * group:(h + 1) * group] = p @ kv[1][:, h]
            lse[i, h * group:(h + 1) * group] = total
            if weights is not None:
                weights[i, h, first:n] += p.sum(0)
    return {"out": out, "lse": lse, "weights": weights}


def exact_append(s):
    c = s["case"]
    h, heads, bs, half = c["q_heads"], c["kv_heads"], c["block"], c["rotary"] // 2
    x = s["qkv"].double()
    if c["norms"]:
        x[:, :h + heads] *= torch.rsqrt(x[:, :h + heads].pow(2).sum(-1, keepdim=True) / c["dim"] + EPS)
        x[:, :h] *= s["q_norm"].double()
        x[:, h:h + heads] *= s["k_norm"].double()
    f = torch.arange(half, device=DEV)
    low, high = (f, f + half) if c["halves"] else (2 * f, 2 * f + 1)
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), s["positions"][0].double()[:, None] * s["inv_freq"].double())
    z = torch.complex(x[:, :h + heads, low], x[:, :h + heads, high]) * turn[:, None]
    x[:, :h + heads, low] = z.real
    x[:, :h + heads, high] = z.imag
    if c["op"] == "pack":
        return {"q_out": x[:, :h], "k_read": stands_for(x[:, h:h + heads].float().to(s["qkv"].dtype)), "v_read": stands_for(s["qkv"][:, h + heads:])}
    pool = s["pool"].double()
    if c["layout"]:
        pool = pool.permute(1, 2, 0, 3, 4, 5)
    row = 0
    for i, (n, new) in enumerate(zip(s["lens"].tolist(), news(c))):
        slot = torch.arange(n - new, n, device=DEV)
        block = s["tables"][i].long()[slot // bs]
        pool[s["layer"], 0, block, slot % bs] = x[row:row + new, h:h + heads]
        pool[s["layer"], 1, block, slot % bs] = x[row:row + new, h + heads:]
        row += new
    if c["layout"]:
        pool = pool.permute(2, 0, 1, 3, 4, 5)
    return {"q_out": x[:, :h], "pool": pool}


def stands_for(x):
    """The values that the cache in 4 bits holds for 16-bit rows: group by group."""
    r = torch.empty(x.shape, dtype=torch.float64, device=DEV)
    for a in range(0, x.shape[-1], 32):
        y = x[..., a:a + 32].double()
        lo, hi = y.min(-1, keepdim=True).values, y.max(-1, keepdim=True).values
        step = torch.maximum((hi - lo).float() / 15, lo.float().abs() / 2 ** 20).bfloat16().double()
        code = torch.where(step > 0, torch.floor((y - lo) / step.clamp(min=1e-300) + 0.5), 0.0).clamp(0, 15)
        r[..., a:a + 32] = lo + step * code
    return r
