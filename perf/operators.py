"""Workloads of the operators on the paged KV cache, each with its plain form in elementary torch operations.

    append   rotary positions with several axes (time, height, width) on the new tokens' q and k; k and v go into the cache
    attend   attention of one new token per sequence over the paged cache; every slot's attention weight joins a running sum
    evict    the cache shrinks to the slots with the largest accumulated weight, the newest ones and the first ones

``run`` computes a case in its plain form, or, where ``own`` is true, with the calls a user makes of the package.  The cache
is the package's device pool: [layer][K|V][block][block_size][kv_heads][head_dim], or block-first, with scattered blocks.
"""
import math
import statistics

import torch

own = False
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
_handles = {}


def listed():
    return [
        # one user's first steps on the 8B shape (32 query heads, 8 KV heads of 128): launch latency is all there is
        attend("attend one short", seqs=1, q_heads=32, kv_heads=8, dim=128, block=16, median=37, most=37),
        # the 8B shape under load: 64 requests, lengths lognormal around 1k up to 8k, two idle places in the batch
        attend("attend 64 requests", seqs=64, q_heads=32, kv_heads=8, dim=128, block=16, median=1024, most=8192, idle=2),
        # the 70B shape: 32 requests around 2k up to 16k, eight query heads to a KV head; no weights are wanted
        attend("attend 70B shape", seqs=32, q_heads=64, kv_heads=8, dim=128, block=16, median=2048, most=16384, weights=False),
        # one rank's shard of a model split eight ways, one long document in blocks of 64: the length has to be split
        attend("attend one long shard", seqs=1, q_heads=8, kv_heads=1, dim=128, block=64, median=131072, most=131072, dtype="f16"),
        # odd sizes: heads of 80, five query heads to a KV head, blocks of 24, a sliding window, block-first pool
        attend("attend odd window", seqs=7, q_heads=15, kv_heads=3, dim=80, block=24, median=700, most=5000, window=333, layout=1),
        # one new token for one request: rotation and the write into the cache, nothing but latency
        append("append one token", seqs=1, each=1, before=99, q_heads=32, kv_heads=8, dim=128, block=16),
        # one decode step of 64 requests on the 70B shape
        append("append decode step", seqs=64, each=1, before=2048, q_heads=64, kv_heads=8, dim=128, block=16),
        # the prompts of four requests, text with images between: the 8B shape, 16k tokens in all
        append("append prompts", seqs=4, each=4096, before=0, q_heads=32, kv_heads=8, dim=128, block=16),
        # two layers, one request of 100 slots that shrinks to 64
        evict("evict one small", layers=2, seqs=1, kv_heads=8, dim=128, block=16, length=100, keep=64, recent=16, sink=4),
        # all 32 layers of the 8B shape in a steady state: every 256 tokens eight requests go back to 2048 slots
        evict("evict steady state", layers=32, seqs=8, kv_heads=8, dim=128, block=16, length=2304, keep=2048, recent=256, sink=4),
        # the first eviction after long prompts: 16k slots become 4k in four layers of three requests
        evict("evict after prompts", layers=4, seqs=3, kv_heads=8, dim=128, block=16, length=16384, keep=4096, recent=512, sink=4),
        # one rank's shard of a long document, one layer at a time: few heads, many slots
        evict("evict long shard", layers=1, seqs=1, kv_heads=1, dim=128, block=64, length=131072, keep=8192, recent=1024, sink=4, dtype="f16"),
    ]


def attend(name, **case):
    return {"name": name, "op": "attend", "idle": 0, "window": 0, "weights": True, "dtype": "bf16", "layout": 0, **case}


def append(name, **case):
    return {"name": name, "op": "append", "rotary": case["dim"], "halves": True, "dtype": "bf16", "layout": 0, **case}


def evict(name, **case):
    return {"name": name, "op": "evict", "dtype": "bf16", "layout": 0, **case}


def draw(rng):
    def log(a, b):
        return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))

    op = rng.choice(["attend", "attend", "append", "evict"])
    kv_heads, dim = rng.choice([1, 2, 3, 5, 8]), rng.choice([64, 80, 96, 128, 128, 256])
    common = {"kv_heads": kv_heads, "dim": dim, "block": rng.choice([8, 16, 16, 24, 32, 64]), "dtype": rng.choice(["bf16", "bf16", "f16"]),
              "layout": rng.choice([0, 0, 1])}
    row = kv_heads * dim  # values of one plane's row
    if op == "attend":
        seqs = log(1, 128)
        median = max(1, min(log(1, 65536), (1 << 27) // (seqs * row)))
        common |= {"q_heads": kv_heads * rng.choice([1, 2, 4, 5, 7, 8, 16]), "seqs": seqs, "median": median, "most": median * rng.choice([1, 3, 8]),
                   "idle": rng.choice([0, 0, 1]) if seqs > 1 else 0, "window": rng.choice([0, 0, 0, log(1, 4096)]), "weights": rng.random() < 0.6}
        c = attend("", **common)
        if seqs * c["most"] * row > 1 << 29:
            c["most"] = median
    elif op == "append":
        seqs, each = log(1, 64), rng.choice([1, 1, log(2, 4096)])
        each = max(1, min(each, (1 << 24) // (seqs * row)))
        c = append("", **common, q_heads=kv_heads * rng.choice([1, 2, 4, 5, 7, 8]), seqs=seqs, each=each, before=rng.choice([0, log(1, 8192)]),
                   rotary=rng.choice([dim, dim // 2]), halves=rng.random() < 0.7)
        c["before"] = min(c["before"], (1 << 27) // (seqs * row))
    else:
        layers, seqs = log(1, 32), log(1, 16)
        length = max(20, min(log(20, 65536), (1 << 28) // (layers * seqs * row)))
        keep = rng.randint(8, length - 1)
        c = evict("", **common, layers=layers, seqs=seqs, length=length, keep=keep, recent=rng.randint(0, keep // 2), sink=rng.choice([0, 1, 4]))
    del c["name"]
    size = {"attend": "median", "append": "each", "evict": "length"}[op]
    while work(c)["bytes"] > 4e8 and c[size] > 40:  # no more than the largest listed ones
        c[size] = c[size] * 3 // 4
        if op == "evict":
            c["keep"], c["recent"] = max(8, c["keep"] * 3 // 4), c["recent"] // 3
    return c


# ---- lengths of a case's sequences: fixed by the case, dealt out by the seed ----------------------------------------


def lengths(case):
    n = case["seqs"]
    if case["op"] == "attend":
        live = n - case["idle"]  # lognormal quantiles, sigma 1; idle places of the batch hold no tokens
        z = [statistics.NormalDist().inv_cdf((i + 0.5) / live) for i in range(live)]
        return [min(case["most"], max(1, round(case["median"] * math.exp(x)))) for x in z] + [0] * case["idle"]
    if case["op"] == "append":  # prompts of unequal length: the last ones are shorter
        return [case["before"] + new for new in news(case)]
    span = case["length"] - case["keep"]  # evict: from the full length down; with four or more, one is short enough to stay whole
    lens = [case["length"] - (span * i) // (2 * n) for i in range(n)]
    return lens[:-1] + [max(1, case["keep"] - 3)] if n >= 4 else lens


def news(case):
    return [max(1, case["each"] - (case["each"] * i) // (3 * case["seqs"])) for i in range(case["seqs"])]


def sections(case):
    """The axis of every rotated frequency: time first, then height, then width, 2 : 3 : 3."""
    half = case["rotary"] // 2
    first, second = half // 4, half // 4 + (half - half // 4) // 2
    return [0 if f < first else 1 if f < second else 2 for f in range(half)]


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
    new = torch.tensor(news(case), device=DEV) if case["op"] == "append" else None
    if case["op"] != "append":
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
    shape = (blocks, layers, 2, bs, heads, dim) if case["layout"] else (layers, 2, blocks, bs, heads, dim)
    s["pool"] = torch.empty(shape, dtype=dt, device=DEV).normal_(generator=g)
    if case["op"] == "attend":
        s["q"] = normal(n, case["q_heads"], dim, scale=2.0)
        s["out"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros(n, case["q_heads"], device=DEV)
        s["had"] = s["weights"] = None
        if case["weights"]:  # what earlier steps added up
            s["had"] = torch.rand(n, heads, max(1, longest), generator=g, device=DEV).square_()
            s["weights"] = torch.zeros_like(s["had"])
    elif case["op"] == "append":
        t, half = int(new.sum()), case["rotary"] // 2
        # as a projection leaves them: one buffer of q, k and v side by side
        s["qkv"] = normal(t, case["q_heads"] + 2 * heads, dim)
        s["q_out"] = torch.zeros(t, case["q_heads"], dim, dtype=dt, device=DEV)
        s["inv_freq"] = (10000.0 ** (-torch.arange(half, device=DEV, dtype=torch.float64) / half)).float()
        s["starts"] = torch.cat([new.new_zeros(1), new.cumsum(0)]).to(torch.int32)
        at = torch.arange(t, device=DEV) - torch.repeat_interleave(s["starts"][:-1].long(), new) + case["before"]
        image = (at // 256) % 2 == 1  # images of 16 x 16 patches between runs of text
        base = at - at % 256
        offset = torch.randint(0, 4096, (1,), generator=g, device=DEV)
        s["positions"] = (offset + torch.stack([torch.where(image, base, at), torch.where(image, base + at % 256 // 16, at),
                                                torch.where(image, base + at % 16, at)])).to(torch.int32)
        s["numbers"] = at.to(torch.int32)
        s["axis_of"] = sections(case)
        s["weights"] = torch.rand(n, heads, longest, generator=g, device=DEV)
        s["order"] = torch.zeros(n, heads, longest, dtype=torch.int32, device=DEV)
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
        s["cache"] = binding.KVCache(s["pool"].data_ptr(), layers, bs, heads, dim, blocks, device_layout=case["layout"], dtype=case["dtype"])
    return s


# ---- one pass -------------------------------------------------------------------------------------------------------


def run(s):
    return globals()[("own_" if own else "plain_") + s["case"]["op"]](s)


def own_attend(s):
    s["ops"].kv_attend(s["cache"], s["layer"], s["q"], s["tables"], s["lens"], s["longest"], out=s["out"], lse=s["lse"], window=s["case"]["window"],
                       weights_in=s["had"], weights_out=s["weights"])
    return outputs(s, "out", "lse", "weights")


def own_append(s):
    h, k = s["case"]["q_heads"], s["case"]["kv_heads"]
    qkv = s["qkv"]
    s["ops"].kv_append(s["cache"], s["layer"], qkv[:, :h], qkv[:, h:h + k], qkv[:, h + k:], s["tables"], s["lens"], positions=s["positions"],
                       inv_freq=s["inv_freq"], axis_of=s["axis_of"], halves=s["case"]["halves"], q_out=s["q_out"], seq_starts=s["starts"],
                       weights=s["weights"], order=s["order"], token_order=s["numbers"])
    return outputs(s, "q_out", "pool", "weights", "order")


def own_evict(s):
    c = s["case"]
    s["ops"].kv_evict(s["cache"], s["tables"], s["lens"], s["longest"], keep=c["keep"], recent=c["recent"], sink=c["sink"], weights=s["had"], order=s["ages"],
                      seen=s["seen"], weights_out=s["weights"], order_out=s["order"], lens_out=s["new_lens"])
    return outputs(s, "pool", "weights", "order", "new_lens")


def outputs(s, *names):
    return {k: s[k] for k in names if s[k] is not None}


def planes(s, layer):
    """K and V of one layer as [block][row][head][dim], whatever the pool's layout."""
    p = s["pool"]
    return (p[:, layer, 0], p[:, layer, 1]) if s["case"]["layout"] else (p[layer, 0], p[layer, 1])


def plain_attend(s):
    c, n = s["case"], max(1, s["longest"])
    bs, heads, group, dim = c["block"], c["kv_heads"], c["q_heads"] // c["kv_heads"], c["dim"]
    slot = torch.arange(n, device=DEV)
    lens = s["lens"].long()[:, None]
    live = slot < lens
    seen = live & (slot >= lens - c["window"]) if c["window"] else live
    block = s["tables"].long()[:, slot // bs].clamp(min=0)
    k, v = (torch.where(seen[..., None, None], p[block, slot % bs], 0).float() for p in planes(s, s["layer"]))  # [seq][slot][head][dim]
    q = s["q"].float().reshape(-1, heads, group, dim)
    x = torch.einsum("bhgd,bnhd->bhgn", q, k) * dim ** -0.5
    x = x.masked_fill(~seen[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    e = (x - top.masked_fill(top == -math.inf, 0.0)).exp()
    total = e.sum(-1, keepdim=True)
    p = torch.where(total > 0, e / total, 0.0)
    out = torch.einsum("bhgn,bnhd->bhgd", p, v).reshape(s["q"].shape).to(s["q"].dtype)
    r = {"out": out, "lse": (top + total.log()).reshape(s["lse"].shape)}
    if c["weights"]:
        r["weights"] = torch.where(live[:, None], s["had"] + p.sum(2), s["weights"])
    return r


def plain_append(s):
    c = s["case"]
    h, kh, bs = c["q_heads"], c["kv_heads"], c["block"]
    qkv = s["qkv"].float()
    angle = s["positions"][torch.tensor(s["axis_of"], device=DEV)].float().T * s["inv_freq"]  # [token][frequency]
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]
    rot, rest = qkv[:, :h + kh, :c["rotary"]], qkv[:, :h + kh, c["rotary"]:]
    if c["halves"]:
        x, y = rot.chunk(2, -1)
        rot = torch.cat([x * cos - y * sin, x * sin + y * cos], -1)
    else:
        x, y = rot[..., 0::2], rot[..., 1::2]
        rot = torch.stack([x * cos - y * sin, x * sin + y * cos], -1).flatten(-2)
    qk = torch.cat([rot, rest], -1).to(s["qkv"].dtype)
    token = torch.arange(len(qkv), device=DEV)
    starts = s["starts"].long()
    seq = torch.searchsorted(starts[1:], token, right=True)
    slot = s["lens"].long()[seq] - (starts[seq + 1] - token)
    block = s["tables"].long()[seq, slot // bs]
    kp, vp = planes(s, s["layer"])
    kp[block, slot % bs] = qk[:, h:]
    vp[block, slot % bs] = s["qkv"][:, h + kh:]
    s["weights"][seq, :, slot] = 0.0
    s["order"][seq, :, slot] = s["numbers"][:, None]
    return {"q_out": qk[:, :h], "pool": s["pool"], "weights": s["weights"], "order": s["order"]}


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
    small = live & (lens <= keep)
    stays = stays | small
    hole = ~stays & live & (slot < keep)
    comes = stays & (slot >= keep)
    # the holes and the slots that move, both in ascending order, meet pairwise
    l, b, h, to = hole.nonzero(as_tuple=True)
    src = comes.nonzero(as_tuple=True)[3]
    take = slot.expand(score.shape).clone()
    take[l, b, h, to] = src
    take = take[..., :keep]
    tables = s["tables"].long()
    p = s["pool"]
    planed = p if c["layout"] else p.permute(2, 0, 1, 3, 4, 5)  # [block][layer][K|V][row][head][dim]
    planed[tables[b, to // bs], l, :, to % bs, h] = planed[tables[b, src // bs], l, :, src % bs, h]
    kept = slot[:keep] < lens
    r = {"pool": p, "new_lens": s["lens"].clamp(max=keep)}
    width = min(n, keep)
    for name, old in (("weights", s["had"]), ("order", s["ages"])):
        new = s[name].clone()
        new[..., :width] = torch.where(kept[..., :width], old.gather(-1, take), new[..., :width])
        r[name] = new
    return r


# ---- what a pass cannot do without ----------------------------------------------------------------------------------


def work(case):
    heads, dim, lens = case["kv_heads"], case["dim"], lengths(case)
    if case["op"] == "attend":
        slots = sum(min(n, case["window"]) if case["window"] else n for n in lens)
        ends = case["seqs"] * case["q_heads"]
        weights = 8 * sum(lens) * heads if case["weights"] else 0
        return {"bytes": 4 * slots * heads * dim + weights + ends * (4 * dim + 4) + 4 * sum(-(-n // case["block"]) for n in lens),
                "flops": 4 * slots * case["q_heads"] * dim}
    if case["op"] == "append":
        t = sum(news(case))
        return {"bytes": t * (4 * (case["q_heads"] + 2 * heads) * dim + 8 * heads + 16), "flops": 3 * t * case["rotary"] * (case["q_heads"] + heads)}
    total = 0.0
    for n in lens:
        total += 8 * n + 8 * min(n, case["keep"])  # weight and age of each slot, and of each that stays
        if n > case["keep"]:  # rows that move: the protected new ones, and their share of the others
            tail = n - case["keep"]
            newest = min(case["recent"], tail)
            moved = newest + (tail - newest) * max(0, case["keep"] - case["recent"] - case["sink"]) / max(1, n - case["recent"] - case["sink"])
            total += 8 * dim * moved
    return {"bytes": total * heads * case["layers"], "flops": 0}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "attend":
        return exact_attend(s)
    if case["op"] == "append":
        return exact_append(s)
    return None  # rows, weights and ages are moved, none is computed


def exact_attend(s):
    c = s["case"]
    heads, group, dim, bs = c["kv_heads"], c["q_heads"] // c["kv_heads"], c["dim"], c["block"]
    kp, vp = planes(s, s["layer"])
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device=DEV)
    weights = s["weights"].double() if c["weights"] else None
    for i, n in enumerate(s["lens"].tolist()):
        if n == 0:
            continue
        first = max(0, n - c["window"]) if c["window"] else 0
        ids = s["tables"][i, : -(-n // bs)].long()
        k, v = (p[ids].flatten(0, 1)[first:n].double() for p in (kp, vp))  # [slot][head][dim]
        if weights is not None:
            weights[i, :, :n] = s["had"][i, :, :n].double()
        for h in range(heads):
            q = s["q"][i, h * group:(h + 1) * group].double()
            x = q @ k[:, h].T / math.sqrt(dim)
            total = torch.logsumexp(x, 1)
            p = torch.exp(x - total[:, None])
            out[i, h * group:(h + 1) * group] = p @ v[:, h]
            lse[i, h * group:(h + 1) * group] = total
            if weights is not None:
                weights[i, h, first:n] += p.sum(0)
    return {"out": out, "lse": lse, "weights": weights}


def exact_append(s):
    c = s["case"]
    h, heads, bs, half = c["q_heads"], c["kv_heads"], c["block"], c["rotary"] // 2
    x = s["qkv"].double()
    y = x.clone()
    f = torch.arange(half, device=DEV)
    low, high = (f, f + half) if c["halves"] else (2 * f, 2 * f + 1)
    for a in range(3):
        pick = torch.tensor([q for q in range(half) if s["axis_of"][q] == a], dtype=torch.long, device=DEV)
        turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), s["positions"][a].double()[:, None] * s["inv_freq"].double()[pick])
        z = torch.complex(x[:, :h + heads, low[pick]], x[:, :h + heads, high[pick]]) * turn[:, None]
        y[:, :h + heads, low[pick]] = z.real
        y[:, :h + heads, high[pick]] = z.imag
    pool = s["pool"].double()
    if c["layout"]:
        pool = pool.permute(1, 2, 0, 3, 4, 5)
    weights, row = s["weights"].double(), 0
    for i, (n, new) in enumerate(zip(s["lens"].tolist(), news(c))):
        slot = torch.arange(n - new, n, device=DEV)
        block = s["tables"][i].long()[slot // bs]
        pool[s["layer"], 0, block, slot % bs] = y[row:row + new, h:h + heads]
        pool[s["layer"], 1, block, slot % bs] = y[row:row + new, h + heads:]
        weights[i, :, slot] = 0.0
        row += new
    if c["layout"]:
        pool = pool.permute(2, 0, 1, 3, 4, 5)
    return {"q_out": y[:, :h], "pool": pool, "weights": weights, "order": None}
