"""The operators on the device cache against plain statements in 64 bits: kv_append, kv_attend, kv_evict."""
import ctypes as C
import math

import pytest
import torch

import ops_reference as R
from paper_2601_20309_b200 import binding as B

pytestmark = pytest.mark.gpu
NAN = float("nan")


@pytest.fixture(scope="module")
def ops():
    with B.KVOps(0) as o:
        yield o


def randn(g, *shape, dtype="bf16", scale=1.0):
    return (torch.randn(*shape, generator=g) * scale).to(R.TYPES[dtype]).cuda()


# ---- attend ---------------------------------------------------------------------------------------------------------


def run_attend(ops, c, q, window=0, weights=True, layer=1, scale=0.0, max_len=None):
    n, heads = q.shape[:2]
    out = torch.full_like(q, NAN)
    lse = torch.full((n, heads), NAN, device="cuda")
    w_in = w_out = None
    if weights:
        w_in = torch.rand(n, c.heads, c.longest + 5, device="cuda")
        w_out = torch.full_like(w_in, -3.0)
    ops.kv_attend(c.handle(B), layer, q, c.tables, c.lens, max_len or c.longest, out=out, lse=lse, window=window, scale=scale,
                  weights_in=w_in, weights_out=w_out)
    ops.kv_ops_sync()
    return out.double().cpu(), lse.double().cpu(), w_in, w_out


def check_attend(c, q, got, window=0, layer=1, scale=None):
    out, lse, w_in, w_out = got
    group = q.shape[1] // c.heads
    for i, row in enumerate(R.attend(c, layer, q, window, scale)):
        n = c.lens_list[i]
        for g, (o, z, p, score, bound, total) in enumerate(row):
            assert ((out[i, g] - o).abs() <= bound).all(), (i, g, n, float(((out[i, g] - o).abs() - bound).max()))
            if z == -math.inf:
                assert lse[i, g] == -math.inf
            else:
                assert abs(lse[i, g] - z) <= score + 2.0 ** -20 * (1 + abs(z)), (i, g, n)
        if w_out is not None:
            wi, wo = w_in.double().cpu(), w_out.double().cpu()
            for h in range(c.heads):
                part = row[h * group:(h + 1) * group]
                want = wi[i, h, :n] + sum(p for _, _, p, _, _, _ in part)
                tol = sum(p * (2 * s + 2.0 ** -18) for _, _, p, s, _, _ in part) + 2.0 ** -22 * want.abs()
                assert ((wo[i, h, :n] - want).abs() <= tol).all(), (i, h, n)
                assert (wo[i, h, n:] == -3.0).all()


# lengths around tiles, blocks and splits; head dimensions below, at and above the usual ones; groups that fill no tile
ATTEND = [
    # lens, q_heads, kv_heads, dim, bs, dtype, layout, window
    ([1], 1, 1, 64, 16, "bf16", 0, 0),
    ([0], 4, 2, 128, 16, "bf16", 0, 0),
    ([37], 32, 8, 128, 16, "bf16", 0, 0),
    ([1, 15, 16, 17, 31, 32, 33], 8, 8, 128, 16, "bf16", 0, 0),
    ([127, 0, 128, 129, 300, 1000, 2500], 32, 8, 128, 16, "bf16", 0, 0),
    ([63, 64, 65, 0, 511, 513], 16, 8, 128, 64, "f16", 1, 0),
    ([5, 700, 23, 25], 15, 3, 80, 24, "bf16", 1, 333),
    ([200, 7, 90], 14, 2, 96, 8, "f16", 0, 16),
    ([4099], 8, 1, 128, 64, "bf16", 0, 0),
    ([9000, 3], 16, 1, 128, 32, "f16", 0, 0),
    ([700, 40, 0, 12], 40, 5, 64, 16, "bf16", 0, 0),
    ([150, 333], 4, 2, 256, 16, "bf16", 0, 0),
    ([150, 333], 12, 2, 192, 7, "f16", 1, 100),
    ([50, 170], 26, 13, 72, 5, "bf16", 0, 0),
    ([400, 61], 71, 1, 64, 16, "bf16", 0, 0),
    ([90, 1300], 48, 2, 128, 16, "bf16", 0, 0),
    ([100, 260], 40, 40, 128, 16, "f16", 0, 0),
    ([33, 70, 129], 12, 12, 8, 1, "bf16", 0, 0),
    ([130, 260], 6, 3, 112, 3, "bf16", 0, 1),
    ([3] * 300, 4, 2, 64, 16, "bf16", 0, 0),
    ([(i * 37) % 200 for i in range(150)], 8, 4, 128, 16, "f16", 0, 0),
]


@pytest.mark.parametrize("lens,hq,hk,dim,bs,dtype,layout,window", ATTEND)
@pytest.mark.parametrize("weights", [True, False])
def test_attend(ops, lens, hq, hk, dim, bs, dtype, layout, window, weights):
    c = R.Cache(lens, hk, dim, bs, dtype, layout, seed=len(lens) + dim)
    q = randn(c.g, len(lens), hq, dim, dtype=dtype, scale=2.0)
    before = c.pool.clone()
    got = run_attend(ops, c, q, window, weights)
    check_attend(c, q, got, window)
    assert torch.equal(before.view(torch.int16), c.pool.view(torch.int16))      # the cache is only read


@pytest.mark.parametrize("spread", [0.05, 8.0])
def test_attend_flat_and_peaked_scores(ops, spread):
    c = R.Cache([1500, 260], 2, 128, 16, seed=3)
    q = randn(c.g, 2, 8, 128, scale=spread)
    check_attend(c, q, run_attend(ops, c, q, scale=0.3), scale=0.3)


def test_attend_growing_maximum(ops):
    """Scores that rise from slot to slot, so that every tile moves the running maximum; and that fall."""
    for sign in (1.0, -1.0):
        c = R.Cache([1100, 40], 1, 64, 16, seed=4)
        for i, n in enumerate(c.lens_list):
            k = torch.zeros(n, 1, 64)
            k[:, 0, 0] = torch.arange(n) * sign / 16
            c.write(i, 1, 0, k.to(c.tdtype))
        q = torch.zeros(2, 4, 64, dtype=c.tdtype, device="cuda")
        q[:, :, 0] = torch.tensor([1.0, 2.0, 8.0, 0.5])
        check_attend(c, q, run_attend(ops, c, q, scale=1.0), scale=1.0)


def test_attend_strides_and_reuse_in_place(ops):
    """q as a slice of q, k, v side by side, out in rows of a wider buffer, tables and weights in wider ones; weights in place."""
    c = R.Cache([70, 0, 33], 2, 128, 16, seed=5)
    wide = randn(c.g, 3, 8 + 4, 128)
    q = wide[:, 1:9]
    store = torch.full((3, 10, 136), 7.0, dtype=c.tdtype, device="cuda")
    out = store[:, 1:9, 3:131]
    tables = torch.full((3, 40), -1, dtype=torch.int32, device="cuda")
    tables[:, 2:2 + c.width] = c.tables
    big = torch.rand(3, 5, 300, device="cuda")
    w = big[:, 1:3, 2:]
    had, kept = w.clone(), big.clone()
    ops.kv_attend(c.handle(B), 0, q, tables[:, 2:], c.lens, 70, out=out, weights_in=w, weights_out=w)
    ops.kv_ops_sync()
    plain = out.double().cpu(), None, had, w.clone()
    for i, row in enumerate(R.attend(c, 0, q)):
        for g, (o, _, _, _, bound, _) in enumerate(row):
            assert ((plain[0][i, g] - o).abs() <= bound).all()
        for h in range(2):
            n = c.lens_list[i]
            want = had[i, h, :n].double().cpu() + sum(p for _, _, p, _, _, _ in row[4 * h:4 * h + 4])
            assert torch.allclose(w[i, h, :n].double().cpu(), want, rtol=1e-5, atol=1e-6)
            assert torch.equal(w[i, h, n:], had[i, h, n:])
    kept[:, 1:3, 2:] = w
    assert torch.equal(big, kept)
    edge = store.clone()
    edge[:, 1:9, 3:131] = 7.0
    assert (edge == 7.0).all()
    ref = out.clone()
    ops.kv_attend(c.handle(B), 0, q, c.tables, c.lens, 70, out=q)               # out over q
    ops.kv_ops_sync()
    assert torch.equal(q, ref)


def test_attend_infinities_and_nan_in_live_slots(ops):
    c = R.Cache([40, 40, 40, 40, 40], 2, 64, 16, seed=6)
    q = randn(c.g, 5, 4, 64).abs() + 0.5
    rows = [c.read(i, 1, 0).cpu() for i in range(5)]
    rows[0][:, 0] = -math.inf           # every score of head 0 is -inf: nothing is left
    rows[1][7, 0] = -math.inf           # one slot of weight 0
    rows[2][7, 0, 3] = NAN              # poisons head 0 and no other
    rows[3][39, 1] = math.inf           # inf - inf
    for i in range(5):
        c.write(i, 1, 0, rows[i])
    v = c.read(4, 1, 1).cpu()
    v[11, 1, 5] = math.inf
    c.write(4, 1, 1, v)
    out, lse, w_in, w_out = run_attend(ops, c, q)
    ref = R.attend(c, 1, q)
    for i, g in [(i, g) for i in range(5) for g in range(4)]:
        o, z, p, score, bound, _ = ref[i][g]
        if (i, g) in ((2, 0), (2, 1), (3, 2), (3, 3)):
            assert out[i, g].isnan().all() and lse[i, g].isnan()
            continue
        fin = o.isfinite()
        assert ((out[i, g] - o)[fin].abs() <= bound[fin]).all() and torch.equal(out[i, g].isfinite(), fin), (i, g)
        assert out[i, g, ~fin].tolist() == o[~fin].tolist()
    assert (out[0, :2] == 0).all() and (lse[0, :2] == -math.inf).all()
    assert torch.equal(w_out[0, 0, :40], w_in[0, 0, :40])
    assert w_out[1, 0, 7] == w_in[1, 0, 7]
    assert w_out[2, 0, :40].isnan().all() and w_out[3, 1, :40].isnan().all()
    assert w_out[2, 1, :40].isfinite().all() and w_out[3, 0, :40].isfinite().all()


def test_attend_offsets_beyond_32_bits(ops):
    blocks = (5 << 30) // (4 * 64 * 4 * 128 * 2) + 1                    # 5 GiB: V of layer 1 begins at 3.75 GiB and ends beyond 2^32
    for layout in (0, 1):
        c = R.Cache([700, 90], 4, 128, 64, layout=layout, seed=7, blocks=blocks)
        q = randn(c.g, 2, 16, 128)
        check_attend(c, q, run_attend(ops, c, q))


def test_attend_one_long_sequence(ops):
    c = R.Cache([70001], 1, 64, 16, seed=8, layers=1)
    q = randn(c.g, 1, 4, 64)
    check_attend(c, q, run_attend(ops, c, q, layer=0), layer=0)


def test_attend_gives_the_same_bits_twice_and_under_a_loose_bound(ops):
    c = R.Cache([2500, 17, 800, 1], 8, 128, 16, seed=9, width=400)
    q = randn(c.g, 4, 32, 128)
    a, b, d = run_attend(ops, c, q), run_attend(ops, c, q), run_attend(ops, c, q, max_len=6000, weights=False)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert torch.allclose(a[0], d[0], atol=2.0 ** -6)
    check_attend(c, q, d)


def test_attend_on_a_stream_and_in_a_graph():
    s = torch.cuda.Stream()
    c = R.Cache([400, 33, 0], 2, 128, 16, seed=10)
    q = randn(c.g, 3, 8, 128)
    with B.KVOps(0, s.cuda_stream) as o:
        o.kv_ops_reserve(o.kv_attend_workspace(c.handle(B), 3, 8, 400))
        out = torch.zeros_like(q)
        w = torch.zeros(3, 2, 400, device="cuda")
        torch.cuda.synchronize()
        cache = c.handle(B)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.stream(s):
            o.kv_attend(cache, 1, q, c.tables, c.lens, 400, out=out, weights_out=w)
            o.kv_ops_sync()
            first = out.clone(), w.clone()
            torch.cuda.synchronize()
            with torch.cuda.graph(g, stream=s):
                o.kv_attend(cache, 1, q, c.tables, c.lens, 400, out=out, weights_out=w)
        q2 = randn(c.g, 3, 8, 128)
        q.copy_(q2)
        c.lens_list = [390, 33, 5]
        c.tables_cpu[2, 0] = c.tables_cpu[1, 0]
        c.tables.copy_(c.tables_cpu)
        c.lens.copy_(torch.tensor(c.lens_list))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for i, row in enumerate(R.attend(c, 1, q)):
            for h, (want, _, _, _, bound, _) in enumerate(row):
                assert ((out[i, h].double().cpu() - want).abs() <= bound).all()
        assert not torch.equal(first[0], out)
        del g
        torch.cuda.synchronize()


def test_bad_ids_and_lengths_are_skipped_and_reported():
    c = R.Cache([100, 100, 60], 2, 64, 16, seed=11)
    q = randn(c.g, 3, 4, 64)
    good = c.tables.clone()
    with B.KVOps(0) as o:
        c.tables[1, 3] = c.nb                       # one block outside the pool: its 16 slots count as masked
        out = torch.full_like(q, NAN)
        o.kv_attend(c.handle(B), 1, q, c.tables, c.lens, 100, out=out)
        assert o.kv_ops_sync(check=False) == B.KV_ERR_RANGE
        assert "block id" in o.kv_ops_last_error()
        assert o.kv_ops_sync(check=False) == B.KV_ERR_RANGE                     # sticky, like the pool's
        got = out.double().cpu()
        ref = R.attend(c_with(c, good), 1, q)
        for i in (0, 2):
            for g, (want, _, _, _, bound, _) in enumerate(ref[i]):
                assert ((got[i, g] - want).abs() <= bound).all()
        k, v = (c_with(c, good).read(1, 1, kv).double().cpu() for kv in range(2))
        live = torch.tensor([s for s in range(100) if s // 16 != 3])
        for g in range(4):
            p = ((k[live, g // 2] * q[1, g].double().cpu()).sum(-1) / 8).softmax(0)
            assert torch.allclose(got[1, g], p @ v[live, g // 2], atol=0.02)
    for bad in (-1, 101):
        with B.KVOps(0) as o:
            c.lens[2] = bad
            lse = torch.zeros(3, 4, device="cuda")
            o.kv_attend(c.handle(B), 1, q, good, c.lens, 100, out=out, lse=lse)
            assert o.kv_ops_sync(check=False) == B.KV_ERR_RANGE
            assert "length" in o.kv_ops_last_error()
            assert (out[2] == 0).all() and (lse[2] == -math.inf).all()
            assert lse[:2].isfinite().all()


def c_with(c, tables):
    c.tables_cpu = tables.cpu()
    return c


# ---- append ---------------------------------------------------------------------------------------------------------

APPEND = [
    # before, new, q_heads, kv_heads, dim, bs, dtype, layout, rotary, halves, axes
    ([0], [1], 4, 2, 64, 16, "bf16", 0, 64, True, 1),
    ([99], [1], 32, 8, 128, 16, "bf16", 0, 128, True, 3),
    ([15, 16, 17, 40], [1, 1, 1, 1], 8, 8, 128, 16, "f16", 1, 128, False, 3),
    ([0, 3, 30], [70, 1, 33], 16, 2, 128, 16, "bf16", 0, 128, True, 3),
    ([10, 0, 5], [20, 1, 50], 15, 3, 80, 24, "bf16", 1, 40, True, 2),
    ([7, 0], [5, 9], 6, 3, 72, 5, "f16", 0, 30, False, 4),
    ([0, 100], [300, 2], 8, 1, 256, 64, "bf16", 0, 256, False, 3),
    ([0], [40], 10, 5, 8, 3, "bf16", 0, 2, True, 1),
    ([4, 4], [3, 4], 4, 4, 96, 16, "f16", 0, 0, True, 1),
    ([0] * 150, [1] * 150, 4, 2, 64, 16, "bf16", 0, 64, True, 3),
    ([0, 9], [5, 3], 3, 1, 8, 16, "bf16", 0, 0, True, 1),
    ([0, 9], [5, 3], 3, 1, 8, 16, "f16", 0, 8, False, 1),
    ([20, 0], [3000, 900], 6, 3, 128, 16, "bf16", 0, 96, False, 2),
    ([3] * 70, [i % 5 + 1 for i in range(70)], 7, 7, 112, 16, "bf16", 0, 112, True, 3),
]


def append_case(before, new, hq, hk, dim, bs, dtype, layout, rotary, axes, far=0, seed=1):
    lens = [a + b for a, b in zip(before, new)]
    c = R.Cache(lens, hk, dim, bs, dtype, layout, seed=seed)
    t = sum(new)
    half = rotary // 2
    a = {"qkv": randn(c.g, t, hq + 2 * hk, dim, dtype=dtype), "inv_freq": (10000.0 ** (-torch.arange(half) / max(1, half))).float().cuda(),
         "positions": (torch.randint(0, 3000, (axes, t), generator=c.g, dtype=torch.int32) + far).cuda(),
         "axis_of": [(5 * f // max(1, half) + f) % axes for f in range(half)],
         "starts": torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32).cuda(),
         "numbers": torch.randint(0, 1 << 30, (t,), generator=c.g, dtype=torch.int32).cuda()}
    return c, a


def check_append(c, a, before, new, hq, rotary, halves, q_out, pool_before, layer=1):
    """A turned value is off by its rounding, and by a few float32 units of the pair's size (sine and cosine 2^-21, two products)."""
    hk, u = c.heads, R.UNIT[c.dtype]
    x = a["qkv"].double().cpu()
    angle = a["positions"].double().cpu()[torch.tensor(a["axis_of"], dtype=torch.long)].T * a["inv_freq"].double().cpu()
    y = R.rotate(x[:, :hq + hk], angle[:, None], halves)
    size = x[:, :hq + hk].abs().amax(-1, keepdim=True) * 2
    bound = u * y.abs() + 2.0 ** -19 * size + (2.0 ** -25 if c.dtype == "f16" else 0.0)
    if q_out is not None:
        assert ((q_out.double().cpu() - y[:, :hq]).abs() <= bound[:, :hq]).all()
        if rotary < c.dim:
            assert torch.equal(q_out[..., rotary:], a["qkv"][:, :hq, rotary:])
    row = 0
    after = c.pool.clone()
    for i, n in enumerate(new):
        slots = torch.arange(before[i], before[i] + n)
        b, r = c.where(i, slots)
        k, v = (c.plane(layer, kv)[b, r] for kv in range(2))
        assert ((k.double().cpu() - y[row:row + n, hq:]).abs() <= bound[row:row + n, hq:]).all(), i
        assert torch.equal(v, a["qkv"][row:row + n, hq + hk:])
        for kv in range(2):
            p = (after[:, layer, kv] if c.layout else after[layer, kv])
            p[b, r] = (pool_before[:, layer, kv] if c.layout else pool_before[layer, kv])[b, r]
        row += n
    assert torch.equal(after.view(torch.int16), pool_before.view(torch.int16))  # nothing else was written


@pytest.mark.parametrize("before,new,hq,hk,dim,bs,dtype,layout,rotary,halves,axes", APPEND)
def test_append(ops, before, new, hq, hk, dim, bs, dtype, layout, rotary, halves, axes):
    c, a = append_case(before, new, hq, hk, dim, bs, dtype, layout, rotary, axes)
    n, t = len(new), sum(new)
    q_out = torch.full((t, hq, dim), NAN, dtype=c.tdtype, device="cuda")
    w = torch.full((n, hk, c.longest + 3), 5.0, device="cuda")
    order = torch.full((n, hk, c.longest + 3), -9, dtype=torch.int32, device="cuda")
    start = c.pool.clone()
    qkv = a["qkv"]
    ops.kv_append(c.handle(B), 1, qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:], c.tables, c.lens, positions=a["positions"], inv_freq=a["inv_freq"],
                  axis_of=a["axis_of"], halves=halves, q_out=q_out, seq_starts=a["starts"], weights=w, order=order, token_order=a["numbers"])
    ops.kv_ops_sync()
    check_append(c, a, before, new, hq, rotary, halves, q_out, start)
    row = 0
    for i in range(n):
        live = torch.zeros(w.shape[2], dtype=torch.bool)
        live[before[i]:before[i] + new[i]] = True
        assert (w[i][:, live.cuda()] == 0).all() and (w[i][:, ~live.cuda()] == 5).all()
        assert (order[i][:, live.cuda()] == a["numbers"][row:row + new[i]]).all() and (order[i][:, ~live.cuda()] == -9).all()
        row += new[i]


def test_append_far_positions_keep_their_angle(ops):
    """At positions around two million a float32 product is off by a tenth of a radian; the call's is not."""
    c, a = append_case([5, 0], [1, 30], 8, 2, 128, 16, "f16", 0, 128, 3, far=2_000_000)
    q_out = torch.zeros(31, 8, 128, dtype=c.tdtype, device="cuda")
    start, qkv = c.pool.clone(), a["qkv"]
    ops.kv_append(c.handle(B), 1, qkv[:, :8], qkv[:, 8:10], qkv[:, 10:], c.tables, c.lens, positions=a["positions"], inv_freq=a["inv_freq"],
                  axis_of=a["axis_of"], q_out=q_out, seq_starts=a["starts"])
    ops.kv_ops_sync()
    check_append(c, a, [5, 0], [1, 30], 8, 128, True, q_out, start)


@pytest.mark.parametrize("shift", [0, 1, 4])
def test_append_in_place_strides_and_unaligned_rows(ops, shift):
    """q turned in place in a wider buffer whose rows start anywhere; no axis list; one token per sequence; numbers from the positions."""
    c, a = append_case([3, 16, 0], [1, 1, 1], 5, 3, 80, 16, "bf16", 0, 80, 2)
    a["axis_of"] = [0] * 40
    store = torch.zeros(3, 12, 80 + 7, dtype=c.tdtype, device="cuda")
    view = store[:, :11, shift:shift + 80]
    view.copy_(a["qkv"])
    start = c.pool.clone()
    order = torch.zeros(3, 3, 17, dtype=torch.int32, device="cuda")
    ops.kv_append(c.handle(B), 1, view[:, :5], view[:, 5:8], view[:, 8:], c.tables, c.lens, positions=a["positions"], inv_freq=a["inv_freq"], q_out=view[:, :5],
                  order=order)
    ops.kv_ops_sync()
    check_append(c, a, [3, 16, 0], [1, 1, 1], 5, 80, True, view[:, :5], start)
    assert torch.equal(view[:, 5:], a["qkv"][:, 5:])
    for i, s in enumerate((3, 16, 0)):
        assert (order[i, :, s] == a["positions"][0, i]).all()
    edge = store.clone()
    edge[:, :11, shift:shift + 80] = 0
    assert (edge == 0).all()


def test_append_without_q_idle_places_and_bad_ids():
    c, a = append_case([3, 16, 20], [1, 1, 1], 4, 2, 64, 16, "bf16", 0, 64, 1)
    qkv = a["qkv"]
    lens, tables = c.lens.clone(), c.tables.clone()
    start = c.pool.clone()
    with B.KVOps(0) as o:                               # no q at all; the middle sequence is an idle place: not written, not an error
        lens[1] = 0
        o.kv_append(c.handle(B), 1, None, qkv[:, 4:6], qkv[:, 6:], tables, lens, positions=a["positions"], inv_freq=a["inv_freq"])
        assert o.kv_ops_sync() == 0
        after = c.pool.clone()
        b, r = c.where(1, torch.tensor([16]))
        assert torch.equal(after.view(torch.int16)[:, :, b, r], start.view(torch.int16)[:, :, b, r])
        c.plane(1, 0)[b, r] = R.rotate(qkv[1:2, 4:6].double().cpu(), (a["positions"][0, 1].cpu() * a["inv_freq"].double().cpu()), True).to(c.tdtype).cuda()
        c.plane(1, 1)[b, r] = qkv[1:2, 6:]
        check_append(c, a, [3, 16, 20], [1, 1, 1], 4, 64, True, None, start)
    for what in ("block", "length"):
        c.pool.copy_(start)
        lens, tables = c.lens.clone(), c.tables.clone()
        if what == "block":
            tables[2, 1] = -1
        else:
            lens[2] = -5
        q_out = torch.zeros(3, 4, 64, dtype=c.tdtype, device="cuda")
        with B.KVOps(0) as o:
            o.kv_append(c.handle(B), 1, qkv[:, :4], qkv[:, 4:6], qkv[:, 6:], tables, lens, positions=a["positions"], inv_freq=a["inv_freq"], q_out=q_out)
            assert o.kv_ops_sync(check=False) == B.KV_ERR_RANGE
        b, r = c.where(2, torch.tensor([20]))
        assert torch.equal(c.plane(1, 0)[b, r].view(torch.int16), (start[1, 0])[b, r].view(torch.int16))
        assert (q_out[2] != 0).any()


def test_append_does_not_write_past_the_rows_of_weights_and_order():
    c, a = append_case([3, 16, 20], [1, 1, 1], 4, 2, 64, 16, "bf16", 0, 64, 1)
    qkv, start = a["qkv"], c.pool.clone()
    big = torch.full((3, 2, 40), 5.0, device="cuda")
    with B.KVOps(0) as o:
        o.kv_append(c.handle(B), 1, None, qkv[:, 4:6], qkv[:, 6:], c.tables, c.lens, positions=a["positions"], inv_freq=a["inv_freq"], weights=big[:, :, :17])
        assert o.kv_ops_sync(check=False) == B.KV_ERR_RANGE             # slots 3 and 16 fit, slot 20 does not
    assert (big[0, :, 3] == 0).all() and (big[1, :, 16] == 0).all()
    assert (big[2] == 5).all() and (big[:, :, 17:] == 5).all()
    b, r = c.where(2, torch.tensor([20]))
    assert torch.equal(c.pool.view(torch.int16)[1, :, b, r], start.view(torch.int16)[1, :, b, r])


def test_append_offsets_beyond_32_bits(ops):
    blocks = (5 << 30) // (4 * 64 * 4 * 128 * 2) + 1
    for layout in (0, 1):
        c = R.Cache([130, 64], 4, 128, 64, layout=layout, seed=7, blocks=blocks)
        x = randn(c.g, 2, 8, 128)
        ops.kv_append(c.handle(B), 1, None, x[:, :4], x[:, 4:], c.tables, c.lens, positions=torch.zeros(1, 2, dtype=torch.int32, device="cuda"),
                      inv_freq=torch.ones(64, device="cuda"))
        ops.kv_ops_sync()
        for i, s in enumerate((129, 63)):
            b, r = c.where(i, torch.tensor([s]))
            assert torch.equal(c.plane(1, 0)[b, r][0], x[i, :4]) and torch.equal(c.plane(1, 1)[b, r][0], x[i, 4:])


# ---- evict ----------------------------------------------------------------------------------------------------------

EVICT = [
    # lens, kv_heads, dim, bs, dtype, layout, layers, keep, recent, sink
    ([2], 1, 64, 16, "bf16", 0, 1, 1, 0, 0),
    ([100], 8, 128, 16, "bf16", 0, 2, 64, 16, 4),
    ([64, 65, 63, 0, 128, 1], 2, 128, 16, "f16", 1, 3, 64, 8, 0),
    ([300, 257, 299], 3, 80, 24, "bf16", 0, 2, 256, 100, 3),
    ([1000, 31], 2, 72, 5, "f16", 0, 2, 30, 10, 20),
    ([700], 5, 256, 64, "bf16", 1, 1, 699, 0, 0),
    ([2500, 40, 2049], 1, 64, 16, "bf16", 0, 2, 2048, 1, 4),
    ([5000, 4100], 2, 8, 1, "bf16", 0, 1, 500, 500, 0),
    ([9000], 1, 128, 64, "f16", 0, 1, 4500, 64, 4),
    ([130] * 60, 2, 64, 16, "bf16", 0, 4, 100, 5, 1),
    ([17000, 9], 2, 64, 64, "bf16", 0, 1, 1000, 10, 1),
]


# lengths past what one CTA, a cluster of small CTAs and a cluster of large ones hold as keys; a loose bound of the length
LONG = [([4097, 5], 2, 8, 16, 4000, 40, 4, 0), ([40000, 300, 20000], 1, 8, 16, 15000, 0, 0, 0), ([140001], 1, 8, 64, 70000, 128, 4, 0),
        ([140001], 1, 8, 64, 300, 0, 0, 0), ([300, 200], 3, 64, 16, 120, 7, 3, 40000), ([300], 1, 64, 16, 290, 7, 3, 200000), ([9000] * 40, 4, 8, 16, 8900, 0, 1, 0)]


@pytest.mark.parametrize("kind", ["plain", "ties", "special"])
@pytest.mark.parametrize("lens,heads,dim,bs,keep,recent,sink,bound", LONG)
def test_evict_long(ops, lens, heads, dim, bs, keep, recent, sink, bound, kind):
    c = R.Cache(lens, heads, dim, bs, layers=1, seed=keep, width=-(-max(bound, max(lens)) // bs))
    w, order = metadata(c, kind, c.g)
    w, order = (torch.nn.functional.pad(x, (0, max(0, bound - x.shape[-1]))) for x in (w, order))
    seen = [n + 2 for n in lens]
    pool, w2, o2 = expect_evict(c, w, order, keep, recent, sink, seen)
    wd, od = w.cuda(), order.cuda()
    w_out = torch.full((1, len(lens), heads, keep), -5.0, device="cuda")
    o_out = torch.full(w_out.shape, -5, dtype=torch.int32, device="cuda")
    ops.kv_evict(c.handle(B), c.tables, c.lens, bound or c.longest, keep=keep, recent=recent, sink=sink, weights=wd, order=od,
                 seen=torch.tensor(seen, dtype=torch.int32).cuda(), weights_out=w_out, order_out=o_out)
    ops.kv_ops_sync()
    assert torch.equal(c.pool.view(torch.int16), pool.view(torch.int16))
    for i, n in enumerate(lens):
        m = min(n, keep)
        assert torch.equal(w_out[:, i, :, :m].cpu().view(torch.int32), w2[:, i, :, :m].contiguous().view(torch.int32))
        assert torch.equal(o_out[:, i, :, :m].cpu(), o2[:, i, :, :m])
        assert (w_out[:, i, :, m:] == -5).all()


def metadata(c, kind, g):
    shape = (c.layers, len(c.lens_list), c.heads, c.longest + 3)
    w = torch.rand(shape, generator=g)
    if kind == "ties":
        w = (w * 4).floor() / 4 * torch.where(torch.rand(shape, generator=g) < 0.1, -1.0, 1.0)   # many equals, -0 among them
    elif kind == "special":
        pick = torch.randint(0, 8, shape, generator=g)
        for n, x in enumerate((NAN, math.inf, -math.inf, -0.0, 1e-42, -3.5)):
            w[pick == n] = x
    order = torch.rand(shape, generator=g).argsort(-1).to(torch.int32)
    return w, order


def expect_evict(c, w, order, keep, recent, sink, seen):
    """(pool, weights, order) after the call, by the definition."""
    pool, w2, o2 = c.pool.clone(), w.clone(), order.clone()
    planed = pool if c.layout else pool.permute(2, 0, 1, 3, 4, 5)
    source = c.pool if c.layout else c.pool.permute(2, 0, 1, 3, 4, 5)
    for l in range(c.layers):
        for i, n in enumerate(c.lens_list):
            for h in range(c.heads):
                pairs = R.evict(w[l, i, h], order[l, i, h], n, keep, recent, sink, seen[i])
                if not pairs:
                    continue
                d, s = (torch.tensor(x) for x in zip(*pairs))
                db, dr = c.where(i, d)
                sb, sr = c.where(i, s)
                planed[db, l, :, dr, h] = source[sb, l, :, sr, h]
                w2[l, i, h, d], o2[l, i, h, d] = w[l, i, h, s], order[l, i, h, s]
    return pool, w2, o2


@pytest.mark.parametrize("kind", ["plain", "ties", "special"])
@pytest.mark.parametrize("lens,heads,dim,bs,dtype,layout,layers,keep,recent,sink", EVICT)
def test_evict(ops, lens, heads, dim, bs, dtype, layout, layers, keep, recent, sink, kind):
    c = R.Cache(lens, heads, dim, bs, dtype, layout, layers=layers, seed=keep)
    w, order = metadata(c, kind, c.g)
    seen = [n + 2 for n in lens]
    pool, w2, o2 = expect_evict(c, w, order, keep, recent, sink, seen)
    wd, od = w.cuda(), order.cuda()
    w_out = torch.full((layers, len(lens), heads, keep + 2), -5.0, device="cuda")
    o_out = torch.full(w_out.shape, -5, dtype=torch.int32, device="cuda")
    new = torch.full((len(lens),), -1, dtype=torch.int32, device="cuda")
    start = c.pool.clone()
    args = dict(keep=keep, recent=recent, sink=sink, weights=wd, order=od, seen=torch.tensor(seen, dtype=torch.int32).cuda())
    ops.kv_evict(c.handle(B), c.tables, c.lens, c.longest, weights_out=w_out, order_out=o_out, lens_out=new, **args)
    ops.kv_ops_sync()
    assert torch.equal(c.pool.view(torch.int16), pool.view(torch.int16))
    assert torch.equal(wd.cpu().view(torch.int32), w.view(torch.int32)) and torch.equal(od.cpu(), order)    # inputs only read
    for i, n in enumerate(lens):
        m = min(n, keep)
        assert int(new[i]) == m
        assert torch.equal(w_out[:, i, :, :m].cpu().view(torch.int32), w2[:, i, :, :m].contiguous().view(torch.int32))
        assert torch.equal(o_out[:, i, :, :m].cpu(), o2[:, i, :, :m])
        assert (w_out[:, i, :, m:] == -5).all() and (o_out[:, i, :, m:] == -5).all()
    # in place: the same rows, and nothing beside them
    c.pool.copy_(start)
    ops.kv_evict(c.handle(B), c.tables, c.lens, c.longest, **args)
    ops.kv_ops_sync()
    assert torch.equal(c.pool.view(torch.int16), pool.view(torch.int16))
    assert torch.equal(wd.cpu().view(torch.int32), w2.view(torch.int32)) and torch.equal(od.cpu(), o2)


@pytest.mark.parametrize("lens,keep,layers,heads", [([101, 98, 37, 3], 50, 2, 3), ([1000, 999, 997], 601, 1, 2), ([130, 257, 61, 256] * 10, 99, 4, 4)])
def test_evict_rows_of_whole_quads(ops, lens, keep, layers, heads):
    """Weights and ages whose rows are 16-byte aligned (read four at a time), lengths and numbers to keep that end inside a quad."""
    c = R.Cache(lens, heads, 64, 16, layers=layers, seed=keep)
    bound = -(-c.longest // 4) * 4
    w, order = (torch.nn.functional.pad(x[..., :c.longest], (0, bound + 4 - c.longest)).contiguous() for x in metadata(c, "ties", c.g))
    seen = [n + 1 for n in lens]
    pool, w2, o2 = expect_evict(c, w, order, keep, 7, 2, seen)
    wd, od = w.cuda(), order.cuda()
    c.tables = torch.nn.functional.pad(c.tables, (0, 1), value=-1)       # wide enough for the rounded bound
    w_out = torch.full((layers, len(lens), heads, -(-keep // 4) * 4), -5.0, device="cuda")
    o_out = torch.full(w_out.shape, -5, dtype=torch.int32, device="cuda")
    ops.kv_evict(c.handle(B), c.tables, c.lens, bound, keep=keep, recent=7, sink=2, weights=wd, order=od, seen=torch.tensor(seen, dtype=torch.int32).cuda(),
                 weights_out=w_out, order_out=o_out)
    ops.kv_ops_sync()
    assert torch.equal(c.pool.view(torch.int16), pool.view(torch.int16))
    for i, n in enumerate(lens):
        m = min(n, keep)
        assert torch.equal(w_out[:, i, :, :m].cpu().view(torch.int32), w2[:, i, :, :m].contiguous().view(torch.int32))
        assert torch.equal(o_out[:, i, :, :m].cpu(), o2[:, i, :, :m])
        assert (w_out[:, i, :, m:] == -5).all() and (o_out[:, i, :, m:] == -5).all()


def test_evict_some_layers_without_order(ops):
    """Layers 1 and 2 of four; ages are the slots' own numbers; strided weights; seen = lens."""
    c = R.Cache([90, 70], 2, 64, 16, layers=4, seed=12)
    big = torch.rand(2, 3, 2, 100, generator=c.g)
    slots = torch.arange(100, dtype=torch.int32).expand(2, 2, 2, 100)
    want = c.pool.clone()
    for l in range(2):
        for i, n in enumerate(c.lens_list):
            for h in range(2):
                for d, s in R.evict(big[l, i, h], slots[l, i, h], n, 48, 20, 5, n):
                    (db, dr), (sb, sr) = (c.where(i, torch.tensor([x])) for x in (d, s))
                    want[l + 1, :, db, dr, h] = c.pool[l + 1, :, sb, sr, h]
    w = big.cuda()
    ops.kv_evict(c.handle(B), c.tables, c.lens, 90, keep=48, recent=20, sink=5, weights=w[:, :2], first_layer=1)
    ops.kv_ops_sync()
    assert torch.equal(c.pool.view(torch.int16), want.view(torch.int16))
    assert torch.equal(w[:, 2].cpu(), big[:, 2])


def test_evict_bad_ids_are_skipped_and_reported():
    c = R.Cache([100, 100], 2, 64, 16, layers=1, seed=13)
    w, order = metadata(c, "plain", c.g)
    want = expect_evict(c, w, order, 50, 0, 0, [100, 100])[0]
    bad = c.tables.clone()
    bad[1, 5] = c.nb + 4
    with B.KVOps(0) as o:
        o.kv_evict(c.handle(B), bad, c.lens, 100, keep=50, weights=w.cuda(), order=order.cuda())
        assert o.kv_ops_sync(check=False) == B.KV_ERR_RANGE
    b, _ = c.where(0, torch.arange(100))
    assert torch.equal(c.pool[:, :, b].view(torch.int16), want[:, :, b].view(torch.int16))


def test_evict_offsets_beyond_32_bits(ops):
    blocks = (5 << 30) // (4 * 64 * 4 * 128 * 2) + 1
    for layout in (0, 1):
        c = R.Cache([130, 64], 4, 128, 64, layout=layout, seed=14, blocks=blocks)
        w = torch.rand(2, 2, 4, 130, generator=c.g)
        rows = c.read(0, 1, 1)
        ops.kv_evict(c.handle(B), c.tables, c.lens, 130, keep=65, weights=w.cuda())
        ops.kv_ops_sync()
        for h in range(4):
            for d, s in R.evict(w[1, 0, h], torch.arange(130), 130, 65, 0, 0, 130):
                rows[d, h] = rows[s, h]
        assert torch.equal(c.read(0, 1, 1), rows)


# ---- refusals -------------------------------------------------------------------------------------------------------


def test_refusals_launch_nothing(ops):
    c = R.Cache([40, 40], 2, 64, 16, seed=15)
    q = randn(c.g, 2, 4, 64)
    out = torch.full_like(q, 3.0)
    h = c.handle(B)
    start = c.pool.clone()
    L = B.lib()

    def attend(code, **changes):
        a = B.kv_attend_args_t(layer=1, num_seqs=2, q_heads=4, max_len=40, table_width=c.width, q=q.data_ptr(), q_seq_stride=256, q_head_stride=64,
                               out=out.data_ptr(), out_seq_stride=256, out_head_stride=64, block_tables=c.tables.data_ptr(), table_stride=c.width,
                               lens=c.lens.data_ptr())
        for k, v in changes.items():
            setattr(a, k, v)
        assert L.kv_attend(ops._h, h.address, C.addressof(a)) == code, changes
        assert code == 0 or len(ops.kv_ops_last_error()) > 5

    attend(B.KV_ERR_INVALID_ARG, q=None)
    attend(B.KV_ERR_INVALID_ARG, out=None)
    attend(B.KV_ERR_INVALID_ARG, lens=None)
    attend(B.KV_ERR_INVALID_ARG, block_tables=None)
    attend(B.KV_ERR_INVALID_ARG, num_seqs=-1)
    attend(B.KV_ERR_INVALID_ARG, q_heads=3)
    attend(B.KV_ERR_INVALID_ARG, q_heads=0)
    attend(B.KV_ERR_INVALID_ARG, window=-1)
    attend(B.KV_ERR_INVALID_ARG, max_len=-1)
    attend(B.KV_ERR_INVALID_ARG, max_len=c.width * 16 + 1)
    attend(B.KV_ERR_INVALID_ARG, table_width=0)
    attend(B.KV_ERR_INVALID_ARG, weights_in=out.data_ptr())
    attend(B.KV_ERR_RANGE, layer=2)
    attend(B.KV_ERR_RANGE, layer=-1)
    attend(0, num_seqs=0, q=None)
    assert L.kv_attend(None, h.address, 0) == B.KV_ERR_INVALID_ARG and L.kv_attend(ops._h, None, 0) == B.KV_ERR_INVALID_ARG
    assert L.kv_attend(ops._h, h.address, 0) == B.KV_ERR_INVALID_ARG
    base = c.pool.data_ptr()
    for code, kw in ((B.KV_ERR_UNSUPPORTED, dict(head_dim=60)), (B.KV_ERR_UNSUPPORTED, dict(head_dim=264)), (B.KV_ERR_INVALID_ARG, dict(device_base=base + 8)),
                     (B.KV_ERR_INVALID_ARG, dict(device_base=None)), (B.KV_ERR_INVALID_ARG, dict(block_size=0)), (B.KV_ERR_INVALID_ARG, dict(num_gpu_blocks=0)),
                     (B.KV_ERR_INVALID_ARG, dict(device_layout=2)), (B.KV_ERR_INVALID_ARG, dict(dtype=2)), (B.KV_ERR_INVALID_ARG, dict(num_layers=0))):
        bad = c.handle(B)
        for k, v in kw.items():
            setattr(bad.c, k, v)
        full = B.kv_attend_args_t(num_seqs=2, q_heads=4, max_len=40)
        assert L.kv_attend(ops._h, bad.address, C.addressof(full)) == code
        a = B.kv_append_args_t(num_seqs=1, num_tokens=1, num_axes=1)
        assert L.kv_append(ops._h, bad.address, C.addressof(a)) == code
        e = B.kv_evict_args_t(num_layers=1, num_seqs=1, keep=4)
        assert L.kv_evict(ops._h, bad.address, C.addressof(e)) == code
    with pytest.raises(ValueError):
        ops.kv_attend(h, 1, q.float(), c.tables, c.lens, 40, out=out)
    with pytest.raises(ValueError):
        ops.kv_attend(h, 1, q.cpu(), c.tables, c.lens, 40, out=out)
    with pytest.raises(ValueError):
        ops.kv_attend(h, 1, q, c.tables.long(), c.lens, 40, out=out)
    with pytest.raises(ValueError):
        ops.kv_attend(h, 1, q, c.tables, c.lens, 40, out=out[:1])
    with pytest.raises(ValueError):
        ops.kv_attend(h, 1, q, c.tables, c.lens, 40, out=out, weights_out=torch.zeros(2, 2, 39, device="cuda"))
    with pytest.raises(B.KVError):
        ops.kv_attend(h, 5, q, c.tables, c.lens, 40, out=out)

    k = randn(c.g, 2, 2, 64)
    pos = torch.zeros(1, 2, dtype=torch.int32, device="cuda")
    freq = torch.ones(32, device="cuda")

    def append(code, freq=freq, pos=pos, **kw):
        assert ops.kv_append(h, kw.pop("layer", 1), kw.pop("q", q), k, k, c.tables, c.lens, positions=pos, inv_freq=freq, check=False, **kw) == code

    append(B.KV_ERR_RANGE, layer=9, q_out=out)
    append(B.KV_ERR_INVALID_ARG, q_out=None)
    append(B.KV_ERR_INVALID_ARG, freq=torch.ones(33, device="cuda"), q_out=out)
    append(B.KV_ERR_RANGE, axis_of=[0] * 31 + [1], q_out=out)
    append(B.KV_ERR_INVALID_ARG, pos=pos.expand(5, 2).contiguous(), q_out=out)
    with pytest.raises(ValueError):
        append(0, axis_of=[0] * 5, q_out=out)
    with pytest.raises(ValueError):
        append(0, q_out=out, token_order=pos[0].long(), order=torch.zeros(2, 2, 50, dtype=torch.int32, device="cuda"))

    w = torch.rand(2, 2, 2, 40, device="cuda")
    age = torch.zeros(2, 2, 2, 40, dtype=torch.int32, device="cuda")

    def evict(code, **kw):
        assert ops.kv_evict(h, c.tables, c.lens, 40, check=False, **{"weights": w, "keep": 10, **kw}) == code, kw

    evict(B.KV_ERR_INVALID_ARG, keep=0)
    evict(B.KV_ERR_INVALID_ARG, recent=8, sink=3)
    evict(B.KV_ERR_INVALID_ARG, recent=-1)
    evict(B.KV_ERR_RANGE, first_layer=1)
    evict(B.KV_ERR_RANGE, first_layer=-1)
    evict(B.KV_ERR_INVALID_ARG, order_out=age)
    evict(B.KV_ERR_INVALID_ARG, order=age, weights_out=torch.zeros_like(w))
    evict(B.KV_ERR_INVALID_ARG, order=age, order_out=torch.zeros_like(age), weights_out=w)
    evict(B.KV_ERR_INVALID_ARG, lens_out=c.lens)
    with pytest.raises(ValueError):
        evict(0, weights=w[..., :39])
    with pytest.raises(ValueError):
        evict(0, weights=w.double())
    assert ops.kv_ops_sync() == 0
    assert (out == 3.0).all() and torch.equal(start.view(torch.int16), c.pool.view(torch.int16))
    assert B.lib().kv_ops_create(0, None, None) == B.KV_ERR_INVALID_ARG
    assert ops.kv_ops_reserve(-1, check=False) == B.KV_ERR_INVALID_ARG
    with pytest.raises(B.KVError):
        B.KVOps(99)


def test_workspace_does_not_grow_inside_a_capture():
    c = R.Cache([5000], 1, 64, 16, seed=16, layers=1)
    q = randn(c.g, 1, 4, 64)
    out = torch.zeros_like(q)
    w = torch.zeros(1, 1, 5000, device="cuda")
    s = torch.cuda.Stream()
    with B.KVOps(0, s.cuda_stream) as o:
        need = o.kv_attend_workspace(c.handle(B), 1, 4, 5000)
        assert need > 0
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            with torch.cuda.graph(g, stream=s):
                assert o.kv_attend(c.handle(B), 0, q, c.tables, c.lens, 5000, out=out, weights_out=w, check=False) == B.KV_ERR_NOMEM
                out.add_(1)
        o.kv_ops_reserve(need)
        o.kv_attend(c.handle(B), 0, q, c.tables, c.lens, 5000, out=out, weights_out=w)
        assert o.kv_ops_sync() == 0
        check_attend(c, q, (out.double().cpu(), torch.tensor([[r[1] for r in R.attend(c, 0, q)[0]]]), None, None), layer=0)
        del g


def test_pool_gives_its_cache():
    for layout in (0, 1):
        c = R.Cache([40], 2, 64, 16, layout=layout, seed=17)
        with B.KVPool(2, 16, 2, 64, c.nb, 4, c.pool.data_ptr(), device_layout=layout) as pool:
            h, want = pool.kv_pool_cache("bf16"), c.handle(B)
            assert bytes(h.c) == bytes(want.c) and (h.heads, h.dim, h.dtype) == (2, 64, "bf16")
