"""The operators on a cache in 4 bits, and norms in front of the rotation, against plain statements in 64 bits."""
import math

import pytest
import torch

import ops_reference as R
import ops_reference_q4 as Q
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
    for i, row in enumerate(Q.attend(c, layer, q, window, scale)):
        n = c.lens_list[i]
        for g, (o, z, p, score, bound) in enumerate(row):
            assert ((out[i, g] - o).abs() <= bound).all(), (i, g, n, float(((out[i, g] - o).abs() - bound).max()), float(bound.max()))
            if z == -math.inf:
                assert lse[i, g] == -math.inf
            else:
                assert abs(lse[i, g] - z) <= score + 2.0 ** -20 * (1 + abs(z)), (i, g, n)
        if w_out is not None:
            wi, wo = w_in.double().cpu(), w_out.double().cpu()
            for h in range(c.heads):
                part = row[h * group:(h + 1) * group]
                want = wi[i, h, :n] + sum(p for _, _, p, _, _ in part)
                tol = sum(p * (2 * s + 2.0 ** -18) for _, _, p, s, _ in part) + 2.0 ** -22 * want.abs()
                assert ((wo[i, h, :n] - want).abs() <= tol).all(), (i, h, n)
                assert (wo[i, h, n:] == -3.0).all()


# lengths around tiles, blocks and splits; heads of every padding; groups that fill no tile, one, two and more; blocks in which tiles end
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
    ([150, 333], 12, 2, 192, 12, "f16", 1, 100),
    ([50, 170], 26, 13, 72, 4, "bf16", 0, 0),
    ([400, 61], 71, 1, 64, 20, "bf16", 0, 0),
    ([90, 1300], 48, 2, 128, 16, "bf16", 0, 0),
    ([90, 260], 18, 1, 256, 20, "f16", 0, 0),
    ([100, 260], 40, 40, 128, 16, "f16", 0, 0),
    ([33, 70, 129], 12, 12, 8, 4, "bf16", 0, 0),
    ([130, 260], 6, 3, 40, 28, "f16", 0, 1),
    ([3] * 300, 4, 2, 64, 16, "bf16", 0, 0),
    ([(i * 37) % 200 for i in range(150)], 8, 4, 128, 16, "f16", 0, 0),
    # steps of whole blocks of several tiles, and blocks that steps do not hold: with a window, of three tiles, longer than a step
    ([1500, 90, 4], 4, 1, 64, 32, "bf16", 1, 0),
    ([900, 333], 8, 2, 128, 64, "f16", 0, 0),
    ([900, 333], 8, 2, 128, 64, "bf16", 0, 300),
    ([500, 90], 8, 8, 128, 48, "f16", 1, 0),
    ([2100, 5], 16, 1, 256, 128, "bf16", 0, 0),
    ([1100], 9, 1, 128, 512, "bf16", 0, 0),
    ([600, 70], 10, 5, 128, 32, "bf16", 0, 0),
]


@pytest.mark.parametrize("lens,hq,hk,dim,bs,dtype,layout,window", ATTEND)
@pytest.mark.parametrize("weights", [True, False])
def test_attend(ops, lens, hq, hk, dim, bs, dtype, layout, window, weights):
    c = Q.Cache(lens, hk, dim, bs, dtype, layout, seed=len(lens) + dim)
    q = randn(c.g, len(lens), hq, dim, dtype=dtype, scale=2.0)
    before = c.pool.clone()
    got = run_attend(ops, c, q, window, weights)
    check_attend(c, q, got, window)
    assert torch.equal(before, c.pool)      # the cache is only read


@pytest.mark.parametrize("spread", [0.05, 8.0])
def test_attend_flat_and_peaked_scores(ops, spread):
    c = Q.Cache([1500, 260], 2, 128, 16, seed=3)
    q = randn(c.g, 2, 8, 128, scale=spread)
    check_attend(c, q, run_attend(ops, c, q, scale=0.3), scale=0.3)


def test_attend_growing_maximum(ops):
    """Scores that rise from slot to slot, so that the reference moves again and again; and that fall."""
    for sign in (1.0, -1.0):
        c = Q.Cache([1100, 40], 1, 64, 16, seed=4)
        for i, n in enumerate(c.lens_list):
            k = torch.zeros(n, 1, 64)
            k[:, 0, 0] = torch.arange(n) * sign / 16
            c.write(i, 1, 0, k.to(c.tdtype))
        q = torch.zeros(2, 4, 64, dtype=c.tdtype, device="cuda")
        q[:, :, 0] = torch.tensor([1.0, 2.0, 8.0, 0.5])
        check_attend(c, q, run_attend(ops, c, q, scale=1.0), scale=1.0)


@pytest.mark.parametrize("dtype,low,high", [("bf16", 1e-9, 1e9), ("f16", 1e-4, 3e4), ("bf16", 1e9, 1e-9)])
def test_attend_values_that_grow(ops, dtype, low, high):
    """V's sizes, and with them the steps, change by many powers of two along a row, up and down."""
    c = Q.Cache([700, 30], 2, 128, 16, dtype, seed=5)
    for i, n in enumerate(c.lens_list):
        size = torch.logspace(math.log10(low), math.log10(high), n)[:, None, None]
        c.write(i, 1, 1, (torch.randn(n, 2, 128, generator=c.g) * size / 4).to(c.tdtype))
    q = randn(c.g, 2, 8, 128, dtype=dtype)
    check_attend(c, q, run_attend(ops, c, q))


@pytest.mark.parametrize("what", [0.0, 3.0, -65504.0, 1e-30])
def test_attend_groups_of_one_value(ops, what):
    c = Q.Cache([90], 1, 128, 16, seed=6)
    c.write(0, 1, 1, torch.full((90, 1, 128), what).to(c.tdtype))
    q = randn(c.g, 1, 4, 128)
    check_attend(c, q, run_attend(ops, c, q))


def test_attend_not_finite(ops):
    """A group of V that is not finite makes its 32 elements NaN and no others; one of K its row; what is masked nothing."""
    c = Q.Cache([200, 200, 200], 1, 128, 16, seed=7)
    v = c.rows[(0, 1, 1)].clone()
    v[150, 0, 40] = math.inf
    c.write(0, 1, 1, v)
    k = c.rows[(1, 1, 0)].clone()
    k[17, 0, 0] = NAN
    c.write(1, 1, 0, k)
    v = c.rows[(2, 1, 1)].clone()
    k = c.rows[(2, 1, 0)].clone()
    v[:100] = NAN
    k[:100] = NAN
    c.write(2, 1, 1, v)
    c.write(2, 1, 0, k)
    q = randn(c.g, 3, 4, 128)
    out, lse, _, _ = run_attend(ops, c, q, weights=False)
    nan = torch.isnan(out)
    assert nan[0, :, 32:64].all() and not nan[0, :, :32].any() and not nan[0, :, 64:].any()
    assert nan[1].all() and torch.isnan(lse[1]).all()
    window, lse, _, _ = run_attend(ops, c, q, window=100, weights=False)
    assert not torch.isnan(window[2]).any()
    c.write(0, 1, 1, torch.randn(200, 1, 128, generator=c.g).to(c.tdtype))
    c.write(1, 1, 0, torch.randn(200, 1, 128, generator=c.g).to(c.tdtype))
    v[:100] = 0
    k[:100] = 0
    c.write(2, 1, 1, v)
    c.write(2, 1, 0, k)
    again, lse2, _, _ = run_attend(ops, c, q, window=100, weights=False)
    assert torch.equal(window[2], again[2]) and torch.equal(lse[2], lse2[2])
    q[1, 2, 5] = math.inf
    out, _, _, _ = run_attend(ops, c, q, weights=False)
    assert torch.isnan(out[1, 2]).all() and not torch.isnan(out[1, [0, 1, 3]]).any()


def test_attend_f16_is_as_fine_as_its_type(ops):
    """Over many slots the roundings of the products are as small as the output's: each has 2^-11 / sqrt(3) of the value at the lower end of a
    power of two, less elsewhere, and together stay below 2^-11 in the mean."""
    c = Q.Cache([20000], 1, 128, 64, "f16", seed=20, layers=1)
    q = randn(c.g, 1, 8, 128, dtype="f16")
    out, _, _, _ = run_attend(ops, c, q, weights=False, layer=0)
    want = torch.stack([row[0] for row in Q.attend(c, 0, q)[0]])
    assert float((out[0] - want).norm() / want.norm()) <= 2.0 ** -11


def test_attend_long_row(ops):
    """140001 slots in blocks beyond 4 GiB: 64-bit offsets, a row in many pieces."""
    c = Q.Cache([140001], 1, 64, 64, "f16", seed=8, layers=1, blocks=950_000)
    assert c.pool.numel() > 1 << 32
    q = randn(c.g, 1, 2, 64, dtype="f16")
    check_attend(c, q, run_attend(ops, c, q, layer=0), layer=0)


def test_attend_strides(ops):
    """Rows of q and out at odd places, in place."""
    for dtype in ("bf16", "f16"):
        c = Q.Cache([50, 333], 2, 80, 16, dtype, seed=9)
        wide = randn(c.g, 2, 13, 91, dtype=dtype)
        for q in (wide[:, 1:9, 3:83], wide[:, ::3][:, :4, 8:88]):
            want, _, _, _ = run_attend(ops, c, q.contiguous(), weights=False)
            room = torch.zeros(2, 13, 91, dtype=c.tdtype, device="cuda")
            out = room[:, 2:2 + q.shape[1], 5:85]
            ops.kv_attend(c.handle(B), 1, q, c.tables, c.lens, c.longest, out=out)
            ops.kv_ops_sync()
            assert torch.equal(out.double().cpu(), want)
            assert (room[:, :2] == 0).all() and (room[..., :5] == 0).all() and (room[..., 85:] == 0).all()
            mine = q.clone()
            ops.kv_attend(c.handle(B), 1, mine, c.tables, c.lens, c.longest, out=mine)
            ops.kv_ops_sync()
            assert torch.equal(mine.double().cpu(), want)


def test_attend_bad_ids_and_lengths():
    with B.KVOps(0) as ops:
        c = Q.Cache([100, 100, 100], 2, 128, 16, seed=10)
        q = randn(c.g, 3, 8, 128)
        good, _, _, _ = run_attend(ops, c, q, weights=False)
        tables = c.tables.clone()
        tables[1, 3] = c.nb
        lens = c.lens.clone()
        lens[2] = 101
        out, lse = torch.full_like(q, NAN), torch.full((3, 8), NAN, device="cuda")
        ops.kv_attend(c.handle(B), 1, q, tables, lens, 100, out=out, lse=lse)
        assert ops.kv_ops_sync(check=False) == B.KV_ERR_RANGE
        assert torch.equal(out[0].double().cpu(), good[0])
        assert (out[2] == 0).all() and (lse[2] == -math.inf).all()
        # the slots of the bad block are masked
        (klo, ks, kc), (vlo, vs, vc) = (c.held(1, 1, plane) for plane in range(2))
        keep = [t for t in range(100) if t // 16 != 3]
        for g in range(8):
            p = ((klo + ks * kc)[keep, g // 4] @ q[1, g].double().cpu() / 128 ** 0.5).softmax(0)
            want = p @ (vlo + vs * vc)[keep, g // 4]
            assert ((out[1, g].double().cpu() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -10 * (p @ (vlo.abs() + vs * vc)[keep, g // 4])).all()


# ---- append ---------------------------------------------------------------------------------------------------------


def turned(x, angle, halves, dim):
    half = angle.shape[-1]
    return R.rotate(x, angle, halves) if half else x


APPEND = [
    # news, before, q_heads, kv_heads, dim, rotary, bs, dtype, layout, halves, norms ("", "q", "k", "qk", "heads", "float")
    ([1], 36, 4, 2, 128, 128, 16, "bf16", 0, True, "qk"),
    ([1, 1, 1], 5, 32, 8, 128, 128, 16, "bf16", 0, True, "qk"),
    ([7, 1, 30], 0, 6, 2, 64, 64, 8, "f16", 1, False, "heads"),
    ([40, 3], 11, 4, 4, 80, 80, 24, "bf16", 0, True, "float"),
    ([9, 20], 2, 3, 1, 80, 40, 12, "f16", 0, True, "qk"),
    ([9, 20], 2, 3, 1, 96, 48, 12, "bf16", 0, False, "k"),
    ([5, 17], 0, 2, 2, 256, 256, 16, "bf16", 1, True, "qk"),
    ([5, 17], 0, 2, 2, 256, 2, 16, "f16", 0, False, "q"),
    ([12], 3, 5, 5, 72, 72, 4, "bf16", 0, True, "qk"),
    ([12], 3, 5, 5, 72, 36, 4, "bf16", 0, True, "heads"),
    ([33], 0, 2, 1, 8, 8, 4, "f16", 0, True, "qk"),
    ([21, 2], 0, 2, 1, 128, 0, 16, "bf16", 0, True, "qk"),
    ([21, 2], 0, 2, 1, 128, 128, 16, "bf16", 0, True, ""),
    ([200, 777, 1], 64, 8, 2, 128, 64, 16, "bf16", 0, True, "qk"),
]


@pytest.mark.parametrize("news,before,hq,hk,dim,rotary,bs,dtype,layout,halves,norms", APPEND)
@pytest.mark.parametrize("q4", [True, False])
def test_append(ops, news, before, hq, hk, dim, rotary, bs, dtype, layout, halves, norms, q4):
    lens = [before + n for n in news]
    c = (Q if q4 else R).Cache(lens, hk, dim, bs, dtype, layout, seed=dim + sum(news))
    t, half = sum(news), rotary // 2
    x = randn(c.g, t, hq + 2 * hk, dim, dtype=dtype, scale=3.0)
    freq = (10000.0 ** (-torch.arange(half, dtype=torch.float64) / max(1, half))).float()
    pos = torch.randint(0, 100000, (1, t), generator=c.g, dtype=torch.int32)
    wtype = torch.float32 if norms == "float" else c.tdtype
    of = {"heads": lambda h: (1 + 0.3 * torch.randn(h, dim, generator=c.g)).to(wtype), "": None}.get(norms, lambda h: (1 + 0.3 * torch.randn(dim, generator=c.g)).to(wtype))
    qw = of(hq) if norms not in ("", "k") else None
    kw = of(hk) if norms not in ("", "q") else None
    eps = 1e-5
    starts = torch.tensor([0] + torch.tensor(news).cumsum(0).tolist(), dtype=torch.int32)
    q_out = torch.full((t, hq, dim), NAN, dtype=c.tdtype, device="cuda")
    want = c.pool.clone()
    ops.kv_append(c.handle(B), 1, x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:], c.tables, c.lens, positions=pos.cuda(), inv_freq=freq.cuda(), halves=halves,
                  q_out=q_out, seq_starts=starts.cuda(), q_norm=qw.cuda() if qw is not None else None, k_norm=kw.cuda() if kw is not None else None, norm_eps=eps)
    ops.kv_ops_sync()
    angle = (pos[0].double()[:, None] * freq.double())[:, None]
    y = x.double().cpu()
    q = turned(Q.normed(y[:, :hq], qw.double() if qw is not None else None, eps), angle, halves, dim)
    k = turned(Q.normed(y[:, hq:hq + hk], kw.double() if kw is not None else None, eps), angle, halves, dim)
    # float32: a sum of dim squares and its root, four products, sine and cosine: 2^-18 of the row's largest; then one rounding
    def near(have, exact):
        size = exact.abs().amax(-1, keepdim=True) + 1e-30
        return ((have.double().cpu() - exact).abs() <= R.UNIT[dtype] * exact.abs() + 2.0 ** -18 * size + (2.0 ** -24 if dtype == "f16" else 0)).all()
    assert near(q_out, q)
    at = 0
    for i, n in enumerate(news):
        rows = torch.arange(before, before + n)
        b, r = c.where(i, rows)
        for plane, new in ((0, k[at:at + n]), (1, y[at:at + n, hq + hk:])):
            if q4:
                codes, words = Q.pack(new.float().to(c.tdtype), plane, dtype)
                saved, c.pool = c.pool, want
                cp, wp = c.parts(1, plane)
                cp[b, :, r] = codes.cuda()
                wp[b, :, r] = words.cuda()
                c.pool = saved
            else:
                have = c.plane(1, plane)[b, r]
                assert near(have, new) if plane == 0 else torch.equal(have.cpu(), new.to(c.tdtype))
                (want[:, 1, plane] if layout else want[1, plane])[b, r] = have
        at += n
    assert torch.equal(want.view(torch.uint8), c.pool.view(torch.uint8))      # the codes of the formula, and nothing else was touched


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_pack_of_hard_rows(ops, dtype):
    """Ties between codes, groups of one value, of zeros, of both signs of zero, of subnormal numbers, of the largest, and such that are not finite."""
    t = R.TYPES[dtype]
    info = torch.finfo(t)
    g = torch.Generator().manual_seed(11)
    rows = []
    for s in (1.0, 0.5, 2.0 ** -10, 3.0, 7 / 8):
        half_steps = torch.randint(0, 31, (40, 128), generator=g).float() / 2 * s
        half_steps[:, ::32] = 0
        half_steps[:, 1::32] = 15 * s
        rows.append(half_steps - torch.randint(0, 4, (40, 1), generator=g))
    rows += [torch.full((3, 128), x) for x in (0.0, -0.0, 1.0, -3.0, info.tiny, info.max, -info.max)]
    rows += [torch.randn(20, 128, generator=g) * x for x in (info.tiny, info.smallest_normal * 2.0 ** -4, info.max / 8)]
    odd = torch.randn(12, 128, generator=g)
    odd[0, 5], odd[1, 33], odd[2, 127], odd[3, :32], odd[4, 64] = NAN, math.inf, -math.inf, math.inf, NAN
    odd[5, :2] = torch.tensor([info.max, -info.max])
    rows.append(odd)
    v = torch.cat(rows).to(t)[:, None]
    n = len(v)
    c = Q.Cache([n], 1, 128, 16, dtype, seed=12)
    ops.kv_append(c.handle(B), 1, None, v.cuda(), v.cuda(), c.tables, c.lens, positions=torch.zeros(1, n, dtype=torch.int32, device="cuda"),
                  inv_freq=torch.zeros(0, device="cuda"), seq_starts=torch.tensor([0, n], dtype=torch.int32, device="cuda"))
    ops.kv_ops_sync()
    b, r = c.where(0, torch.arange(n))
    for plane in range(2):
        codes, words = Q.pack(v, plane, dtype)
        have_codes, have_words = (p[b, :, r].cpu() for p in c.parts(1, plane))
        # -0 and +0 are the same lowest value
        zero = lambda w: w.contiguous().view(torch.int32).where((w.contiguous().view(torch.int32) & 0x7FFF) != 0, w.contiguous().view(torch.int32) & ~0x8000)  # noqa: E731
        bad = (zero(have_words) != zero(words)).any(-1)[:, 0].nonzero()[:, 0].tolist()
        assert not bad, (plane, bad[:5], v[bad[0], 0], have_words[bad[0]], words[bad[0]])
        bad = (have_codes != codes).any(-1)[:, 0].nonzero()[:, 0].tolist()
        assert not bad, (plane, bad[:5], v[bad[0], 0], have_codes[bad[0]], codes[bad[0]])
    k, w = torch.zeros_like(v).cuda(), torch.zeros_like(v).cuda()
    ops.kv_read(c.handle(B), 1, c.tables, c.lens, k_out=k, v_out=w, seq_starts=torch.tensor([0, n], dtype=torch.int32, device="cuda"))
    ops.kv_ops_sync()
    lo, step, code = Q.quantise(v)
    exact = (lo + step * code)
    want = exact.float().to(t)
    for have in (k, w):
        assert torch.equal(torch.isnan(have.cpu()), torch.isnan(want))
        assert ((have.cpu() == want) | torch.isnan(want)).all()


# ---- read -----------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dim,bs,dtype,layout", [(128, 16, "bf16", 0), (64, 8, "f16", 1), (80, 24, "bf16", 0), (256, 4, "f16", 0), (8, 4, "bf16", 0), (200, 16, "bf16", 1)])
@pytest.mark.parametrize("q4", [True, False])
def test_read(ops, dim, bs, dtype, layout, q4):
    lens, news = [70, 5, 0, 33], [70, 3, 0, 1]
    c = (Q if q4 else R).Cache(lens, 3, dim, bs, dtype, layout, seed=dim)
    starts = torch.tensor([2, 72, 75, 75, 76], dtype=torch.int32)           # two tokens in front and two behind that are nobody's
    for room in (dim, dim + 16, dim + 3):
        k, v = (torch.full((78, 5, room), 7.0, dtype=c.tdtype, device="cuda") for _ in range(2))
        with B.KVOps(0) as own:                                             # tokens of no sequence are reported
            own.kv_read(c.handle(B), 1, c.tables, c.lens, k_out=k[:, 1:4, :dim], v_out=v[:, 2:5, room - dim:], seq_starts=starts.cuda())
            own.kv_ops_sync(check=False)
        for plane, (have, h0, d0) in enumerate(((k, 1, 0), (v, 2, room - dim))):
            want = torch.full((78, 5, room), 7.0, dtype=c.tdtype)
            for i, n in enumerate(news):
                if n:
                    if q4:
                        lo, step, code = c.held(i, 1, plane)
                        rows = (lo + step * code).float().to(c.tdtype)
                    else:
                        rows = c.read(i, 1, plane).cpu()
                    want[starts[i]:starts[i] + n, h0:h0 + 3, d0:d0 + dim] = rows[-n:]
            assert torch.equal(have.cpu(), want), (plane, room)
    last = torch.full((4, 3, dim), 7.0, dtype=c.tdtype, device="cuda")
    ops.kv_read(c.handle(B), 1, c.tables, c.lens, v_out=last)
    ops.kv_ops_sync()
    assert (last[2] == 7).all() and torch.equal(last[3], v[75, 2:5, room - dim:]) and torch.equal(last[0], v[71, 2:5, room - dim:])


@pytest.mark.parametrize("dim,heads,q4", [(8, 1, False), (16, 1, False), (24, 1, False), (8, 2, False), (8, 1, True), (16, 1, True)])
def test_read_of_the_smallest_rows(ops, dim, heads, q4):
    """One thread may have a token's whole row."""
    lens = [70, 300]
    c = (Q if q4 else R).Cache(lens, heads, dim, 16, seed=dim + heads)
    k, v = (torch.full((sum(lens) + 1, heads, dim), 7.0, dtype=c.tdtype, device="cuda") for _ in range(2))
    starts = torch.tensor([0, 70, 370], dtype=torch.int32, device="cuda")
    ops.kv_read(c.handle(B), 1, c.tables, c.lens, k_out=k[:-1], v_out=v[:-1], seq_starts=starts)
    ops.kv_ops_sync()
    for plane, have in enumerate((k, v)):
        assert (have[-1] == 7).all()
        for i, n in enumerate(lens):
            if q4:
                lo, step, code = c.held(i, 1, plane)
                want = (lo + step * code).float().to(c.tdtype)
            else:
                want = c.read(i, 1, plane).cpu()
            assert torch.equal(have[70 * i:70 * i + n].cpu(), want), (plane, i)


# ---- evict ----------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("lens,keep,recent,sink,heads,dim,bs,dtype,layout", [
    ([40, 24, 100], 24, 4, 2, 2, 128, 16, "bf16", 0),
    ([130, 90, 7], 50, 10, 1, 3, 64, 8, "f16", 1),
    ([1000, 800], 300, 64, 4, 1, 80, 20, "bf16", 0),
    ([9000], 4000, 100, 4, 1, 256, 16, "f16", 0),
    ([2300, 2200], 2048, 256, 4, 8, 128, 16, "bf16", 0),
])
def test_evict(ops, lens, keep, recent, sink, heads, dim, bs, dtype, layout):
    c = Q.Cache(lens, heads, dim, bs, dtype, layout, layers=2, seed=dim + keep)
    n, longest = len(lens), max(lens)
    w = torch.rand(2, n, heads, longest, generator=c.g)
    w[torch.rand(w.shape, generator=c.g) < 0.2] = 0.0
    order = torch.arange(longest, dtype=torch.int32).expand(2, n, heads, -1).contiguous()
    wd, od, new = w.cuda(), order.cuda(), torch.zeros(n, dtype=torch.int32, device="cuda")
    want = c.pool.clone()
    saved = c.pool.clone()
    ops.kv_evict(c.handle(B), c.tables, c.lens, longest, keep=keep, recent=recent, sink=sink, weights=wd, order=od, lens_out=new)
    ops.kv_ops_sync()
    have, c.pool = c.pool, want
    source = saved
    for layer in range(2):
        for i in range(n):
            for h in range(heads):
                pairs = R.evict(w[layer, i, h], order[layer, i, h], lens[i], keep, recent, sink, lens[i])
                if not pairs:
                    continue
                d, s = (torch.tensor(x) for x in zip(*pairs))
                (bd, rd), (bs_, rs) = c.where(i, d), c.where(i, s)
                for plane in range(2):
                    c.pool = source
                    parts = [p[bs_, h, rs].clone() for p in c.parts(layer, plane)]
                    c.pool = want
                    for p, rows in zip(c.parts(layer, plane), parts):
                        p[bd, h, rd] = rows
    assert torch.equal(have, want)
    assert new.tolist() == [min(x, keep) for x in lens]
