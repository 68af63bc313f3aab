"""Attention over a cache in 4 bits at the ends of its number range: scores of any size, V of very different sizes, and what is left of the
weights' bits.  Keys here are of one value per group, so that scores are known exactly and bounds need no term for them."""
import math

import pytest
import torch

import ops_reference as R
import ops_reference_q4 as Q
from paper_2601_20309_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    with B.KVOps(0) as o:
        yield o


def cache(scores, v, dtype="bf16", heads=1, bs=16, dim=128):
    """One sequence per row of `scores`, a list of lists: K's first group holds a slot's score in every element, the others 0; V as given,
    [slots, heads, dim] per sequence."""
    c = Q.Cache([len(s) for s in scores], heads, dim, bs, dtype, layers=1, seed=1)
    for i, s in enumerate(scores):
        k = torch.zeros(len(s), heads, dim)
        k[:, :, :32] = torch.tensor(s)[:, None, None]
        assert torch.equal(k, k.to(c.tdtype).float())
        c.write(i, 0, 0, k.to(c.tdtype))
        c.write(i, 0, 1, v[i].to(c.tdtype))
    return c


def run(ops, c, factors, weights=False):
    """Query head g's scores are factors[g] times the slots'.  (out, lse, weights out)"""
    q = torch.zeros(len(c.lens_list), len(factors), c.dim, dtype=c.tdtype, device="cuda")
    q[:, :, 0] = torch.tensor(factors)
    out, lse = torch.full_like(q, math.nan), torch.full(q.shape[:2], math.nan, device="cuda")
    w = torch.zeros(len(c.lens_list), c.heads, c.longest, device="cuda") if weights else None
    ops.kv_attend(c.handle(B), 0, q, c.tables, c.lens, c.longest, out=out, lse=lse, scale=1.0, weights_out=w)
    ops.kv_ops_sync()
    return out.double().cpu(), lse.double().cpu(), w.double().cpu() if weights else None


def expected(c, scores, factor, i, h):
    """(out, lse, p, p * step per slot and element, the same times what a code counts in a product: 0 to 15, or -8 to 7; size of the terms) in float64."""
    s = torch.tensor(scores[i], dtype=torch.float64) * factor
    top = s.max()
    e = (s - top).exp()
    p = e / e.sum()
    lo, step, code = (x[:, h] for x in c.held(i, 0, 1))
    count = torch.maximum(code, (code - 8).abs())
    return (p @ (lo + step * code), float(top + e.sum().log()), p, p[:, None] * step, p[:, None] * step * count, p @ (lo.abs() + 8 * step + step * count))


def check(c, scores, factors, got, left, centred=False):
    """`left`: what a weight times a step may be off by, of itself (2^-11: a rounding to float16).  Besides, and per slot, 2^-25 of a unit in which
    the row's largest product is 2^8 or more, times a code of up to 15; exponentials, sums and the scores' one rounding 2^-18 (the largest weight's
    score is off by 2^-23 of itself, and that of weights that count by no more than 2^-23 * (its size)); the output's rounding.  `centred`: codes count from -8
    to 7."""
    out, lse, w = got
    group = len(factors) // c.heads
    for i in range(len(scores)):
        total = torch.zeros(c.heads, len(scores[i]), dtype=torch.float64)
        for g, f in enumerate(factors):
            o, z, p, ps, terms, size = expected(c, scores, f, i, g // group)
            near = 2.0 ** -18 + 2.0 ** -22 * max(abs(f * s) for s in scores[i])
            if centred:
                lo, step, code = (x[:, g // group] for x in c.held(i, 0, 1))
                terms = ps * (code - 8).abs()
            bound = R.UNIT[c.dtype] * o.abs() + left * terms.sum(0) + near * size + len(scores[i]) * 15 * 2.0 ** -33 * ps.max() + (2.0 ** -25 if c.dtype == "f16" else 0)
            bad = (out[i, g] - o).abs() - bound
            assert (bad <= 0).all(), (i, g, float(bad.max()), float(bound.max()), out[i, g], o)
            assert abs(lse[i, g] - z) <= 2.0 ** -20 * (1 + abs(z)), (i, g, float(lse[i, g]), z)
            total[g // group] += p
        if w is not None:
            assert ((w[i, :, :len(scores[i])] - total).abs() <= 2.0 ** -17 * total + 2.0 ** -126).all()


@pytest.mark.parametrize("key,factor,size", [(32768.0, 50.0 * 128, 0.008), (32768.0, 33.0 * 128, 0.008 / 128), (61440.0, 60000.0, 1.0), (61440.0, 60000.0, 1e-4)])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_scores_of_any_size(ops, dtype, key, factor, size):
    """Scores of 2e8 to 4e9: all the same, and one of them the largest."""
    if dtype == "bf16":
        key, factor = (float(torch.tensor(x).to(torch.bfloat16)) for x in (key, factor))
    n = 100
    scores = [[key] * n, [key / 2] * 37 + [key] + [key / 2] * (n - 38)]
    g = torch.Generator().manual_seed(2)
    v = [torch.randn(n, 1, 128, generator=g) * size for _ in scores]
    c = cache(scores, v, dtype)
    check(c, scores, [factor, -factor], run(ops, c, [factor, -factor]), 2.0 ** -11)


@pytest.mark.parametrize("power", [47, 60, 95, -60, -95])
@pytest.mark.parametrize("n", [40, 300, 3000])
def test_sums_and_weights_know_nothing_of_v(ops, power, n):
    """V is 0 in the first slots and large or small behind them, in one CTA and in parts that meet: the slots in front keep their weight."""
    g = torch.Generator().manual_seed(3)
    scores = [(torch.randint(-32, 32, (n,), generator=g) / 16).tolist(), (torch.arange(n) // 64 / 4).tolist(), [1.0] * n]
    scores[0][n - 1] = 6.0
    v = [torch.randn(n, 2, 128, generator=g) * 2.0 ** power for _ in scores]
    for i, first in enumerate((n // 2, n - 3, 5)):
        v[i][:first] = 0.0
    c = cache(scores, v, heads=2)
    factors = [1.0, 0.25, -1.0, 0.0]
    check(c, scores, factors, run(ops, c, factors, weights=True), 2.0 ** -11)


@pytest.mark.parametrize("power", [10, 26, 36, 80])
@pytest.mark.parametrize("n,where", [(64, 0), (64, 40), (700, 0), (700, 333), (700, 699), (6000, 5000)])
def test_a_slot_without_weight_takes_nothing_from_the_others(ops, power, n, where):
    """One slot scores far below all others and its V is 2^power times theirs; and one that was the largest until the others came."""
    g = torch.Generator().manual_seed(4)
    low = (torch.randint(-16, 16, (n,), generator=g) / 8).tolist()
    low[where] = -300.0
    late = [300.0] * n
    late[0] = 0.0
    v = [torch.randn(n, 1, 128, generator=g) for _ in range(2)]
    v[0][where] *= 2.0 ** power
    v[1][0] *= 2.0 ** power
    c = cache([low, late], v)
    check(c, [low, late], [1.0, 0.5, 2.0], run(ops, c, [1.0, 0.5, 2.0], weights=True), 2.0 ** -11)


@pytest.mark.parametrize("power", [20, 60])
def test_a_small_weight_of_a_large_value_counts(ops, power):
    """Products of the same size from weights and steps of very different sizes, in either order; the maximum rises in every step."""
    n = 500
    for turn in (1, -1):
        scores = [torch.linspace(-power, 0, n).mul(16).round().div(16).tolist()[::turn]]
        g = torch.Generator().manual_seed(5)
        v = [torch.randn(n, 1, 128, generator=g) * torch.exp(-torch.tensor(scores[0]))[:, None, None]]
        scores = [torch.tensor(scores[0]).to(torch.bfloat16).float().tolist()]
        c = cache(scores, v)
        check(c, scores, [1.0, 0.5], run(ops, c, [1.0, 0.5], weights=True), 2.0 ** -11)


@pytest.mark.parametrize("n", [5, 40, 333, 5000])
def test_f16_outputs_have_the_weights_in_float32(ops, n):
    """What the rounding of a weight times a step to float16 leaves is there too: 2^-22 of it is lost at most."""
    g = torch.Generator().manual_seed(6)
    scores = [(torch.randint(-64, 64, (n,), generator=g) / 32).tolist() for _ in range(2)]
    c = cache(scores, [torch.randn(n, 2, 128, generator=g) for _ in range(2)], "f16", heads=2)
    check(c, scores, [1.0, 0.5, 1.5, -1.0], run(ops, c, [1.0, 0.5, 1.5, -1.0]), 2.0 ** -22, centred=True)


def test_one_rounding_of_all_weights(ops):
    """Every sixteenth slot has a larger score and V of zeros, the others one score and one step (V is -1 or 1), so that their weights are rounded alike,
    by up to 2^-11.  In f16 that is 2^-11 of the sum of what they are multiplied with at most, not of the sum of its sizes: V adds up to little.  (In
    bf16 it is 2^-11 of the sizes, as for weights that are rounded each in its own way.)"""
    n = 4000
    g = torch.Generator().manual_seed(7)
    scores = [[4.25 if t % 16 == 0 else 0.25 for t in range(n)]]
    v = [torch.randint(0, 2, (n, 1, 128), generator=g).float() * 2 - 1]
    v[0][::16] = 0.0
    c = cache(scores, v, "f16")
    factors = torch.tensor([0.1 + 0.05 * k for k in range(16)]).to(torch.float16).float().tolist()
    out, _, _ = run(ops, c, factors)
    lo, step, code = (x[:, 0] for x in c.held(0, 0, 1))
    for k, f in enumerate(factors):
        o, _, p, ps, _, _ = expected(c, scores, f, 0, 0)
        # exponentials: 2^-18 of the output (all alike); float32 sums: 2^-20 of the terms' sizes
        bound = (2.0 ** -11 + 2.0 ** -18) * o.abs() + 2.0 ** -25 + 2.0 ** -11 * (ps * (code - 8)).sum(0).abs() + 2.0 ** -20 * (p[:, None] * (lo.abs() + 8 * step)).sum(0) + n * 15 * 2.0 ** -33 * ps.max()
        assert ((out[0, k] - o).abs() <= bound).all(), (k, float(((out[0, k] - o).abs() - bound).max()), float(bound.max()))


@pytest.mark.parametrize("dtype,tiny", [("bf16", 2.0 ** -100), ("f16", 2.0 ** -24)])
@pytest.mark.parametrize("n", [5, 45])
def test_scores_too_small_for_float32_are_alike(ops, dtype, tiny, n):
    """A factor that is 0 in float32 makes nothing of the slots that are masked."""
    g = torch.Generator().manual_seed(8)
    c = cache([[1.0] * n], [torch.randn(n, 1, 128, generator=g)], dtype)
    q = torch.full((1, 2, 128), tiny, dtype=c.tdtype, device="cuda")
    out, lse = torch.full_like(q, math.nan), torch.full((1, 2), math.nan, device="cuda")
    ops.kv_attend(c.handle(B), 0, q, c.tables, c.lens, n, out=out, lse=lse, scale=2.0 ** -140)
    ops.kv_ops_sync()
    o, z, _, _, terms, size = expected(c, [[0.0] * n], 1.0, 0, 0)
    assert ((out[0].double().cpu() - o).abs() <= R.UNIT[dtype] * o.abs() + 2.0 ** -11 * terms.sum(0) + 2.0 ** -18 * size).all()
    assert ((lse.double().cpu() - z).abs() <= 2.0 ** -20 * (1 + z)).all()


@pytest.mark.parametrize("n", [40, 300, 3000])
def test_v_at_the_lower_limit(ops, n):
    """Elements around 2^-108, steps of 2^-112 and more: products keep their bits."""
    g = torch.Generator().manual_seed(9)
    scores = [(torch.randint(-32, 32, (n,), generator=g) / 8).tolist()]
    c = cache(scores, [torch.randn(n, 1, 128, generator=g) * 2.0 ** -108])
    assert float(c.held(0, 0, 1)[1].min()) >= 2.0 ** -112
    check(c, scores, [1.0, 0.5, -1.0], run(ops, c, [1.0, 0.5, -1.0], weights=True), 2.0 ** -11)


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_f16_scores_have_float32s_bits(ops, dim):
    """lse of one slot is its score, the sum of 2 G float32 sums, s * sum of q * code and lo * sum of q.  Each comes from two instructions that add 16
    products, and is added to the others: a dozen truncations at its own size at most, by 2^-23 of it, whose mean square is 2^-46 / 3 each if their
    errors are as good as independent: 16 * 2^-48 of the sizes' squares in all, over 2048 scores."""
    n = 64
    c = Q.Cache([1] * n, 2, dim, 16, "f16", seed=10, layers=1)
    q = torch.randn(n, 32, dim, generator=c.g).to(torch.float16).cuda()
    out, lse = torch.zeros_like(q), torch.zeros(n, 32, device="cuda")
    ops.kv_attend(c.handle(B), 0, q, c.tables, c.lens, 1, out=out, lse=lse)
    ops.kv_ops_sync()
    far, sizes = 0.0, 0.0
    for i in range(n):
        lo, step, code = (x[0].repeat_interleave(16, 0) for x in c.held(i, 0, 0))
        x = q[i].double().cpu()
        far += float(((lse[i].double().cpu() - ((lo + step * code) * x).sum(-1) / dim ** 0.5) ** 2).sum())
        groups = ((y * x).unflatten(-1, (-1, 32)).sum(-1) for y in (step * code, lo))
        sizes += float(sum((y ** 2).sum() for y in groups)) / dim
    assert far <= 16 * 2.0 ** -48 * sizes, ((far / n / 32) ** 0.5, (sizes / n / 32) ** 0.5)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n", [1, 50, 3000])
def test_zeros_that_are_the_lowest_of_their_group(ops, dtype, n):
    """V is 0 in every other element and not negative elsewhere: the outputs of those elements are 0 in bf16, where code and lowest value are, and no more
    than what is lost of 2^-22 of eight steps, and of float32 sums of them, in f16."""
    g = torch.Generator().manual_seed(11)
    scores = [(torch.randint(-64, 64, (n,), generator=g) / 32).tolist()]
    v = torch.randn(n, 1, 128, generator=g).abs()
    v[..., ::2] = 0.0
    c = cache(scores, [v], dtype)
    factors = [1.0, 0.3125, -1.0, 1.5]
    out, lse, _ = got = run(ops, c, factors)
    check(c, scores, factors, got, 2.0 ** -11 if dtype == "bf16" else 2.0 ** -22)
    for k, f in enumerate(factors):
        _, _, _, ps, _, _ = expected(c, scores, f, 0, 0)
        most = 0.0 if dtype == "bf16" else (2.0 ** -22 + 2.0 ** -20) * 8 * ps.sum(0)[::2] + n * 15 * 2.0 ** -33 * ps.max() + 2.0 ** -25
        assert (out[0, k, ::2].abs() <= most).all()
