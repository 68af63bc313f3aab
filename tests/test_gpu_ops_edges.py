"""Edges of the operators on the device cache: values that are not finite, weights far below the largest, slots in front of a
window, tokens of no sequence, strides that are never used, tensors that want gradients, tables without entries."""
import math

import pytest
import torch

import ops_reference as R
from paper_2601_20309_b200 import binding as B

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def ops():
    with B.KVOps(0) as o:
        yield o


def randn(g, *shape, dtype="bf16", scale=1.0):
    return (torch.randn(*shape, generator=g) * scale).to(R.TYPES[dtype]).cuda()


# ---- weights far below the largest ----------------------------------------------------------------------------------


def one_peak(ops, dtype, seqs, heads, n):
    """One slot of score 18 in front of n - 1 slots of score 0: each has exp(-18) = 2^-26 of the largest weight, together they
    are x = (n - 1) exp(-18) of it.  The first slot's V is 0, the others' 1000.  160 sequences share their blocks: as many
    rows as SMs, hardly any of them cut."""
    c = R.Cache([n], heads, 64, 16, dtype, layers=1)
    k, v = torch.zeros(n, heads, 64), torch.full((n, heads, 64), 1000.0)
    k[0, :, 0] = 18.0
    v[0] = 0.0
    c.write(0, 0, 0, k.to(c.tdtype))
    c.write(0, 0, 1, v.to(c.tdtype))
    q = torch.zeros(seqs, heads, 64, dtype=c.tdtype, device="cuda")
    q[..., 0] = 1.0
    out, lse = torch.full_like(q, NAN), torch.full((seqs, heads), NAN, device="cuda")
    ops.kv_attend(c.handle(B), 0, q, c.tables.expand(seqs, -1).contiguous(), c.lens.expand(seqs).contiguous(), n, out=out, lse=lse, scale=1.0)
    ops.kv_ops_sync()
    return out.double(), lse.double(), (n - 1) * math.exp(-18.0)


PEAKS = [(1, 1, 500), (160, 8, 20000), (1, 8, 40000)]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("seqs,heads,n", PEAKS)
def test_the_sum_of_a_row_keeps_many_small_weights(ops, dtype, seqs, heads, n):
    """lse = 18 + log(1 + x), to the bound of all lse tests: an uncompensated sum of a long row is off by twice as much."""
    _, lse, x = one_peak(ops, dtype, seqs, heads, n)
    assert (lse - (18.0 + math.log1p(x))).abs().max().item() <= 2.0 ** -20 * 19


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("seqs,heads,n", PEAKS)
def test_the_output_keeps_many_small_weights(ops, dtype, seqs, heads, n):
    """out = 1000 x / (1 + x).  Bound: the weights' rounding and the output's, u each, the exponential's and the sums' error
    2^-18, and half of the smallest f16 number."""
    out, _, x = one_peak(ops, dtype, seqs, heads, n)
    want = 1000.0 * x / (1 + x)
    assert (out - want).abs().max().item() <= (2 * R.UNIT[dtype] + 2.0 ** -18) * want + 2.0 ** -25


# ---- values that are not finite -------------------------------------------------------------------------------------


@pytest.mark.parametrize("n,others", [(40, 0), (40, 3), (300, 200), (6000, 0), (6000, 40)])
@pytest.mark.parametrize("weights", [True, False])
def test_no_score_left_gives_zero_whatever_v_holds(ops, n, others, weights):
    """All scores of head 0 are -inf and its V rows hold infinities and NaN: out 0, lse -inf, weights as they were."""
    c = R.Cache([n] + [50] * others, 2, 64, 16, seed=n)
    k, v = c.read(0, 1, 0).cpu(), c.read(0, 1, 1).cpu()
    k[:, 0] = -INF
    v[3, 0, 5], v[n // 2, 0, 6], v[n - 1, 0, 63] = INF, NAN, -INF
    c.write(0, 1, 0, k)
    c.write(0, 1, 1, v)
    q = randn(c.g, 1 + others, 4, 64).abs() + 0.5
    out, lse = torch.full_like(q, 7.0), torch.full((1 + others, 4), 7.0, device="cuda")
    w = torch.rand(1 + others, 2, c.longest, device="cuda") if weights else None
    w_out = torch.full_like(w, -3.0) if weights else None
    ops.kv_attend(c.handle(B), 1, q, c.tables, c.lens, c.longest, out=out, lse=lse, weights_in=w, weights_out=w_out)
    ops.kv_ops_sync()
    assert (out[0, :2] == 0).all() and (lse[0, :2] == -INF).all()
    assert out[0, 2:].isfinite().all() and lse[0, 2:].isfinite().all() and out[1:].isfinite().all()
    if weights:
        assert torch.equal(w_out[0, 0, :n], w[0, 0, :n])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n,run,others", [(100, 30, 0), (900, 500, 0), (6000, 3000, 0), (6000, 3000, 150)])
def test_v_of_a_slot_without_weight_counts_wherever_the_row_is_cut(ops, dtype, n, run, others):
    """A run of slots of score -inf, weight 0, with one infinity and one NaN in their V: 0 * inf makes those two elements NaN, in
    rows that one CTA has and in rows that are cut (inside the run as well) alike; all other elements are as ever."""
    c = R.Cache([n] + [60] * others, 1, 64, 16, dtype, seed=run)
    k, v = c.read(0, 1, 0).cpu(), c.read(0, 1, 1).cpu()
    first = n // 4
    k[first:first + run] = -INF
    v[first + run // 2, 0, 5], v[first + run // 3, 0, 40] = INF, NAN
    c.write(0, 1, 0, k)
    c.write(0, 1, 1, v)
    q = randn(c.g, 1 + others, 2, 64, dtype=dtype).abs() + 0.5
    out = torch.full_like(q, 7.0)
    ops.kv_attend(c.handle(B), 1, q, c.tables, c.lens, n, out=out)
    ops.kv_ops_sync()
    rest = [d for d in range(64) if d not in (5, 40)]
    assert out[0][:, [5, 40]].isnan().all()
    v[first + run // 2, 0, 5] = v[first + run // 3, 0, 40] = 0.0        # for the statement in 64 bits
    c.write(0, 1, 1, v)
    for i, row in enumerate(R.attend(c, 1, q)):
        for g, (o, _, _, _, bound, _) in enumerate(row):
            d = rest if i == 0 else list(range(64))
            assert ((out[i, g].double().cpu() - o)[d].abs() <= bound[d]).all(), (i, g)


@pytest.mark.parametrize("n,window", [(40, 10), (700, 333), (6000, 333)])
@pytest.mark.parametrize("in_place", [True, False])
def test_slots_before_the_window_keep_their_weight_when_the_sum_is_nan(ops, n, window, in_place):
    """A NaN in K makes the row's sum NaN, and with it the weights inside the window; in front of it nothing changes."""
    c = R.Cache([n], 1, 64, 16, seed=n)
    k = c.read(0, 1, 0).cpu()
    k[n - 3, 0, 9] = NAN
    c.write(0, 1, 0, k)
    q = randn(c.g, 1, 2, 64)
    w = torch.rand(1, 1, n, device="cuda")
    had = w.clone()
    w_out = w if in_place else torch.full_like(w, -3.0)
    out = torch.zeros_like(q)
    ops.kv_attend(c.handle(B), 1, q, c.tables, c.lens, n, out=out, window=window, weights_in=w, weights_out=w_out)
    ops.kv_ops_sync()
    assert torch.equal(w_out[..., :n - window], had[..., :n - window])
    assert w_out[..., n - window:].isnan().all() and out.isnan().all()


# ---- tokens of no sequence ------------------------------------------------------------------------------------------


def test_tokens_in_front_of_the_first_start_are_not_written():
    """seq_starts = [2, 5]: tokens 0 and 1 belong to no sequence.  They are skipped and reported; 2, 3 and 4 go to the last slots."""
    c = R.Cache([20], 2, 64, 16, seed=1)
    kv = randn(c.g, 5, 4, 64)
    start = c.pool.clone()
    w = torch.full((1, 2, 20), 5.0, device="cuda")
    with B.KVOps(0) as o:
        o.kv_append(c.handle(B), 1, None, kv[:, :2], kv[:, 2:], c.tables, c.lens, positions=torch.zeros(1, 5, dtype=torch.int32, device="cuda"),
                    inv_freq=torch.ones(32, device="cuda"), seq_starts=torch.tensor([2, 5], dtype=torch.int32).cuda(), weights=w)
        assert o.kv_ops_sync(check=False) == B.KV_ERR_RANGE
    assert torch.equal(c.read(0, 1, 0)[17:], kv[2:, :2]) and torch.equal(c.read(0, 1, 1)[17:], kv[2:, 2:])
    assert (w[..., :17] == 5).all() and (w[..., 17:] == 0).all()
    b, r = c.where(0, torch.arange(17, 20))
    for side in range(2):
        c.plane(1, side)[b, r] = start[1, side][b, r]
    assert torch.equal(c.pool.view(torch.int16), start.view(torch.int16))


# ---- strides that are never used ------------------------------------------------------------------------------------


def test_strides_of_dimensions_of_size_one_do_not_count(ops):
    """One sequence (one layer) cut out of a larger array beside a fresh one: their strides differ where nothing steps."""
    c = R.Cache([40], 2, 64, 16, seed=2)
    q = randn(c.g, 1, 4, 64)
    out = torch.zeros_like(q)
    big = torch.rand(6, 2, 40, device="cuda")
    had, fresh = big[::3][1:], torch.zeros(1, 2, 40, device="cuda")
    assert had.stride() != fresh.stride() and had.shape == fresh.shape
    ops.kv_attend(c.handle(B), 1, q, c.tables, c.lens, 40, out=out, weights_in=had, weights_out=fresh)
    ops.kv_ops_sync()
    p = [row[2] for row in R.attend(c, 1, q)[0]]
    want = had[0].double().cpu() + torch.stack([p[0] + p[1], p[2] + p[3]])
    assert torch.allclose(fresh[0].double().cpu(), want, rtol=1e-4, atol=1e-6)

    order = torch.full((1, 2, 40), -9, dtype=torch.int32, device="cuda")
    kv = randn(c.g, 1, 4, 64)
    ops.kv_append(c.handle(B), 1, None, kv[:, :2], kv[:, 2:], c.tables, c.lens, positions=torch.zeros(1, 1, dtype=torch.int32, device="cuda"),
                  inv_freq=torch.ones(32, device="cuda"), weights=had, order=order, token_order=torch.tensor([77], dtype=torch.int32).cuda())
    ops.kv_ops_sync()
    assert (had[0, :, 39] == 0).all() and (order[0, :, 39] == 77).all() and (order[0, :, :39] == -9).all()

    layers = torch.rand(4, 1, 2, 40, device="cuda")
    w, ages = layers[2:3], torch.arange(40, dtype=torch.int32, device="cuda").expand(3, 2, 1, 2, 40).contiguous()[1:2, 1]
    w_out, o_out = torch.zeros(3, 5, 2, 24, device="cuda")[1:2, 4:], torch.zeros(1, 1, 2, 24, dtype=torch.int32, device="cuda")
    assert w.stride() != ages.stride() and w_out.stride() != o_out.stride()
    before = w.clone()
    ops.kv_evict(c.handle(B), c.tables, c.lens, 40, keep=24, recent=4, sink=2, weights=w, order=ages, weights_out=w_out, order_out=o_out, first_layer=1)
    ops.kv_ops_sync()
    for h in range(2):
        want = list(range(24))
        for d, s in R.evict(before[0, 0, h].cpu(), torch.arange(40), 40, 24, 4, 2, 40):
            want[d] = s
        assert o_out[0, 0, h].tolist() == want and torch.equal(w_out[0, 0, h], before[0, 0, h, want])


# ---- tensors that want gradients ------------------------------------------------------------------------------------


def test_tensors_that_want_gradients_are_refused_where_they_would_be_recorded(ops):
    """The operators have no backward pass: with gradients on, such a tensor would leave the graph without a word."""
    c = R.Cache([40, 7], 2, 64, 16, seed=3)
    q, kv = randn(c.g, 2, 4, 64), randn(c.g, 2, 4, 64)
    out = torch.full_like(q, 3.0)
    start = c.pool.clone()
    pos, freq = torch.zeros(1, 2, dtype=torch.int32, device="cuda"), torch.ones(32, device="cuda")
    leaf, kv_leaf, freq_leaf = (x.clone().requires_grad_() for x in (q, kv, freq))
    h = c.handle(B)
    for bad in (dict(q=leaf), dict(q=leaf * 2), dict(out=leaf)):
        a = {"q": q, "out": out, **bad}
        with pytest.raises(ValueError, match="grad"):
            ops.kv_attend(h, 1, a["q"], c.tables, c.lens, 40, out=a["out"])
    for k, v, f in ((kv_leaf[:, :2], kv[:, 2:], freq), (kv[:, :2], kv_leaf[:, 2:], freq), (kv[:, :2], kv[:, 2:], freq_leaf)):
        with pytest.raises(ValueError, match="grad"):
            ops.kv_append(h, 1, None, k, v, c.tables, c.lens, positions=pos, inv_freq=f)
    with pytest.raises(ValueError, match="grad"):
        ops.kv_evict(h, c.tables, c.lens, 40, keep=10, weights=torch.rand(2, 2, 2, 40, device="cuda", requires_grad=True))
    ops.kv_ops_sync()
    assert (out == 3).all() and torch.equal(c.pool.view(torch.int16), start.view(torch.int16))
    ops.kv_attend(h, 1, q, c.tables, c.lens, 40, out=out)
    for guard in (torch.no_grad, torch.inference_mode):
        with guard():
            got = torch.zeros_like(q)
            ops.kv_attend(h, 1, leaf, c.tables, c.lens, 40, out=got)
            ops.kv_ops_sync()
            assert torch.equal(got, out)
    got = torch.zeros_like(q)
    ops.kv_attend(h, 1, leaf.detach(), c.tables, c.lens, 40, out=got)
    ops.kv_ops_sync()
    assert torch.equal(got, out)


# ---- nothing in the cache yet ---------------------------------------------------------------------------------------


def test_tables_without_entries_for_a_batch_without_tokens(ops):
    """All places of the batch are idle and no block has been handed out: tables of width 0, max_len 0."""
    c = R.Cache([5], 2, 64, 16, seed=4)
    tables, lens = torch.empty(3, 0, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    q, kv = randn(c.g, 3, 4, 64), randn(c.g, 3, 4, 64)
    out, lse = torch.full_like(q, 3.0), torch.zeros(3, 4, device="cuda")
    start = c.pool.clone()
    ops.kv_attend(c.handle(B), 1, q, tables, lens, 0, out=out, lse=lse)
    assert (out == 0).all() and (lse == -INF).all()
    turned = torch.zeros_like(q)
    ops.kv_append(c.handle(B), 1, q, kv[:, :2], kv[:, 2:], tables, lens, positions=torch.zeros(1, 3, dtype=torch.int32, device="cuda"),
                  inv_freq=torch.ones(32, device="cuda"), q_out=turned)
    assert ops.kv_ops_sync() == 0
    assert torch.equal(turned, q) and torch.equal(c.pool.view(torch.int16), start.view(torch.int16))
    assert ops.kv_attend(c.handle(B), 1, q, tables, lens, 1, out=out, check=False) == B.KV_ERR_INVALID_ARG


# ---- bad block ids --------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("n,keep,quads", [(100, 50, False), (100, 52, True), (400, 150, False), (3000, 2000, False), (5000, 700, False)])
def test_evict_drops_exactly_the_pairs_of_a_bad_block(n, keep, quads, layout):
    """Bad ids in a block of holes and in a block of sources: their rows, weights and ages stay, all other pairs move.  Up to 64
    rows move in the selecting kernel, more in a second one; lengths for each kind of selection."""
    c = R.Cache([n, n - 1], 2, 64, 16, layout=layout, layers=2, seed=n)
    g, width = c.g, n if quads else n + 3
    w = torch.rand(2, 2, 2, width, generator=g)
    order = torch.rand(2, 2, 2, width, generator=g).argsort(-1).to(torch.int32)
    lost = {1, (keep + n) // 32}                # of sequence 1: a block of holes, a block of sources
    bad = c.tables.clone()
    bad[1, 1], bad[1, (keep + n) // 32] = c.nb, -3
    want, w2, o2 = c.pool.clone(), w.clone(), order.clone()
    planed, source = (p if layout else p.permute(2, 0, 1, 3, 4, 5) for p in (want, c.pool))
    dropped = 0
    for l in range(2):
        for i in range(2):
            for h in range(2):
                pairs = R.evict(w[l, i, h], order[l, i, h], c.lens_list[i], keep, 5, 2, n + 1)
                fine = [(d, s) for d, s in pairs if i == 0 or not {d // 16, s // 16} & lost]
                dropped += len(pairs) - len(fine)
                d, s = (torch.tensor(x) for x in zip(*fine))
                (db, dr), (sb, sr) = c.where(i, d), c.where(i, s)
                planed[db, l, :, dr, h] = source[sb, l, :, sr, h]
                w2[l, i, h, d], o2[l, i, h, d] = w[l, i, h, s], order[l, i, h, s]
    assert dropped > 0
    wd, od = w.cuda(), order.cuda()
    w_out, o_out = torch.full((2, 2, 2, keep), -5.0, device="cuda"), torch.full((2, 2, 2, keep), -5, dtype=torch.int32, device="cuda")
    seen = torch.full((2,), n + 1, dtype=torch.int32, device="cuda")
    start = c.pool.clone()
    args = dict(keep=keep, recent=5, sink=2, weights=wd, order=od, seen=seen)
    with B.KVOps(0) as o:
        for outputs in (dict(weights_out=w_out, order_out=o_out), {}):
            c.pool.copy_(start)
            o.kv_evict(c.handle(B), bad, c.lens, n, **args, **outputs)
            assert o.kv_ops_sync(check=False) == B.KV_ERR_RANGE
            assert torch.equal(c.pool.view(torch.int16), want.view(torch.int16))
            got_w, got_o = (w_out, o_out) if outputs else (wd, od)
            m = keep if outputs else width
            assert torch.equal(got_w.cpu(), w2[..., :m]) and torch.equal(got_o.cpu(), o2[..., :m])


# ---- sizes at the limit of 32 bits ----------------------------------------------------------------------------------


def test_a_call_whose_steps_do_not_round_up_within_32_bits_is_refused(ops):
    """42966 sequences of 49981 steps (128 slots each, one KV head) are 2^31 - 2 steps: rounded up to whole pieces they would wrap."""
    cache = B.KVCache(1 << 20, 1, 1 << 14, 1, 64, 1 << 20)
    with pytest.raises(B.KVError) as e:
        ops.kv_attend_workspace(cache, 42966, 1, 49981 * 128 - 15, weights=False)
    assert e.value.code == B.KV_ERR_UNSUPPORTED
    assert ops.kv_attend_workspace(cache, 42966, 1, 49970 * 128 - 15, weights=False) > 0
