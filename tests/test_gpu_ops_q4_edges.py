"""Cache in 4 bits and norms: refusals, streams and graphs, idle places and bad blocks, far offsets, the operators together, the decode loop."""
import ctypes as C
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


def freq_of(dim):
    return (10000.0 ** (-torch.arange(dim // 2, dtype=torch.float64) / (dim // 2))).float().cuda()


def values(c, i, layer, plane):
    lo, step, code = c.held(i, layer, plane)
    return lo + step * code


# ---- refusals -------------------------------------------------------------------------------------------------------


def test_refusals(ops):
    c = Q.Cache([40], 2, 64, 16, seed=1)
    h = c.handle(B)
    x = torch.randn(1, 8, 64, device="cuda").to(torch.bfloat16)
    pos, freq = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), freq_of(64)
    one = torch.ones(64, device="cuda")

    def append(match, error=ValueError, **more):
        with pytest.raises(error, match=match):
            ops.kv_append(h, 0, x[:, :4], x[:, 4:6], x[:, 6:], c.tables, c.lens, positions=pos, inv_freq=freq,
                          **{"q_out": x[:, :4], **more})

    append("differ in type", q_norm=one, k_norm=one.to(torch.bfloat16))
    append("must be float32 or bf16", q_norm=one.double())
    append("must have shape", q_norm=one[:32])
    append("must have shape", k_norm=torch.ones(4, 64, device="cuda"))
    append("must be a tensor", q_norm=1.0)
    append("must be on cuda", k_norm=one.cpu())
    append("last dimension", k_norm=torch.ones(128, device="cuda")[::2])
    append("requires grad", k_norm=torch.ones(64, device="cuda", requires_grad=True))
    append("eps", B.KVError, k_norm=one, norm_eps=-1.0)
    append("eps", B.KVError, k_norm=one, norm_eps=NAN)
    with pytest.raises(ValueError, match="q_norm without q"):
        ops.kv_append(h, 0, None, x[:, 4:6], x[:, 6:], c.tables, c.lens, positions=pos, inv_freq=freq, q_norm=one)
    with pytest.raises(ValueError, match="k_out or v_out"):
        ops.kv_read(h, 0, c.tables, c.lens)
    with pytest.raises(ValueError, match="must be bf16"):
        ops.kv_read(h, 0, c.tables, c.lens, k_out=torch.zeros(1, 2, 64, device="cuda"))
    with pytest.raises(ValueError, match="must have shape"):
        ops.kv_read(h, 0, c.tables, c.lens, k_out=x[:, :3])
    with pytest.raises(ValueError, match="must have shape"):
        ops.kv_read(h, 0, c.tables, c.lens, k_out=x[:, :2], v_out=torch.zeros(2, 2, 64, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(B.KVError, match="every sequence has one token"):
        ops.kv_read(h, 0, c.tables, c.lens, k_out=torch.zeros(2, 2, 64, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(B.KVError, match="no such layer"):
        ops.kv_read(h, 2, c.tables, c.lens, k_out=x[:, :2])
    for bs in (1, 6, 10):
        bad = B.KVCache(c.pool.data_ptr(), 2, bs, 2, 64, 3, dtype="bf16_q4")
        with pytest.raises(B.KVError, match="multiple of 4 tokens"):
            ops.kv_attend(bad, 0, x[:, :4], c.tables, c.lens, 1, out=x[:, :4])
    with pytest.raises(B.KVError, match="16-byte aligned"):
        ops.kv_attend(B.KVCache(c.pool.data_ptr() + 8, 2, 16, 2, 64, 3, dtype="bf16_q4"), 0, x[:, :4], c.tables, c.lens, 40, out=x[:, :4])
    L, bad = B.lib(), B.kv_norm_args_t(one.data_ptr(), None, 0, 0, 7, 1e-6)
    a = B.kv_append_args_t()
    a.num_seqs = a.num_tokens = a.num_axes = a.q_heads = 1
    a.q = a.k = a.v = x.data_ptr()
    assert L.kv_append_normed(ops._h, h.address, C.addressof(a), C.addressof(bad)) == B.KV_ERR_INVALID_ARG
    bad = B.kv_norm_args_t(one.data_ptr(), None, -64, 0, 1, 1e-6)
    assert L.kv_append_normed(ops._h, h.address, C.addressof(a), C.addressof(bad)) == B.KV_ERR_INVALID_ARG
    a.q = None
    assert L.kv_append_normed(ops._h, h.address, C.addressof(a), C.addressof(B.kv_norm_args_t(one.data_ptr(), None, 0, 0, 1, 1e-6))) == B.KV_ERR_INVALID_ARG
    ops.kv_ops_sync()


def test_pool_cache_of_4_bits():
    store = torch.zeros(4 * 2 * 2 * 16 * 2 * 40, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    with B.KVPool(2, 16, 2, 40, 4, 4, store.data_ptr()) as pool:
        assert pool.kv_pool_cache("bf16_q4").dim == 128 and pool.kv_pool_cache("f16_q4", 80).dim == 80
        for dim in (64, 136, 100):
            with pytest.raises(ValueError, match="do not hold"):
                pool.kv_pool_cache("bf16_q4", dim)
    with B.KVPool(2, 16, 2, 64, 4, 4, store.data_ptr()) as pool:
        with pytest.raises(B.KVError, match="kv_cache_row_units"):
            pool.kv_pool_cache("bf16_q4")
        assert pool.kv_pool_cache("bf16", 64).dim == 64


def test_nothing_to_do(ops):
    c = Q.Cache([5], 2, 64, 16, seed=2)
    before = c.pool.clone()
    none = torch.zeros(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    e32 = torch.zeros(0, dtype=torch.int32, device="cuda")
    ops.kv_append(c.handle(B), 0, None, none, none, c.tables[:0], e32, positions=torch.zeros(1, 0, dtype=torch.int32, device="cuda"), inv_freq=freq_of(64))
    ops.kv_read(c.handle(B), 0, c.tables[:0], e32, k_out=none)
    ops.kv_attend(c.handle(B), 0, torch.zeros(0, 4, 64, dtype=torch.bfloat16, device="cuda"), c.tables[:0], e32, 0, out=torch.zeros(0, 4, 64, dtype=torch.bfloat16, device="cuda"))
    ops.kv_ops_sync()
    assert torch.equal(before, c.pool)


# ---- what is nobody's, and what is wrong ----------------------------------------------------------------------------


@pytest.mark.parametrize("q4", [True, False])
def test_append_leaves_what_is_not_its_own(q4):
    """An idle sequence, tokens in front of the first and behind the last, a bad block, a length beyond the table: their rows of the cache
    stay, their q is worked on all the same, the rest is written."""
    c = (Q if q4 else R).Cache([20, 40, 33, 50], 3, 64, 16, seed=3)
    g = torch.Generator().manual_seed(4)
    lens = torch.tensor([20, 0, 33, 500], dtype=torch.int32, device="cuda")
    tables = c.tables.clone()
    tables[2, 1] = -5
    starts = torch.tensor([1, 4, 6, 26, 28], dtype=torch.int32, device="cuda")
    x = torch.randn(30, 10, 64, generator=g).to(torch.bfloat16).cuda()
    q = torch.full((30, 4, 64), NAN, dtype=torch.bfloat16, device="cuda")
    one = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    before = c.pool.clone()
    weights, order = torch.full((4, 3, 60), 9.0, device="cuda"), torch.full((4, 3, 60), 9, dtype=torch.int32, device="cuda")
    with B.KVOps(0) as ops:
        ops.kv_append(c.handle(B), 1, x[:, :4], x[:, 4:7], x[:, 7:], tables, lens, positions=torch.arange(30, dtype=torch.int32, device="cuda")[None],
                      inv_freq=freq_of(64), q_out=q, seq_starts=starts, q_norm=one, k_norm=one, weights=weights, order=order)
        assert ops.kv_ops_sync(check=False) == B.KV_ERR_RANGE
    assert not torch.isnan(q).any()
    written = {(0, s) for s in (17, 18, 19)} | {(2, s) for s in range(13, 33) if s // 16 != 1}
    changed = set()
    now, c.pool = c.pool, before
    for i, n in enumerate(c.lens_list):
        b, r = c.where(i, torch.arange(n))
        for s in range(n):
            same = True
            for plane in range(2):
                for pool in (before, now):
                    c.pool = pool
                    parts = [p[b[s], :, r[s]] for p in c.parts(1, plane)] if q4 else [c.plane(1, plane)[b[s], r[s]]]
                    if pool is before:
                        old = [p.clone() for p in parts]
                    else:
                        same &= all(torch.equal(p.view(torch.uint8), o.view(torch.uint8)) for p, o in zip(parts, old))
            if not same:
                changed.add((i, s))
    assert changed == written
    assert {(i, s) for i in range(4) for s in range(60) if (weights[i, :, s] == 0).all()} == written
    assert all((order[i, :, s] != 9).all() for i, s in written if s != 19) and (weights == 9).sum() == (60 * 4 - len(written)) * 3


def test_far_offsets(ops):
    """Append, read, attention and eviction in a pool of more than 4 GiB."""
    c = Q.Cache([90, 70], 1, 128, 64, seed=5, layers=1, blocks=450_000)
    assert c.pool.numel() > 1 << 32 and int(c.tables_cpu.max()) > 400_000
    g = torch.Generator().manual_seed(6)
    x = torch.randn(2, 3, 128, generator=g).to(torch.bfloat16).cuda()
    ops.kv_append(c.handle(B), 0, None, x[:, 1:2], x[:, 2:], c.tables, c.lens, positions=torch.zeros(1, 2, dtype=torch.int32, device="cuda"), inv_freq=freq_of(128))
    k, v = torch.zeros(2, 1, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 1, 128, dtype=torch.bfloat16, device="cuda")
    ops.kv_read(c.handle(B), 0, c.tables, c.lens, k_out=k, v_out=v)
    ops.kv_ops_sync()
    for have, rows in ((k, x[:, 1:2]), (v, x[:, 2:])):
        lo, step, code = Q.quantise(rows.cpu())
        assert torch.equal(have.cpu(), (lo + step * code).float().to(torch.bfloat16))
    rows = [values(c, 0, 0, plane) for plane in range(2)]
    w = torch.rand(1, 2, 1, 90, generator=g)
    pairs = R.evict(w[0, 0, 0], range(90), 90, 40, 4, 0, 90)
    ops.kv_evict(c.handle(B), c.tables, c.lens, 90, keep=40, recent=4, weights=w.cuda())
    ops.kv_ops_sync()
    for plane in range(2):
        for d, s in pairs:
            rows[plane][d] = rows[plane][s]
        assert torch.equal(values(c, 0, 0, plane)[:40], rows[plane][:40])


# ---- streams and graphs ---------------------------------------------------------------------------------------------


def test_captured_and_replayed_on_a_side_stream():
    """One decode step (append with norms, attention with weights) and an eviction as a graph, replayed three times on new inputs,
    against the same calls one by one."""
    lens, heads, dim = [300, 17, 0, 40], 2, 128
    g = torch.Generator().manual_seed(7)
    xs = [torch.randn(4, 12, dim, generator=g).to(torch.bfloat16).cuda() for _ in range(3)]
    one = (1 + 0.1 * torch.randn(dim, generator=g)).cuda()
    stream = torch.cuda.Stream()
    results = []
    for captured in (False, True):
        c = Q.Cache(lens, heads, dim, 16, seed=8, width=20)
        x, n = xs[0].clone(), c.lens.clone()
        q, out = torch.zeros(4, 8, dim, dtype=torch.bfloat16, device="cuda"), torch.zeros(4, 8, dim, dtype=torch.bfloat16, device="cuda")
        w = torch.zeros(2, 4, heads, 320, device="cuda")
        pos, freq = torch.full((1, 4), 50, dtype=torch.int32, device="cuda"), freq_of(dim)
        got = []
        torch.cuda.synchronize()
        with torch.cuda.stream(stream), B.KVOps(0, stream.cuda_stream) as ops:
            def step():
                for layer in range(2):
                    ops.kv_append(c.handle(B), layer, x[:, :8], x[:, 8:10], x[:, 10:], c.tables, n, positions=pos, inv_freq=freq, q_out=q, weights=w[layer],
                                  q_norm=one, k_norm=one)
                    ops.kv_attend(c.handle(B), layer, q, c.tables, n, 320, out=out, weights_in=w[layer], weights_out=w[layer])
                ops.kv_evict(c.handle(B), c.tables, n, 320, keep=256, recent=8, weights=w)
            ops.kv_ops_reserve(1 << 24)
            graph = torch.cuda.CUDAGraph()
            if captured:
                with torch.cuda.graph(graph, stream=stream):
                    step()
            for new in xs:
                x.copy_(new)
                graph.replay() if captured else step()
                got.append((out.clone(), w.clone(), c.pool.clone()))
            ops.kv_ops_sync()
        torch.cuda.synchronize()
        del graph
        results.append(got)
    for a, b in zip(*results):
        assert all(torch.equal(p.view(torch.uint8), r.view(torch.uint8)) for p, r in zip(a, b))


def test_two_contexts_at_once():
    """The same calls on two streams at the same time, each with its context, give what they give alone."""
    c = Q.Cache([3000, 1200, 60], 4, 128, 16, seed=9)
    q = torch.randn(3, 16, 128, generator=c.g).to(torch.bfloat16).cuda()
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    contexts = [B.KVOps(0, s.cuda_stream) for s in streams]
    outs = [[torch.zeros_like(q) for _ in range(8)] for _ in streams]
    for k in range(8):
        for s, o, out in zip(streams, contexts, outs):
            o.kv_attend(c.handle(B), 1, q, c.tables, c.lens, 3000, out=out[k])
    for o in contexts:
        o.kv_ops_sync()
        o.destroy()
    assert all(torch.equal(x, outs[0][0]) for out in outs for x in out)


def test_attend_scale_of_either_sign(ops):
    c = Q.Cache([200], 1, 64, 16, seed=10)
    q = torch.randn(1, 4, 64, generator=c.g).to(torch.bfloat16).cuda()
    for dtype in ("plus", "minus"):
        a, b = torch.zeros_like(q), torch.zeros_like(q)
        sign = 1.0 if dtype == "plus" else -1.0
        ops.kv_attend(c.handle(B), 1, q, c.tables, c.lens, 200, out=a, scale=0.3 * sign)
        ops.kv_attend(c.handle(B), 1, -q, c.tables, c.lens, 200, out=b, scale=-0.3 * sign)
        ops.kv_ops_sync()
        assert torch.equal(a, b)
        want = (values(c, 0, 1, 0)[:, 0] @ q[0].double().cpu().T * 0.3 * sign).softmax(0).T @ values(c, 0, 1, 1)[:, 0]
        size = values(c, 0, 1, 1).abs().max()
        assert ((a[0].double().cpu() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -9 * size).all()


def test_norms_with_several_axes_and_in_place(ops):
    """Three rotary axes, q_out = q, per-head weights in float32; the tokens' weights and ages are set as without norms."""
    c = R.Cache([12, 30], 2, 64, 16, seed=11)
    g = torch.Generator().manual_seed(12)
    x = torch.randn(7, 8, 64, generator=g).to(torch.bfloat16).cuda()
    axis_of = [f % 3 for f in range(32)]
    pos = torch.randint(0, 5000, (3, 7), generator=g, dtype=torch.int32)
    qw, kw = 1 + 0.2 * torch.randn(4, 64, generator=g), 1 + 0.2 * torch.randn(2, 64, generator=g)
    y = x.double().cpu()
    weights, order = torch.ones(2, 2, 40, device="cuda"), torch.zeros(2, 2, 40, dtype=torch.int32, device="cuda")
    ops.kv_append(c.handle(B), 0, x[:, :4], x[:, 4:6], x[:, 6:], c.tables, c.lens, positions=pos.cuda(), inv_freq=freq_of(64), axis_of=axis_of, q_out=x[:, :4],
                  seq_starts=torch.tensor([0, 2, 7], dtype=torch.int32, device="cuda"), weights=weights, order=order,
                  token_order=torch.arange(100, 107, dtype=torch.int32, device="cuda"), q_norm=qw.cuda(), k_norm=kw.cuda(), norm_eps=0.0)
    ops.kv_ops_sync()
    angle = (pos.double()[torch.tensor(axis_of)] * freq_of(64).double().cpu()[:, None]).T[:, None]
    q = R.rotate(Q.normed(y[:, :4], qw.double(), 0.0), angle, True)
    k = R.rotate(Q.normed(y[:, 4:6], kw.double(), 0.0), angle, True)
    have = torch.cat([c.read(0, 0, 0)[10:], c.read(1, 0, 0)[25:]]).double().cpu()
    for h, w in ((x[:, :4].double().cpu(), q), (have, k)):
        assert ((h - w).abs() <= 2.0 ** -8 * w.abs() + 2.0 ** -18 * w.abs().amax(-1, keepdim=True)).all()
    assert torch.equal(torch.cat([c.read(0, 0, 1)[10:], c.read(1, 0, 1)[25:]]), x[:, 6:])
    assert order[0, 0, 10:12].tolist() == [100, 101] and order[1, 1, 25:30].tolist() == [102, 103, 104, 105, 106]
    assert (weights[0, :, 10:12] == 0).all() and (weights[1, :, 25:30] == 0).all() and weights.sum() == 160 - 14


def test_norm_of_zeros_and_of_large_rows(ops):
    """A row of zeros stays zeros with eps and is NaN without; rows near the type's largest and smallest are normed like others."""
    for q4 in (False, True):
        c = (Q if q4 else R).Cache([4], 1, 64, 16, seed=13)
        x = torch.zeros(4, 3, 64)
        x[1:] = torch.randn(3, 3, 64, generator=torch.Generator().manual_seed(14)) * torch.tensor([1e15, 1e-15, 1.0])[:, None, None]
        x = x.to(torch.bfloat16).cuda()
        one = torch.ones(64, device="cuda")
        for eps in (1e-6, 0.0):
            q = torch.zeros(4, 1, 64, dtype=torch.bfloat16, device="cuda")
            ops.kv_append(c.handle(B), 0, x[:, :1], x[:, 1:2], x[:, 2:], c.tables, c.lens, positions=torch.zeros(1, 4, dtype=torch.int32, device="cuda"),
                          inv_freq=freq_of(64), q_out=q, seq_starts=torch.tensor([0, 4], dtype=torch.int32, device="cuda"), q_norm=one, k_norm=one, norm_eps=eps)
            k = torch.zeros(4, 1, 64, dtype=torch.bfloat16, device="cuda")
            ops.kv_read(c.handle(B), 0, c.tables, c.lens, k_out=k, seq_starts=torch.tensor([0, 4], dtype=torch.int32, device="cuda"))
            ops.kv_ops_sync()
            if eps:
                assert (q[0] == 0).all() and (k[0] == 0).all()
            else:
                assert torch.isnan(q[0]).all() and torch.isnan(k[0]).all()
            want = Q.normed(x[:, :1].double().cpu(), torch.ones(64).double(), eps)
            assert ((q[1:].double().cpu() - want[1:]).abs() <= 2.0 ** -8 * want[1:].abs() + 2.0 ** -18 * want[1:].abs().amax(-1, keepdim=True)).all()


# ---- together -------------------------------------------------------------------------------------------------------


def test_prompt_rotation_decode_and_eviction_together():
    """On a pool's cache: a prompt is appended, its blocks go to the host and come back into other blocks, a token is decoded, the cache shrinks,
    another token is decoded, the rows are read."""
    heads, dim, bs, n = 2, 80, 16, 90
    units = B.kv_cache_row_units("bf16_q4", dim)
    g = torch.Generator().manual_seed(15)
    store = torch.zeros(2, 2, 16, bs, heads, units, dtype=torch.bfloat16, device="cuda")
    freq, one = freq_of(dim), (1 + 0.1 * torch.randn(dim, generator=g)).to(torch.bfloat16).cuda()
    torch.cuda.synchronize()
    with B.KVPool(2, bs, heads, units, 16, 8, store.data_ptr()) as pool, B.KVOps(0, torch.cuda.current_stream().cuda_stream) as ops:
        cache = pool.kv_pool_cache("bf16_q4", dim)
        ids, moved = [3, 9, 1, 14, 6, 11], [0, 2, 4, 5, 7, 8]
        table = torch.tensor([ids], dtype=torch.int32, device="cuda")
        x = torch.randn(n, 4 + 2 * heads, dim, generator=g).to(torch.bfloat16).cuda()
        lens = torch.tensor([n], dtype=torch.int32, device="cuda")
        weights = torch.zeros(2, 1, heads, 96, device="cuda")
        for layer in range(2):
            ops.kv_append(cache, layer, None, x[:, 4:6], x[:, 6:], table, lens, positions=torch.arange(n, dtype=torch.int32, device="cuda")[None], inv_freq=freq,
                          k_norm=one, seq_starts=torch.tensor([0, n], dtype=torch.int32, device="cuda"), weights=weights[layer])
        read = torch.zeros(2, n, heads, dim, dtype=torch.bfloat16, device="cuda")
        ops.kv_read(cache, 1, table, lens, k_out=read[0], v_out=read[1], seq_starts=torch.tensor([0, n], dtype=torch.int32, device="cuda"))
        ops.kv_ops_sync()
        pool.kv_swap_out(ids, list(range(6)))
        pool.kv_sync()
        store[:, :, ids] = -1
        torch.cuda.synchronize()
        pool.kv_swap_in(list(range(6)), moved)
        pool.kv_stream_wait(torch.cuda.current_stream().cuda_stream)
        table = torch.tensor([moved], dtype=torch.int32, device="cuda")
        back = torch.zeros_like(read)
        ops.kv_read(cache, 1, table, lens, k_out=back[0], v_out=back[1], seq_starts=torch.tensor([0, n], dtype=torch.int32, device="cuda"))
        ops.kv_ops_sync()
        assert torch.equal(read, back)
        k, v = back.double().cpu()
        out = torch.zeros(1, 4, dim, dtype=torch.bfloat16, device="cuda")
        q = torch.randn(1, 4, dim, generator=g).to(torch.bfloat16).cuda()

        def check(k, v):
            for h in range(4):
                p = (k[:, h // 2] @ q[0, h].double().cpu() / dim ** 0.5).softmax(0)
                # what kv_read gives is rounded once more: 2^-9 of every score's terms and of the values
                score = 2.0 ** -9 * float((k[:, h // 2].abs() @ q[0, h].double().cpu().abs()).max()) / dim ** 0.5
                assert ((out[0, h].double().cpu() - p @ v[:, h // 2]).abs() <= (2.0 ** -7 + 2 * score) * (p @ v[:, h // 2].abs()) + 2.0 ** -9 * float(v.abs().max())).all()
        for layer in range(2):
            ops.kv_attend(cache, layer, q, table, lens, n, out=out, weights_in=weights[layer], weights_out=weights[layer])
        ops.kv_ops_sync()
        check(k, v)
        pairs = [R.evict(weights[1, 0, h].cpu(), range(n), n, 48, 8, 2, n) for h in range(heads)]
        ops.kv_evict(cache, table, lens, n, keep=48, recent=8, sink=2, weights=weights, lens_out=(short := torch.zeros_like(lens)))
        for h, moves in enumerate(pairs):
            for d, s in moves:
                k[d, h], v[d, h] = k[s, h], v[s, h]
        ops.kv_attend(cache, 1, q, table, short, 48, out=out)
        ops.kv_ops_sync()
        assert short.tolist() == [48]
        check(k[:48], v[:48])


def test_decoder_in_4_bits_matches_a_plain_cache():
    """The decode loop with norms on a 4-bit cache against lists of rows that are quantised by the definition, rotation included."""
    from paper_2601_20309_b200.decode import Decoder
    layers, hq, hk, dim, places = 2, 4, 2, 64, 3
    g = torch.Generator().manual_seed(16)
    qw, kw = (1 + 0.2 * torch.randn(layers, dim, generator=g) for _ in range(2))
    d = Decoder(layers, 16, hq, hk, dim, 30, 60, places, 64, bits=4, q_norm=qw.cuda(), k_norm=kw.cuda(), norm_eps=1e-5)
    inv = freq_of(dim).double().cpu()
    rows = {}

    def append(req, layer, x, pos):
        angle = (pos.double()[0][:, None] * inv)[:, None]
        q = R.rotate(Q.normed(x[:, :hq].double(), qw[layer].double(), 1e-5), angle, True)
        k = R.rotate(Q.normed(x[:, hq:hq + hk].double(), kw[layer].double(), 1e-5), angle, True).float().to(torch.bfloat16)
        for plane, new in enumerate((k, x[:, hq + hk:])):
            lo, step, code = Q.quantise(new)
            rows.setdefault((req, layer, plane), []).append((lo, step * code))
        return q.float().to(torch.bfloat16).double()

    try:
        for req, n in ((5, 20), (2, 7)):
            x = torch.randn(layers, n, hq + 2 * hk, dim, generator=g).to(torch.bfloat16)
            pos = torch.randint(0, 50, (1, n), generator=g, dtype=torch.int32)
            d.add(req, x.cuda(), pos.cuda())
            for layer in range(layers):
                append(req, layer, x[layer], pos)
        for step in range(24):
            x = torch.randn(layers, places, hq + 2 * hk, dim, generator=g).to(torch.bfloat16)
            pos = torch.randint(0, 200, (1, places), generator=g, dtype=torch.int32)
            got = d.step(x.cuda(), pos.cuda()).double().cpu()
            for req, row in d.place_of.items():
                for layer in range(layers):
                    if not d.running[row]:
                        assert (got[layer, row] == 0).all()
                        continue
                    q = append(req, layer, x[layer, row:row + 1], pos[:, row:row + 1])[0]
                    (klo, kc), (vlo, vc) = (tuple(torch.cat([r[part] for r in rows[req, layer, plane]]) for part in range(2)) for plane in range(2))
                    k, v = klo + kc, vlo + vc
                    for h in range(hq):
                        p = (k[:, h // 2] @ q[h] / 8).softmax(0)
                        # q's rounding may fall to the other side of a middle: 2^-8 of a term's size at most, in each score
                        score = 2.0 ** -8 * float((k[:, h // 2].abs() * q[h].abs()).amax(-1).max()) / 8
                        bound = (2.0 ** -8 + 2.0 ** -11 + 4 * score) * (p @ (vlo.abs() + vc)[:, h // 2])
                        assert ((got[layer, row, h] - p @ v[:, h // 2]).abs() <= bound).all(), (step, req, layer, h)
            if step % 9 == 4:
                d.rotate([5], [])
            elif step % 9 == 7:
                d.rotate([], [5])
        assert d.pool.kv_get_stats()["kernel_launches"] >= 0 and math.isfinite(float(got.sum()))
    finally:
        d.close()


def test_decoder_takes_16_or_4_bits():
    from paper_2601_20309_b200.decode import Decoder
    with pytest.raises(ValueError, match="16 or 4"):
        Decoder(1, 16, 2, 1, 64, 4, 4, 1, 16, bits=8)
    with pytest.raises(ValueError, match="no cache for heads"):
        Decoder(1, 16, 2, 1, 100, 4, 4, 1, 16, bits=4)
