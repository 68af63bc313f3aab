"""The decode loop at its edges: no blocks left, no room left, calls under another stream than the one it was made on."""
import pytest
import torch

from paper_2601_20309_b200 import binding as B
from test_gpu_decode import Plain

pytestmark = pytest.mark.gpu
LAYERS, HQ, HK, DIM = 2, 4, 2, 64


def make(blocks, places, max_tokens, lens, seed, **kw):
    """A decoder and the plain cache beside it, with a request per entry of `lens` (id: tokens)."""
    from paper_2601_20309_b200.decode import Decoder
    d = Decoder(LAYERS, 16, HQ, HK, DIM, blocks, 4 * blocks, places, max_tokens, sections=(8, 12, 12), **kw)
    m = Plain(LAYERS, HQ, HK, DIM, kw.get("keep", 0), 0, 0, 0, d.axis_of)
    g = torch.Generator().manual_seed(seed)
    for req, n in lens.items():
        x, pos = torch.randn(LAYERS, n, HQ + 2 * HK, DIM, generator=g).to(torch.bfloat16), torch.randint(0, 50, (3, n), generator=g, dtype=torch.int32)
        d.add(req, x.cuda(), pos.cuda())
        for layer in range(LAYERS):
            m.append(req, layer, x[layer], pos)
        m.seen[req] = n
    return d, m, g


def token(g, places):
    return torch.randn(LAYERS, places, HQ + 2 * HK, DIM, generator=g).to(torch.bfloat16), torch.randint(0, 200, (3, places), generator=g, dtype=torch.int32)


def compare(d, m, got, x, pos, away=()):
    """One token of every running request went in: outputs, weights and ages against the plain cache.  K may be off by a rounding, where
    the turned value lies near the middle of two: a score by 2^-8 of sum |q k| / 8, which widens the bound as a relative
    error of every weight."""
    for req, row in d.place_of.items():
        if req in away:
            assert (got[:, row] == 0).all()
            continue
        for layer in range(LAYERS):
            q = m.append(req, layer, x[layer, row:row + 1], pos[:, row:row + 1])
            out, bound = m.attend(req, layer, q[0])
            for h in range(HQ):
                k, v = (torch.stack(rows[(layer, req, h // (HQ // HK))]) for rows in (m.k, m.v))
                p = (k @ q[0, h] / 8).softmax(0)
                score = 2.0 ** -8 * float((k * q[0, h]).abs().sum(1).max()) / 8
                assert ((got[layer, row, h] - out[h]).abs() <= bound[h] + 2 * score * (p @ v.abs())).all(), (req, layer, h)
        m.seen[req] += 1


def state(d):
    torch.cuda.synchronize()
    info = {r: d.table.kv_req_info(r) for r in d.place_of}
    return dict(d.place_of), list(d.held), list(d.seen), list(d.running), info, d.table.kv_table_get_stats()["free_gpu_blocks"], \
        d.store.clone(), d.weights.clone(), d.order.clone()


def same(a, b):
    return a[:6] == b[:6] and all(torch.equal(x, y) for x, y in zip(a[6:], b[6:]))


def test_a_step_that_finds_no_block_changes_nothing():
    """Two requests need a block, one is left.  The step is refused whole; after a preemption it goes through as if nothing had been."""
    d, m, g = make(5, 3, 64, {1: 16, 2: 16, 3: 20}, 1)
    try:
        before = state(d)
        x, pos = token(g, 3)
        for _ in range(3):
            with pytest.raises(B.KVError) as e:
                d.step(x.cuda(), pos.cuda())
            assert e.value.code == B.KV_ERR_NOMEM
            assert same(before, state(d))
        d.rotate([3], [])
        compare(d, m, d.step(x.cuda(), pos.cuda()).double().cpu(), x, pos, away=[3])
        assert d.held[:2] == [17, 17] and d.seen[:2] == [17, 17] and d.table.kv_req_info(1)["tokens"] == 17
        x, pos = token(g, 3)
        compare(d, m, d.step(x.cuda(), pos.cuda()).double().cpu(), x, pos, away=[3])
    finally:
        d.close()


def test_a_step_beyond_the_rows_or_with_wrong_tensors_changes_nothing():
    d, m, g = make(12, 3, 32, {1: 31, 2: 5}, 2)
    try:
        x, pos = token(g, 3)
        before = state(d)
        for bad_x, bad_pos in ((x.float(), pos), (x[:, :2], pos), (x, pos.long()), (x, pos[:, :2]), (x[:, :, :5], pos), (x[:1], pos),
                           (x.clone().requires_grad_(), pos)):
            with pytest.raises(ValueError):
                d.step(bad_x.cuda(), bad_pos.cuda())
            assert same(before, state(d))
        compare(d, m, d.step(x.cuda(), pos.cuda()).double().cpu(), x, pos)
        before = state(d)
        with pytest.raises(ValueError, match="max_tokens"):
            d.step(x.cuda(), pos.cuda())                    # request 1 holds 32 tokens
        assert same(before, state(d))
        d.rotate([1], [])
        x, pos = token(g, 3)
        compare(d, m, d.step(x.cuda(), pos.cuda()).double().cpu(), x, pos, away=[1])
    finally:
        d.close()


def test_a_request_that_does_not_fit_is_not_added():
    d, m, g = make(6, 2, 64, {1: 20}, 3)
    try:
        before = state(d)
        x, pos = torch.randn(LAYERS, 70, HQ + 2 * HK, DIM, generator=g).to(torch.bfloat16).cuda(), torch.zeros(3, 70, dtype=torch.int32, device="cuda")
        for error, n, y, p in ((ValueError, 65, x, pos), (ValueError, 30, x.float(), pos), (ValueError, 30, x, pos.long()), (ValueError, 30, x[:1], pos),
                               (ValueError, 30, x[:, :, :5], pos), (ValueError, 30, x, pos[:, :20]),
                               (ValueError, 30, x.clone().requires_grad_(), pos)):
            with pytest.raises(error):
                d.add(2, y[:, :n], p[:, :n])
            assert same(before, state(d)), n
        with pytest.raises(B.KVError):
            d.add(1, x[:, :8], pos[:, :8])                  # it is there already
        assert same(before, state(d))
        d.add(2, x[:, :30], pos[:, :30])
        before = state(d)
        with pytest.raises(ValueError):
            d.add(3, x[:, :8], pos[:, :8])                  # no place left
        assert same(before, state(d))
    finally:
        d.close()


@pytest.mark.parametrize("busy", ["caller", "own"])
def test_calls_under_another_stream(busy):
    """Made on one stream, fed and read under another, with one of the two a few milliseconds behind: what the caller made is there
    before the kernels read it, tables and lengths are there and stay, results are there when the caller's stream goes on."""
    s, own = torch.cuda.Stream(), torch.cuda.Stream()
    with torch.cuda.stream(own):
        d, m, g = make(24, 3, 64, {1: 30, 2: 7}, 4, keep=32, slack=4, recent=4, sink=2)
    m.keep, m.slack, m.recent, m.sink = 32, 4, 4, 2
    torch.cuda.synchronize()
    try:
        for step in range(8):
            x, pos = token(g, 3)
            with torch.cuda.stream(s if busy == "caller" else own):
                torch.cuda._sleep(10_000_000)
            with torch.cuda.stream(s):
                xd, pd = x.cuda(), pos.cuda()
                got = d.step(xd, pd).clone()
                del xd, pd
                torch.full((1 << 20,), 0x7FFFFFFF, dtype=torch.int32, device="cuda")       # takes what the allocator has back
            s.synchronize()
            compare(d, m, got.double().cpu(), x, pos)
            for req in [r for r, row in d.place_of.items() if len(m.w[(0, r, 0)]) >= 36]:
                m.evict(req)
            assert all(d.held[row] == len(m.w[(0, req, 0)]) for req, row in d.place_of.items())
        with torch.cuda.stream(s):
            x, pos = torch.randn(LAYERS, 20, HQ + 2 * HK, DIM, generator=g).to(torch.bfloat16), torch.randint(0, 50, (3, 20), generator=g, dtype=torch.int32)
            d.add(5, x.cuda(), pos.cuda())
        for layer in range(LAYERS):
            m.append(5, layer, x[layer], pos)
        m.seen[5] = 20
        with torch.cuda.stream(s):
            d.rotate([1], [])
            x, pos = token(g, 3)
            got = d.step(x.cuda(), pos.cuda()).clone()
        s.synchronize()
        compare(d, m, got.double().cpu(), x, pos, away=[1])
    finally:
        d.close()
