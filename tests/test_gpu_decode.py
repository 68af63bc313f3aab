"""The decode loop (pool, block table, kv_append, kv_attend, kv_evict together) against a plain cache of lists in 64 bits."""
import pytest
import torch

import ops_reference as R

pytestmark = pytest.mark.gpu


class Plain:
    """Per layer, request and KV head: the rows of K and V as the cache's type holds them, their weights and ages."""

    def __init__(self, layers, q_heads, kv_heads, dim, keep, slack, recent, sink, axis_of):
        self.layers, self.q_heads, self.kv_heads, self.dim = layers, q_heads, kv_heads, dim
        self.keep, self.slack, self.recent, self.sink, self.axis_of = keep, slack, recent, sink, axis_of
        self.k, self.v, self.w, self.age, self.seen = {}, {}, {}, {}, {}

    def turn(self, x, positions):
        half = self.dim // 2
        inv = (10000.0 ** (-torch.arange(half, dtype=torch.float64) / half)).float().double()
        angle = positions.double()[torch.tensor(self.axis_of)] * inv[:, None]
        return R.rotate(x.double(), angle.T[:, None], True)

    def append(self, req, layer, x, positions):
        h, n = self.q_heads, self.kv_heads
        y = self.turn(x[:, :h + n], positions)
        k = y[:, h:].to(torch.bfloat16).double()
        for g in range(n):
            key = (layer, req, g)
            self.k.setdefault(key, []).extend(k[:, g])
            self.v.setdefault(key, []).extend(x[:, h + n + g].double())
            self.w.setdefault(key, []).extend([0.0] * len(x))
            self.age.setdefault(key, []).extend(range(self.seen.get(req, 0), self.seen.get(req, 0) + len(x)))
        return y[:, :h].to(torch.bfloat16).double()

    def attend(self, req, layer, q):
        out = torch.zeros(self.q_heads, self.dim, dtype=torch.float64)
        bound = torch.zeros_like(out)
        for g in range(self.q_heads):
            key = (layer, req, g // (self.q_heads // self.kv_heads))
            k, v = torch.stack(self.k[key]), torch.stack(self.v[key])
            p = (k @ q[g] / self.dim ** 0.5).softmax(0)
            out[g], bound[g] = p @ v, 2 * R.UNIT["bf16"] * (p @ v.abs())
            self.w[key] = [a + float(b) for a, b in zip(self.w[key], p)]
        return out, bound

    def evict(self, req):
        for key in [k for k in self.k if k[1] == req]:
            n = len(self.w[key])
            for d, s in R.evict(self.w[key], self.age[key], n, self.keep, self.recent, self.sink, self.seen[req]):
                for rows in (self.k, self.v, self.w, self.age):
                    rows[key][d] = rows[key][s]
            for rows in (self.k, self.v, self.w, self.age):
                del rows[key][self.keep:]


def test_decode_with_eviction_and_rotation_matches_a_plain_cache():
    from paper_2601_20309_b200.decode import Decoder
    layers, hq, hk, dim, keep, slack, places = 2, 4, 2, 64, 24, 8, 4
    d = Decoder(layers, 16, hq, hk, dim, 40, 80, places, 64, keep=keep, slack=slack, recent=6, sink=2, sections=(8, 12, 12))
    m = Plain(layers, hq, hk, dim, keep, slack, 6, 2, d.axis_of)
    g = torch.Generator().manual_seed(5)
    evictions = 0
    try:
        for req, n in ((7, 30), (3, 5), (9, 17)):
            x = torch.randn(layers, n, hq + 2 * hk, dim, generator=g).to(torch.bfloat16)
            pos = torch.randint(0, 50, (3, n), generator=g, dtype=torch.int32)
            d.add(req, x.cuda(), pos.cuda())
            for layer in range(layers):
                m.append(req, layer, x[layer], pos)
            m.seen[req] = n
        away = []
        for step in range(40):
            x = torch.randn(layers, places, hq + 2 * hk, dim, generator=g).to(torch.bfloat16)
            pos = torch.randint(0, 200, (3, places), generator=g, dtype=torch.int32)
            got = d.step(x.cuda(), pos.cuda()).double().cpu()
            for req, row in d.place_of.items():
                if req in away:
                    assert (got[:, row] == 0).all()
                    continue
                for layer in range(layers):
                    q = m.append(req, layer, x[layer, row:row + 1], pos[:, row:row + 1])
                    out, bound = m.attend(req, layer, q[0])
                    # a score is off by a rounding of K's type where the turned value lies near the middle of two: widened by that
                    assert ((got[layer, row] - out).abs() <= bound + 0.02).all(), (step, req, layer)
                m.seen[req] += 1
                if len(m.w[(0, req, 0)]) >= keep + slack:
                    # ages agree exactly after each eviction: the same slots were kept
                    m.evict(req)
                    evictions += 1
                    for layer in range(layers):
                        for h in range(hk):
                            assert d.order[layer, row, h, :keep].tolist() == m.age[(layer, req, h)], (step, req, layer, h)
                assert d.held[row] == len(m.w[(0, req, 0)])
            if step % 7 == 3:
                away = [7, 9] if not away else []
                d.rotate(away, [] if away else [7, 9])
        assert evictions >= 3
        held = sum(-(-d.held[r] // 16) for r in d.place_of.values() if d.running[r])
        assert d.table.kv_table_get_stats()["free_gpu_blocks"] == 40 - held
    finally:
        d.close()
