"""Attention over a cache in 4 bits when a wait inside its kernel runs out: the call ends, the context says so, the GPU is as before."""
import math

import pytest
import torch

import ops_reference_q4 as Q
from paper_2601_20309_b200 import binding as B

pytestmark = pytest.mark.gpu

# whole blocks by bulk copies, in one CTA's rows and in pieces; blocks that tiles end in (other warps load), with a window; one head and several
# ways of it, several heads; heads of 256 whose loading warps give registers away
SHAPES = [
    # lens, q_heads, kv_heads, dim, bs, dtype, window
    ([37], 8, 2, 128, 16, "bf16", 0),
    ([700, 0, 90, 3000], 32, 8, 128, 16, "bf16", 0),
    ([9000], 8, 1, 128, 64, "f16", 0),
    ([700, 2000, 40], 15, 3, 80, 24, "bf16", 333),
    ([5000, 100], 4, 1, 64, 20, "f16", 0),
    ([900, 300], 16, 1, 256, 16, "bf16", 0),
    ([300, 400], 12, 4, 256, 12, "f16", 100),
]


def call(ops, c, q, window, weights):
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], device="cuda")
    w = torch.zeros(len(c.lens_list), c.heads, c.longest, device="cuda") if weights else None
    ops.kv_attend(c.handle(B), 0, q, c.tables, c.lens, c.longest, out=out, lse=lse, window=window, weights_out=w)
    return out, lse, w


@pytest.mark.parametrize("lens,hq,hk,dim,bs,dtype,window", SHAPES)
@pytest.mark.parametrize("weights", [True, False])
def test_a_wait_that_runs_out_ends_the_call(lens, hq, hk, dim, bs, dtype, window, weights):
    c = Q.Cache(lens, hk, dim, bs, dtype, seed=1, layers=1)
    q = torch.randn(len(lens), hq, dim, generator=c.g).to(c.tdtype).cuda()
    before = c.pool.clone()
    with B.KVOps(0) as good:
        want = call(good, c, q, window, weights)
        good.kv_ops_sync()
        # without looking: the first wait of every warp runs out
        with B.KVOps(0) as ops:
            ops.kv_ops_set_wait_limit(0, 0)
            for _ in range(3):
                call(ops, c, q, window, weights)
            assert ops.kv_ops_sync(check=False) == B.KV_ERR_TIMEOUT
            ops.kv_ops_set_wait_limit(64, 2 * 10 ** 9)          # sticky
            assert ops.kv_ops_sync(check=False) == B.KV_ERR_TIMEOUT
            with pytest.raises(B.KVError, match="ran out"):
                ops.kv_ops_sync()
        # one to eight looks: some warps come through and others do not; where all do, the results are those of any other call
        for polls in (1, 2, 3, 5, 8) * 4:
            with B.KVOps(0) as ops:
                ops.kv_ops_set_wait_limit(polls, 0)
                got = call(ops, c, q, window, weights)
                status = ops.kv_ops_sync(check=False)
                assert status in (B.KV_OK, B.KV_ERR_TIMEOUT)
                if status == B.KV_OK:
                    assert all(x is None or torch.equal(x, y) for x, y in zip(got, want))
        again = call(good, c, q, window, weights)
        good.kv_ops_sync()
    assert all(x is None or torch.equal(x, y) for x, y in zip(again, want))
    assert torch.equal(before, c.pool)
    assert not any(math.isnan(float(x.float().sum())) for x in want if x is not None)


def test_wait_limit_arguments():
    with B.KVOps(0) as ops:
        assert ops.kv_ops_set_wait_limit(16, 61 * 10 ** 9, check=False) == B.KV_ERR_INVALID_ARG
        assert ops.kv_ops_set_wait_limit(4, 10 ** 9) == B.KV_OK           # a shorter but ample limit changes nothing
        c = Q.Cache([300], 2, 128, 16, seed=2, layers=1)
        q = torch.randn(1, 8, 128, generator=c.g).to(c.tdtype).cuda()
        call(ops, c, q, 0, True)
        ops.kv_ops_sync()


def test_a_timeout_outranks_a_bad_length():
    """A context that has skipped a sequence before says so, and says that results are not to be used once a wait has run out."""
    c = Q.Cache([300, 20], 2, 128, 16, seed=3, layers=1)
    q = torch.randn(2, 8, 128, generator=c.g).to(c.tdtype).cuda()
    with B.KVOps(0) as ops:
        lens, right = torch.tensor([300, 500], dtype=torch.int32, device="cuda"), c.lens
        c.lens = lens
        call(ops, c, q, 0, False)
        assert ops.kv_ops_sync(check=False) == B.KV_ERR_RANGE
        c.lens = right
        call(ops, c, q, 0, False)
        assert ops.kv_ops_sync(check=False) == B.KV_ERR_RANGE
        ops.kv_ops_set_wait_limit(0, 0)
        call(ops, c, q, 0, False)
        with pytest.raises(B.KVError, match="ran out") as e:
            ops.kv_ops_sync()
        assert e.value.code == B.KV_ERR_TIMEOUT
        # and a bad length afterwards does not hide it
        ops.kv_ops_set_wait_limit(64, 2 * 10 ** 9)
        c.lens = lens
        call(ops, c, q, 0, False)
        assert ops.kv_ops_sync(check=False) == B.KV_ERR_TIMEOUT
        c.lens = right
