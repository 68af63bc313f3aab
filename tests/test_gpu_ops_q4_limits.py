"""Norms of rows at the limits the header names, keys included; tokens of no sequence are reported by kv_read; the numbers of heads the calls take."""
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


def angles(dim):
    return torch.zeros(dim // 2, device="cuda")


@pytest.mark.parametrize("dim", [64, 80, 256])
@pytest.mark.parametrize("q4", [False, True])
def test_norms_at_their_limits(ops, dim, q4):
    """Rows of elements of 2^59 and of 2^-60, rows with one element that is not 0, and rows of both sizes: q and k, from the float32 and the float64 path."""
    g = torch.Generator().manual_seed(1)
    sign = torch.randint(0, 2, (8, dim), generator=g) * 2.0 - 1
    x = sign.clone()
    x[0] *= 2.0 ** 59
    x[1] *= 2.0 ** -60
    x[2] *= 2.0 ** 59 * (0.25 + 0.75 * torch.rand(dim, generator=g))
    x[3] *= 2.0 ** -60 * (1 + torch.rand(dim, generator=g))
    x[4], x[5] = 0.0, 0.0
    x[4, dim - 1], x[5, 3] = 2.0 ** 59, 2.0 ** -60
    x[6, : dim // 2] *= 2.0 ** 59
    x[6, dim // 2:] *= 2.0 ** -60
    x = x.to(torch.bfloat16)[:, None].expand(8, 3, dim).contiguous().cuda()
    c = (Q if q4 else R).Cache([8], 1, dim, 16, seed=2)
    w = (1 + 0.2 * torch.randn(dim, generator=g)).cuda()
    starts = torch.tensor([0, 8], dtype=torch.int32, device="cuda")
    for eps in (0.0, 2.0 ** -130):
        q, k = (torch.full((8, 1, dim), math.nan, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        ops.kv_append(c.handle(B), 0, x[:, :1], x[:, 1:2], x[:, 2:], c.tables, c.lens, positions=torch.zeros(1, 8, dtype=torch.int32, device="cuda"),
                      inv_freq=angles(dim), q_out=q, seq_starts=starts, q_norm=w, k_norm=w, norm_eps=eps)
        ops.kv_read(c.handle(B), 0, c.tables, c.lens, k_out=k, seq_starts=starts)
        ops.kv_ops_sync()
        want = Q.normed(x[:, :1].double().cpu(), w.double().cpu(), eps)
        # sums, root and factors in float32, 2^-18 of the row's largest; one rounding
        near = 2.0 ** -8 * want.abs() + 2.0 ** -18 * want.abs().amax(-1, keepdim=True)
        assert ((q.double().cpu() - want).abs() <= near).all()
        if q4:
            lo, step, code = Q.quantise(want.float().to(torch.bfloat16))
            assert torch.equal(k.cpu(), (lo + step * code).float().to(torch.bfloat16))
        else:
            assert ((k.double().cpu() - want).abs() <= near).all()


@pytest.mark.parametrize("q4", [False, True])
def test_read_reports_tokens_of_no_sequence(q4):
    c = (Q if q4 else R).Cache([20, 9], 2, 64, 16, seed=3)
    for starts, status in (([0, 20, 29], B.KV_OK), ([1, 20, 29], B.KV_ERR_RANGE), ([0, 20, 28], B.KV_ERR_RANGE), ([0, 21, 29], B.KV_ERR_RANGE)):
        k = torch.full((29, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda")
        with B.KVOps(0) as ops:
            ops.kv_read(c.handle(B), 0, c.tables, c.lens, k_out=k, seq_starts=torch.tensor(starts, dtype=torch.int32, device="cuda"))
            assert ops.kv_ops_sync(check=False) == status, starts
        nobody = [t for t in range(29) if t < starts[0] or t >= starts[2] or (starts[1] == 21 and t == 0)]
        assert (k[nobody] == 7).all() and not (k[[t for t in range(29) if t not in nobody]] == 7).all(-1).any()


def test_numbers_of_heads(ops):
    """kv_read takes up to 512 KV heads, kv_append up to 4096 rows per token, q's, k's and v's together; both refuse more."""
    lens = torch.ones(1, dtype=torch.int32, device="cuda")
    tables = torch.zeros(1, 1, dtype=torch.int32, device="cuda")
    store = torch.zeros(2 * 4 * 2048 * 20, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()

    def rows(heads):
        return torch.randn(1, heads, 8, device="cuda").to(torch.bfloat16)

    def append(heads, q_heads):
        cache = B.KVCache(store.data_ptr(), 1, 4, heads, 8, 1, dtype="bf16_q4")
        q = rows(q_heads) if q_heads else None
        ops.kv_append(cache, 0, q, rows(heads), rows(heads), tables, lens, positions=torch.zeros(1, 1, dtype=torch.int32, device="cuda"), inv_freq=angles(8), q_out=q)

    cache = B.KVCache(store.data_ptr(), 1, 4, 512, 8, 1, dtype="bf16_q4")
    k, out = rows(512), rows(512)
    ops.kv_append(cache, 0, None, k, k, tables, lens, positions=torch.zeros(1, 1, dtype=torch.int32, device="cuda"), inv_freq=angles(8))
    ops.kv_read(cache, 0, tables, lens, k_out=out)
    ops.kv_ops_sync()
    lo, step, code = Q.quantise(k.cpu())
    assert torch.equal(out.cpu(), (lo + step * code).float().to(torch.bfloat16))
    append(2048, 0)
    append(1000, 2096)
    ops.kv_ops_sync()
    with pytest.raises(B.KVError, match="too many heads"):
        append(2048, 1)
    with pytest.raises(B.KVError, match="too many heads"):
        ops.kv_read(B.KVCache(store.data_ptr(), 1, 4, 513, 8, 1, dtype="bf16_q4"), 0, tables, lens, k_out=rows(513))
