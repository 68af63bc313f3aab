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
