"""Host side of the cache in 4 bits that needs no GPU: struct layout, row sizes, null arguments; and the reference itself against a
row worked out by hand."""
import ctypes as C

import torch

import ops_reference_q4 as Q
from paper_2601_20309_b200 import binding as B


def test_struct_sizes_match_the_header_layout():
    assert C.sizeof(B.kv_norm_args_t) == 40
    assert C.sizeof(B.kv_read_args_t) == 104


def test_row_units():
    for dim, groups in ((8, 2), (64, 2), (72, 4), (80, 4), (128, 4), (136, 8), (256, 8)):
        assert B.kv_cache_row_units("bf16", dim) == B.kv_cache_row_units("f16", dim) == dim
        assert B.kv_cache_row_units("bf16_q4", dim) == B.kv_cache_row_units("f16_q4", dim) == 10 * groups
    for dim in (0, -8, 4, 100, 264):
        assert B.kv_cache_row_units("bf16_q4", dim) == 0
    assert B.lib().kv_cache_row_units(9, 128) == 0


def test_null_arguments_are_refused_without_a_device():
    L = B.lib()
    assert L.kv_append_normed(None, None, None, None) == B.KV_ERR_INVALID_ARG
    assert L.kv_read(None, None, None) == B.KV_ERR_INVALID_ARG


def test_pack_by_hand():
    """64 elements 0, 1/4, .. as f16: group 0 runs from 0 to 31/4, step 31/60 rounded to bf16 = 0.515625, group 1 from 8."""
    x = (torch.arange(64) / 4).to(torch.float16).reshape(1, 1, 64)
    lo, step, code = Q.quantise(x)
    assert lo[0, 0, [0, 63]].tolist() == [0.0, 8.0] and step[0, 0, 0] == 0.515625
    assert code[0, 0, :5].tolist() == [0, 0, 1, 1, 2] and code[0, 0, 31] == 15
    k, w = Q.pack(x, 0, "f16")
    v, _ = Q.pack(x, 1, "f16")
    # K: byte 0 has elements 0 and 1, byte 4 (group 1's first word) elements 32 and 33, byte 8 elements 8 and 9
    assert k[0, 0, 0] == 0 and k[0, 0, 1] == 1 + 16 * 1 and k[0, 0, 8] == int(code[0, 0, 8]) + 16 * int(code[0, 0, 9])
    # V: half word 0 has elements 0 to 3, half word 1 elements 32 to 35, half word 2 elements 4 to 7
    assert v[0, 0, 1] == 1 + 16 * 1 and v[0, 0, 2] == int(code[0, 0, 32]) + 16 * int(code[0, 0, 33]) and v[0, 0, 4] == 2 + 16 * int(code[0, 0, 5])
    assert w[0, 0].view(torch.int16)[1].item() == torch.tensor(0.515625, dtype=torch.bfloat16).view(torch.int16).item()
    assert w[0, 0].view(torch.int16)[2].item() == torch.tensor(8.0, dtype=torch.float16).view(torch.int16).item()


def test_quantised_values_are_within_half_a_step():
    x = torch.randn(50, 3, 80, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    lo, step, code = Q.quantise(x)
    # the step is rounded by 2^-9 of it, so the highest element may lie 15 * 2^-9 steps beyond the last code
    assert ((lo + step * code - x.double()).abs() <= step * (0.5 + 15 * 2.0 ** -9)).all()
