"""Host side of the operators on the device cache that needs no GPU: struct layout, the block table's shrink."""
import ctypes as C
import random

from oracle.kv_block_table import BlockTableModel
from paper_2601_20309_b200 import binding as B


def test_struct_sizes_match_the_header_layout():
    assert C.sizeof(B.kv_cache_t) == 40
    assert C.sizeof(B.kv_attend_args_t) == 144
    assert C.sizeof(B.kv_append_args_t) == 360
    assert C.sizeof(B.kv_evict_args_t) == 160


def test_null_arguments_are_refused_without_a_device():
    L = B.lib()
    assert L.kv_ops_destroy(None) == B.KV_ERR_INVALID_ARG and L.kv_ops_sync(None) == B.KV_ERR_INVALID_ARG
    assert L.kv_attend(None, None, None) == B.KV_ERR_INVALID_ARG
    assert L.kv_append(None, None, None) == B.KV_ERR_INVALID_ARG
    assert L.kv_evict(None, None, None) == B.KV_ERR_INVALID_ARG
    assert L.kv_pool_cache(None, 0, None) == B.KV_ERR_INVALID_ARG
    assert L.kv_req_shrink(None, 1, 1) == B.KV_ERR_INVALID_ARG
    assert len(L.kv_ops_last_error(None)) > 3


def test_shrink_by_hand():
    """Blocks of 16; a request of 100 tokens owns 7 device blocks, 6 of them copied out; at 40 tokens it owns 3 and no copy counts."""
    t = B.KVTable(num_gpu_blocks=20, num_host_blocks=20, block_size=16)
    t.kv_req_add(1, 100)
    assert t.kv_eager_rotate(100) == 6
    assert t.kv_req_shrink(1, 101, check=False) == B.KV_ERR_INVALID_ARG
    assert t.kv_req_shrink(1, 0, check=False) == B.KV_ERR_INVALID_ARG
    assert t.kv_req_shrink(2, 5, check=False) == B.KV_ERR_INVALID_ARG
    first = t.kv_req_blocks(1)[0][:3].tolist()
    t.kv_req_shrink(1, 40)
    i = t.kv_req_info(1)
    assert (i["tokens"], i["num_blocks"], i["synced_blocks"], i["host_blocks"], i["dirty_blocks"]) == (40, 3, 0, 3, 1)
    assert t.kv_req_blocks(1)[0].tolist() == first
    s = t.kv_table_get_stats()
    assert (s["free_gpu_blocks"], s["free_host_blocks"]) == (17, 17)
    t.kv_req_append(1, 9)
    assert t.kv_req_info(1)["num_blocks"] == 4
    t.kv_req_preempt(1)
    assert t.kv_table_get_stats()["preempt_blocks_moved"] == 4                  # every host copy was stale
    assert t.kv_req_shrink(1, 5, check=False) == B.KV_ERR_INVALID_ARG           # it is not on the GPU
    t.kv_req_finish(1)
    s = t.kv_table_get_stats()
    assert (s["free_gpu_blocks"], s["free_host_blocks"]) == (20, 20)


def test_shrink_in_random_histories_matches_the_model():
    for seed in range(30):
        rng = random.Random(seed)
        t, m = B.KVTable(num_gpu_blocks=60, num_host_blocks=90, block_size=8), BlockTableModel(60, 90, 8)
        for step in range(120):
            rid = rng.randrange(8)
            op = rng.choice(["add", "append", "append", "shrink", "shrink", "eager", "rotate", "finish"])
            if op == "add":
                n = rng.randrange(1, 120)
                assert t.kv_req_add(rid, n, check=False) == m.add(rid, n)
            elif op == "append":
                n = rng.randrange(1, 30)
                assert t.kv_req_append(rid, n, check=False) == m.append(rid, n)
            elif op == "shrink":
                n = rng.randrange(0, 100)
                assert t.kv_req_shrink(rid, n, check=False) == m.shrink(rid, n)
            elif op == "eager":
                n = rng.randrange(0, 12)
                assert t.kv_eager_rotate(n) == len(m.eager(n))
            elif op == "rotate":
                on = [r for r in m.reqs if m.reqs[r].on_gpu and rng.random() < 0.4]
                off = [r for r in m.reqs if not m.reqs[r].on_gpu and rng.random() < 0.6]
                assert t.kv_req_rotate(on, off, check=False) == m.rotate(on, off)[0]
            else:
                assert t.kv_req_finish(rid, check=False) == m.finish(rid)
            s = t.kv_table_get_stats()
            assert (s["free_gpu_blocks"], s["free_host_blocks"], s["requests"]) == (m.free_gpu, m.free_host, len(m.reqs)), (seed, step, op)
            held = [g for r in m.reqs for g in t.kv_req_blocks(r)[0].tolist() if g >= 0]
            assert len(held) == len(set(held)) == 60 - m.free_gpu
            for r, q in m.reqs.items():
                i = t.kv_req_info(r)
                assert (i["tokens"], i["num_blocks"], bool(i["on_gpu"])) == (q.tokens, len(q.version), q.on_gpu)
                assert i["synced_blocks"] == sum(q.host_valid(b) for b in range(len(q.version)))
