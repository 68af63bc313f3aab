"""Host side of the operators on the device cache at its edges, without a GPU: the block table when host memory runs out inside a
shrink, error texts of several threads."""
import ctypes as C
import os
import subprocess
import threading

from paper_2601_20309_b200 import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# The table's source with a pool that does nothing and an operator new that fails on demand: the n-th allocation from now on.
PROGRAM = r"""
#include "paper_2601_20309_b200/csrc/kv_table.cu"
#include <cstdlib>

static long fail_in = -1;
static int64_t done = 0;             // 1: the pool's transfers have finished
void *operator new(size_t n)
{
    if (fail_in >= 0 && fail_in-- == 0) throw std::bad_alloc();
    if (void *p = malloc(n)) return p;
    throw std::bad_alloc();
}
void operator delete(void *p) noexcept { free(p); }
void operator delete(void *p, size_t) noexcept { free(p); }

extern "C" {
int32_t kv_pool_progress(kv_pool_t *, int64_t *a, int64_t *b, int64_t *c, int64_t *d)
{
    if (a) *a = 1;               // a swap-out was issued and has not finished: released blocks are pending ones
    if (b) *b = done;
    if (c) *c = 0;
    if (d) *d = 0;
    return KV_OK;
}
int32_t kv_pool_shape(kv_pool_t *, kv_pool_shape_t *s)
{
    s->num_gpu_blocks = 200;
    s->num_host_blocks = 300;
    s->block_size = 16;
    return KV_OK;
}
int32_t kv_sync(kv_pool_t *)
{
    done = 1;
    return KV_OK;
}
int32_t kv_swap_out(kv_pool_t *, const int32_t *, const int32_t *, int64_t) { return KV_OK; }
int32_t kv_rotate(kv_pool_t *, const int32_t *, const int32_t *, int64_t, const int32_t *, const int32_t *, int64_t) { return KV_OK; }
const char *kv_last_error(kv_pool_t *) { return ""; }
}

static bool check(bool ok, const char *what, long at)
{
    if (!ok) printf("%s (allocation %ld)\n", what, at);
    return ok;
}

int main()
{
    bool ok = true, failed = false;
    int dummy;
    for (long at = 0; at < 200; ++at) {
        kv_table_t *t = nullptr;
        done = 0;
        ok &= kv_table_create((kv_pool_t *)&dummy, &t) == KV_OK;
        // request 1 between others whose host blocks come back, so that its own merge with free ones or stand alone
        int64_t n = 0;
        for (int r = 0; r < 5; ++r) {
            ok &= kv_req_add(t, r, 16 * 20) == KV_OK;
            ok &= kv_eager_rotate(t, 7, &n) == KV_OK && n == 7;
        }
        for (int k = 0; k < 10; ++k) kv_eager_rotate(t, 6, &n);
        kv_req_finish(t, 0);
        kv_req_finish(t, 3);
        kv_table_stats_t before, after;
        kv_table_get_stats(t, &before);
        kv_req_info_t info;
        kv_req_info(t, 1, &info);
        const int64_t host = info.host_blocks;
        ok &= check(info.synced_blocks > 5, "the request has copies", at);
        fail_in = at;
        const int32_t rc = kv_req_shrink(t, 1, 40);
        fail_in = -1;
        kv_req_info(t, 1, &info);
        kv_table_get_stats(t, &after);
        ok &= check(info.synced_blocks == 0, "a stale copy counts as valid", at);
        ok &= check(after.free_gpu_blocks + info.num_blocks == before.free_gpu_blocks + 20, "device blocks are lost", at);
        ok &= check(after.free_host_blocks + info.host_blocks == before.free_host_blocks + host, "host blocks are lost", at);
        if (rc != KV_OK) {
            failed = true;
            ok &= check(rc == KV_ERR_NOMEM && info.num_blocks >= 3 && info.tokens >= 40, "not a whole request", at);
            ok &= check(kv_req_shrink(t, 1, 40) == KV_OK, "a second try", at);
        }
        kv_req_info(t, 1, &info);
        ok &= check(info.tokens == 40 && info.num_blocks == 3 && info.synced_blocks == 0, "shrunk", at);
        for (int r : {1, 2, 4}) kv_req_finish(t, r);
        kv_table_get_stats(t, &after);
        ok &= check(after.free_gpu_blocks == 200 && after.free_host_blocks == 300 && after.free_host_extents == 1, "all blocks are back, in one run", at);
        // the free host blocks that are counted are there: one request takes them all
        ok &= check(kv_req_add(t, 9, 16 * 200) == KV_OK && kv_eager_rotate(t, 200, &n) == KV_OK && n == 200, "taken again", at);
        kv_table_destroy(t);
        if (rc == KV_OK) break;
    }
    ok &= check(failed, "an allocation failed", -1);
    return ok ? 0 : 1;
}
"""


def test_a_shrink_without_memory_loses_nothing_and_leaves_no_stale_copy(tmp_path):
    source, exe = tmp_path / "shrink.cpp", tmp_path / "shrink"
    source.write_text(PROGRAM)
    built = subprocess.run(["g++", "-O1", "-std=c++17", "-x", "c++", f"-I{ROOT}", "-o", exe, source], capture_output=True, text=True)
    assert built.returncode == 0, built.stderr
    run = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert run.returncode == 0, run.stdout


def test_the_error_text_of_a_failed_create_belongs_to_its_thread():
    """One context per device is often made by one thread per device: what went wrong in one is not told to another."""
    L = B.lib()
    texts = {}

    def other():
        texts["before"] = L.kv_ops_last_error(None)
        assert L.kv_ops_create(0, None, None) == B.KV_ERR_INVALID_ARG
        texts["after"] = L.kv_ops_last_error(None)

    handle = C.c_void_p()
    assert L.kv_ops_create(1 << 20, None, C.byref(handle)) != B.KV_OK and not handle
    mine = L.kv_ops_last_error(None)
    t = threading.Thread(target=other)
    t.start()
    t.join()
    assert texts == {"before": b"no error", "after": b"null argument"}
    assert L.kv_ops_last_error(None) == mine != b"null argument"
