// Host side of the operators on the device cache: argument checks, workspace, launches.
#include "../../include/duplexkv.h"

#include <algorithm>
#include <cstdio>
#include <cstring>
#include <new>
#include <vector>

#include "kv_append.cuh"
#include "kv_append_rows.cuh"
#include "kv_attend.cuh"
#include "kv_attend_q4.cuh"
#include "kv_evict.cuh"
#include "kv_read.cuh"

struct kv_ops {
    int device = 0, sms = 0;
    cudaStream_t stream = nullptr;
    uint8_t *ws = nullptr;
    size_t ws_bytes = 0;
    std::vector<void *> outgrown;    // earlier workspaces: captured graphs may hold them
    unsigned *status_host = nullptr, *status_dev = nullptr;
    int32_t sticky = KV_OK;
    unsigned wait_polls = KV_OPS_WAIT_POLLS;      // kv_ops_set_wait_limit
    unsigned long long wait_ns = KV_OPS_WAIT_NS;
    bool attend_ready[2][2][3][2] = {};   // [4 bits][bf16][head dimension][query tiles]: shared-memory limit raised
    char err[256];
};

namespace {

thread_local char g_ops_err[256] = "no error";

int32_t fail(kv_ops *o, int32_t code, const char *msg)
{
    snprintf(o ? o->err : g_ops_err, 256, "%s", msg);
    return code;
}

int32_t fail_cuda(kv_ops *o, cudaError_t e, const char *what)
{
    (void)cudaGetLastError();
    snprintf(o ? o->err : g_ops_err, 256, "%s: %s", what, cudaGetErrorString(e));
    if (o && o->sticky == KV_OK) o->sticky = KV_ERR_CUDA;
    return KV_ERR_CUDA;
}

// the context's device is current while one of these lives
struct OnDevice {
    int before = -1;
    explicit OnDevice(int device)
    {
        int now = -1;
        if (cudaGetDevice(&now) == cudaSuccess && now != device && cudaSetDevice(device) == cudaSuccess) before = now;
    }
    ~OnDevice()
    {
        if (before >= 0) (void)cudaSetDevice(before);
    }
};

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline bool is_bf16(const kv_cache_t *c) { return c->dtype == KV_DT_BF16 || c->dtype == KV_DT_BF16_Q4; }
inline bool is_q4(int32_t dtype) { return dtype == KV_DT_BF16_Q4 || dtype == KV_DT_F16_Q4; }
inline int q4_groups(int head_dim) { return head_dim <= 64 ? 2 : head_dim <= 128 ? 4 : 8; }
inline int64_t align256(int64_t a) { return (a + 255) / 256 * 256; }

int32_t grow_workspace(kv_ops *o, int64_t bytes)
{
    if (bytes < 0) return fail(o, KV_ERR_INVALID_ARG, "negative size");
    if ((size_t)bytes <= o->ws_bytes) return KV_OK;
    cudaStreamCaptureStatus st = cudaStreamCaptureStatusNone;
    if (cudaStreamIsCapturing(o->stream, &st) != cudaSuccess) (void)cudaGetLastError();
    if (st != cudaStreamCaptureStatusNone) return fail(o, KV_ERR_NOMEM, "the workspace cannot grow during stream capture: kv_ops_reserve it first");
    const size_t want = std::max<size_t>((size_t)bytes, o->ws_bytes + o->ws_bytes / 2);
    void *p = nullptr;
    try {
        o->outgrown.reserve(o->outgrown.size() + 1);
    } catch (...) {
        return fail(o, KV_ERR_NOMEM, "out of host memory");
    }
    if (cudaMalloc(&p, want) != cudaSuccess) {
        (void)cudaGetLastError();
        return fail(o, KV_ERR_NOMEM, "no device memory for the operators' workspace");
    }
    if (o->ws) o->outgrown.push_back(o->ws);
    o->ws = (uint8_t *)p;
    o->ws_bytes = want;
    return KV_OK;
}

// the checks that all calls share, and the address rule
int32_t make_view(kv_ops *o, const kv_cache_t *c, KvView &v)
{
    if (!c || !c->device_base) return fail(o, KV_ERR_INVALID_ARG, "no cache");
    if (c->num_layers <= 0 || c->block_size <= 0 || c->kv_heads <= 0 || c->head_dim <= 0 || c->num_gpu_blocks <= 0 || c->num_gpu_blocks > INT32_MAX)
        return fail(o, KV_ERR_INVALID_ARG, "bad cache shape");
    if (c->device_layout != KV_DEV_LAYER_FIRST && c->device_layout != KV_DEV_BLOCK_FIRST) return fail(o, KV_ERR_INVALID_ARG, "unknown device layout");
    if (c->dtype != KV_DT_BF16 && c->dtype != KV_DT_F16 && !is_q4(c->dtype)) return fail(o, KV_ERR_INVALID_ARG, "unknown element type");
    if (c->head_dim % 8 || c->head_dim > 256) return fail(o, KV_ERR_UNSUPPORTED, "head_dim must be a multiple of 8, at most 256");
    if ((uintptr_t)c->device_base % 16) return fail(o, KV_ERR_INVALID_ARG, "the cache must be 16-byte aligned");
    if (is_q4(c->dtype) && c->block_size % 4) return fail(o, KV_ERR_UNSUPPORTED, "a cache in 4 bits needs blocks of a multiple of 4 tokens");
    const int64_t row = (int64_t)c->kv_heads * kv_cache_row_units(c->dtype, c->head_dim) * 2, seg = row * c->block_size;
    if (seg > INT32_MAX) return fail(o, KV_ERR_UNSUPPORTED, "a plane of one block exceeds 2 GiB");
    v.base = (uint8_t *)c->device_base;
    v.blk_stride = c->device_layout == KV_DEV_BLOCK_FIRST ? seg * 2 * c->num_layers : seg;
    v.plane_stride = c->device_layout == KV_DEV_BLOCK_FIRST ? seg : seg * c->num_gpu_blocks;
    v.groups = is_q4(c->dtype) ? q4_groups(c->head_dim) : 0;
    v.row_stride = v.groups ? 16 * v.groups : (int)row;
    v.head_stride = v.groups ? 20 * v.groups * c->block_size : c->head_dim * 2;
    v.bs = c->block_size;
    v.nb = (int)c->num_gpu_blocks;
    v.heads = c->kv_heads;
    v.dim = c->head_dim;
    v.status = o->status_dev;
    return KV_OK;
}

int32_t set_tables(kv_ops *o, KvView &v, const int32_t *tables, int64_t stride, int32_t width, const int32_t *lens, int64_t max_len)
{
    // before any token there is a batch without blocks: tables of no entries
    if ((!tables && (width || max_len)) || !lens) return fail(o, KV_ERR_INVALID_ARG, "block_tables and lens are needed");
    if (width < 0 || stride < 0) return fail(o, KV_ERR_INVALID_ARG, "bad block table shape");
    if (max_len < 0 || max_len > INT32_MAX / 2) return fail(o, KV_ERR_INVALID_ARG, "bad max_len");
    if (max_len > (int64_t)width * v.bs) return fail(o, KV_ERR_INVALID_ARG, "the block tables are too narrow for max_len");
    v.tables = tables;
    v.table_stride = stride;
    v.lens = lens;
    v.max_len = max_len;
    return KV_OK;
}

int32_t launched(kv_ops *o, const char *what)
{
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? KV_OK : fail_cuda(o, e, what);
}

// ---- attend

struct AttendPlan {
    int dp, nt, warps;                       // kernel shape: padded head dimension, tiles of 8 query heads, warps per CTA
    size_t smem;
    int64_t lse, part_of, part_ml, part_o, total;   // workspace offsets (the scores lie at 0)
};

constexpr int64_t ATTEND_SMEM = 227 * 1024 - 4096;   // what a CTA may have, less the kernel's static share
// Rows of up to this many steps are never split.  A step of one warp takes about 0.9 us, the second kernel 4 to 7 (the more
// with weights to add up): 4 sequences of 500 slots with weights 13.5 us whole, 17.6 split; 1 of 900 without 14.7 whole, 12.1 split.
// Near the limit with weights few whole rows lose already: of 900 slots one takes 21.6 us whole and 16.7 split, 16 take 26.8 and 29.1
constexpr int ATTEND_ALONE_STEPS = 4, ATTEND_ALONE_STEPS_WEIGHTS = 8;
// In 4 bits a step is two tiles of each warp, and the limit the same with weights and without: one sequence of 1000 slots (4 steps) 14.5 us
// whole and 14.7 split, with weights 17.6 and 19.7; of 2000 (8 steps) 23.9 and 15.0, 33.4 and 20.1; 64 of 100 (4 steps) 12.3 and 15.7
constexpr int ATTEND_ALONE_STEPS_Q4 = 4;
// No piece is shorter: with 1 step one sequence of 2000 slots takes 22.5 us, with 2 18.8, with 4 18.8; seven windows of 333 12.8, 14.9, 17.9
constexpr int ATTEND_MIN_STEPS = 2;
// CTAs of the join per piece that put rows together.  With weights there are KV_JOIN_SHARES others beside them: 64 sequences 90.6 us
// with 1, 90.2 with 2, 90.0 with 4; one of 131072 slots 27.8, 28.0, 29.0.  Without: 32 sequences of the 70B shape 86.0, 82.8, 81.2
// (8: 84.5); 64 sequences 80.0, 78.6, 78.1 (82.2); one of 131072 slots 25.0, 25.3, 25.3 (27.0)
constexpr int ATTEND_ROW_CTAS_WEIGHTS = 1, ATTEND_ROW_CTAS = 4;

int32_t plan_attend(kv_ops *o, const kv_cache_t *c, const kv_attend_args_t *a, KvAttend &k, AttendPlan &p)
{
    if (!a) return fail(o, KV_ERR_INVALID_ARG, "no arguments");
    int32_t rc = make_view(o, c, k.c);
    if (rc != KV_OK) return rc;
    if (a->layer < 0 || a->layer >= c->num_layers) return fail(o, KV_ERR_RANGE, "no such layer");
    if (a->num_seqs < 0 || a->num_seqs > 65535 || a->q_heads <= 0 || a->window < 0) return fail(o, KV_ERR_INVALID_ARG, "bad count");
    if (a->q_heads % c->kv_heads) return fail(o, KV_ERR_INVALID_ARG, "q_heads must be a multiple of kv_heads");
    if (a->q_heads / c->kv_heads > KV_MAX_GROUP || c->kv_heads > 65535) return fail(o, KV_ERR_UNSUPPORTED, "too many heads");
    if (a->max_len < 0 || a->max_len > INT32_MAX / 2) return fail(o, KV_ERR_INVALID_ARG, "bad max_len");
    k.group = a->q_heads / c->kv_heads;
    p.dp = c->head_dim <= 64 ? 64 : c->head_dim <= 128 ? 128 : 256;
    // One tile of 8 query heads or two at once; more than 16 walk the cache again for each 16.  32 sequences around 8k slots, 2 KV
    // heads, 377 MB: groups of 8 72 us with one tile and 81 with two, 9 123 and 82, 16 124 and 84; 17 to 32 147, 64 268 us
    // (with weights 8 86, 16 110, 32 235, 64 598)
    p.nt = k.group <= 8 ? 1 : 2;
    const int G = k.c.groups, most = G ? KV_Q4_WARPS : p.dp == 256 ? KV_ATTEND_WARPS / 2 : KV_ATTEND_WARPS;
    // one address per tile where a block holds whole tiles, else one per row: 70B shape 80.4 against 89.2 us, 64 sequences with
    // weights 90.3 against 100.5, one of 131072 slots 27.9 against 28.9
    k.whole_tiles = c->block_size % 16 == 0;
    // KV heads per CTA: as many as there are warps, so that a CTA reads whole rows of the cache.  Short rows that no CTA
    // shares (no second kernel) rather go one head to a CTA while there are SMs for it, with more warps along the row: 1 (16)
    // sequences of 37 slots and 8 KV heads 6.9 (7.2) us, all heads in one CTA 10.6 (10.8); of 130 8.9 (9.3) against 12.3 (15.5); of 16,
    // where one step is all there is, 6.9 (7.2) against 6.7 (6.8).
    auto shape = [&](int heads_wanted) {
        k.hc = 1;
        for (int d = 2; d <= std::min(heads_wanted, G ? KV_Q4_WARPS : KV_ATTEND_WARPS); ++d)
            if (c->kv_heads % d == 0) k.hc = d;
        k.tw = 1;
        while (k.hc * k.tw * 2 <= most && !(G && !k.whole_tiles && k.tw * 2 * kv_q4_sub(G, p.nt) > 8)) k.tw *= 2;   // rows are looked up by a warp: 8 tiles by fours
        p.warps = k.hc * k.tw;
        if (G) k.tw *= kv_q4_sub(G, p.nt);               // a warp takes two tiles at once
        return ceil_div(a->max_len + 15, 16 * k.tw);     // steps of the longest row
    };
    k.group_chunks = (int)ceil_div(k.group, 8 * p.nt);
    const bool one_head = (int64_t)a->num_seqs * c->kv_heads * k.group_chunks <= o->sms;
    int64_t longest = shape(one_head ? 1 : most);
    // query-head chunks of one KV head all add to the same weights: those go through the second kernel
    const bool split = longest > (G ? ATTEND_ALONE_STEPS_Q4 : a->weights_out ? ATTEND_ALONE_STEPS_WEIGHTS : ATTEND_ALONE_STEPS) || (a->weights_out && k.group_chunks > 1);
    if (split && one_head) longest = shape(most);
    k.head_chunks = c->kv_heads / k.hc;
    const int64_t box = p.warps > k.hc ? (int64_t)p.warps / 2 * (G ? kv_q4_box(G, p.nt) : p.nt * (p.dp / 16 + 1) * 4) * 32 * 4 : 0;
    const int64_t stage = G ? (int64_t)k.tw * k.hc * kv_q4_tile(G) : (int64_t)p.warps * 64 * p.dp;
    k.stages = (int)std::min<int64_t>(G ? KV_Q4_STAGES : KV_ATTEND_STAGES, (ATTEND_SMEM - box) / stage);     // the kernels' tables have so many
    if (!split) k.stages = (int)std::max<int64_t>(1, std::min<int64_t>(k.stages, longest));
    p.smem = (size_t)(k.stages * stage + box);
    // the kernels round the number of steps up to their numbers of CTAs in 32 bits
    if (longest * a->num_seqs * k.head_chunks * k.group_chunks > INT32_MAX - KV_JOIN_SHARES * o->sms)
        return fail(o, KV_ERR_UNSUPPORTED, "num_seqs * max_len is too large for one call");
    k.pieces = split ? o->sms : 0;
    k.min_steps = ATTEND_MIN_STEPS;
    // Whole blocks: of 2^n tiles, as many as a step has or fewer, and steps that begin where blocks do.  One sequence of 131072 slots in
    // blocks of 64, 1 KV head: 20.4 us when that was compared, and 26.4 with a bulk copy per tile, plane, codes and words
    const int tiles = c->block_size / 16;
    k.block_tiles = G && k.whole_tiles && (tiles & (tiles - 1)) == 0 && k.tw % tiles == 0 && (tiles == 1 || a->window == 0) ? tiles : 0;
    const int64_t parts = (int64_t)k.pieces * 2 * k.hc * 8 * p.nt;
    p.lse = align256(a->weights_out ? (int64_t)a->num_seqs * a->q_heads * a->max_len * 4 : 0);
    p.part_of = p.lse + align256(split ? (int64_t)a->num_seqs * a->q_heads * 4 : 0);
    p.part_ml = p.part_of + align256((int64_t)k.pieces * 16);
    p.part_o = p.part_ml + align256(parts * 8);
    p.total = p.part_o + parts * c->head_dim * 4;
    return KV_OK;
}

template <typename T> const void *attend_kernel(int dp, int nt, bool q4)
{
    if (q4) {
        if (dp == 64) return nt == 1 ? (const void *)kv_attend_q4<T, 2, 1> : (const void *)kv_attend_q4<T, 2, 2>;
        if (dp == 128) return nt == 1 ? (const void *)kv_attend_q4<T, 4, 1> : (const void *)kv_attend_q4<T, 4, 2>;
        return nt == 1 ? (const void *)kv_attend_q4<T, 8, 1> : (const void *)kv_attend_q4<T, 8, 2>;
    }
    if (dp == 64) return nt == 1 ? (const void *)kv_attend_stream<T, 64, 1> : (const void *)kv_attend_stream<T, 64, 2>;
    if (dp == 128) return nt == 1 ? (const void *)kv_attend_stream<T, 128, 1> : (const void *)kv_attend_stream<T, 128, 2>;
    return nt == 1 ? (const void *)kv_attend_stream<T, 256, 1> : (const void *)kv_attend_stream<T, 256, 2>;
}

}  // namespace

extern "C" {

int32_t kv_cache_row_units(int32_t dtype, int32_t head_dim)
{
    if (head_dim <= 0 || head_dim % 8 || head_dim > 256) return 0;
    if (dtype == KV_DT_BF16 || dtype == KV_DT_F16) return head_dim;
    return is_q4(dtype) ? 10 * q4_groups(head_dim) : 0;
}

const char *kv_ops_last_error(kv_ops_t *o) { return o ? o->err : g_ops_err; }

int32_t kv_ops_create(int32_t device_id, void *stream, kv_ops_t **out)
{
    if (!out) return fail(nullptr, KV_ERR_INVALID_ARG, "null argument");
    *out = nullptr;
    int devices = 0;
    cudaError_t e = cudaGetDeviceCount(&devices);
    if (e != cudaSuccess) return fail_cuda(nullptr, e, "cudaGetDeviceCount");
    if (device_id < 0 || device_id >= devices) return fail(nullptr, KV_ERR_INVALID_ARG, "no such device");
    const OnDevice on(device_id);
    kv_ops *o = new (std::nothrow) kv_ops();
    if (!o) return fail(nullptr, KV_ERR_NOMEM, "out of host memory");
    o->device = device_id;
    o->stream = (cudaStream_t)stream;
    snprintf(o->err, 256, "no error");
    e = cudaDeviceGetAttribute(&o->sms, cudaDevAttrMultiProcessorCount, device_id);
    if (e == cudaSuccess) e = cudaHostAlloc((void **)&o->status_host, 64, cudaHostAllocMapped);
    if (e == cudaSuccess) {
        *o->status_host = 0;
        e = cudaHostGetDevicePointer((void **)&o->status_dev, o->status_host, 0);
    }
    if (e != cudaSuccess) {
        const int32_t rc = fail_cuda(nullptr, e, "kv_ops_create");
        if (o->status_host) cudaFreeHost(o->status_host);
        delete o;
        return rc;
    }
    *out = o;
    return KV_OK;
}

int32_t kv_ops_destroy(kv_ops_t *o)
{
    if (!o) return KV_ERR_INVALID_ARG;
    const OnDevice on(o->device);
    (void)cudaStreamSynchronize(o->stream);
    if (o->ws) cudaFree(o->ws);
    for (void *p : o->outgrown) cudaFree(p);
    if (o->status_host) cudaFreeHost(o->status_host);
    (void)cudaGetLastError();
    delete o;
    return KV_OK;
}

int32_t kv_ops_reserve(kv_ops_t *o, int64_t bytes)
{
    if (!o) return KV_ERR_INVALID_ARG;
    const OnDevice on(o->device);
    return grow_workspace(o, bytes);
}

int32_t kv_ops_set_wait_limit(kv_ops_t *o, uint32_t polls, uint64_t ns)
{
    if (!o) return KV_ERR_INVALID_ARG;
    if (ns > 60000000000ull) return fail(o, KV_ERR_INVALID_ARG, "a wait of more than 60 s");
    o->wait_polls = polls;
    o->wait_ns = ns;
    return KV_OK;
}

int32_t kv_ops_sync(kv_ops_t *o)
{
    if (!o) return KV_ERR_INVALID_ARG;
    const OnDevice on(o->device);
    const cudaError_t e = cudaStreamSynchronize(o->stream);
    if (e != cudaSuccess) return fail_cuda(o, e, "cudaStreamSynchronize");
    const unsigned st = *(volatile unsigned *)o->status_host;
    // results that are not to be used outrank slots that were skipped
    if (st & KV_OPS_TIMEOUT && (o->sticky == KV_OK || o->sticky == KV_ERR_RANGE)) {
        o->sticky = KV_ERR_TIMEOUT;
        snprintf(o->err, 256, "a wait inside a kernel ran out (status 0x%x)", st);
    } else if (st && o->sticky == KV_OK) {
        o->sticky = KV_ERR_RANGE;
        snprintf(o->err, 256, "a kernel met %s and skipped it (status 0x%x)",
                 st & KV_OPS_BAD_BLOCK ? "a block id outside the cache" : "a length outside its bounds", st);
    }
    return o->sticky;
}

int32_t kv_attend_workspace(kv_ops_t *o, const kv_cache_t *cache, const kv_attend_args_t *args, int64_t *bytes)
{
    if (!o || !bytes) return fail(o, KV_ERR_INVALID_ARG, "null argument");
    KvAttend k;
    AttendPlan p;
    const int32_t rc = plan_attend(o, cache, args, k, p);
    if (rc == KV_OK) *bytes = p.total;
    return rc;
}

int32_t kv_attend(kv_ops_t *o, const kv_cache_t *cache, const kv_attend_args_t *a)
{
    if (!o) return fail(nullptr, KV_ERR_INVALID_ARG, "null argument");
    KvAttend k;
    AttendPlan p;
    int32_t rc = plan_attend(o, cache, a, k, p);
    if (rc != KV_OK) return rc;
    if (a->num_seqs == 0) return KV_OK;
    const OnDevice on(o->device);
    if (!a->q || !a->out) return fail(o, KV_ERR_INVALID_ARG, "q and out are needed");
    if (a->weights_in && !a->weights_out) return fail(o, KV_ERR_INVALID_ARG, "weights_in without weights_out");
    if ((rc = set_tables(o, k.c, a->block_tables, a->table_stride, a->table_width, a->lens, a->max_len)) != KV_OK) return rc;
    if ((rc = grow_workspace(o, p.total)) != KV_OK) return rc;
    k.layer = a->layer;
    k.seqs = a->num_seqs;
    k.q_heads = a->q_heads;
    k.window = a->window;
    k.scale2 = (a->scale != 0.f ? a->scale : 1.f / sqrtf((float)cache->head_dim)) * 1.44269504088896340736f;
    k.q = a->q;
    k.q_seq = a->q_seq_stride;
    k.q_head = a->q_head_stride;
    k.q_pairs = (uintptr_t)a->q % 4 == 0 && a->q_seq_stride % 2 == 0 && a->q_head_stride % 2 == 0;
    k.q_vec = (uintptr_t)a->q % 16 == 0 && a->q_seq_stride % 8 == 0 && a->q_head_stride % 8 == 0;
    k.out_vec = (uintptr_t)a->out % 8 == 0 && a->out_seq_stride % 4 == 0 && a->out_head_stride % 4 == 0;
    k.out = a->out;
    k.o_seq = a->out_seq_stride;
    k.o_head = a->out_head_stride;
    k.lse = a->lse;
    k.w_in = a->weights_in;
    k.w_out = a->weights_out;
    k.w_seq = a->w_seq_stride;
    k.w_head = a->w_head_stride;
    k.scores = a->weights_out ? (float *)o->ws : nullptr;
    k.row_lse = (float *)(o->ws + p.lse);
    k.part_of = (int4 *)(o->ws + p.part_of);
    k.part_ml = (float2 *)(o->ws + p.part_ml);
    k.part_o = (float *)(o->ws + p.part_o);
    k.wait_polls = o->wait_polls;
    k.wait_ns = o->wait_ns;

    const bool bf16 = is_bf16(cache), q4 = k.c.groups != 0, wide = q4 && kv_q4_wide(k.c.groups, p.nt);
    const void *kernel = bf16 ? attend_kernel<__nv_bfloat16>(p.dp, p.nt, q4) : attend_kernel<__half>(p.dp, p.nt, q4);
    bool &ready = o->attend_ready[q4][bf16][p.dp / 128][p.nt - 1];
    if (!ready) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(227 * 1024 - 4096));
        if (e != cudaSuccess) return fail_cuda(o, e, "cudaFuncSetAttribute");
        if (wide) {              // registers move between the warps: there must be enough of them at the launch
            cudaFuncAttributes at;
            const cudaError_t f = cudaFuncGetAttributes(&at, kernel);
            if (f != cudaSuccess) return fail_cuda(o, f, "cudaFuncGetAttributes");
            if (!kv_q4_fits(4, at.numRegs) || !kv_q4_fits(8, at.numRegs)) return fail(o, KV_ERR_UNSUPPORTED, "the kernel was built with too few registers");
        }
        ready = true;
    }
    const unsigned threads = 32 * (q4 ? (p.warps + 3) / 4 * 4 + KV_Q4_LOADERS : p.warps);
    void *params[] = {&k};
    const unsigned rows = (unsigned)(k.seqs * k.head_chunks * k.group_chunks);
    cudaError_t e = cudaLaunchKernel(kernel, dim3(k.pieces ? k.pieces : rows), dim3(threads), params, p.smem, o->stream);
    if (e != cudaSuccess) return fail_cuda(o, e, "kv_attend");
    if (k.pieces) {
        // programmatic dependent launch: the join's CTAs come up while the last of the stream's finish
        cudaLaunchAttribute early;
        early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
        early.val.programmaticStreamSerializationAllowed = 1;
        cudaLaunchConfig_t cfg = {};
        const int row_ctas = k.scores ? ATTEND_ROW_CTAS_WEIGHTS : ATTEND_ROW_CTAS;
        cfg.gridDim = dim3(k.pieces * (row_ctas + (k.scores ? KV_JOIN_SHARES : 0)));
        cfg.dynamicSmemBytes = std::max((size_t)kv_join_floats(k.hc, 8 * p.nt, k.pieces), (size_t)k.hc * k.group) * 4;
        cfg.blockDim = dim3(KV_JOIN_THREADS);
        cfg.stream = o->stream;
        cfg.attrs = &early;
        cfg.numAttrs = 1;
        e = bf16 ? cudaLaunchKernelEx(&cfg, kv_attend_join<__nv_bfloat16>, k, 8 * p.nt, row_ctas) : cudaLaunchKernelEx(&cfg, kv_attend_join<__half>, k, 8 * p.nt, row_ctas);
        if (e != cudaSuccess) return fail_cuda(o, e, "kv_attend");
    }
    return KV_OK;
}

int32_t kv_append(kv_ops_t *o, const kv_cache_t *cache, const kv_append_args_t *a) { return kv_append_normed(o, cache, a, nullptr); }

int32_t kv_append_normed(kv_ops_t *o, const kv_cache_t *cache, const kv_append_args_t *a, const kv_norm_args_t *norms)
{
    if (!o) return fail(nullptr, KV_ERR_INVALID_ARG, "null argument");
    if (!a) return fail(o, KV_ERR_INVALID_ARG, "no arguments");
    KvAppend k;
    int32_t rc = make_view(o, cache, k.c);
    if (rc != KV_OK) return rc;
    if (a->layer < 0 || a->layer >= cache->num_layers) return fail(o, KV_ERR_RANGE, "no such layer");
    if (a->num_seqs < 0 || a->num_tokens < 0 || a->num_tokens > INT32_MAX || (a->q && a->q_heads <= 0)) return fail(o, KV_ERR_INVALID_ARG, "bad count");
    if (a->rotary_dim < 0 || a->rotary_dim > cache->head_dim || a->rotary_dim % 2) return fail(o, KV_ERR_INVALID_ARG, "rotary_dim must be even, at most head_dim");
    if (a->pair_style != 0 && a->pair_style != 1) return fail(o, KV_ERR_INVALID_ARG, "unknown pair_style");
    if (a->num_axes < 1 || a->num_axes > 4) return fail(o, KV_ERR_INVALID_ARG, "num_axes must be 1 to 4");
    for (int f = 0; f < a->rotary_dim / 2; ++f)
        if (a->axis_of[f] >= a->num_axes) return fail(o, KV_ERR_RANGE, "axis_of names an axis that positions does not have");
    const bool normed = norms && (norms->q_weight || norms->k_weight);
    if (normed) {
        if (!(norms->eps >= 0.f) || !(norms->eps < INFINITY)) return fail(o, KV_ERR_INVALID_ARG, "eps must be a number and not negative");
        if (norms->weight_float != 0 && norms->weight_float != 1) return fail(o, KV_ERR_INVALID_ARG, "unknown type of the norms' weights");
        if (norms->q_head_stride < 0 || norms->k_head_stride < 0) return fail(o, KV_ERR_INVALID_ARG, "negative stride of the norms' weights");
        if (norms->q_weight && !a->q) return fail(o, KV_ERR_INVALID_ARG, "weights of a norm of q without q");
    }
    if (a->num_tokens == 0 || a->num_seqs == 0) return KV_OK;
    const OnDevice on(o->device);
    if (!a->seq_starts && a->num_tokens != a->num_seqs) return fail(o, KV_ERR_INVALID_ARG, "without seq_starts every sequence has one token");
    if (!a->k || !a->v) return fail(o, KV_ERR_INVALID_ARG, "k and v are needed");
    if (a->q && !a->q_out) return fail(o, KV_ERR_INVALID_ARG, "q without q_out");
    if (a->rotary_dim && (!a->positions || !a->inv_freq)) return fail(o, KV_ERR_INVALID_ARG, "rotation needs positions and inv_freq");
    if (a->order && !a->token_order && !a->positions) return fail(o, KV_ERR_INVALID_ARG, "order needs token_order or positions");
    if ((rc = set_tables(o, k.c, a->block_tables, a->table_stride, a->table_width, a->lens,
                         std::min<int64_t>((int64_t)a->table_width * cache->block_size, INT32_MAX / 2))) != KV_OK) return rc;
    k.layer = a->layer;
    k.num_seqs = a->num_seqs;
    k.q_heads = a->q_heads;
    k.rotary = a->rotary_dim;
    k.pairs_style = a->pair_style;
    k.q = a->q;
    k.k = a->k;
    k.v = a->v;
    k.q_tok = a->q_token_stride;
    k.q_head = a->q_head_stride;
    k.k_tok = a->k_token_stride;
    k.k_head = a->k_head_stride;
    k.v_tok = a->v_token_stride;
    k.v_head = a->v_head_stride;
    k.q_out = a->q_out;
    k.qo_tok = a->qo_token_stride;
    k.qo_head = a->qo_head_stride;
    k.positions = a->positions;
    k.axis_stride = a->axis_stride;
    k.inv_freq = a->inv_freq;
    k.starts = a->seq_starts;
    k.weights = a->weights;
    k.order = a->order;
    k.m_seq = a->m_seq_stride;
    k.m_head = a->m_head_stride;
    k.token_order = a->token_order;
    k.num_slots = a->num_slots;
    memcpy(k.axis_of, a->axis_of, sizeof(k.axis_of));
    k.num_tokens = a->num_tokens;
    // 16 bytes at a time where every row begins on 16 bytes and the pairs that turn together are whole packs of eight, 8 bytes
    // likewise (a rotation of 40 of 80 elements turns halves of 20), else element by element: 14.3k prompt tokens 65, 80 and 204 us,
    // 64 tokens of a decode step 4.9, 5.6 and 10.0
    const int turning = a->pair_style ? a->rotary_dim : a->rotary_dim / 2;
    const auto packs = [&](int64_t v) {
        const auto fits = [v](const void *q, int64_t x, int64_t y) { return (uintptr_t)q % (2 * v) == 0 && x % v == 0 && y % v == 0; };
        return turning % v == 0 && (cache->head_dim - a->rotary_dim) % v == 0 && fits(a->k, a->k_token_stride, a->k_head_stride) &&
               fits(a->v, a->v_token_stride, a->v_head_stride) &&
               (!a->q || (fits(a->q, a->q_token_stride, a->q_head_stride) && fits(a->q_out, a->qo_token_stride, a->qo_head_stride)));
    };
    const int v = packs(8) ? 8 : packs(4) ? 4 : 1;
    k.units = (v > 1 && a->pair_style ? a->rotary_dim / v : a->rotary_dim / 2 / v) + (cache->head_dim - a->rotary_dim) / v;
    // a row number below 2^32 / rows is divided by rows exactly with the reciprocal
    const int64_t rows = (int64_t)(a->q ? a->q_heads : 0) + 2 * cache->kv_heads;
    if (rows > 4096) return fail(o, KV_ERR_UNSUPPORTED, "too many heads");
    // tokens per CTA: up to eight CTAs per SM, then more tokens.  With 4 / 8 / 16 CTAs per SM 2000 tokens of 32 + 8 + 8 heads take
    // 12.2 / 14.1 / 17.9 us, 3500 18.9 / 20.1 / 21.3, 6900 36.5 / 35.2 / 36.0, 14.3k 67.1 / 65.0 / 63.5; up to 500 all the same
    k.per = (int)std::min<int64_t>(AP_TOKENS, ceil_div(a->num_tokens, 8 * o->sms));
    k.by_rows = (unsigned)ceil_div(int64_t(1) << 32, rows);
    const bool bf16 = is_bf16(cache);
    if (normed || k.c.groups) {
        KvAppendRows r;
        r.q_w = normed ? norms->q_weight : nullptr;
        r.k_w = normed ? norms->k_weight : nullptr;
        r.q_w_head = normed ? norms->q_head_stride : 0;
        r.k_w_head = normed ? norms->k_head_stride : 0;
        r.w_float = normed ? norms->weight_float : 0;
        r.eps = normed ? norms->eps : 0.f;
        r.turns = (int)ceil_div(a->rotary_dim, 16);
        const int lanes = std::max(r.turns + (int)ceil_div(cache->head_dim - a->rotary_dim, 16), 2 * k.c.groups);
        r.lanes_log2 = 0;
        while (1 << r.lanes_log2 < lanes) ++r.lanes_log2;
        const int q4 = k.c.groups != 0, per_token = r.turns * (q4 ? 192 : 64), at_once = AP_THREADS >> r.lanes_log2;
        if (per_token) k.per = std::min(k.per, 32 * 1024 / per_token);       // with the keys in passing and the weights 46 KB at most
        const int abreast = 32 >> r.lanes_log2, warps = AP_THREADS / 32;
        const int groups = (int)(ceil_div(a->q ? a->q_heads : 0, abreast) + 2 * ceil_div(cache->kv_heads, abreast));
        r.splits = 1;
        r.per_split = groups;
        // Few tokens: their rows all at once, as far as there are SMs.  64 tokens of 64 + 8 + 8 heads with norms 5.1 us so, 7.0 with one CTA per token
        if (k.per == 1) {
            r.splits = (int)std::max<int64_t>(1, std::min<int64_t>(ceil_div(groups, warps), 4 * o->sms / a->num_tokens));
            r.per_split = (int)ceil_div(groups, r.splits);
            r.splits = (int)ceil_div(groups, r.per_split);
        }
        // The number of runs a CTA's tokens are cut into: whichever gives the shortest way for the busiest warp, a task's beginning counted
        // as a token's work
        r.chunk = k.per;
        for (int runs = 2; runs <= k.per; ++runs) {
            const auto way = [&](int64_t chunk) { return ceil_div(groups * ceil_div(k.per, chunk), warps) * (chunk + 1); };
            if (way(ceil_div(k.per, runs)) < way(r.chunk)) r.chunk = (int)ceil_div(k.per, runs);
        }
        r.by_groups = (unsigned)ceil_div(int64_t(1) << 32, groups);
        r.by_dim = 1.f / cache->head_dim;
        r.p = k;
        const size_t smem = (size_t)k.per * per_token + (q4 ? (size_t)at_once * k.c.groups * 64 : 0);
        // Whole rows: heads of 64, 128 or 256, every lane's elements aligned and of one kind.  14.3k prompt tokens with norms 74.6 us so and 91.1
        // with guards and four elements at a time, into 4 bits and read back 133 and 163; one token 8.1 and 8.6
        const bool whole = v == 8 && lanes * 16 == cache->head_dim && lanes == 1 << r.lanes_log2 && lanes >= 4 && lanes <= 16;
        const auto pick = [&](auto t) {
            using T = decltype(t);
            using Kernel = void (*)(KvAppendRows);
            const Kernel kernels[2][5] = {
                {kv_append_rows<T, 1, false, 0>, kv_append_rows<T, 4, false, 0>, kv_append_rows<T, 8, false, 2>, kv_append_rows<T, 8, false, 3>, kv_append_rows<T, 8, false, 4>},
                {kv_append_rows<T, 1, true, 0>, kv_append_rows<T, 4, true, 0>, kv_append_rows<T, 8, true, 2>, kv_append_rows<T, 8, true, 3>, kv_append_rows<T, 8, true, 4>}};
            return kernels[q4][whole ? r.lanes_log2 : v >= 4 ? 1 : 0];
        };
        const auto kernel = bf16 ? pick(__nv_bfloat16()) : pick(__half());
        kernel<<<(unsigned)(ceil_div(a->num_tokens, k.per) * r.splits), AP_THREADS, smem, o->stream>>>(r);
        return launched(o, "kv_append");
    }
    const unsigned grid = (unsigned)ceil_div(a->num_tokens, k.per);
    const size_t smem = (size_t)k.per * (a->rotary_dim / 2) * sizeof(float2);
    const auto kernel = bf16 ? (v == 8   ? kv_append_tokens<__nv_bfloat16, 8>
                                : v == 4 ? kv_append_tokens<__nv_bfloat16, 4>
                                         : kv_append_tokens<__nv_bfloat16, 1>)
                             : (v == 8 ? kv_append_tokens<__half, 8> : v == 4 ? kv_append_tokens<__half, 4> : kv_append_tokens<__half, 1>);
    kernel<<<grid, AP_THREADS, smem, o->stream>>>(k);
    return launched(o, "kv_append");
}

int32_t kv_read(kv_ops_t *o, const kv_cache_t *cache, const kv_read_args_t *a)
{
    if (!o) return fail(nullptr, KV_ERR_INVALID_ARG, "null argument");
    if (!a) return fail(o, KV_ERR_INVALID_ARG, "no arguments");
    KvRead k;
    int32_t rc = make_view(o, cache, k.c);
    if (rc != KV_OK) return rc;
    if (a->layer < 0 || a->layer >= cache->num_layers) return fail(o, KV_ERR_RANGE, "no such layer");
    if (a->num_seqs < 0 || a->num_tokens < 0 || a->num_tokens > INT32_MAX) return fail(o, KV_ERR_INVALID_ARG, "bad count");
    if (cache->kv_heads > 512) return fail(o, KV_ERR_UNSUPPORTED, "too many heads");
    if (a->num_tokens == 0 || a->num_seqs == 0) return KV_OK;
    const OnDevice on(o->device);
    if (!a->seq_starts && a->num_tokens != a->num_seqs) return fail(o, KV_ERR_INVALID_ARG, "without seq_starts every sequence has one token");
    if (!a->k && !a->v) return fail(o, KV_ERR_INVALID_ARG, "k or v is needed");
    if ((rc = set_tables(o, k.c, a->block_tables, a->table_stride, a->table_width, a->lens,
                         std::min<int64_t>((int64_t)a->table_width * cache->block_size, INT32_MAX / 2))) != KV_OK) return rc;
    k.layer = a->layer;
    k.num_seqs = a->num_seqs;
    k.num_tokens = a->num_tokens;
    k.k = a->k;
    k.v = a->v;
    k.k_tok = a->k_token_stride;
    k.k_head = a->k_head_stride;
    k.v_tok = a->v_token_stride;
    k.v_head = a->v_head_stride;
    k.starts = a->seq_starts;
    k.units = k.c.groups ? 4 : (int)ceil_div(cache->head_dim, 16);
    const int per_token = k.units * cache->kv_heads;
    k.by_units = per_token == 1 ? 0 : (unsigned)ceil_div(int64_t(1) << 32, per_token);     // 2^32 has no place in 32 bits
    k.per = (int)std::min<int64_t>(RD_TOKENS, ceil_div(a->num_tokens, 8 * o->sms));
    const auto fits = [](const void *p, int64_t x, int64_t y) { return (uintptr_t)p % 16 == 0 && x % 8 == 0 && y % 8 == 0; };
    const bool vec = (!a->k || fits(a->k, a->k_token_stride, a->k_head_stride)) && (!a->v || fits(a->v, a->v_token_stride, a->v_head_stride));
    const auto pick = [&](auto t) {
        using T = decltype(t);
        using Kernel = void (*)(KvRead);
        const Kernel kernels[2][4] = {{kv_read_rows<T, false, 0>, kv_read_rows<T, false, 2>, kv_read_rows<T, false, 4>, kv_read_rows<T, false, 8>},
                                      {kv_read_rows<T, true, 0>, kv_read_rows<T, true, 2>, kv_read_rows<T, true, 4>, kv_read_rows<T, true, 8>}};
        return kernels[vec][k.c.groups == 8 ? 3 : k.c.groups / 2];
    };
    const auto kernel = is_bf16(cache) ? pick(__nv_bfloat16()) : pick(__half());
    kernel<<<(unsigned)ceil_div(a->num_tokens, k.per), AP_THREADS, 0, o->stream>>>(k);
    return launched(o, "kv_read");
}

}  // extern "C"

namespace {

struct EvictPlan {
    int64_t problems, cap, count, holes, srcs, total;
    int threads, cluster;                       // EV_SMALL_THREADS: kv_evict_small
    bool regs, fused;
};

// Up to here kv_evict_small has the lowest latency.  16 problems with four warps each / 256 threads / 1024: of 300 slots 9.1 / 15.3 /
// 19.1 us (its rows in the same kernel), 600 15.3 / 15.8 / 19.1, 1000 15.2 / 15.9 / 19.1, 2000 17.6 / 17.1 / 19.7, 4000 21.9 / 19.5 / 20.9
constexpr int EVICT_SHORT = 1024;

int32_t plan_evict(kv_ops *o, const kv_cache_t *c, const kv_evict_args_t *a, KvEvict &k, EvictPlan &p)
{
    if (!a) return fail(o, KV_ERR_INVALID_ARG, "no arguments");
    int32_t rc = make_view(o, c, k.c);
    if (rc != KV_OK) return rc;
    if (a->num_layers < 0 || a->num_seqs < 0 || a->num_seqs > 65535 || a->num_layers > 65535 || a->keep < 1 || a->recent < 0 || a->sink < 0)
        return fail(o, KV_ERR_INVALID_ARG, "bad count");
    if (a->first_layer < 0 || (int64_t)a->first_layer + a->num_layers > c->num_layers) return fail(o, KV_ERR_RANGE, "no such layers");
    if ((int64_t)a->recent + a->sink > a->keep) return fail(o, KV_ERR_INVALID_ARG, "recent + sink exceeds keep");
    if (a->max_len < 0 || a->max_len > INT32_MAX / 2) return fail(o, KV_ERR_INVALID_ARG, "bad max_len");
    p.problems = (int64_t)a->num_layers * a->num_seqs * c->kv_heads;
    if (p.problems * EV_CLUSTER > INT32_MAX) return fail(o, KV_ERR_UNSUPPORTED, "too many (layer, sequence, head) problems in one call");
    p.cap = std::max<int64_t>(0, std::min<int64_t>(a->keep, a->max_len - a->keep));
    // Four warps per problem where problems are short, or enough of them to fill the GPU: of 2304 slots 64 take 18.8 us so and 17.5 with
    // 256 threads, 256 28.9 / 27.6, 512 42.9 / 44.9, 592 45.7 / 47.4, 2048 110 / 132; of 8000 slots 64 take 52.6 and 40.6 with 1024
    // threads, 256 111 / 111, 592 200 / 221, 1024 270 / 302.  Else 256 threads hold 4096 keys and 1024 threads 16384 (16 problems of 4000
    // slots 19.5 us with 256 and 20.9 with 1024, 256 of them 54.5 / 64.4).  A cluster of eight such CTAs holds 131072, and beyond that the
    // keys are read again in every round: one problem of 40000 slots 79 us in one CTA that reads again, 66 in two, 32 in four that
    // hold them; of 131072 247, 165, 98, and 45 in eight; of 140000 86 in eight that read again
    p.threads = a->max_len <= EVICT_SHORT || (a->max_len <= EV_SMALL_SLOTS && p.problems >= 4 * o->sms) ? EV_SMALL_THREADS
                : a->max_len <= 256 * EV_KEYS                                                       ? 256
                                                                                                      : 1024;
    p.cluster = 1;
    while (p.threads == 1024 && p.cluster < EV_CLUSTER && (int64_t)p.cluster * p.threads * EV_KEYS < a->max_len) p.cluster *= 2;
    p.regs = a->max_len <= (int64_t)p.cluster * p.threads * EV_KEYS;
    // Rows in the same kernel, or in a second one: 16 problems of 500 slots and 40 rows 11.3 / 16.2 us, 100 rows 11.5 / 14.9, 200 14.9 / 15.0,
    // 400 18.6 / 14.9; 2048 problems of 2048 slots and 64 rows 54.9 / 61.4, 256 101 / 110.  The limit keeps the lists at 512 bytes per CTA
    p.fused = p.threads == EV_SMALL_THREADS && p.cap <= EV_FUSED_ROWS;
    p.count = 0;
    p.holes = align256(p.problems * 4);
    p.srcs = p.holes + align256(p.problems * p.cap * 4);
    p.total = p.srcs + p.problems * p.cap * 4;
    return KV_OK;
}

}  // namespace

extern "C" {

int32_t kv_evict_workspace(kv_ops_t *o, const kv_cache_t *cache, const kv_evict_args_t *args, int64_t *bytes)
{
    if (!o || !bytes) return fail(o, KV_ERR_INVALID_ARG, "null argument");
    KvEvict k;
    EvictPlan p;
    const int32_t rc = plan_evict(o, cache, args, k, p);
    if (rc == KV_OK) *bytes = p.total;
    return rc;
}

int32_t kv_evict(kv_ops_t *o, const kv_cache_t *cache, const kv_evict_args_t *a)
{
    if (!o) return fail(nullptr, KV_ERR_INVALID_ARG, "null argument");
    KvEvict k;
    EvictPlan p;
    int32_t rc = plan_evict(o, cache, a, k, p);
    if (rc != KV_OK) return rc;
    if (p.problems == 0) return KV_OK;
    const OnDevice on(o->device);
    if (!a->weights) return fail(o, KV_ERR_INVALID_ARG, "weights are needed");
    if (a->order_out && !a->order) return fail(o, KV_ERR_INVALID_ARG, "order_out without order");
    if (a->order && !a->order_out != !a->weights_out) return fail(o, KV_ERR_INVALID_ARG, "weights and order go to outputs both, or are both changed in place");
    if (a->order && a->weights_out && (a->weights_out == a->weights) != (a->order_out == a->order))
        return fail(o, KV_ERR_INVALID_ARG, "weights and order go to outputs both, or are both changed in place");
    if (a->lens_out == a->lens) return fail(o, KV_ERR_INVALID_ARG, "lens_out must not be lens");
    if ((rc = set_tables(o, k.c, a->block_tables, a->table_stride, a->table_width, a->lens, a->max_len)) != KV_OK) return rc;
    if ((rc = grow_workspace(o, p.total)) != KV_OK) return rc;
    k.first_layer = a->first_layer;
    k.layers = a->num_layers;
    k.seqs = a->num_seqs;
    k.keep = a->keep;
    k.recent = a->recent;
    k.sink = a->sink;
    k.w = a->weights;
    k.order = a->order;
    k.m_layer = a->m_layer_stride;
    k.m_seq = a->m_seq_stride;
    k.m_head = a->m_head_stride;
    k.seen = a->seen;
    const bool apart = a->weights_out && a->weights_out != a->weights;
    k.w_out = apart ? a->weights_out : (float *)a->weights;
    k.order_out = apart ? a->order_out : (int *)a->order;
    k.o_layer = apart ? a->o_layer_stride : a->m_layer_stride;
    k.o_seq = apart ? a->o_seq_stride : a->m_seq_stride;
    k.o_head = apart ? a->o_head_stride : a->m_head_stride;
    k.lens_out = a->lens_out;
    k.count = (int *)(o->ws + p.count);
    k.holes = (int *)(o->ws + p.holes);
    k.srcs = (int *)(o->ws + p.srcs);
    k.cap = (int)p.cap;
    k.problems = (int)p.problems;
    k.fused = p.fused;
    const auto quad = [](const void *q, int64_t x, int64_t y, int64_t z) { return (uintptr_t)q % 16 == 0 && x % 4 == 0 && y % 4 == 0 && z % 4 == 0; };
    // a quad that begins below the length must end inside its row: the last row of the array has max_len entries at least.  2048 problems
    // of 2304 slots 109.8 us by quads, 111.0 one by one
    k.quads = a->max_len % 4 == 0 && quad(k.w, k.m_layer, k.m_seq, k.m_head) && quad(k.order, 0, 0, 0) && quad(k.w_out, k.o_layer, k.o_seq, k.o_head) &&
              quad(k.order_out, 0, 0, 0);
    const int units = cache->head_dim / 4;
    k.units_shift = units & (units - 1) ? -1 : __builtin_ctz(units);
    cudaLaunchAttribute attr;
    cudaLaunchConfig_t cfg = {};
    cfg.stream = o->stream;
    cfg.attrs = &attr;
    cudaError_t e;
    if (p.threads == EV_SMALL_THREADS) {
        cfg.gridDim = dim3((unsigned)p.problems);
        cfg.blockDim = dim3(EV_SMALL_THREADS);
        cfg.dynamicSmemBytes = ceil_div(a->max_len, 4 * EV_SMALL_THREADS) * 16 * EV_SMALL_THREADS;
        e = k.c.groups ? cudaLaunchKernelEx(&cfg, kv_evict_small<true>, k) : cudaLaunchKernelEx(&cfg, kv_evict_small<false>, k);
    } else {
        attr.id = cudaLaunchAttributeClusterDimension;
        attr.val.clusterDim.x = p.cluster;
        attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
        cfg.numAttrs = 1;
        cfg.gridDim = dim3((unsigned)(p.problems * p.cluster));
        cfg.blockDim = dim3(p.threads);
        e = p.threads == 256 ? cudaLaunchKernelEx(&cfg, kv_evict_select<256, true>, k)
            : p.regs         ? cudaLaunchKernelEx(&cfg, kv_evict_select<1024, true>, k)
                             : cudaLaunchKernelEx(&cfg, kv_evict_select<1024, false>, k);
    }
    if (e != cudaSuccess) return fail_cuda(o, e, "kv_evict");
    if (!p.fused && p.cap > 0) {
        // an ordinary launch: its CTAs waiting on the SMs beside the first kernel's cost more than the gap (137 against 123 us
        // in a steady state of 32 layers and 8 sequences)
        cfg.numAttrs = 0;
        cfg.dynamicSmemBytes = 0;
        cfg.gridDim = dim3((unsigned)ceil_div(p.cap, 32), (unsigned)std::min<int64_t>(ceil_div(p.problems, EV_MOVE_WARPS), 65535));
        cfg.blockDim = dim3(EV_MOVE_WARPS * 32);
        e = k.c.groups ? cudaLaunchKernelEx(&cfg, kv_evict_move<true>, k) : cudaLaunchKernelEx(&cfg, kv_evict_move<false>, k);
        if (e != cudaSuccess) return fail_cuda(o, e, "kv_evict");
    }
    return KV_OK;
}

}  // extern "C"
