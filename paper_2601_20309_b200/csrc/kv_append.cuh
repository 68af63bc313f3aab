// New tokens into the paged cache: rotary positions with several axes on q and k, then k and v into their slots.
//
// A token's angles are the same for all its heads, so they are worked out once per token: position * inv_freq is exact
// in float64 (31 + 24 bits against 53, one rounding at most), reduced to a fraction of a turn there, and only then
// goes to float32 for sine and cosine: at position 10^5 a float32 product would be off by 4e-3 radians already.
//
// What bounds it: for prompts the bytes of q, k and v, read and written once; for a decode step the chain of loads.  A CTA
// takes up to AP_TOKENS tokens.  Every thread first sends off its first loads of rows, and the tokens' angles and slots (a
// search, a length, a block id: loads that wait for one another) are worked out while they travel, all tokens at once;
// then only rows stream through, four packs of 16 bytes, or of 16 bytes and their partners, per thread in flight.
#pragma once
#include "kv_ops.cuh"

struct KvAppend {
    KvView c;
    int layer, num_seqs, q_heads, rotary, pairs_style;
    long long num_tokens;
    const void *q, *k, *v;
    long long q_tok, q_head, k_tok, k_head, v_tok, v_head;
    void *q_out;
    long long qo_tok, qo_head;
    const int *positions;
    long long axis_stride;
    const float *inv_freq;
    const int *starts;
    float *weights;
    int *order;
    long long m_seq, m_head;
    const int *token_order;
    int vec;             // elements a thread moves at once: 8, or 1 where rows are not 16-byte aligned or odd in size
    int units;           // work items of a row: packs of `vec` elements with those they turn with, then packs that pass
    int per;             // tokens per CTA
    unsigned by_units, by_token;     // 2^32 / d, rounded up (0 for d = 1), for d = units and d = units * rows
    uint8_t axis_of[128];
};

// the sequence that token t belongs to: the last one that starts at or before it.  A warp looks at 32 places at once
__device__ __forceinline__ int kv_seq_of(const int *starts, int num_seqs, long long t)
{
    const int lane = threadIdx.x & 31;
    int lo = 0, n = num_seqs;        // the answer lies in [lo, lo + n)
    while (n > 1) {
        const int step = (n + 31) / 32, at = lo + lane * step;
        const unsigned v = __ballot_sync(~0u, lane * step < n && starts[at] <= t);
        const int last = v ? 31 - __clz(v) : 0;
        lo += last * step;
        n = min(step, n - last * step);
    }
    return lo;
}

constexpr int AP_THREADS = 256, AP_ITEMS = 2, AP_TOKENS = 16;

// e / d by the rounded-up reciprocal (0 for d = 1): exact for e < 2^32 / d
__device__ __forceinline__ int kv_divide(int e, unsigned reciprocal) { return reciprocal ? (int)__umulhi((unsigned)e, reciprocal) : e; }

template <typename T, int V> struct KvPack;
template <typename T> struct __align__(16) KvPack<T, 8> { T e[8]; };
template <typename T> struct KvPack<T, 1> { T e[1]; };

template <typename T, int V>
__global__ void __launch_bounds__(AP_THREADS) kv_append_tokens(const __grid_constant__ KvAppend a)
{
    using Pack = KvPack<T, V>;
    extern __shared__ float2 turn[];             // [token][frequency]: cosine and sine
    __shared__ uint8_t *kv_row[AP_TOKENS];       // K of the token's slot, or nullptr
    __shared__ long long meta[AP_TOKENS];
    const int tid = threadIdx.x, dim = a.c.dim, half = a.rotary >> 1, heads = a.c.heads, q_heads = a.q ? a.q_heads : 0;
    // a row: `turns` items that turn (in the halves style a pack and its partners, else a pack of pairs), then packs that pass
    const bool halves = a.pairs_style == 0;
    const int turns = halves ? half / V : V == 1 ? half : a.rotary / V, units = a.units, rows = q_heads + 2 * heads;
    const long long first = (long long)blockIdx.x * a.per;
    const int tokens = (int)min((long long)a.per, a.num_tokens - first), items = tokens * rows * units;
    for (int e0 = tid; e0 - tid < items; e0 += AP_THREADS * AP_ITEMS) {
        Pack x[AP_ITEMS], y[AP_ITEMS];
        int token[AP_ITEMS], row[AP_ITEMS], lo[AP_ITEMS], hi[AP_ITEMS];
#pragma unroll
        for (int n = 0; n < AP_ITEMS; ++n) {
            const int e = e0 + n * AP_THREADS;
            row[n] = -1;
            if (e < items) {
                token[n] = a.per == 1 ? 0 : kv_divide(e, a.by_token);
                const int f = e - token[n] * rows * units, u = f - kv_divide(f, a.by_units) * units;
                row[n] = kv_divide(f, a.by_units);
                const bool pair = u < turns;
                lo[n] = pair ? halves || V > 1 ? u * V : 2 * u : a.rotary + (u - turns) * V;
                hi[n] = pair ? halves ? lo[n] + half : V == 1 ? lo[n] + 1 : -1 : -1;
                const long long t = first + token[n];
                const T *from = row[n] < q_heads           ? (const T *)a.q + t * a.q_tok + row[n] * a.q_head
                                : row[n] < q_heads + heads ? (const T *)a.k + t * a.k_tok + (row[n] - q_heads) * a.k_head
                                                           : (const T *)a.v + t * a.v_tok + (row[n] - q_heads - heads) * a.v_head;
                x[n] = *(const Pack *)(from + lo[n]);
                if (hi[n] >= 0) y[n] = *(const Pack *)(from + hi[n]);
            }
        }
        if (e0 == tid) {             // the first time: angles and slots
            for (int f = tid; f < tokens * half; f += AP_THREADS) {
                const int k = f / half, q = f - k * half;
                const double cycles = (double)a.positions[a.axis_of[q] * a.axis_stride + first + k] * (double)a.inv_freq[q] * 0.15915494309189533577;
                sincospif((float)(2.0 * (cycles - rint(cycles))), &turn[f].y, &turn[f].x);
            }
            for (int k = tid >> 5; k < tokens; k += AP_THREADS / 32) {
                const long long t = first + k;
                const int i = a.starts ? kv_seq_of(a.starts, a.num_seqs, t) : (int)t;
                const long long left = a.starts ? a.starts[i + 1] - t : 1;       // this token and those behind it
                const int n = a.c.len(i);
                const long long s = n - left;
                const bool ok = left > 0 && s >= 0;
                if ((tid & 31) == 0) {
                    if (!ok && n > 0) atomicOr(a.c.status, KV_OPS_BAD_LEN);
                    kv_row[k] = ok ? a.c.slot(i, (int)s, a.layer * 2) : nullptr;
                    meta[k] = i * a.m_seq + s;
                }
            }
            __syncthreads();
        }
#pragma unroll
        for (int n = 0; n < AP_ITEMS; ++n) {
            if (row[n] < 0) continue;
            const bool is_v = row[n] >= q_heads + heads;
            T *to;
            if (row[n] < q_heads) to = (T *)a.q_out + (first + token[n]) * a.qo_tok + row[n] * a.qo_head;
            else if (kv_row[token[n]]) to = (T *)(kv_row[token[n]] + (is_v ? a.c.plane_stride : 0)) + (row[n] - q_heads - (is_v ? heads : 0)) * dim;
            else continue;
            if (!is_v && lo[n] < a.rotary) {
                const float2 *cs = turn + token[n] * half + (halves ? lo[n] : lo[n] >> 1);
                if (halves || V == 1) {
#pragma unroll
                    for (int d = 0; d < V; ++d) {
                        const float u = kv_float(x[n].e[d]), w = kv_float(y[n].e[d]);
                        x[n].e[d] = kv_round<T>(u * cs[d].x - w * cs[d].y);
                        y[n].e[d] = kv_round<T>(u * cs[d].y + w * cs[d].x);
                    }
                } else {
#pragma unroll
                    for (int d = 0; d < V / 2; ++d) {
                        const float u = kv_float(x[n].e[2 * d]), w = kv_float(x[n].e[2 * d + 1]);
                        x[n].e[2 * d] = kv_round<T>(u * cs[d].x - w * cs[d].y);
                        x[n].e[2 * d + 1] = kv_round<T>(u * cs[d].y + w * cs[d].x);
                    }
                }
            }
            *(Pack *)(to + lo[n]) = x[n];
            if (hi[n] >= 0) *(Pack *)(to + hi[n]) = y[n];
        }
    }
    if (a.weights || a.order)
        for (int e = tid; e < tokens * heads; e += AP_THREADS) {
            const int k = e / heads, h = e - k * heads;
            if (!kv_row[k]) continue;
            if (a.weights) a.weights[meta[k] + h * a.m_head] = 0.f;
            if (a.order) a.order[meta[k] + h * a.m_head] = a.token_order ? a.token_order[first + k] : a.positions[first + k];
        }
}
