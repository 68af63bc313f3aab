// New tokens into the paged cache: rotary positions with several axes on q and k, then k and v into their slots.
//
// A token's angles are the same for all its heads, so they are worked out once per token: position * inv_freq is exact
// in float64 (31 + 24 bits against 53, one rounding at most), reduced to a fraction of a turn there, and only then
// goes to float32 for sine and cosine: at position 10^5 a float32 product would be off by 4e-3 radians already.
//
// What bounds it: for prompts the bytes of q, k and v, read and written once; for a decode step the chain of loads.  A CTA
// takes up to AP_TOKENS tokens.  Every thread first sends off its first loads of rows, and the tokens' angles and slots (a
// search, a length, a block id: loads that wait for one another) are worked out while they travel, all tokens at once;
// then only rows stream through, two packs of 16 bytes and their partners per thread in flight, at a place in the row that
// is the same all along, so that nothing but the row's address is worked out per row.
//
// Measured: 14.3k prompt tokens of 32 + 8 + 8 heads of 128, 353 MB: 65 us, 5.4 TB/s, 83 % of the floor (with one row per thread
// 69 us, three 76, four 73; with the place worked out per pack 78; one token per CTA 186).  One token 4.0 us, 64 tokens of
// 64 + 8 + 8 heads 5.0 us, where the first form's search by one thread and loads behind the angles took 9.7 and 14.4.
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
    int num_slots;       // of weights and order
    int units;           // threads of a row: packs of `vec` elements with those they turn with, then packs that pass
    int per;             // tokens per CTA
    unsigned by_rows;    // 2^32 / rows of a token, rounded up
    uint8_t axis_of[128];
};

constexpr int AP_THREADS = 256, AP_ROWS = 2, AP_TOKENS = 16;

// what a thread moves at once: eight or four elements as pairs, or one element
template <typename T, int V> struct __align__(V * 2) KvPack { unsigned w[V / 2]; };
template <typename T> struct KvPack<T, 1> { T e; };

template <typename T, int V>
__global__ void __launch_bounds__(AP_THREADS) kv_append_tokens(const __grid_constant__ KvAppend a)
{
    using Pack = KvPack<T, V>;
    extern __shared__ __align__(16) float2 turn[];       // [token][frequency]: cosine and sine
    __shared__ uint8_t *kv_row[AP_TOKENS];               // K of the token's slot, or nullptr
    __shared__ long long meta[AP_TOKENS];
    const int tid = threadIdx.x, dim = a.c.dim, half = a.rotary >> 1, heads = a.c.heads, q_heads = a.q ? a.q_heads : 0, rows = q_heads + 2 * heads;
    const bool halves = a.pairs_style == 0;
    // A thread has the same place in every row it works on: unit u.  The first `turns` units turn: a pack and its partners
    // (halves style), a pack of pairs, or a single pair; the others pass.
    const int turns = halves ? half / V : V == 1 ? half : a.rotary / V, lanes = AP_THREADS / a.units, u = tid % a.units, mine = tid / a.units;
    const bool turned = u < turns;
    const int lo = turned ? halves || V > 1 ? u * V : 2 * u : a.rotary + (u - turns) * V, hi = !turned ? -1 : halves ? lo + half : V == 1 ? lo + 1 : -1;
    // frequencies of a unit lie two by two, side by side with the other units': a warp's reads of them do not collide
    const int per_unit = V == 1 ? 1 : halves ? V : V / 2;
    const long long first = (long long)blockIdx.x * a.per;
    const int tokens = (int)min((long long)a.per, a.num_tokens - first), total = tokens * rows;
    for (int r0 = mine; r0 - mine < total; r0 += lanes * AP_ROWS) {
        Pack x[AP_ROWS], y[AP_ROWS];
        int token[AP_ROWS], row[AP_ROWS];
#pragma unroll
        for (int n = 0; n < AP_ROWS; ++n) {
            const int r = r0 + n * lanes;
            row[n] = -1;
            if (r < total && mine < lanes) {
                token[n] = (int)__umulhi((unsigned)r, a.by_rows);
                row[n] = r - token[n] * rows;
                const long long t = first + token[n];
                const T *from = row[n] < q_heads           ? (const T *)a.q + t * a.q_tok + row[n] * a.q_head
                                : row[n] < q_heads + heads ? (const T *)a.k + t * a.k_tok + (row[n] - q_heads) * a.k_head
                                                           : (const T *)a.v + t * a.v_tok + (row[n] - q_heads - heads) * a.v_head;
                x[n] = *(const Pack *)(from + lo);
                if (hi >= 0) y[n] = *(const Pack *)(from + hi);
            }
        }
        if (r0 == mine) {            // the first time: angles and slots
            for (int f = tid; f < tokens * half; f += AP_THREADS) {
                const int k = f / half, q = f - k * half;
                const double cycles = (double)a.positions[a.axis_of[q] * a.axis_stride + first + k] * (double)a.inv_freq[q] * 0.15915494309189533577;
                float2 cs;
                sincospif((float)(2.0 * (cycles - rint(cycles))), &cs.y, &cs.x);
                turn[k * half + (V == 1 ? q : (q % per_unit / 2 * turns + q / per_unit) * 2 + q % 2)] = cs;
            }
            for (int k = tid >> 5; k < tokens; k += AP_THREADS / 32) {
                const long long t = first + k;
                const int i = a.starts ? kv_seq_of(a.starts, a.num_seqs, t) : (int)t;
                const long long left = a.starts ? a.starts[i + 1] - t : 1;       // this token and those behind it
                const bool member = !a.starts || a.starts[i] <= t;               // not one in front of the first start
                const int n = a.c.len(i);
                const long long s = n - left;
                const bool ok = member && left > 0 && s >= 0 && (!(a.weights || a.order) || s < a.num_slots);
                if ((tid & 31) == 0) {
                    if (!ok && n > 0) atomicOr(a.c.status, KV_OPS_BAD_LEN);
                    kv_row[k] = ok ? a.c.slot(i, (int)s, a.layer * 2) : nullptr;
                    meta[k] = i * a.m_seq + s;
                }
            }
            __syncthreads();
        }
#pragma unroll
        for (int n = 0; n < AP_ROWS; ++n) {
            if (row[n] < 0) continue;
            const bool is_v = row[n] >= q_heads + heads;
            T *to;
            if (row[n] < q_heads) to = (T *)a.q_out + (first + token[n]) * a.qo_tok + row[n] * a.qo_head;
            else if (kv_row[token[n]]) to = (T *)(kv_row[token[n]] + (is_v ? a.c.plane_stride : 0)) + (row[n] - q_heads - (is_v ? heads : 0)) * dim;
            else continue;
            if (!is_v && turned) {
                const float2 *cs = turn + token[n] * half;
                if constexpr (V == 1) {
                    const float2 c = cs[u];
                    const float p = kv_float(x[n].e), q = kv_float(y[n].e);
                    x[n].e = kv_round<T>(p * c.x - q * c.y);
                    y[n].e = kv_round<T>(p * c.y + q * c.x);
                } else if (halves) {
#pragma unroll
                    for (int j = 0; j < V / 2; ++j) {    // two frequencies
                        const float4 c = *(const float4 *)(cs + (j * turns + u) * 2);
                        const float2 p = kv_unpair(x[n].w[j], T()), q = kv_unpair(y[n].w[j], T());
                        x[n].w[j] = kv_pair(p.x * c.x - q.x * c.y, p.y * c.z - q.y * c.w, T());
                        y[n].w[j] = kv_pair(p.x * c.y + q.x * c.x, p.y * c.w + q.y * c.z, T());
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < V / 4; ++j) {
                        const float4 c = *(const float4 *)(cs + (j * turns + u) * 2);
                        const float2 p = kv_unpair(x[n].w[2 * j], T()), q = kv_unpair(x[n].w[2 * j + 1], T());
                        x[n].w[2 * j] = kv_pair(p.x * c.x - p.y * c.y, p.x * c.y + p.y * c.x, T());
                        x[n].w[2 * j + 1] = kv_pair(q.x * c.z - q.y * c.w, q.x * c.w + q.y * c.z, T());
                    }
                }
            }
            *(Pack *)(to + lo) = x[n];
            if (hi >= 0) *(Pack *)(to + hi) = y[n];
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
