// Eviction by accumulated attention weight: `keep` slots stay, and only those at or above `keep` move, into the holes
// the evicted ones leave below it.  Sources (>= keep) and holes (< keep) never meet, so the moves need no order.
//
// First form: kv_evict_select, one CTA per (layer, sequence, KV head), finds the threshold key by four radix passes of
// eight bits, then walks the slots in order and writes the (hole, source) pairs to the workspace; kv_evict_move copies
// the K and V rows.
#pragma once
#include "kv_ops.cuh"

struct KvEvict {
    KvView c;
    int first_layer, layers, seqs, keep, recent, sink;
    const float *w;
    const int *order;
    long long m_layer, m_seq, m_head;
    const int *seen;
    float *w_out;
    int *order_out;
    long long o_layer, o_seq, o_head;
    int *lens_out;
    int *count;          // [problem]: rows that move
    int *holes, *srcs;   // [problem][cap]
    int cap;
};

// weights as integers of the same order: NaN lowest, -0 equal to +0, protected slots above everything
__device__ __forceinline__ unsigned kv_evict_key(float w, bool held)
{
    if (held) return 0xFFFFFFFFu;
    if (isnan(w)) return 0u;
    const unsigned u = __float_as_uint(w + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ unsigned kv_evict_slot_key(const KvEvict &a, long long at, int t, int newest)
{
    const int age = a.order ? a.order[at + t] : t;
    return kv_evict_key(a.w[at + t], age >= newest || age < a.sink);
}

constexpr int EV_THREADS = 256;

// exclusive prefix sum of one value per thread over the CTA; total to every thread
__device__ __forceinline__ int kv_block_scan(int v, int *total)
{
    __shared__ int part[EV_THREADS / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(~0u, x, o);
        if (lane >= o) x += y;
    }
    if (lane == 31) part[warp] = x;
    __syncthreads();
    int before = 0, all = 0;
    for (int w = 0; w < EV_THREADS / 32; ++w) {
        if (w < warp) before += part[w];
        all += part[w];
    }
    __syncthreads();
    *total = all;
    return before + x - v;
}

__global__ void __launch_bounds__(EV_THREADS) kv_evict_select(const __grid_constant__ KvEvict a)
{
    __shared__ int hist[256];
    __shared__ unsigned s_digit;
    __shared__ int s_need;
    const int h = blockIdx.x, i = blockIdx.y, l = blockIdx.z, tid = threadIdx.x;
    const int problem = (l * a.seqs + i) * a.c.heads + h;
    const int n = a.c.len(i);
    const long long at = l * a.m_layer + i * a.m_seq + h * a.m_head;
    const long long to = l * a.o_layer + i * a.o_seq + h * a.o_head;
    if (l == 0 && h == 0 && tid == 0 && a.lens_out) a.lens_out[i] = min(n, a.keep);
    const bool apart = a.w_out != a.w;
    if (n <= a.keep) {
        if (apart)
            for (int t = tid; t < n; t += EV_THREADS) {
                a.w_out[to + t] = a.w[at + t];
                if (a.order_out) a.order_out[to + t] = a.order[at + t];
            }
        if (tid == 0) a.count[problem] = 0;
        return;
    }
    const int newest = (a.seen ? a.seen[i] : n) - a.recent;
    // the key of rank keep - 1 from above, eight bits at a time; need = how many of the keys that begin with the
    // prefix found so far still stay
    unsigned prefix = 0;
    int need = a.keep;
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int b = tid; b < 256; b += EV_THREADS) hist[b] = 0;
        __syncthreads();
        for (int t = tid; t < n; t += EV_THREADS) {
            const unsigned k = kv_evict_slot_key(a, at, t, newest);
            if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255], 1);
        }
        __syncthreads();
        if (tid == 0) {
            int left = need, b = 255;
            while (b > 0 && hist[b] < left) left -= hist[b--];
            s_digit = b;
            s_need = left;
        }
        __syncthreads();
        prefix |= s_digit << shift;
        need = s_need;
        __syncthreads();
    }
    int ties = 0, nh = 0, ns = 0;
    for (int t0 = 0; t0 < n; t0 += EV_THREADS) {
        const int t = t0 + tid;
        const unsigned k = t < n ? kv_evict_slot_key(a, at, t, newest) : 0u;
        const bool tie = t < n && k == prefix;
        int all;
        const int rank = ties + kv_block_scan(tie, &all);
        ties += all;
        const bool stays = t < n && (k > prefix || (tie && rank < need));
        const bool hole = t < a.keep && !stays, src = t >= a.keep && stays;
        const int ph = nh + kv_block_scan(hole, &all);
        nh += all;
        const int ps = ns + kv_block_scan(src, &all);
        ns += all;
        if (hole) a.holes[(long long)problem * a.cap + ph] = t;
        if (src) a.srcs[(long long)problem * a.cap + ps] = t;
        if (apart && stays && t < a.keep) {
            a.w_out[to + t] = a.w[at + t];
            if (a.order_out) a.order_out[to + t] = a.order[at + t];
        }
    }
    __syncthreads();
    for (int m = tid; m < nh; m += EV_THREADS) {
        const int d = a.holes[(long long)problem * a.cap + m], s = a.srcs[(long long)problem * a.cap + m];
        a.w_out[to + d] = a.w[at + s];
        if (a.order_out) a.order_out[to + d] = a.order[at + s];
    }
    if (tid == 0) a.count[problem] = nh;
}

__global__ void __launch_bounds__(256) kv_evict_move(const __grid_constant__ KvEvict a)
{
    const int problem = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int h = problem % a.c.heads, i = problem / a.c.heads % a.seqs, l = problem / a.c.heads / a.seqs + a.first_layer;
    const int n = a.count[problem];
    for (int m = blockIdx.y * 8 + warp; m < n; m += gridDim.y * 8) {
        const int d = a.holes[(long long)problem * a.cap + m], s = a.srcs[(long long)problem * a.cap + m];
        for (int kv = 0; kv < 2; ++kv) {
            const uint8_t *from = a.c.slot(i, s, l * 2 + kv);
            uint8_t *into = a.c.slot(i, d, l * 2 + kv);
            if (!from || !into) continue;
            for (int b = lane * 16; b < a.c.dim * 2; b += 512)
                *(uint4 *)(into + (long long)h * a.c.head_stride + b) = *(const uint4 *)(from + (long long)h * a.c.head_stride + b);
        }
    }
}
