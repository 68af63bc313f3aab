// New tokens into the paged cache: rotary positions with several axes on q and k, then k and v into their slots.
//
// A token's angles are the same for all its heads, so they are worked out once per token: position * inv_freq is exact
// in float64 (31 + 24 bits against 53, one rounding at most), reduced to a fraction of a turn there, and only then
// goes to float32 for sine and cosine: at position 10^5 a float32 product would be off by 4e-3 radians already.
#pragma once
#include "kv_ops.cuh"

struct KvAppend {
    KvView c;
    int layer, num_seqs, q_heads, rotary, pairs_style;
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
    uint8_t axis_of[128];
};

// the sequence that token t belongs to: the last one that starts at or before it
__device__ __forceinline__ int kv_seq_of(const int *starts, int num_seqs, long long t)
{
    int lo = 0, hi = num_seqs;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (starts[mid] <= t) lo = mid;
        else hi = mid;
    }
    return lo;
}

template <typename T>
__global__ void __launch_bounds__(128) kv_append_tokens(const __grid_constant__ KvAppend a)
{
    __shared__ float cs[128], sn[128];
    __shared__ uint8_t *kv_row[2];
    __shared__ int where[2];
    const long long t = blockIdx.x;
    const int tid = threadIdx.x, dim = a.c.dim, half = a.rotary >> 1, heads = a.c.heads;
    if (tid < half) {
        const double turns = (double)a.positions[a.axis_of[tid] * a.axis_stride + t] * (double)a.inv_freq[tid] * 0.15915494309189533577;
        sincospif((float)(2.0 * (turns - rint(turns))), &sn[tid], &cs[tid]);
    }
    if (tid == 0) {
        const int i = a.starts ? kv_seq_of(a.starts, a.num_seqs, t) : (int)t;
        const long long left = a.starts ? a.starts[i + 1] - t : 1;   // this token and those behind it
        const int n = a.c.len(i);
        const long long s = n - left;
        const bool ok = left > 0 && s >= 0;
        if (!ok && n > 0) atomicOr(a.c.status, KV_OPS_BAD_LEN);
        kv_row[0] = ok ? a.c.slot(i, (int)s, a.layer * 2) : nullptr;
        kv_row[1] = kv_row[0] ? a.c.slot(i, (int)s, a.layer * 2 + 1) : nullptr;
        where[0] = i;
        where[1] = (int)s;
    }
    __syncthreads();
    for (int e = tid; e < (a.q ? a.q_heads : 0) * half; e += 128) {
        const int g = e / half, f = e % half;
        const int lo = a.pairs_style ? 2 * f : f, hi = a.pairs_style ? 2 * f + 1 : f + half;
        const T *q = (const T *)a.q + t * a.q_tok + g * a.q_head;
        T *o = (T *)a.q_out + t * a.qo_tok + g * a.qo_head;
        const float x = kv_float(q[lo]), y = kv_float(q[hi]);
        o[lo] = kv_round<T>(x * cs[f] - y * sn[f]);
        o[hi] = kv_round<T>(x * sn[f] + y * cs[f]);
    }
    for (int e = tid; e < (a.q ? a.q_heads : 0) * (dim - a.rotary); e += 128) {
        const int g = e / (dim - a.rotary), d = a.rotary + e % (dim - a.rotary);
        ((T *)a.q_out)[t * a.qo_tok + g * a.qo_head + d] = ((const T *)a.q)[t * a.q_tok + g * a.q_head + d];
    }
    if (!kv_row[0]) return;
    for (int e = tid; e < heads * half; e += 128) {
        const int h = e / half, f = e % half;
        const int lo = a.pairs_style ? 2 * f : f, hi = a.pairs_style ? 2 * f + 1 : f + half;
        const T *k = (const T *)a.k + t * a.k_tok + h * a.k_head;
        T *o = (T *)kv_row[0] + h * dim;
        const float x = kv_float(k[lo]), y = kv_float(k[hi]);
        o[lo] = kv_round<T>(x * cs[f] - y * sn[f]);
        o[hi] = kv_round<T>(x * sn[f] + y * cs[f]);
    }
    for (int e = tid; e < heads * (dim - a.rotary); e += 128) {
        const int h = e / (dim - a.rotary), d = a.rotary + e % (dim - a.rotary);
        ((T *)kv_row[0])[h * dim + d] = ((const T *)a.k)[t * a.k_tok + h * a.k_head + d];
    }
    for (int e = tid; e < heads * dim; e += 128)
        ((T *)kv_row[1])[e] = ((const T *)a.v)[t * a.v_tok + (e / dim) * a.v_head + e % dim];
    for (int h = tid; h < heads; h += 128) {
        const long long at = where[0] * a.m_seq + h * a.m_head + where[1];
        if (a.weights) a.weights[at] = 0.f;
        if (a.order) a.order[at] = a.token_order ? a.token_order[t] : a.positions[t];
    }
}
