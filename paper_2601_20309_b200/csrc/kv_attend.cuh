// Attention of one new token per sequence over the paged cache.
//
// First form: one CTA per (sequence, query head).  Scores go to the workspace, their maximum and the sum of
// exponentials are taken over the whole row, then every thread sums one element of the output over the slots.  K and V
// are read once per query head.
#pragma once
#include "kv_ops.cuh"

struct KvAttend {
    KvView c;
    int layer, q_heads, group, window;
    float scale;
    const void *q;
    long long q_seq, q_head;
    void *out;
    long long o_seq, o_head;
    float *lse;
    const float *w_in;
    float *w_out;
    long long w_seq, w_head;
    float *scores;       // [seq][q_head][max_len]
    float *row_lse;      // [seq][q_head]
};

template <typename T>
__global__ void __launch_bounds__(128) kv_attend_rows(const __grid_constant__ KvAttend a)
{
    __shared__ float qs[256], red[4];
    const int g = blockIdx.x, i = blockIdx.y, h = g / a.group, dim = a.c.dim;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int n = a.c.len(i), first = a.window > 0 && n > a.window ? n - a.window : 0;
    float *sc = a.scores + ((long long)i * a.q_heads + g) * a.c.max_len;
    for (int d = tid; d < dim; d += 128) qs[d] = kv_float(((const T *)a.q)[i * a.q_seq + g * a.q_head + d]);
    __syncthreads();
    float top = -INFINITY;
    for (int t = first + warp; t < n; t += 4) {
        const T *k = (const T *)a.c.slot(i, t, a.layer * 2);
        float s = 0.f;
        if (k)
            for (int d = lane; d < dim; d += 32) s += qs[d] * kv_float(k[h * dim + d]);
#pragma unroll
        for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(~0u, s, o);
        s = k ? s * a.scale : -INFINITY;
        if (lane == 0) sc[t] = s;
        top = isnan(s) || isnan(top) ? NAN : fmaxf(top, s);
    }
    if (lane == 0) red[warp] = top;
    __syncthreads();
    for (int w = 0; w < 4; ++w) top = isnan(red[w]) || isnan(top) ? NAN : fmaxf(top, red[w]);
    const float ref = top == -INFINITY ? 0.f : top;
    __syncthreads();
    float sum = 0.f;
    for (int t = first + tid; t < n; t += 128) sum += expf(sc[t] - ref);
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
    if (lane == 0) red[warp] = sum;
    __syncthreads();
    sum = red[0] + red[1] + red[2] + red[3];
    const float lse = sum == 0.f ? -INFINITY : ref + logf(sum);
    if (tid == 0) {
        a.row_lse[(long long)i * a.q_heads + g] = lse;
        if (a.lse) a.lse[(long long)i * a.q_heads + g] = lse;
    }
    for (int d = tid; d < dim; d += 128) {
        float o = 0.f;
        if (sum != 0.f) {
            for (int t = first; t < n; ++t) {
                const T *v = (const T *)a.c.slot(i, t, a.layer * 2 + 1);
                if (v) o += expf(sc[t] - ref) * kv_float(v[h * dim + d]);
            }
            o /= sum;
        }
        ((T *)a.out)[i * a.o_seq + g * a.o_head + d] = kv_round<T>(o);
    }
}

// weights_out = weights_in + the slot's attention weight, summed over the query heads of its KV head in their order
__global__ void __launch_bounds__(256) kv_attend_weights(const __grid_constant__ KvAttend a)
{
    const int i = blockIdx.z, h = blockIdx.y;
    const int n = a.c.len(i), first = a.window > 0 && n > a.window ? n - a.window : 0;
    for (long long t = blockIdx.x * 256 + threadIdx.x; t < n; t += (long long)gridDim.x * 256) {
        const long long at = i * a.w_seq + h * a.w_head + t;
        float w = 0.f;
        if (t >= first)
            for (int g = h * a.group; g < (h + 1) * a.group; ++g) {
                const float lse = a.row_lse[(long long)i * a.q_heads + g];
                if (lse != -INFINITY) w += expf(a.scores[((long long)i * a.q_heads + g) * a.c.max_len + t] - lse);
            }
        a.w_out[at] = (a.w_in ? a.w_in[at] : 0.f) + w;
    }
}
