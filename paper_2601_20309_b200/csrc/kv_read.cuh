// Rows of K and V out of the paged cache, side by side and in 16 bits: the inverse of an append, for what takes plain tensors
// (the attention of a prompt that arrives in pieces, an export).  element = lo + s * code, one fused operation, one rounding.
//
// What bounds it: the bytes written, 3.2 times those read from a cache in 4 bits.  A thread writes 16 neighbouring elements of one
// head of K and of V; the tokens' slots (a search, a length, a block id) are found once per CTA.
#pragma once
#include "kv_append.cuh"

struct KvRead {
    KvView c;
    int layer, num_seqs;
    long long num_tokens;
    void *k, *v;                 // either may be nullptr
    long long k_tok, k_head, v_tok, v_head;
    const int *starts;
    int per;                     // tokens per CTA
    int units;                   // runs of 16 elements of a head
    unsigned by_units;           // 2^32 / (units * heads), rounded up
};

constexpr int RD_TOKENS = 32;

template <typename T, bool VEC, bool Q4>
__global__ void __launch_bounds__(AP_THREADS) kv_read_rows(const __grid_constant__ KvRead a)
{
    __shared__ const uint8_t *kv_row[RD_TOKENS];
    __shared__ int to_words[RD_TOKENS];
    const int tid = threadIdx.x, dim = a.c.dim, per_token = a.units * a.c.heads;
    const long long first = (long long)blockIdx.x * a.per;
    const int tokens = (int)min((long long)a.per, a.num_tokens - first), total = tokens * per_token;
    for (int k = tid >> 5; k < tokens; k += AP_THREADS / 32) {
        const long long t = first + k;
        const int i = a.starts ? kv_seq_of(a.starts, a.num_seqs, t) : (int)t;
        const long long left = a.starts ? a.starts[i + 1] - t : 1;
        const bool member = !a.starts || a.starts[i] <= t;
        const int n = a.c.len(i);
        const long long s = n - left;
        const bool ok = member && left > 0 && s >= 0;
        if ((tid & 31) == 0) {
            if (!ok && n > 0) atomicOr(a.c.status, KV_OPS_BAD_LEN);
            kv_row[k] = ok ? a.c.slot(i, (int)s, a.layer * 2) : nullptr;
            if (Q4) to_words[k] = ok ? a.c.to_words((int)s) : 0;
        }
    }
    __syncthreads();
    for (int f = tid; f < total; f += AP_THREADS) {
        const int token = (int)__umulhi((unsigned)f, a.by_units), rest = f - token * per_token, h = rest / a.units, u = rest - h * a.units;
        const uint8_t *row = kv_row[token];
        if (!row) continue;
        row += (long long)h * a.c.head_stride;
        const int runs = min(2, (dim - 16 * u) >> 3);    // of eight elements
        unsigned w[2][8];
        if constexpr (Q4) {
            const int G = a.c.groups, g = u >> 1;
            unsigned codes[2][2], word[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) codes[0][j] = ((const unsigned *)row)[((u & 1) * 2 + j) * G + g];
            word[0] = ((const unsigned *)(row + to_words[token]))[g];
            row += a.c.plane_stride;
#pragma unroll
            for (int j = 0; j < 2; ++j)
                codes[1][j] = ((const unsigned short *)row)[((u & 1) * 4 + 2 * j) * G + g] |
                              (unsigned)((const unsigned short *)row)[((u & 1) * 4 + 2 * j + 1) * G + g] << 16;
            word[1] = ((const unsigned *)(row + to_words[token]))[g];
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                // a code in the lowest bits of a 16-bit word is code * 2^-24 in float16, four bits further code * 2^-20
                const float lo = kv_unpair(word[p], T()).x, s = __uint_as_float(word[p] & 0xffff0000u);
                const auto at = [&](float code, float unit) { return fmaf(s, code * unit, lo); };
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const unsigned c = codes[p][j], d = c >> 8;
                    const float2 x0 = kv_unpair(c & 0x000f000fu, __half()), x1 = kv_unpair(c & 0x00f000f0u, __half());     // elements 0 and 4, 1 and 5
                    const float2 x2 = kv_unpair(d & 0x000f000fu, __half()), x3 = kv_unpair(d & 0x00f000f0u, __half());     // 2 and 6, 3 and 7
                    w[p][4 * j] = kv_pair(at(x0.x, 0x1p24f), at(x1.x, 0x1p20f), T());
                    w[p][4 * j + 1] = kv_pair(at(x2.x, 0x1p24f), at(x3.x, 0x1p20f), T());
                    w[p][4 * j + 2] = kv_pair(at(x0.y, 0x1p24f), at(x1.y, 0x1p20f), T());
                    w[p][4 * j + 3] = kv_pair(at(x2.y, 0x1p24f), at(x3.y, 0x1p20f), T());
                }
            }
        } else {
#pragma unroll
            for (int p = 0; p < 2; ++p, row += a.c.plane_stride)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    if (j < runs) {
                        const uint4 v = ((const uint4 *)row)[2 * u + j];
                        w[p][4 * j] = v.x, w[p][4 * j + 1] = v.y, w[p][4 * j + 2] = v.z, w[p][4 * j + 3] = v.w;
                    }
        }
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            void *base = p ? a.v : a.k;
            if (!base) continue;
            T *to = (T *)base + (first + token) * (p ? a.v_tok : a.k_tok) + h * (p ? a.v_head : a.k_head) + 16 * u;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                if (j >= runs) continue;
                if (VEC) ((uint4 *)to)[j] = make_uint4(w[p][4 * j], w[p][4 * j + 1], w[p][4 * j + 2], w[p][4 * j + 3]);
                else
#pragma unroll
                    for (int e = 0; e < 8; ++e) ((unsigned short *)to)[8 * j + e] = (unsigned short)(w[p][4 * j + (e >> 1)] >> (16 * (e & 1)));
            }
        }
    }
}
