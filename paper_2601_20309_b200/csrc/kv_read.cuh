// Rows of K and V out of the paged cache, side by side and in 16 bits: the inverse of an append, for what takes plain tensors
// (the attention of a prompt that arrives in pieces, an export).  element = lo + s * code, one fused operation, one rounding.
//
// What bounds it: the bytes written, 3.2 times those read from a cache in 4 bits.  A thread writes 16 neighbouring elements of one
// head of K and of V, or, in 4 bits, eight of every group, which is what G neighbouring words of codes hold; the tokens' slots (a
// search, a length, a block id) are found once per CTA.  14.3k tokens of 8 heads of 128, 77 MB: 17 us, 4.5 TB/s (23 us with 16
// neighbouring elements per thread here too: loads of 2 and 4 bytes).
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
    int units;                   // threads of a row and head
    unsigned by_units;           // 2^32 / (units * heads), rounded up; 0: units * heads is 1
};

constexpr int RD_TOKENS = 32;

// G: groups of a cache in 4 bits, 0: 16 bits
template <typename T, bool VEC, int G>
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
            if (G) to_words[k] = ok ? a.c.to_words((int)s) : 0;
        }
    }
    __syncthreads();
    for (int f = tid; f < total; f += AP_THREADS) {
        const int token = a.by_units ? (int)__umulhi((unsigned)f, a.by_units) : f, rest = f - token * per_token, h = rest / a.units, u = rest - h * a.units;
        const uint8_t *row = kv_row[token];
        if (!row) continue;
        row += (long long)h * a.c.head_stride;
        T *k_to = a.k ? (T *)a.k + (first + token) * a.k_tok + h * a.k_head : nullptr, *v_to = a.v ? (T *)a.v + (first + token) * a.v_tok + h * a.v_head : nullptr;
        auto put = [](T *to, const uint4 &v) {           // eight elements
            if (VEC) *(uint4 *)to = v;
            else {
                const unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int e = 0; e < 8; ++e) ((unsigned short *)to)[e] = (unsigned short)(w[e >> 1] >> (16 * (e & 1)));
            }
        };
        if constexpr (G == 0) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int d = 16 * u + 8 * j;
                if (d >= dim) continue;
                if (k_to) put(k_to + d, *(const uint4 *)(row + 2 * d));
                if (v_to) put(v_to + d, *(const uint4 *)(row + a.c.plane_stride + 2 * d));
            }
        } else {
            // elements 32 g + 8 u .. + 7 of every group g: G words of K's codes side by side, as many half words twice of V's
            unsigned codes[2][G], words[2][G];
            kv_words(codes[0], row + 4 * G * u);
            kv_words(codes[1], row + a.c.plane_stride + 4 * G * u);
            kv_words(words[0], row + to_words[token]);
            kv_words(words[1], row + a.c.plane_stride + to_words[token]);
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                T *to = p ? v_to : k_to;
                if (!to) continue;
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    if (32 * g + 8 * u >= dim) continue;
                    const unsigned c = p ? __byte_perm(codes[1][g >> 1], codes[1][G / 2 + (g >> 1)], g & 1 ? 0x7632 : 0x5410) : codes[0][g], d = c >> 8;
                    // a code in the lowest bits of a 16-bit word is code * 2^-24 in float16, four bits further code * 2^-20
                    const float lo = kv_unpair(words[p][g], T()).x, s = __uint_as_float(words[p][g] & 0xffff0000u);
                    const auto at = [&](float code, float unit) { return fmaf(s, code * unit, lo); };
                    const float2 x0 = kv_unpair(c & 0x000f000fu, __half()), x1 = kv_unpair(c & 0x00f000f0u, __half());     // elements 0 and 4, 1 and 5
                    const float2 x2 = kv_unpair(d & 0x000f000fu, __half()), x3 = kv_unpair(d & 0x00f000f0u, __half());     // 2 and 6, 3 and 7
                    put(to + 32 * g + 8 * u, make_uint4(kv_pair(at(x0.x, 0x1p24f), at(x1.x, 0x1p20f), T()), kv_pair(at(x2.x, 0x1p24f), at(x3.x, 0x1p20f), T()),
                                                        kv_pair(at(x0.y, 0x1p24f), at(x1.y, 0x1p20f), T()), kv_pair(at(x2.y, 0x1p24f), at(x3.y, 0x1p20f), T())));
                }
            }
        }
    }
}
