// New tokens into the paged cache where a row is more than its elements one by one: norms of q and k over the elements of a head
// before the rotation, and rows that the cache holds in 4 bits.
//
//   norm      y_d = x_d / sqrt(mean x^2 + eps) * w_d, for the heads of q and of k whose weights are given; then the rotation of
//             kv_append.cuh.  Float32 throughout, one rounding at the end.
//   4 bits    per group of 32 elements: lo = the lowest, s = (highest - lo) * float32(1/15), at least |lo| 2^-20, rounded to bf16;
//             code = floor((x - lo) / s + 1/2), at most 15.  lo is an element, so it is exact; s is never 0 beside a lo that is
//             not, which gives the attention a bound of lo by s.  A group with an element that is not finite, or whose range is not,
//             has NaN for both and reads as NaN.
//
// The 4-bit cache holds the codes of exactly what the 16-bit cache would hold: the row rounded to the cache's type.  A key that the
// rotation leaves next to a border between two codes, or between two values of the type, falls to the side the formula says: norm
// and rotation of keys run in float64 there (a third of the SM's rate, 8 of 48 rows), and the border itself is decided exactly: with
// n the code by a reciprocal, the remainder d - n s is exact in one fused operation, and moves n by one where it leaves [-s/2, s/2).
//
// A row belongs to 2^k lanes of a warp, 16 elements each in two runs of eight: what turns together where halves turn, neighbours
// elsewhere.  Sums over a row are shuffles among its lanes.  A key to be packed crosses shared memory once, from its
// pairs to neighbours, since groups are neighbours.  Angles and slots as in kv_append_tokens: once per token, behind the first loads.
#pragma once
#include "kv_append.cuh"

struct KvAppendRows {
    KvAppend p;
    const void *q_w, *k_w;       // weights of the norms, nullptr: none
    long long q_w_head, k_w_head;    // from a head's weights to the next's, 0: the same for all
    int w_float;                 // weights are float32, else of the cache's type
    float eps;
    int lanes_log2;              // lanes of a row
    int turns;                   // lanes that hold what turns
};

// a word of a group that is not finite
template <typename T> __device__ __forceinline__ unsigned kv_nan_word();
template <> __device__ __forceinline__ unsigned kv_nan_word<__nv_bfloat16>() { return 0x7fc07fc0u; }
template <> __device__ __forceinline__ unsigned kv_nan_word<__half>() { return 0x7fc07e00u; }

// Word and codes of 16 elements (as pairs), half of a group whose other half the neighbouring lane has; `count` of them exist.
// The codes come as 4 bits each, in order.  `mask`: the lanes that take part.
template <typename T> __device__ __forceinline__ unsigned kv_quantise(const unsigned (&x)[8], int count, unsigned mask, unsigned (&codes)[2])
{
    float lo = INFINITY, hi = -INFINITY;
    bool bad = false;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float2 v = kv_unpair(x[j], T());
        if (2 * j < count) {
            lo = fminf(lo, fminf(v.x, v.y));
            hi = fmaxf(hi, fmaxf(v.x, v.y));
            bad |= !(fabsf(v.x) < INFINITY) || !(fabsf(v.y) < INFINITY);
        }
    }
    lo = fminf(lo, __shfl_xor_sync(mask, lo, 1));
    hi = fmaxf(hi, __shfl_xor_sync(mask, hi, 1));
    bad |= __shfl_xor_sync(mask, (int)bad, 1) != 0;
    codes[0] = codes[1] = 0;
    if (lo > hi && !bad) return 0;                       // a group of nothing
    const float raw = fmaxf((hi - lo) * (1.f / 15.f), fabsf(lo) * 0x1p-20f);
    const __nv_bfloat16 rounded = __float2bfloat16(raw);
    float s = __bfloat162float(rounded);
    if (bad || !(s < INFINITY)) return kv_nan_word<T>();
    const unsigned word = kv_pair(lo, 0.f, T()) | (unsigned)__bfloat16_as_ushort(rounded) << 16;
    if (s == 0.f) return word;
    const float lift = s < 0x1p-100f ? 0x1p60f : 1.f;    // a reciprocal that is a number
    s *= lift;
    const float inv = 1.f / s, border = 0.5f * s;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float2 v = kv_unpair(x[j], T());
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const float d = ((e ? v.y : v.x) - lo) * lift;
            float n = floorf(fmaf(d, inv, 0.5f));
            const float left = fmaf(-n, s, d);
            n += (left >= border ? 1.f : 0.f) - (left < -border ? 1.f : 0.f);
            const unsigned code = 2 * j < count ? (unsigned)fminf(fmaxf(n, 0.f), 15.f) : 0u;
            codes[j >> 2] |= code << (4 * (2 * (j & 3) + e));
        }
    }
    return word;
}

// eight neighbouring elements, the first `n` of them, V at a time
template <int V> __device__ __forceinline__ void kv_load_run(unsigned (&w)[4], const void *from, int n)
{
    w[0] = w[1] = w[2] = w[3] = 0;
    if constexpr (V == 8) {
        if (n > 0) {
            const uint4 v = *(const uint4 *)from;
            w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
        }
    } else if constexpr (V == 4) {
#pragma unroll
        for (int b = 0; b < 2; ++b)
            if (n > 4 * b) {
                const uint2 v = ((const uint2 *)from)[b];
                w[2 * b] = v.x, w[2 * b + 1] = v.y;
            }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) w[e >> 1] |= (unsigned)((const unsigned short *)from)[e] << (16 * (e & 1));
    }
}
template <int V> __device__ __forceinline__ void kv_store_run(void *to, const unsigned (&w)[4], int n)
{
    if constexpr (V == 8) {
        if (n > 0) *(uint4 *)to = make_uint4(w[0], w[1], w[2], w[3]);
    } else if constexpr (V == 4) {
#pragma unroll
        for (int b = 0; b < 2; ++b)
            if (n > 4 * b) ((uint2 *)to)[b] = make_uint2(w[2 * b], w[2 * b + 1]);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) ((unsigned short *)to)[e] = (unsigned short)(w[e >> 1] >> (16 * (e & 1)));
    }
}

constexpr int AR_WEIGHTS = 256;      // elements of a head, at most

// Dynamic shared memory: [token][4][turns] float4 of cosine and sine of two frequencies each; packed caches further have
// [token][8][turns] double2 in front, and [row of the CTA][padded dim] elements behind
template <typename T, int V, bool Q4>
__global__ void __launch_bounds__(AP_THREADS) kv_append_rows(const __grid_constant__ KvAppendRows b)
{
    const KvAppend &a = b.p;
    extern __shared__ __align__(16) uint8_t ar_smem[];
    __shared__ uint8_t *kv_row[AP_TOKENS];               // K of the token's slot, or nullptr
    __shared__ long long meta[AP_TOKENS];
    __shared__ int to_words[AP_TOKENS];
    __shared__ __align__(16) float weight[2][AR_WEIGHTS];
    const int tid = threadIdx.x, dim = a.c.dim, half = a.rotary >> 1, heads = a.c.heads, q_heads = a.q ? a.q_heads : 0, rows = q_heads + 2 * heads;
    const int L = 1 << b.lanes_log2, u = tid & (L - 1), mine = tid >> b.lanes_log2, lanes = AP_THREADS >> b.lanes_log2, turns = b.turns;
    const unsigned mask = (L == 32 ? ~0u : (1u << L) - 1) << (tid & 31 & ~(L - 1));      // the lanes of this row
    const bool halves = a.pairs_style == 0;
    double2 *wide = (double2 *)ar_smem;
    float4 *turn = (float4 *)(ar_smem + (Q4 ? a.per * 8 * turns * 16 : 0));
    T *cross = (T *)(ar_smem + a.per * turns * (Q4 ? 192 : 64)) + mine * a.c.groups * 32;

    // the two runs of the lane in a row of q or k, and in one of v
    const bool turned = u < turns;
    const int b0 = turned ? (halves ? 8 * u : 16 * u) : a.rotary + 16 * (u - turns), b1 = turned && halves ? half + 8 * u : b0 + 8;
    const int end0 = turned ? (halves ? half : a.rotary) : dim, end1 = turned ? a.rotary : dim;
    const int n0 = min(max(end0 - b0, 0), 8), n1 = min(max(end1 - b1, 0), 8);
    const int v0 = 16 * u, vn0 = min(max(dim - v0, 0), 8), vn1 = min(max(dim - v0 - 8, 0), 8);

    const long long first = (long long)blockIdx.x * a.per;
    const int tokens = (int)min((long long)a.per, a.num_tokens - first), total = tokens * rows;
    for (int r0 = mine; r0 - mine < total; r0 += lanes * AP_ROWS) {
        unsigned x[AP_ROWS][4], y[AP_ROWS][4];
        int token[AP_ROWS], row[AP_ROWS];
#pragma unroll
        for (int n = 0; n < AP_ROWS; ++n) {
            const int r = r0 + n * lanes;
            row[n] = -1;
            token[n] = 0;
            if (r < total) {
                token[n] = (int)__umulhi((unsigned)r, a.by_rows);
                row[n] = r - token[n] * rows;
                const long long t = first + token[n];
                const bool is_v = row[n] >= q_heads + heads;
                const T *from = row[n] < q_heads ? (const T *)a.q + t * a.q_tok + row[n] * a.q_head
                                : is_v           ? (const T *)a.v + t * a.v_tok + (row[n] - q_heads - heads) * a.v_head
                                                 : (const T *)a.k + t * a.k_tok + (row[n] - q_heads) * a.k_head;
                kv_load_run<V>(x[n], from + (is_v ? v0 : b0), is_v ? vn0 : n0);
                kv_load_run<V>(y[n], from + (is_v ? v0 + 8 : b1), is_v ? vn1 : n1);
            }
        }
        if (r0 == mine) {            // the first time: weights that all heads share, angles and slots
            for (int d = tid; d < 2 * dim; d += AP_THREADS) {
                const int of_k = d >= dim, e = d - of_k * dim;
                const void *w = of_k ? b.k_w : b.q_w;
                if (w && (of_k ? b.k_w_head : b.q_w_head) == 0) weight[of_k][e] = b.w_float ? ((const float *)w)[e] : kv_float(((const T *)w)[e]);
            }
            for (int f = tid; f < tokens * half; f += AP_THREADS) {
                const int k = f / half, q = f - k * half, lane = q >> 3, j = q & 7;
                const double cycles = (double)a.positions[a.axis_of[q] * a.axis_stride + first + k] * (double)a.inv_freq[q] * 0.15915494309189533577;
                const double turned_by = 2.0 * (cycles - rint(cycles));
                float2 cs;
                if constexpr (Q4) {
                    double2 z;
                    sincospi(turned_by, &z.y, &z.x);
                    wide[(k * 8 + j) * turns + lane] = z;
                    cs = make_float2((float)z.x, (float)z.y);
                } else
                    sincospif((float)turned_by, &cs.y, &cs.x);
                ((float2 *)(turn + (k * 4 + (j >> 1)) * turns + lane))[j & 1] = cs;
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
                    if (Q4) to_words[k] = ok ? a.c.to_words((int)s) : 0;
                }
            }
            __syncthreads();
        }
#pragma unroll
        for (int n = 0; n < AP_ROWS; ++n) {
            if (row[n] < 0) continue;            // all lanes of the row
            const bool is_q = row[n] < q_heads, is_v = row[n] >= q_heads + heads;
            const int h = row[n] - (is_q ? 0 : is_v ? q_heads + heads : q_heads);
            uint8_t *slot = kv_row[token[n]];
            if (!is_q && !slot) continue;
            const void *wp = is_q ? b.q_w : is_v ? nullptr : b.k_w;
            const long long w_head = is_q ? b.q_w_head : b.k_w_head;
            const float *ws = weight[is_q ? 0 : 1];
            auto norm_weight = [&](int e) {
                if (w_head == 0) return ws[e];
                return b.w_float ? ((const float *)wp)[h * w_head + e] : kv_float(((const T *)wp)[h * w_head + e]);
            };
            if (Q4 && !is_q && !is_v) {          // a key in float64
                double r = 1.0;
                if (wp) {
                    double sum = 0.0;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float2 p = kv_unpair(x[n][j], T()), q = kv_unpair(y[n][j], T());
                        sum = fma((double)p.x, (double)p.x, fma((double)p.y, (double)p.y, sum));
                        sum = fma((double)q.x, (double)q.x, fma((double)q.y, (double)q.y, sum));
                    }
                    for (int o = L >> 1; o; o >>= 1) sum += __shfl_xor_sync(mask, sum, o);
                    r = 1.0 / sqrt(sum / dim + (double)b.eps);
                }
                // elements p and q of the two runs, or neighbours p.x and p.y
                auto normed = [&](float v, int e, bool on) { return wp && on ? (double)v * r * (double)norm_weight(e) : (double)v; };
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 p = kv_unpair(x[n][j], T()), q = kv_unpair(y[n][j], T());
                    double p0 = normed(p.x, b0 + 2 * j, 2 * j < n0), p1 = normed(p.y, b0 + 2 * j + 1, 2 * j + 1 < n0);
                    double q0 = normed(q.x, b1 + 2 * j, 2 * j < n1), q1 = normed(q.y, b1 + 2 * j + 1, 2 * j + 1 < n1);
                    if (turned) {
                        const double2 *cs = wide + token[n] * 8 * turns + u;
                        auto rotate = [](double &f, double &g, double2 c) {
                            const double t = f * c.x - g * c.y;
                            g = f * c.y + g * c.x;
                            f = t;
                        };
                        if (halves) {
                            if (2 * j < n0) rotate(p0, q0, cs[2 * j * turns]);
                            if (2 * j + 1 < n0) rotate(p1, q1, cs[(2 * j + 1) * turns]);
                        } else {
                            if (2 * j < n0) rotate(p0, p1, cs[j * turns]);
                            if (2 * j < n1) rotate(q0, q1, cs[(4 + j) * turns]);
                        }
                    }
                    x[n][j] = kv_pair((float)p0, (float)p1, T());
                    y[n][j] = kv_pair((float)q0, (float)q1, T());
                }
            } else if (!is_v) {
                float r = 1.f;
                if (wp) {
                    float sum = 0.f;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float2 p = kv_unpair(x[n][j], T()), q = kv_unpair(y[n][j], T());
                        sum += p.x * p.x + p.y * p.y + (q.x * q.x + q.y * q.y);
                    }
                    for (int o = L >> 1; o; o >>= 1) sum += __shfl_xor_sync(mask, sum, o);
                    r = 1.f / sqrtf(sum / dim + b.eps);
                }
                auto normed = [&](float v, int e, bool on) { return wp && on ? v * r * norm_weight(e) : v; };
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 p = kv_unpair(x[n][j], T()), q = kv_unpair(y[n][j], T());
                    float p0 = normed(p.x, b0 + 2 * j, 2 * j < n0), p1 = normed(p.y, b0 + 2 * j + 1, 2 * j + 1 < n0);
                    float q0 = normed(q.x, b1 + 2 * j, 2 * j < n1), q1 = normed(q.y, b1 + 2 * j + 1, 2 * j + 1 < n1);
                    if (turned) {
                        const float4 *cs = turn + token[n] * 4 * turns + u;
                        auto rotate = [](float &f, float &g, float cosine, float sine) {
                            const float t = f * cosine - g * sine;
                            g = f * sine + g * cosine;
                            f = t;
                        };
                        if (halves) {
                            if (2 * j < n0) {
                                const float4 c = cs[j * turns];
                                rotate(p0, q0, c.x, c.y);
                                if (2 * j + 1 < n0) rotate(p1, q1, c.z, c.w);
                            }
                        } else {
                            if (2 * j < n0) {
                                const float4 c = cs[(j >> 1) * turns];
                                rotate(p0, p1, j & 1 ? c.z : c.x, j & 1 ? c.w : c.y);
                            }
                            if (2 * j < n1) {
                                const float4 c = cs[(2 + (j >> 1)) * turns];
                                rotate(q0, q1, j & 1 ? c.z : c.x, j & 1 ? c.w : c.y);
                            }
                        }
                    }
                    x[n][j] = kv_pair(p0, p1, T());
                    y[n][j] = kv_pair(q0, q1, T());
                }
            }
            if (is_q || !Q4) {
                T *to = is_q ? (T *)a.q_out + (first + token[n]) * a.qo_tok + h * a.qo_head
                             : (T *)(slot + (is_v ? a.c.plane_stride : 0) + (long long)h * a.c.head_stride);
                kv_store_run<V>(to + (is_v ? v0 : b0), x[n], is_v ? vn0 : n0);
                kv_store_run<V>(to + (is_v ? v0 + 8 : b1), y[n], is_v ? vn1 : n1);
                continue;
            }
            if constexpr (Q4) {
                unsigned e[8], codes[2];
                if (!is_v) {                     // from pairs to neighbours
                    __syncwarp(mask);            // what an earlier key left is read
                    kv_store_run<V>(cross + b0, x[n], n0);
                    kv_store_run<V>(cross + b1, y[n], n1);
                    __syncwarp(mask);
                    if (vn0 > 0) kv_load_run<8>(x[n], cross + v0, 8);
                    if (vn1 > 0) kv_load_run<8>(y[n], cross + v0 + 8, 8);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    e[j] = x[n][j];
                    e[4 + j] = y[n][j];
                }
                const unsigned word = kv_quantise<T>(e, vn0 + vn1, mask, codes);
                const int G = a.c.groups, g = u >> 1;
                if (g >= G) continue;
                uint8_t *at = slot + (is_v ? a.c.plane_stride : 0) + (long long)h * a.c.head_stride;
                if (is_v) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) ((unsigned short *)at)[((u & 1) * 4 + k) * G + g] = (unsigned short)(codes[k >> 1] >> (16 * (k & 1)));
                } else {
#pragma unroll
                    for (int k = 0; k < 2; ++k) ((unsigned *)at)[((u & 1) * 2 + k) * G + g] = codes[k];
                }
                if ((u & 1) == 0) ((unsigned *)(at + to_words[token[n]]))[g] = word;
            }
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
