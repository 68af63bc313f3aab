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
    int splits, per_split;       // CTAs that share a token's rows (where there are few tokens), rows of each
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
        unsigned pair = 0;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const float d = ((e ? v.y : v.x) - lo) * lift, t = __fadd_rd(fmaf(d, inv, 0.5f), 0x1p23f);   // 2^23 + the code, rounded down
            const float left = fmaf(0x1p23f - t, s, d);
            int n = __float_as_int(t) - __float_as_int(0x1p23f);
            if (left >= border) ++n;
            if (left < -border) --n;
            pair |= (unsigned)min(max(n, 0), 15) << (4 * e);
        }
        codes[j >> 2] |= (2 * j < count ? pair : 0u) << (8 * (j & 3));
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

constexpr int AR_WEIGHTS = 256 + 16;         // elements of a head, at most, and those of the last run that are none

// Dynamic shared memory: [token][4][turns] float4 of cosine and sine of two frequencies each; packed caches further have
// [token][8][turns] double2 in front, and [row of the CTA][padded dim] elements behind
template <typename T, int V, bool Q4>
__global__ void __launch_bounds__(AP_THREADS, Q4 ? 3 : 4) kv_append_rows(const __grid_constant__ KvAppendRows b)
{
    const KvAppend &a = b.p;
    extern __shared__ __align__(16) uint8_t ar_smem[];
    __shared__ uint8_t *kv_row[AP_TOKENS];               // K of the token's slot, or nullptr
    __shared__ long long meta[AP_TOKENS];
    __shared__ int to_words[AP_TOKENS];
    __shared__ __align__(16) float weight[2][AR_WEIGHTS];
    __shared__ __align__(16) double k_weight[Q4 ? AR_WEIGHTS : 2];
    const int tid = threadIdx.x, dim = a.c.dim, half = a.rotary >> 1, heads = a.c.heads, q_heads = a.q ? a.q_heads : 0;
    const int split = b.splits > 1 ? blockIdx.x % b.splits : 0, row0 = split * b.per_split, rows = min(b.per_split, q_heads + 2 * heads - row0);
    const int L = 1 << b.lanes_log2, u = tid & (L - 1), mine = tid >> b.lanes_log2, lanes = AP_THREADS >> b.lanes_log2, turns = b.turns;
    const unsigned mask = (L == 32 ? ~0u : (1u << L) - 1) << (tid & 31 & ~(L - 1));      // the lanes of this row
    const bool halves = a.pairs_style == 0;
    double2 *wide = (double2 *)ar_smem;
    float4 *turn = (float4 *)(ar_smem + (Q4 ? a.per * 8 * turns * 16 : 0));
    T *cross = (T *)(ar_smem + a.per * turns * (Q4 ? 192 : 64)) + mine * a.c.groups * 32;

    // The two runs of the lane in a row of q or k, and in one of v.  What a run has beyond its elements is zero, is worked on like them and
    // goes nowhere
    const bool turned = u < turns;
    const int b0 = turned ? (halves ? 8 * u : 16 * u) : a.rotary + 16 * (u - turns), b1 = turned && halves ? half + 8 * u : b0 + 8;
    const int end0 = turned ? (halves ? half : a.rotary) : dim, end1 = turned ? a.rotary : dim;
    const int n0 = min(max(end0 - b0, 0), 8), n1 = min(max(end1 - b1, 0), 8);
    const int w0 = n0 ? b0 : 0, w1 = n1 ? b1 : 0;        // where their weights are
    const int v0 = 16 * u, vn0 = min(max(dim - v0, 0), 8), vn1 = min(max(dim - v0 - 8, 0), 8);

    const long long first = (long long)(blockIdx.x / b.splits) * a.per;
    const int tokens = (int)min((long long)a.per, a.num_tokens - first), total = tokens * rows;
    unsigned x[4], y[4], x1[4], y1[4];                   // of the row at hand, and of the next one
    int token1, row1;
    auto fetch = [&](int r) {
        row1 = -1;
        if (r >= total) return;
        token1 = b.splits > 1 ? 0 : (int)__umulhi((unsigned)r, a.by_rows);
        row1 = row0 + r - token1 * rows;
        const long long t = first + token1;
        const bool is_v = row1 >= q_heads + heads;
        const T *from = row1 < q_heads ? (const T *)a.q + t * a.q_tok + row1 * a.q_head
                        : is_v         ? (const T *)a.v + t * a.v_tok + (row1 - q_heads - heads) * a.v_head
                                       : (const T *)a.k + t * a.k_tok + (row1 - q_heads) * a.k_head;
        kv_load_run<V>(x1, from + (is_v ? v0 : b0), is_v ? vn0 : n0);
        kv_load_run<V>(y1, from + (is_v ? v0 + 8 : b1), is_v ? vn1 : n1);
    };
    fetch(mine);
    // weights that all heads share, angles and slots, while that is on its way
    const bool has_k = row0 + rows > q_heads && row0 < q_heads + heads;
    for (int d = tid; d < 2 * dim; d += AP_THREADS) {
        const int of_k = d >= dim, e = d - of_k * dim;
        const void *w = of_k ? b.k_w : b.q_w;
        if (w && (of_k ? b.k_w_head : b.q_w_head) == 0) {
            const float v = b.w_float ? ((const float *)w)[e] : kv_float(((const T *)w)[e]);
            if (Q4 && of_k) k_weight[e] = (double)v;
            else weight[of_k][e] = v;
        }
    }
    for (int f = tid; f < tokens * half; f += AP_THREADS) {
        const int k = f / half, q = f - k * half, lane = q >> 3, j = q & 7;
        const double cycles = (double)a.positions[a.axis_of[q] * a.axis_stride + first + k] * (double)a.inv_freq[q] * 0.15915494309189533577;
        const double turned_by = 2.0 * (cycles - rint(cycles));
        if (Q4 && has_k) {
            double2 z;
            sincospi(turned_by, &z.y, &z.x);
            wide[(k * 8 + j) * turns + lane] = z;
        }
        float2 cs;
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
    for (int r = mine; r < total; r += lanes) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x[j] = x1[j];
            y[j] = y1[j];
        }
        const int token = token1, row = row1;
        fetch(r + lanes);
        const bool is_q = row < q_heads, is_v = row >= q_heads + heads;
        const int h = row - (is_q ? 0 : is_v ? q_heads + heads : q_heads);
        uint8_t *slot = kv_row[token];
        if (!is_q && !slot) continue;            // all lanes of the row
        if (Q4 && !is_q && !is_v) {              // a key in float64
            double rn = 1.0;
            if (b.k_w) {
                double sum = 0.0, sum2 = 0.0;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 f = kv_unpair(x[j], T()), g = kv_unpair(y[j], T());
                    const double f0 = f.x, f1 = f.y, g0 = g.x, g1 = g.y;
                    sum = fma(f0, f0, sum);
                    sum2 = fma(f1, f1, sum2);
                    sum = fma(g0, g0, sum);
                    sum2 = fma(g1, g1, sum2);
                }
                sum += sum2;
                for (int o = L >> 1; o; o >>= 1) sum += __shfl_xor_sync(mask, sum, o);
                rn = 1.0 / sqrt(sum / dim + (double)b.eps);
            }
            const double2 *cs = wide + token * 8 * turns + u;
            const bool own = b.k_w && b.k_w_head != 0;
            auto weigh = [&](float v, int e) {   // elements of the last run that are none have any weight
                if (!b.k_w) return (double)v;
                const double w = !own ? k_weight[e] : e >= dim ? 0.0 : b.w_float ? (double)((const float *)b.k_w)[h * b.k_w_head + e] : (double)kv_float(((const T *)b.k_w)[h * b.k_w_head + e]);
                return (double)v * rn * w;
            };
            auto rotate = [](double &f, double &g, double2 c) {
                const double t = f * c.x - g * c.y;
                g = f * c.y + g * c.x;
                f = t;
            };
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 f = kv_unpair(x[j], T()), g = kv_unpair(y[j], T());
                double f0 = weigh(f.x, w0 + 2 * j), f1 = weigh(f.y, w0 + 2 * j + 1), g0 = weigh(g.x, w1 + 2 * j), g1 = weigh(g.y, w1 + 2 * j + 1);
                if (turned) {
                    if (halves) {
                        rotate(f0, g0, cs[2 * j * turns]);
                        rotate(f1, g1, cs[(2 * j + 1) * turns]);
                    } else {
                        rotate(f0, f1, cs[j * turns]);
                        rotate(g0, g1, cs[(4 + j) * turns]);
                    }
                }
                x[j] = kv_pair((float)f0, (float)f1, T());
                y[j] = kv_pair((float)g0, (float)g1, T());
            }
        } else if (!is_v) {
            float f[8], g[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 p = kv_unpair(x[j], T()), q = kv_unpair(y[j], T());
                f[2 * j] = p.x, f[2 * j + 1] = p.y, g[2 * j] = q.x, g[2 * j + 1] = q.y;
            }
            const void *wp = is_q ? b.q_w : b.k_w;
            if (wp) {
                float sum = 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) sum = fmaf(f[j], f[j], fmaf(g[j], g[j], sum));
                for (int o = L >> 1; o; o >>= 1) sum += __shfl_xor_sync(mask, sum, o);
                const float rn = rsqrtf(sum / dim + b.eps);
                const long long w_head = is_q ? b.q_w_head : b.k_w_head;
                float w[8], z[8];
                if (w_head == 0) {
                    const float *ws = weight[is_q ? 0 : 1];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {        // runs of pairs begin anywhere
                        w[j] = ws[w0 + j];
                        z[j] = ws[w1 + j];
                    }
                } else
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const long long e = h * w_head + b0 + j, e2 = h * w_head + b1 + j;
                        w[j] = j >= n0 ? 0.f : b.w_float ? ((const float *)wp)[e] : kv_float(((const T *)wp)[e]);
                        z[j] = j >= n1 ? 0.f : b.w_float ? ((const float *)wp)[e2] : kv_float(((const T *)wp)[e2]);
                    }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    f[j] *= rn * w[j];
                    g[j] *= rn * z[j];
                }
            }
            if (turned) {
                const float4 *cs = turn + token * 4 * turns + u;
                auto rotate = [](float &p, float &q, float cosine, float sine) {
                    const float t = p * cosine - q * sine;
                    q = p * sine + q * cosine;
                    p = t;
                };
#pragma unroll
                for (int j = 0; j < 4; ++j) {            // two frequencies
                    const float4 c = cs[j * turns];
                    if (halves) {
                        rotate(f[2 * j], g[2 * j], c.x, c.y);
                        rotate(f[2 * j + 1], g[2 * j + 1], c.z, c.w);
                    } else if (j < 2) {
                        rotate(f[4 * j], f[4 * j + 1], c.x, c.y);
                        rotate(f[4 * j + 2], f[4 * j + 3], c.z, c.w);
                    } else {
                        rotate(g[4 * j - 8], g[4 * j - 7], c.x, c.y);
                        rotate(g[4 * j - 6], g[4 * j - 5], c.z, c.w);
                    }
                }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                x[j] = kv_pair(f[2 * j], f[2 * j + 1], T());
                y[j] = kv_pair(g[2 * j], g[2 * j + 1], T());
            }
        }
        if (is_q || !Q4) {
            T *to = is_q ? (T *)a.q_out + (first + token) * a.qo_tok + h * a.qo_head
                         : (T *)(slot + (is_v ? a.c.plane_stride : 0) + (long long)h * a.c.head_stride);
            kv_store_run<V>(to + (is_v ? v0 : b0), x, is_v ? vn0 : n0);
            kv_store_run<V>(to + (is_v ? v0 + 8 : b1), y, is_v ? vn1 : n1);
            continue;
        }
        if constexpr (Q4) {
            unsigned e[8], codes[2];
            if (!is_v) {                         // from pairs to neighbours
                __syncwarp(mask);                // what an earlier key left is read
                kv_store_run<V>(cross + b0, x, n0);
                kv_store_run<V>(cross + b1, y, n1);
                __syncwarp(mask);
                if (vn0 > 0) kv_load_run<8>(x, cross + v0, 8);
                if (vn1 > 0) kv_load_run<8>(y, cross + v0 + 8, 8);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                e[j] = x[j];
                e[4 + j] = y[j];
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
            if ((u & 1) == 0) ((unsigned *)(at + to_words[token]))[g] = word;
        }
    }
    if ((a.weights || a.order) && split == 0)
        for (int e = tid; e < tokens * heads; e += AP_THREADS) {
            const int k = e / heads, h = e - k * heads;
            if (!kv_row[k]) continue;
            if (a.weights) a.weights[meta[k] + h * a.m_head] = 0.f;
            if (a.order) a.order[meta[k] + h * a.m_head] = a.token_order ? a.token_order[first + k] : a.positions[first + k];
        }
}
