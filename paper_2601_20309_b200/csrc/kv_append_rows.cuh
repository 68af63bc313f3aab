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
// and rotation of keys run in float64 there (half of float32's rate, 8 of 48 rows), and the border itself is decided exactly: n
// comes from a reciprocal that is a little too small, so it is never too large; the remainder d - n s is exact in one fused operation, and
// where it reaches s/2 the code is one more.
//
// Split.  A row belongs to 2^k lanes of a warp, 16 elements each in two runs of eight: what turns together where halves turn, neighbours
// elsewhere.  Sums over a row are shuffles among its lanes.  A warp has rows of q, of k or of v, never of two of them, so that it stays
// together; a task is a group of its rows for a run of tokens, so that pointers, weights and kind are found once for all of them; the
// next token's row is on its way while one is worked on.  A key to be packed crosses shared memory once, from its pairs to neighbours, since
// groups are neighbours.  Angles and slots as in kv_append_tokens: once per token, behind the first loads.
//
// What bounds it.  Norms into 16 bits: 353 MB of 14.3k prompt tokens in 74.6 us, 4.7 TB/s, 73 % of the copy peak (the same without norms in
// kv_append_tokens 65 us): 225 instructions per four rows, half of the issue slots; with rows taken one by one 428 and 100 us.  Into
// 4 bits about 110 us: 355 instructions per four rows, of which keys (float64 and codes) and values take two thirds.
// 64 tokens 5.1 us: one launch and the chain of loads.
#pragma once
#include "kv_append.cuh"

struct KvAppendRows {
    KvAppend p;
    const void *q_w, *k_w;       // weights of the norms, nullptr: none
    long long q_w_head, k_w_head;    // from a head's weights to the next's, 0: the same for all
    int w_float;                 // weights are float32, else of the cache's type
    float eps, by_dim;           // by_dim: 1 / head_dim
    int chunk;                   // tokens of a task: rows of some heads for so many tokens in turn
    int lanes_log2;              // lanes of a row
    int turns;                   // lanes that hold what turns
    int splits, per_split;       // CTAs that share a token's groups of rows (where there are few tokens), groups of each
    unsigned by_groups;          // 2^32 / groups of a CTA, rounded up
};

// a word of a group that is not finite
template <typename T> __device__ __forceinline__ unsigned kv_nan_word();
template <> __device__ __forceinline__ unsigned kv_nan_word<__nv_bfloat16>() { return 0x7fc07fc0u; }
template <> __device__ __forceinline__ unsigned kv_nan_word<__half>() { return 0x7fc07e00u; }

// minimum and maximum of pairs, NaN where one is
__device__ __forceinline__ unsigned kv_min2(unsigned a, unsigned b, __nv_bfloat16)
{
    const __nv_bfloat162 v = __hmin2_nan(*(const __nv_bfloat162 *)&a, *(const __nv_bfloat162 *)&b);
    return *(const unsigned *)&v;
}
__device__ __forceinline__ unsigned kv_min2(unsigned a, unsigned b, __half)
{
    const __half2 v = __hmin2_nan(*(const __half2 *)&a, *(const __half2 *)&b);
    return *(const unsigned *)&v;
}
__device__ __forceinline__ unsigned kv_max2(unsigned a, unsigned b, __nv_bfloat16)
{
    const __nv_bfloat162 v = __hmax2_nan(*(const __nv_bfloat162 *)&a, *(const __nv_bfloat162 *)&b);
    return *(const unsigned *)&v;
}
__device__ __forceinline__ unsigned kv_max2(unsigned a, unsigned b, __half)
{
    const __half2 v = __hmax2_nan(*(const __half2 *)&a, *(const __half2 *)&b);
    return *(const unsigned *)&v;
}

// Word and codes of 16 elements (as pairs), half of a group whose other half the neighbouring lane has; `count` of them exist, 0, 8 or 16.
// The codes come as 4 bits each, in order.  By a whole warp.
template <typename T> __device__ __forceinline__ unsigned kv_quantise(const unsigned (&x)[8], int count, unsigned (&codes)[2])
{
    // lowest and highest of the pairs, of the lane, of both lanes; they travel as a pair
    unsigned lo2 = kv_pair(INFINITY, INFINITY, T()), hi2 = lo2 | 0x80008000u;
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (8 * (j / 4) < count) {
            lo2 = kv_min2(lo2, x[j], T());
            hi2 = kv_max2(hi2, x[j], T());
        }
    unsigned low = kv_min2(lo2, lo2 >> 16, T()) & 0xffffu, high = kv_max2(hi2, hi2 >> 16, T()) & 0xffffu;
    const unsigned there = __shfl_xor_sync(~0u, low | high << 16, 1);
    low = kv_min2(low, there, T()) & 0xffffu;
    high = kv_max2(high, there >> 16, T()) & 0xffffu;
    const float lo = kv_unpair(low, T()).x, hi = kv_unpair(high, T()).x, range = hi - lo;
    codes[0] = codes[1] = 0;
    if (range == -INFINITY) return 0;                    // a group of nothing
    const __nv_bfloat16 rounded = __float2bfloat16(fmaxf(range * (1.f / 15.f), fabsf(lo) * 0x1p-20f));
    float s = __bfloat162float(rounded);
    if (!(range < INFINITY) || !(fabsf(lo) < INFINITY) || !(s < INFINITY)) return kv_nan_word<T>();
    const unsigned word = low | (unsigned)__bfloat16_as_ushort(rounded) << 16;
    if (s == 0.f) return word;
    if (s >= 0x1p-100f) {
        // 2^23 + d / s, rounded to the nearest, or the one below where it is near the middle: the reciprocal is a little too small, never too
        // large.  No code is above 15: s is at least the range / 15 less 2^-8 of it
        const float inv = 1.f / s * (1.f - 0x1p-21f), border = 0.5f * s;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float2 v = kv_unpair(x[j], T());
            if (8 * (j / 4) >= count) continue;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float d = (e ? v.y : v.x) - lo, t = fmaf(d, inv, 0x1p23f), left = fmaf(0x1p23f - t, s, d);
                const int at = 4 * (2 * (j & 3) + e);
                codes[j >> 2] += (__float_as_uint(t) - __float_as_uint(0x1p23f)) << at;
                if (left >= border) codes[j >> 2] += 1u << at;
            }
        }
        return word;
    }
    // a step whose reciprocal may not be a number, or that is far from a 15th of the range itself
    s *= 0x1p60f;
#pragma unroll 1
    for (int j = 0; j < count; ++j) {
        const float2 v = kv_unpair(j < 2 ? x[0] : j < 4 ? x[1] : j < 6 ? x[2] : j < 8 ? x[3] : j < 10 ? x[4] : j < 12 ? x[5] : j < 14 ? x[6] : x[7], T());
        const float d = ((j & 1 ? v.y : v.x) - lo) * 0x1p60f;
        int n = (int)fminf(floorf(d / s), 16.f);
        if (fmaf((float)-n, s, d) >= 0.5f * s) ++n;
        codes[j >> 3] |= (unsigned)min(n, 15) << (4 * (j & 7));
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
// LG: 0, or the rows are whole: 2^LG lanes with 16 elements each, aligned
template <typename T, int V, bool Q4, int LG>
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
    // A row has L lanes; a warp has rows of q, of k or of v, never of two of them
    constexpr bool WHOLE = LG > 0;
    const int log2 = WHOLE ? LG : b.lanes_log2, L = 1 << log2, u = tid & (L - 1), turns = b.turns, abreast = 32 >> log2, mine = (tid & 31) >> log2;
    const int q_groups = (q_heads + abreast - 1) >> (5 - log2), kv_groups = (heads + abreast - 1) >> (5 - log2);
    const int split = b.splits > 1 ? blockIdx.x % b.splits : 0, group0 = split * b.per_split, groups = min(b.per_split, q_groups + 2 * kv_groups - group0);
    const bool halves = a.pairs_style == 0;
    double2 *wide = (double2 *)ar_smem;
    float4 *turn = (float4 *)(ar_smem + (Q4 ? a.per * 8 * turns * 16 : 0));
    T *cross = (T *)(ar_smem + a.per * turns * (Q4 ? 192 : 64)) + (tid >> log2) * a.c.groups * 32;

    // The two runs of the lane in a row of q or k, and in one of v.  What a run has beyond its elements is zero, is worked on like them and
    // goes nowhere
    const bool turned = u < turns;
    const int b0 = turned ? (halves ? 8 * u : 16 * u) : a.rotary + 16 * (u - turns), b1 = turned && halves ? half + 8 * u : b0 + 8;
    const int end0 = turned ? (halves ? half : a.rotary) : dim, end1 = turned ? a.rotary : dim;
    const int n0 = WHOLE ? 8 : min(max(end0 - b0, 0), 8), n1 = WHOLE ? 8 : min(max(end1 - b1, 0), 8);
    const int w0 = n0 ? b0 : 0, w1 = n1 ? b1 : 0;        // where their weights are
    const int v0 = 16 * u, vn0 = WHOLE ? 8 : min(max(dim - v0, 0), 8), vn1 = WHOLE ? 8 : min(max(dim - v0 - 8, 0), 8);

    const long long first = (long long)(b.splits > 1 ? blockIdx.x / b.splits : blockIdx.x) * a.per;
    const int tokens = (int)min((long long)a.per, a.num_tokens - first);
    // A task is a group of rows for a run of tokens: pointers, weights and what is to be done stay the same for all of them
    const int warp = tid >> 5, chunks = (tokens + b.chunk - 1) / b.chunk, tasks = groups * chunks;
    unsigned x[4], y[4], x1[4] = {}, y1[4] = {};         // of the token at hand, and of the next one
    const T *from = nullptr;
    long long step = 0;
    int h = 0, t0 = 0, t1 = 0, c0 = 0, c1 = 0, to_second = 0;    // c0, c1: elements of the lane's runs (0: there is no such head)
    bool is_q = false, is_v = false;
    auto fetch = [&]() {
        kv_load_run<V>(x1, from, WHOLE ? 8 : c0);
        kv_load_run<V>(y1, from + to_second, WHOLE ? 8 : c1);
        from += step;
    };
    auto begin = [&](int task) {
        const int chunk = chunks == 1 ? 0 : (int)__umulhi((unsigned)task, b.by_groups), group = group0 + task - chunk * groups;
        t0 = chunk * b.chunk;
        t1 = min(t0 + b.chunk, tokens);
        is_q = group < q_groups;
        is_v = group >= q_groups + kv_groups;
        h = (group - (is_q ? 0 : is_v ? q_groups + kv_groups : q_groups)) * abreast + mine;
        const bool on = h < (is_q ? q_heads : heads);
        c0 = on ? is_v ? vn0 : n0 : 0;
        c1 = on ? is_v ? vn1 : n1 : 0;
        step = is_q ? a.q_tok : is_v ? a.v_tok : a.k_tok;
        to_second = is_v ? 8 : b1 - b0;
        const int there = WHOLE ? min(h, (is_q ? q_heads : heads) - 1) : h;      // of whole rows some head is read in any case
        from = (const T *)(is_q ? a.q : is_v ? a.v : a.k) + (first + t0) * step + there * (is_q ? a.q_head : is_v ? a.v_head : a.k_head) + (is_v ? v0 : b0);
        fetch();
    };
    auto next = [&](int t) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x[j] = x1[j];
            y[j] = y1[j];
        }
        if (t + 1 < t1) fetch();
    };
    if (warp < tasks) begin(warp);
    // weights that all heads share, angles and slots, while that is on its way
    const bool has_k = group0 + groups > q_groups && group0 < q_groups + kv_groups;
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
        float2 cs;
        if (Q4 && has_k) {
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
    auto sum_of_row = [&](auto v) {
#pragma unroll
        for (int o = 1; o < 32; o <<= 1)
            if (o < (WHOLE ? 1 << LG : L)) v += __shfl_xor_sync(~0u, v, o);
        return v;
    };
    for (int task = warp; task < tasks; task += AP_THREADS / 32) {
        if (task != warp) begin(task);
        if (is_q || (!is_v && !Q4)) {            // norm and rotation in float32
            const void *wp = is_q ? b.q_w : b.k_w;
            const long long w_head = is_q ? b.q_w_head : b.k_w_head;
            float w[8], z[8];
            if (wp && w_head == 0) {
                const float *ws = weight[is_q ? 0 : 1];
#pragma unroll
                for (int j = 0; j < 8; j += V == 8 ? 4 : 1)
                    if constexpr (V == 8) {
                        const float4 p = *(const float4 *)(ws + w0 + j), q = *(const float4 *)(ws + w1 + j);
                        w[j] = p.x, w[j + 1] = p.y, w[j + 2] = p.z, w[j + 3] = p.w;
                        z[j] = q.x, z[j + 1] = q.y, z[j + 2] = q.z, z[j + 3] = q.w;
                    } else {                     // runs of pairs begin anywhere
                        w[j] = ws[w0 + j];
                        z[j] = ws[w1 + j];
                    }
            } else if (wp)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const long long e = h * w_head + b0 + j, e2 = h * w_head + b1 + j;
                    w[j] = j >= c0 ? 0.f : b.w_float ? ((const float *)wp)[e] : kv_float(((const T *)wp)[e]);
                    z[j] = j >= c1 ? 0.f : b.w_float ? ((const float *)wp)[e2] : kv_float(((const T *)wp)[e2]);
                }
            const float4 *cs = turn + t0 * 4 * turns + u;
            T *out = is_q ? (T *)a.q_out + (first + t0) * a.qo_tok + h * a.qo_head + b0 : nullptr;
            for (int t = t0; t < t1; ++t, cs += 4 * turns) {
                float f[8], g[8];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 p = kv_unpair(x1[j], T()), q = kv_unpair(y1[j], T());
                    f[2 * j] = p.x, f[2 * j + 1] = p.y, g[2 * j] = q.x, g[2 * j + 1] = q.y;
                }
                if (t + 1 < t1) fetch();
                if (wp) {
                    float sum = 0.f;
#pragma unroll
                    for (int j = 0; j < 8; ++j) sum = fmaf(f[j], f[j], fmaf(g[j], g[j], sum));
                    const float rn = rsqrtf(fmaf(sum_of_row(sum), b.by_dim, b.eps));
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        f[j] *= rn * w[j];
                        g[j] *= rn * z[j];
                    }
                }
                if (turned) {
                    auto rotate = [](float &p, float &q, float cosine, float sine) {
                        const float r = p * cosine - q * sine;
                        q = p * sine + q * cosine;
                        p = r;
                    };
                    if (halves)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {    // two frequencies
                            const float4 c = cs[j * turns];
                            rotate(f[2 * j], g[2 * j], c.x, c.y);
                            rotate(f[2 * j + 1], g[2 * j + 1], c.z, c.w);
                        }
                    else
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const float4 c = cs[j * turns], d = cs[(2 + j) * turns];
                            rotate(f[4 * j], f[4 * j + 1], c.x, c.y);
                            rotate(f[4 * j + 2], f[4 * j + 3], c.z, c.w);
                            rotate(g[4 * j], g[4 * j + 1], d.x, d.y);
                            rotate(g[4 * j + 2], g[4 * j + 3], d.z, d.w);
                        }
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    x[j] = kv_pair(f[2 * j], f[2 * j + 1], T());
                    y[j] = kv_pair(g[2 * j], g[2 * j + 1], T());
                }
                T *to = out;
                if (is_q) out += a.qo_tok;
                else {
                    if (!kv_row[t]) continue;
                    to = (T *)(kv_row[t] + (long long)h * a.c.head_stride) + b0;
                }
                if (WHOLE && c0 == 0) continue;
                kv_store_run<V>(to, x, WHOLE ? 8 : c0);
                kv_store_run<V>(to + to_second, y, WHOLE ? 8 : c1);
            }
            continue;
        }
        const double2 *cs = wide + t0 * 8 * turns + u;
        for (int t = t0; t < t1; ++t, cs += 8 * turns) {
            next(t);
            uint8_t *slot = kv_row[t];
            if (!slot) continue;                 // all lanes
            if (!Q4) {                           // a row of v as it is
                T *to = (T *)(slot + a.c.plane_stride + (long long)h * a.c.head_stride);
                kv_store_run<V>(to + v0, x, c0);
                kv_store_run<V>(to + v0 + 8, y, c1);
                continue;
            }
            if constexpr (Q4) {
                if (!is_v) {                     // a key in float64
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
                        rn = 1.0 / sqrt(sum_of_row(sum + sum2) / dim + (double)b.eps);
                    }
                    auto rotate = [](double &f, double &g, double2 c) {
                        const double r = f * c.x - g * c.y;
                        g = f * c.y + g * c.x;
                        f = r;
                    };
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float2 f = kv_unpair(x[j], T()), g = kv_unpair(y[j], T());
                        double f0 = f.x, f1 = f.y, g0 = g.x, g1 = g.y;
                        if (b.k_w) {             // elements of the last run that are none have any weight
                            if (WHOLE && b.k_w_head == 0) {
                                const double2 p = *(const double2 *)(k_weight + w0 + 2 * j), q = *(const double2 *)(k_weight + w1 + 2 * j);
                                f0 *= rn * p.x;
                                f1 *= rn * p.y;
                                g0 *= rn * q.x;
                                g1 *= rn * q.y;
                            } else if (b.k_w_head == 0) {
                                f0 *= rn * k_weight[w0 + 2 * j];
                                f1 *= rn * k_weight[w0 + 2 * j + 1];
                                g0 *= rn * k_weight[w1 + 2 * j];
                                g1 *= rn * k_weight[w1 + 2 * j + 1];
                            } else {
                                auto own = [&](int e) {
                                    if (e >= dim || h >= heads) return 0.0;
                                    return rn * (b.w_float ? (double)((const float *)b.k_w)[h * b.k_w_head + e] : (double)kv_float(((const T *)b.k_w)[h * b.k_w_head + e]));
                                };
                                f0 *= own(w0 + 2 * j);
                                f1 *= own(w0 + 2 * j + 1);
                                g0 *= own(w1 + 2 * j);
                                g1 *= own(w1 + 2 * j + 1);
                            }
                        }
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
                    // from pairs to neighbours
                    __syncwarp();                // what an earlier key left is read
                    kv_store_run<V>(cross + b0, x, n0);
                    kv_store_run<V>(cross + b1, y, n1);
                    __syncwarp();
                    if (vn0 > 0) kv_load_run<8>(x, cross + v0, 8);
                    if (vn1 > 0) kv_load_run<8>(y, cross + v0 + 8, 8);
                }
                unsigned e[8], codes[2];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    e[j] = x[j];
                    e[4 + j] = y[j];
                }
                const unsigned word = kv_quantise<T>(e, vn0 + vn1, codes);
                const int G = a.c.groups, g = u >> 1;
                if (g >= G || h >= heads) continue;
                uint8_t *at = slot + (is_v ? a.c.plane_stride : 0) + (long long)h * a.c.head_stride;
                if (is_v) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) ((unsigned short *)at)[((u & 1) * 4 + k) * G + g] = (unsigned short)(codes[k >> 1] >> (16 * (k & 1)));
                } else {
#pragma unroll
                    for (int k = 0; k < 2; ++k) ((unsigned *)at)[((u & 1) * 2 + k) * G + g] = codes[k];
                }
                if ((u & 1) == 0) ((unsigned *)(at + to_words[t]))[g] = word;
            }
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
