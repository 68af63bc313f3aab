// Attention of one new token per sequence over the paged cache: kv_attend_stream reads the cache once, kv_attend_join
// joins the pieces of sequences that were split and adds up the weights.
//
// What bounds it: the bytes of K and V.  A slot of one KV head is 4*dim bytes against 4*dim*group operations, so even
// with 16 query heads to a KV head the tensor pipe idles; what matters is that every SM has loads in flight all the time.
//
// Split.  A *row* is (sequence, chunk of `hc` KV heads, chunk of up to 8*NT query heads of each); it is walked in *steps* of
// 16 * tw slots.  All steps of all rows form one line, cut into equal contiguous pieces, one per CTA: lengths may be as
// unequal as they like, every CTA gets the same number of steps, and no plan is made on the host, which does not know
// the lengths.  A piece that covers a whole row writes its output; the at most two pieces of a CTA that do not are left in
// the workspace (running maximum, sum, output sums) for kv_attend_join, which adds them in the order of the slots.
//
// Inside a CTA every warp is on its own: warp = (way, KV head of the chunk), a tile is 16 slots of one head.  It fills its
// own ring of shared-memory stages with cp.async (each row of a tile may lie in another block: the block ids are read one
// tile ahead) and computes from it, so warps never wait for one another except at the end of a row that several ways share.
//
// Mathematics of a tile, on mma.m16n8k16 with the cache as the left operand, so that the few query heads fill the narrow
// side:  S^T[16 slots, 8 heads] = K Q^T;  m, p = exp2(S - m), l in float32 (scale and log2 e are applied to the sums);
// O^T[dim, 8 heads] = alpha O^T + V^T P^T, V^T by transposing ldmatrix, P^T by movmatrix from the score fragment.  P is
// rounded to the cache's type, the only rounding besides the output's; l sums the unrounded p.
// Masked slots (beyond the length, before the window, in a bad block) are never loaded: their K and V are zero-filled, so
// whatever the block holds there cannot reach a sum, and their score is -inf.
#pragma once
#include "kv_ops.cuh"

struct KvAttend {
    KvView c;
    int layer, seqs, q_heads, group, window;
    float scale2;        // scale * log2 e
    const void *q;
    long long q_seq, q_head;
    void *out;
    long long o_seq, o_head;
    float *lse;
    const float *w_in;
    float *w_out;
    long long w_seq, w_head;
    int hc, tw;          // KV heads and ways of a CTA: hc * tw warps
    int head_chunks, group_chunks;
    int stages;
    int pieces;          // CTAs the line of steps is cut for; 0: every row is one CTA's (no join)
    int min_steps;       // no piece is shorter
    int q_pairs;         // q may be read in pairs of elements
    float *scores;       // [seq][kv_head][max_len][group], base 2; nullptr: no weights wanted
    float *row_lse;      // [seq][q_head], base 2
    float2 *part_ml;     // [piece][2][hc][8*NT]: maximum and sum
    float *part_o;       // [piece][2][hc][8*NT][dim]
};

constexpr int KV_ATTEND_WARPS = 8, KV_ATTEND_STAGES = 6;
constexpr float KV_LN2 = 0.69314718055994530942f;

__device__ __forceinline__ float kv_exp2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// what is subtracted from scores before the exponential: a row of nothing but -inf must not become NaN
__device__ __forceinline__ float kv_ref(float m) { return m == -INFINITY ? 0.f : m; }

template <typename T> struct KvMma;
template <> struct KvMma<__nv_bfloat16> {
    static __device__ __forceinline__ void mma(float (&c)[4], const unsigned (&a)[4], unsigned b0, unsigned b1)
    {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    }
    static __device__ __forceinline__ unsigned pack(float lo, float hi)
    {
        const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
        return *(const unsigned *)&v;
    }
};
template <> struct KvMma<__half> {
    static __device__ __forceinline__ void mma(float (&c)[4], const unsigned (&a)[4], unsigned b0, unsigned b1)
    {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    }
    static __device__ __forceinline__ unsigned pack(float lo, float hi)
    {
        const __half2 v = __floats2half2_rn(lo, hi);
        return *(const unsigned *)&v;
    }
};

__device__ __forceinline__ void kv_ldmatrix(unsigned (&r)[4], unsigned addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void kv_ldmatrix_t(unsigned (&r)[4], unsigned addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ unsigned kv_movmatrix_t(unsigned x)
{
    unsigned y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
// 16 bytes to shared memory, or zeros
__device__ __forceinline__ void kv_cp16(unsigned dst, const void *src, bool live)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(live ? 16 : 0) : "memory");
}

// a sequence's slots that count: [first, n), walked from `base` = first rounded down to a tile
struct KvSpan {
    int n, first, base;
    __device__ __forceinline__ KvSpan(const KvAttend &a, int i)
    {
        n = a.c.len(i);
        first = a.window > 0 && n > a.window ? n - a.window : 0;
        base = first & ~15;
    }
    __device__ __forceinline__ int steps(const KvAttend &a) const { return (n - base + 16 * a.tw - 1) / (16 * a.tw); }
};

// Sums the steps of one row over the sequences in front of `upto` and over all of them (every thread gets both).
// Block-wide; `red` holds two values per warp.
__device__ __forceinline__ void kv_attend_sums(const KvAttend &a, int upto, long long *red, long long &before, long long &all)
{
    long long b = 0, s = 0;
    for (int i = threadIdx.x; i < a.seqs; i += blockDim.x) {
        const int k = KvSpan(a, i).steps(a);
        s += k;
        if (i < upto) b += k;
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        s += __shfl_xor_sync(~0u, s, o);
        b += __shfl_xor_sync(~0u, b, o);
    }
    const int warps = blockDim.x >> 5;
    if ((threadIdx.x & 31) == 0) {
        red[threadIdx.x >> 5] = s;
        red[warps + (threadIdx.x >> 5)] = b;
    }
    __syncthreads();
    before = all = 0;
    for (int w = 0; w < warps; ++w) {
        all += red[w];
        before += red[warps + w];
    }
    __syncthreads();
}

__device__ __forceinline__ long long kv_attend_piece(const KvAttend &a, long long total)
{
    const long long q = (total + a.pieces - 1) / a.pieces;
    return q > a.min_steps ? q : a.min_steps;
}

template <typename T, int DP, int NT>
__global__ void __launch_bounds__(KV_ATTEND_WARPS * 32) kv_attend_stream(const __grid_constant__ KvAttend a)
{
    constexpr int ROW = DP * 2, TILE = 16 * ROW, KS = DP / 16, LANES = DP / 8, PASS = 32 / LANES, HEADS = 8 * NT;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ long long red[2 * KV_ATTEND_WARPS];
    __shared__ long long s_at[2];
    __shared__ int4 info[KV_ATTEND_WARPS][KV_ATTEND_STAGES];
    __shared__ float s_lse[KV_ATTEND_WARPS][HEADS];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, warps = blockDim.x >> 5;
    const int hw = warp % a.hc, way = warp / a.hc;
    const int rows_of_seq = a.head_chunks * a.group_chunks;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    // sequences without slots
    for (int i = blockIdx.x; i < a.seqs; i += gridDim.x)
        if (a.c.len(i) == 0) {
            for (int e = tid; e < a.q_heads * a.c.dim; e += blockDim.x)
                ((T *)a.out)[i * a.o_seq + e / a.c.dim * a.o_head + e % a.c.dim] = kv_round<T>(0.f);
            if (a.lse)
                for (int g = tid; g < a.q_heads; g += blockDim.x) a.lse[(long long)i * a.q_heads + g] = -INFINITY;
        }

    // ---- this CTA's piece of the line of steps: the row and step it begins at, and how many steps it has
    int pi, pch, pk;                 // sequence, row of the sequence, step: where the next tile to be loaded lies
    long long todo;
    if (a.pieces == 0) {
        pi = blockIdx.x / rows_of_seq;
        pch = blockIdx.x % rows_of_seq;
        pk = 0;
        todo = KvSpan(a, pi).steps(a);
    } else {
        // every thread sums a run of sequences; the one whose run holds the piece's first step walks it
        const int run = (a.seqs + blockDim.x - 1) / blockDim.x, lo = min(tid * run, a.seqs), hi = min(lo + run, a.seqs);
        long long mine = 0;
        for (int i = lo; i < hi; ++i) mine += KvSpan(a, i).steps(a);
        long long x = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long y = __shfl_up_sync(~0u, x, o);
            if (lane >= o) x += y;
        }
        if (lane == 31) red[warp] = x;
        __syncthreads();
        long long before = 0, total = 0;
        for (int w = 0; w < warps; ++w) {
            if (w < warp) before += red[w];
            total += red[w];
        }
        before = (before + x - mine) * rows_of_seq;
        total *= rows_of_seq;
        const long long piece = kv_attend_piece(a, total), s0 = blockIdx.x * piece;
        todo = min(total, s0 + piece) - s0;
        if (todo <= 0) return;
        if (s0 >= before && s0 < before + mine * rows_of_seq) {
            int i = lo;
            long long left = s0 - before;
            for (; i < hi; ++i) {
                const long long k = (long long)KvSpan(a, i).steps(a) * rows_of_seq;
                if (left < k) break;
                left -= k;
            }
            s_at[0] = i;
            s_at[1] = left;
        }
        __syncthreads();
        pi = (int)s_at[0];
        const int k = KvSpan(a, pi).steps(a);
        pch = (int)(s_at[1] / k);
        pk = (int)(s_at[1] % k);
    }
    if (todo <= 0) return;

    const unsigned ring = (unsigned)__cvta_generic_to_shared(smem) + warp * a.stages * 2 * TILE;
    const uint8_t *kbase = a.c.base + (long long)a.layer * 2 * a.c.plane_stride;
    int4 *my_info = info[warp];

    // ---- producer: the next tile's position, its block ids (lane r holds row r's) and what the consumer has to know
    long long left = todo;
    int psteps, id = -1, off = 0, t0 = 0, flags = 0, ti = 0, tch = 0;
    bool live = false;
    KvSpan span(a, pi);
    psteps = span.steps(a);
    bool fresh = true;               // the tile begins a run of this CTA in its row
    auto peek = [&]() {
        if (left <= 0) return;
        const int h = pch / a.group_chunks * a.hc + hw;
        t0 = span.base + (pk * a.tw + way) * 16;
        const int t = t0 + (lane & 15);
        live = t >= span.first && t < span.n;
        id = -1;
        off = h * a.c.head_stride;
        if (live) {
            id = a.c.tables[pi * a.c.table_stride + t / a.c.bs];
            off += t % a.c.bs * a.c.row_stride;
        }
        ti = pi;
        tch = pch;
        flags = (fresh ? 1 << 16 : 0) | (pk == 0 ? 1 << 18 : 0) | (pk == psteps - 1 ? 1 << 19 : 0);
        fresh = false;
        --left;
        if (left == 0 || pk == psteps - 1) flags |= 1 << 17;
        if (++pk == psteps) {
            pk = 0;
            fresh = true;
            if (++pch == rows_of_seq) {
                pch = 0;
                if (left > 0) {
                    do span = KvSpan(a, ++pi);
                    while (span.n == 0);
                    psteps = span.steps(a);
                }
            }
        }
    };
    long long unissued = todo;
    int put = 0;
    auto issue = [&]() {
        if (unissued > 0) {
            --unissued;
            const bool ok = live && (unsigned)id < (unsigned)a.c.nb;
            if (live && !ok) atomicOr(a.c.status, KV_OPS_BAD_BLOCK);
            const unsigned mask = __ballot_sync(~0u, ok) & 0xffffu;
            if (lane == 0) my_info[put] = make_int4((int)mask | flags, t0, ti, tch);
            const unsigned stage = ring + put * 2 * TILE;
            const int chunk = lane % LANES;
#pragma unroll
            for (int j = 0; j < 16 / PASS; ++j) {
                const int r = j * PASS + lane / LANES;
                const int rid = __shfl_sync(~0u, id, r), roff = __shfl_sync(~0u, off, r);
                const bool on = (mask >> r & 1) && chunk * 8 < a.c.dim;
                const uint8_t *src = on ? kbase + rid * a.c.blk_stride + roff + chunk * 16 : a.c.base;
                const unsigned dst = stage + r * ROW + ((chunk ^ (r & 7)) << 4);
                kv_cp16(dst, src, on);
                kv_cp16(dst + TILE, on ? src + a.c.plane_stride : src, on);
            }
            put = put + 1 == a.stages ? 0 : put + 1;
            peek();
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    peek();
    for (int s = 0; s < a.stages - 1; ++s) issue();

    // ---- consumer
    unsigned qf[NT][KS][2];
    float o[NT][KS][4], m[NT][2], l[NT][2];
    int take = 0;
    bool began = false;              // the run of tiles at hand begins where its row does
    for (long long n = 0; n < todo; ++n) {
        __syncwarp();                // the stage about to be filled is no longer read
        issue();
        // the tile that is computed now was committed stages - 1 groups ago
        switch (a.stages) {
        case 1: asm volatile("cp.async.wait_group 0;" ::: "memory"); break;
        case 2: asm volatile("cp.async.wait_group 1;" ::: "memory"); break;
        case 3: asm volatile("cp.async.wait_group 2;" ::: "memory"); break;
        case 4: asm volatile("cp.async.wait_group 3;" ::: "memory"); break;
        case 5: asm volatile("cp.async.wait_group 4;" ::: "memory"); break;
        default: asm volatile("cp.async.wait_group 5;" ::: "memory"); break;
        }
        __syncwarp();
        const int4 tile = my_info[take];
        const unsigned mask = tile.x & 0xffff, stage = ring + take * 2 * TILE;
        const int h = tile.w / a.group_chunks * a.hc + hw, g0 = tile.w % a.group_chunks * HEADS;   // first query head in the group
        const int heads = min(HEADS, a.group - g0);
        if (tile.x & 1 << 16) {
            began = tile.x & 1 << 18;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const int g = nt * 8 + (lane >> 2);
                const T *q = (const T *)a.q + tile.z * a.q_seq + (long long)(h * a.group + g0 + g) * a.q_head;
#pragma unroll
                for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        const int d = ks * 16 + b * 8 + (lane & 3) * 2;
                        unsigned v = 0;
                        if (g < heads && d < a.c.dim)
                            v = a.q_pairs ? *(const unsigned *)(q + d) : *(const unsigned short *)(q + d) | (unsigned)*(const unsigned short *)(q + d + 1) << 16;
                        qf[nt][ks][b] = v;
                    }
#pragma unroll
                for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[nt][ks][e] = 0.f;
                m[nt][0] = m[nt][1] = -INFINITY;
                l[nt][0] = l[nt][1] = 0.f;
            }
        }
        if (mask) {
            float s[NT][4];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[nt][e] = 0.f;
            {
                const int r = lane & 15, c0 = lane >> 4;
                const unsigned krow = stage + r * ROW;
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    unsigned k[4];
                    kv_ldmatrix(k, krow + (((2 * ks + c0) ^ (r & 7)) << 4));
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) KvMma<T>::mma(s[nt], k, qf[nt][ks][0], qf[nt][ks][1]);
                }
            }
            const bool lo = mask >> (lane >> 2) & 1, hi = mask >> (8 + (lane >> 2)) & 1;
            unsigned pf[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                for (int e = 0; e < 4; ++e) s[nt][e] = (e < 2 ? lo : hi) ? s[nt][e] * a.scale2 : -INFINITY;
                if (a.scores) {
                    const int g = nt * 8 + (lane & 3) * 2;
                    float *to = a.scores + (((long long)tile.z * a.c.heads + h) * a.c.max_len + tile.y + (lane >> 2)) * a.group + g0 + g;
#pragma unroll
                    for (int b = 0; b < 2; ++b, to += 8 * a.group) {
                        if (tile.y + (lane >> 2) + b * 8 >= a.c.max_len) continue;
                        if ((a.group & 1) == 0 && g < heads) *(float2 *)to = make_float2(s[nt][2 * b], s[nt][2 * b + 1]);
                        else
#pragma unroll
                            for (int e = 0; e < 2; ++e)
                                if (g + e < heads) to[e] = s[nt][2 * b + e];
                    }
                }
                float alpha[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float x = fmaxf(s[nt][e], s[nt][e + 2]);
                    x = fmaxf(x, __shfl_xor_sync(~0u, x, 4));
                    x = fmaxf(x, __shfl_xor_sync(~0u, x, 8));
                    x = fmaxf(x, __shfl_xor_sync(~0u, x, 16));
                    x = fmaxf(x, m[nt][e]);
                    const float ref = kv_ref(x);
                    alpha[e] = kv_exp2(m[nt][e] - ref);
                    m[nt][e] = x;
                    s[nt][e] = kv_exp2(s[nt][e] - ref);
                    s[nt][e + 2] = kv_exp2(s[nt][e + 2] - ref);
                    l[nt][e] = l[nt][e] * alpha[e] + (s[nt][e] + s[nt][e + 2]);
                }
                pf[nt][0] = kv_movmatrix_t(KvMma<T>::pack(s[nt][0], s[nt][1]));
                pf[nt][1] = kv_movmatrix_t(KvMma<T>::pack(s[nt][2], s[nt][3]));
                if (__any_sync(~0u, alpha[0] != 1.f || alpha[1] != 1.f))
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[nt][ks][e] *= alpha[e & 1];
            }
            const int r = (lane & 7) + (lane >> 4) * 8, c0 = lane >> 3 & 1;
            const unsigned vrow = stage + TILE + r * ROW;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                unsigned v[4];
                kv_ldmatrix_t(v, vrow + (((2 * ks + c0) ^ (r & 7)) << 4));
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) KvMma<T>::mma(o[nt][ks], v, pf[nt][0], pf[nt][1]);
            }
        }
        take = take + 1 == a.stages ? 0 : take + 1;

        if (tile.x & 1 << 17) {      // the CTA's last step in this row
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int x = 4; x <= 16; x <<= 1) l[nt][e] += __shfl_xor_sync(~0u, l[nt][e], x);
            const bool whole = began && (tile.x & 1 << 19);
            if (a.tw > 1) {          // the ways of a head meet in pairs
                float *box = (float *)(smem + warps * a.stages * 2 * TILE);
                for (int st = a.tw >> 1; st >= 1; st >>= 1) {
                    if (way >= st && way < 2 * st) {
                        float *to = box + ((way - st) * a.hc + hw) * (NT * (KS + 1) * 4) * 32 + lane;
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                to[(nt * 4 + e) * 32] = m[nt][e];
                                to[(nt * 4 + 2 + e) * 32] = l[nt][e];
                            }
#pragma unroll
                            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                                for (int e = 0; e < 4; ++e) to[(NT * 4 + (nt * KS + ks) * 4 + e) * 32] = o[nt][ks][e];
                        }
                    }
                    __syncthreads();
                    if (way < st) {
                        const float *from = box + (way * a.hc + hw) * (NT * (KS + 1) * 4) * 32 + lane;
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            float x[2], y[2];
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const float m2 = from[(nt * 4 + e) * 32], top = fmaxf(m[nt][e], m2), ref = kv_ref(top);
                                x[e] = kv_exp2(m[nt][e] - ref);
                                y[e] = kv_exp2(m2 - ref);
                                m[nt][e] = top;
                                l[nt][e] = l[nt][e] * x[e] + from[(nt * 4 + 2 + e) * 32] * y[e];
                            }
#pragma unroll
                            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                                for (int e = 0; e < 4; ++e)
                                    o[nt][ks][e] = o[nt][ks][e] * x[e & 1] + from[(NT * 4 + (nt * KS + ks) * 4 + e) * 32] * y[e & 1];
                        }
                    }
                    __syncthreads();
                }
            }
            if (way == 0) {
                const long long part = ((long long)blockIdx.x * 2 + (began ? 1 : 0)) * a.hc + hw;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int g = nt * 8 + (lane & 3) * 2 + e;
                        if (g >= heads) continue;
                        const int gq = h * a.group + g0 + g;
                        if (whole) {
                            const float inv = l[nt][e] == 0.f ? 0.f : 1.f / l[nt][e];
                            const float lse2 = l[nt][e] == 0.f ? -INFINITY : m[nt][e] + log2f(l[nt][e]);
                            T *to = (T *)a.out + tile.z * a.o_seq + gq * a.o_head;
#pragma unroll
                            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                                for (int b = 0; b < 2; ++b) {
                                    const int d = ks * 16 + b * 8 + (lane >> 2);
                                    if (d < a.c.dim) to[d] = kv_round<T>(o[nt][ks][2 * b + e] * inv);
                                }
                            if (lane < 4) {
                                if (a.lse) a.lse[(long long)tile.z * a.q_heads + gq] = lse2 * KV_LN2;
                                a.row_lse[(long long)tile.z * a.q_heads + gq] = lse2;
                                if (a.pieces == 0) s_lse[hw][g] = lse2;
                            }
                        } else {
                            float *to = a.part_o + (part * HEADS + g) * a.c.dim;
#pragma unroll
                            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                                for (int b = 0; b < 2; ++b) {
                                    const int d = ks * 16 + b * 8 + (lane >> 2);
                                    if (d < a.c.dim) to[d] = o[nt][ks][2 * b + e];
                                }
                            if (lane < 4) a.part_ml[part * HEADS + g] = make_float2(m[nt][e], l[nt][e]);
                        }
                    }
            }
        }
    }

    // ---- rows that are one CTA's add up their weights here: every thread reads the scores it wrote itself
    if (a.pieces == 0 && a.scores) {
        __syncthreads();
        const int i = blockIdx.x / rows_of_seq, h = blockIdx.x % rows_of_seq / a.group_chunks * a.hc + hw;
        const KvSpan sp(a, i);
        const long long at = i * a.w_seq + h * a.w_head;
        for (int t = way * 32 + lane; t < sp.base; t += a.tw * 32) a.w_out[at + t] = a.w_in ? a.w_in[at + t] : 0.f;
        const int steps = sp.steps(a);
        for (int k = 0; k < steps; ++k) {
            const int t0 = sp.base + (k * a.tw + way) * 16;
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const int t = t0 + b * 8 + (lane >> 2);
                float w = 0.f;
                if (t < sp.n && t >= sp.first) {
                    const float *from = a.scores + (((long long)i * a.c.heads + h) * a.c.max_len + t) * a.group;
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const int g = nt * 8 + (lane & 3) * 2 + e;
                            if (g < a.group && s_lse[hw][g] != -INFINITY) w += kv_exp2(from[g] - s_lse[hw][g]);
                        }
                }
                w += __shfl_xor_sync(~0u, w, 1);
                w += __shfl_xor_sync(~0u, w, 2);
                if ((lane & 3) == 0 && t < sp.n) a.w_out[at + t] = (a.w_in ? a.w_in[at + t] : 0.f) + w;
            }
        }
    }
}

// Joins the pieces of rows that more than one CTA worked on, in the order of the slots, and adds up the weights of all
// rows.  CTA (x, KV head, sequence): query heads x, x + gridDim.x, ... of the group, slots from x * KV_JOIN_SLOTS on.
constexpr int KV_JOIN_SLOTS = 1024, KV_JOIN_THREADS = 256, KV_MAX_GROUP = 256;

template <typename T>
__global__ void __launch_bounds__(KV_JOIN_THREADS) kv_attend_join(const __grid_constant__ KvAttend a, int heads_of_chunk)
{
    __shared__ long long red[2 * KV_JOIN_THREADS / 32];
    __shared__ float lse2[KV_MAX_GROUP];
    __shared__ float box[KV_JOIN_THREADS / 32][256];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int x = blockIdx.x, h = blockIdx.y, i = blockIdx.z;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const KvSpan sp(a, i);
    if (sp.n == 0) return;
    if (x >= a.group && (!a.scores || x * KV_JOIN_SLOTS >= sp.n)) return;
    long long before, total;
    kv_attend_sums(a, i, red, before, total);
    const int rows_of_seq = a.head_chunks * a.group_chunks, steps = sp.steps(a);
    before *= rows_of_seq;
    const long long piece = kv_attend_piece(a, total * rows_of_seq);
    const int hw = h % a.hc;
    for (int gc = 0; gc < a.group_chunks; ++gc) {
        const long long first = before + (long long)(h / a.hc * a.group_chunks + gc) * steps;
        const long long c0 = first / piece, c1 = (first + steps - 1) / piece;
        const int heads = min(heads_of_chunk, a.group - gc * heads_of_chunk);
        // the parts of this row: the first is its CTA's second, all others their CTA's first
        auto part = [&](long long c) { return ((c * 2 + (c == c0 ? 1 : 0)) * a.hc + hw) * heads_of_chunk; };
        for (int g = warp; g < heads; g += KV_JOIN_THREADS / 32) {
            const int gg = gc * heads_of_chunk + g;
            const long long row = (long long)i * a.q_heads + h * a.group + gg;
            if (c0 == c1) {
                if (lane == 0) lse2[gg] = a.row_lse[row];
                continue;
            }
            float top = -INFINITY, sum = 0.f;
            for (long long c = c0 + lane; c <= c1; c += 32) {
                const float2 ml = a.part_ml[part(c) + g];
                const float t = fmaxf(top, ml.x), ref = kv_ref(t);
                sum = sum * kv_exp2(top - ref) + ml.y * kv_exp2(ml.x - ref);
                top = t;
            }
#pragma unroll
            for (int o = 16; o; o >>= 1) {
                const float t2 = __shfl_xor_sync(~0u, top, o), s2 = __shfl_xor_sync(~0u, sum, o);
                const float t = fmaxf(top, t2), ref = kv_ref(t);
                sum = sum * kv_exp2(top - ref) + s2 * kv_exp2(t2 - ref);
                top = t;
            }
            if (lane == 0) {
                lse2[gg] = sum == 0.f ? -INFINITY : top + log2f(sum);
                if (a.lse && x == 0) a.lse[row] = lse2[gg] * KV_LN2;
            }
        }
        __syncthreads();
        if (c0 != c1)
            for (int g = x; g < a.group; g += gridDim.x) {
                if (g / heads_of_chunk != gc) continue;
                float acc[8];
#pragma unroll
                for (int d = 0; d < 8; ++d) acc[d] = 0.f;
                const float z = lse2[g];
                if (z != -INFINITY)
#pragma unroll 4
                    for (long long c = c0 + warp; c <= c1; c += KV_JOIN_THREADS / 32) {
                        const long long p = part(c) + g - gc * heads_of_chunk;
                        const float f = kv_exp2(a.part_ml[p].x - z);
#pragma unroll
                        for (int b = 0; b < 2; ++b)
                            if (b * 128 + lane * 4 < a.c.dim) {
                                const float4 v = *(const float4 *)(a.part_o + p * a.c.dim + b * 128 + lane * 4);
                                acc[4 * b] += f * v.x;
                                acc[4 * b + 1] += f * v.y;
                                acc[4 * b + 2] += f * v.z;
                                acc[4 * b + 3] += f * v.w;
                            }
                    }
#pragma unroll
                for (int d = 0; d < 8; ++d) box[warp][(d >> 2) * 128 + lane * 4 + (d & 3)] = acc[d];
                __syncthreads();
                if (tid < a.c.dim) {
                    float v = 0.f;
#pragma unroll
                    for (int w = 0; w < KV_JOIN_THREADS / 32; ++w) v += box[w][tid];
                    ((T *)a.out)[i * a.o_seq + (h * a.group + g) * a.o_head + tid] = kv_round<T>(v);
                }
                __syncthreads();
            }
    }
    if (!a.scores) return;
    __syncthreads();
    const long long at = i * a.w_seq + h * a.w_head;
    for (int t = x * KV_JOIN_SLOTS + tid; t < min((x + 1) * KV_JOIN_SLOTS, sp.n); t += KV_JOIN_THREADS) {
        float w = 0.f;
        if (t >= sp.first) {
            const float *from = a.scores + (((long long)i * a.c.heads + h) * a.c.max_len + t) * a.group;
            if ((a.group & 3) == 0) {
                for (int g = 0; g < a.group; g += 4) {
                    const float4 s = *(const float4 *)(from + g);
                    const float part[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (lse2[g + e] != -INFINITY) w += kv_exp2(part[e] - lse2[g + e]);
                }
            } else {
                for (int g = 0; g < a.group; ++g)
                    if (lse2[g] != -INFINITY) w += kv_exp2(from[g] - lse2[g]);
            }
        }
        a.w_out[at + t] = (a.w_in ? a.w_in[at + t] : 0.f) + w;
    }
}
