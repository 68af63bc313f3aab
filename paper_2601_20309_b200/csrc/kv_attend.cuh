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
// own ring of shared-memory stages with cp.async (three stages of 8 KiB for heads of 128: 128 KiB in flight per SM; each row of
// a tile may lie in another block, so a copy by rows fits where a TMA box would not, and rows beyond the length are filled
// with zeros on the way) and computes from it, so warps never wait for one another except at the end of a row that
// several ways share.  With eight KV heads the warps of a CTA read whole rows of the cache, 2 KiB each, side by side.
//
// Measured (B200, 148 SMs): 32 sequences around 2k up to 16k slots, 64 query and 8 KV heads of 128, 424 MB: 58 us from the first
// tile to the median CTA's last, 7.3 TB/s; the whole call 81 us (5.2 TB/s, 80 % of the floor): 4 us until loads are under way,
// 6 between the median and the slowest SM, 8 for the second kernel.  64 sequences around 1k up to 8k with weights, 415 MB:
// 90 us.  What was counted on the way there: 730 instructions per tile and warp at 4.4 cycles each kept it at 88 us; one
// address per tile instead of one per row, xor addressing and two score chains brought that to 460 (the compensated sum adds 17).
//
// Mathematics of a tile, on mma.m16n8k16 with the cache as the left operand, so that the few query heads fill the narrow
// side:  S^T[16 slots, 8 heads] = K Q^T;  m, p = exp2(S - m), l in float32 (scale and log2 e are applied to the sums);
// O^T[dim, 8 heads] = alpha O^T + V^T P^T, V^T by transposing ldmatrix, P^T by movmatrix from the score fragment.  P is
// rounded to the cache's type (f16: times 2^14, taken back at the end), the only rounding besides the output's: it lets the
// second product run on the tensor pipe at the cache's width, and over many slots its error averages out below the output's
// own.  l sums the unrounded p, with compensation, since in a long row the small ones would vanish beside one large.  (tcgen05
// would take the cache as its left operand just the same, 128 slots at a time, but a decode step has no use for its rate: the tensor pipe is 8 %
// busy as it is, and the running maximum would have to travel between tensor memory and registers for every tile.)
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
    int whole_tiles;     // the block size is a multiple of 16: a tile lies in one block
    float *scores;       // [seq][kv_head][max_len][group], base 2; nullptr: no weights wanted
    float2 *part_ml;     // [piece][2][hc][8*NT]: maximum and sum
    float *part_o;       // [piece][2][hc][8*NT][dim]
    int4 *part_of;       // [piece]: the row (of all) that the piece begins inside of, its place in the line, its steps (0: none), the length of a piece
    float *row_lse;      // [seq][q_head], base 2, of rows that one CTA has
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
    static constexpr float LIFT = 1.f;
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
    // the weights of the second product go up to this: f16 has no numbers below 2^-24, and many small weights count together, so
    // only those below 2^-28 of the row's largest lose bits, and those below 2^-39 vanish
    static constexpr float LIFT = 16384.f;
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

// The line of steps, searched by a whole CTA: every thread sums the steps of a run of sequences.
struct KvLine {
    int before, mine, total;         // steps in front of the thread's run, in it, and of all sequences (fewer than 2^31)
    int lo, hi;
    // `red` holds one value per warp
    __device__ __forceinline__ KvLine(const KvAttend &a, int *red)
    {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, rows_of_seq = a.head_chunks * a.group_chunks;
        const int run = (a.seqs + blockDim.x - 1) / blockDim.x;
        lo = min((int)threadIdx.x * run, a.seqs);
        hi = min(lo + run, a.seqs);
        mine = 0;
        for (int i = lo; i < hi; ++i) mine += KvSpan(a, i).steps(a);
        mine *= rows_of_seq;
        int x = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(~0u, x, o);
            if (lane >= o) x += y;
        }
        if (lane == 31) red[warp] = x;
        __syncthreads();
        before = total = 0;
        for (int w = 0; w < (int)(blockDim.x >> 5); ++w) {
            if (w < warp) before += red[w];
            total += red[w];
        }
        before += x - mine;
    }
    // the sequence, its row and the step in it that step s < total of the line is; `at` holds two values
    __device__ __forceinline__ void find(const KvAttend &a, int s, int *at, int &i, int &row, int &k) const
    {
        const int rows_of_seq = a.head_chunks * a.group_chunks;
        if (s >= before && s < before + mine) {
            int j = lo;
            int left = s - before;
            for (; j < hi - 1; ++j) {
                const int n = KvSpan(a, j).steps(a) * rows_of_seq;
                if (left < n) break;
                left -= n;
            }
            at[0] = j;
            at[1] = left;
        }
        __syncthreads();
        i = at[0];
        const int steps = KvSpan(a, i).steps(a);
        row = at[1] / steps;
        k = at[1] - row * steps;
    }
};

__device__ __forceinline__ int kv_attend_piece(const KvAttend &a, int total) { return max((total + a.pieces - 1) / a.pieces, a.min_steps); }

// 128 registers where that is enough (one query tile, heads of up to 128): the join's CTAs then fit beside this kernel's
template <typename T, int DP, int NT>
__global__ void __launch_bounds__(KV_ATTEND_WARPS * 32 / (DP == 256 ? 2 : 1), DP * NT <= 128 ? 2 : 1) kv_attend_stream(const __grid_constant__ KvAttend a)
{
    constexpr float LIFT = KvMma<T>::LIFT;
    constexpr int ROW = DP * 2, TILE = 16 * ROW, KS = DP / 16, LANES = DP / 8, PASS = 32 / LANES, HEADS = 8 * NT;
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ int red[KV_ATTEND_WARPS], s_at[2];
    __shared__ int4 info[KV_ATTEND_WARPS][KV_ATTEND_STAGES];
    __shared__ float s_lse[KV_ATTEND_WARPS][HEADS];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, warps = blockDim.x >> 5;
    const int hw = warp % a.hc, way = warp / a.hc;
    const int rows_of_seq = a.head_chunks * a.group_chunks;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    if (a.pieces && tid == 0) a.part_of[blockIdx.x] = make_int4(0, 0, 0, 0);

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
    int todo, s0 = 0, piece = 0;
    if (a.pieces == 0) {
        pi = blockIdx.x / rows_of_seq;
        pch = blockIdx.x % rows_of_seq;
        pk = 0;
        todo = KvSpan(a, pi).steps(a);
    } else {
        const KvLine line(a, red);
        piece = kv_attend_piece(a, line.total);
        s0 = (int)min((long long)blockIdx.x * piece, (long long)line.total);
        todo = min(line.total - s0, piece);
        if (todo <= 0) return;
        line.find(a, s0, s_at, pi, pch, pk);
    }
    if (todo <= 0) return;
    const int k0 = pk;

    const unsigned ring = (unsigned)__cvta_generic_to_shared(smem) + warp * a.stages * 2 * TILE;
    const uint8_t *kbase = a.c.base + (long long)a.layer * 2 * a.c.plane_stride;
    int4 *my_info = info[warp];

    // ---- producer.  The block ids of two tiles of a row are read at once, lane r for row r % 16 of tile r / 16, and used
    // one tile later, so that no load waits for its address.  With blocks of whole tiles one address serves a tile.
    int unseen = todo;               // tiles whose ids have not been read
    int id = -1, off = 0, t0 = 0, ti = 0, tch = 0, have = 0, half = 0, tk = 0, tsteps = 0;
    unsigned masks = 0;
    const uint8_t *rowp = a.c.base;
    bool live = false, exists = false, fresh = true;   // fresh: the next tile begins this CTA's run in its row
    const int chunk = lane % LANES, chunk_on = chunk * 8 < a.c.dim;
    const int lane_off = lane / LANES * a.c.row_stride + chunk * 16;
    KvSpan span(a, pi);
    int psteps = span.steps(a);
    auto peek = [&]() {
        have = min(min(2, psteps - pk), unseen);
        half = 0;
        if (have == 0) return;
        t0 = span.base + (pk * a.tw + way) * 16;
        const int tile = t0 + (lane >> 4) * a.tw * 16, t = tile + (lane & 15);
        live = (lane >> 4) < have && t >= span.first && t < span.n;
        exists = a.whole_tiles ? (lane >> 4) < have && tile < span.n : live;
        if (exists) {
            const int b = t / a.c.bs;
            id = a.c.tables[pi * a.c.table_stride + b];
            off = (pch / a.group_chunks * a.hc + hw) * a.c.head_stride + (t - b * a.c.bs) * a.c.row_stride;
        }
        ti = pi;
        tch = pch;
        tk = pk;
        tsteps = psteps;
        unseen -= have;
        pk += have;
        if (pk == psteps && unseen > 0) {
            pk = 0;
            if (++pch == rows_of_seq) {
                pch = 0;
                do span = KvSpan(a, ++pi);
                while (span.n == 0);
                psteps = span.steps(a);
            }
        }
    };
    int put = 0;
    auto issue = [&]() {
        if (half < have) {
            if (half == 0) {
                const bool known = exists && (unsigned)id < (unsigned)a.c.nb;
                if (live && !known) atomicOr(a.c.status, KV_OPS_BAD_BLOCK);
                masks = __ballot_sync(~0u, live && known);
                rowp = known ? kbase + id * a.c.blk_stride + off : a.c.base;
            }
            const unsigned mask = (masks >> (half * 16)) & 0xffffu;
            const bool ends = tk + half == tsteps - 1;
            if (lane == 0) {
                const int flags = (fresh ? 1 << 16 : 0) | (ends || (unseen == 0 && half == have - 1) ? 1 << 17 : 0) | (tk + half == 0 ? 1 << 18 : 0) |
                                  (ends ? 1 << 19 : 0);
                my_info[put] = make_int4((int)mask | flags, t0 + half * a.tw * 16, ti, tch);
            }
            fresh = ends;
            unsigned dst = ring + put * 2 * TILE + lane / LANES * ROW;
            const unsigned on = chunk_on ? mask >> (lane / LANES) : 0u;
            if (a.whole_tiles) {
                const uint8_t *src = (const uint8_t *)__shfl_sync(~0u, (unsigned long long)rowp, half * 16) + (mask ? lane_off : 0);
                const int step = mask ? PASS * a.c.row_stride : 0;
#pragma unroll
                for (int j = 0; j < 16 / PASS; ++j, src += step) {
                    const unsigned to = dst + j * PASS * ROW + ((chunk ^ (j * PASS + lane / LANES) & 7) << 4);
                    kv_cp16(to, src, on >> (j * PASS) & 1);
                    kv_cp16(to + TILE, src + a.c.plane_stride, on >> (j * PASS) & 1);
                }
            } else {
#pragma unroll 1
                for (int j = 0; j < 16 / PASS; ++j) {
                    const int r = j * PASS + lane / LANES;
                    const uint8_t *src = (const uint8_t *)__shfl_sync(~0u, (unsigned long long)rowp, half * 16 + r);
                    const bool row_on = on >> (j * PASS) & 1;
                    const unsigned to = dst + j * PASS * ROW + ((chunk ^ (r & 7)) << 4);
                    if (row_on) src += chunk * 16;
                    kv_cp16(to, src, row_on);
                    kv_cp16(to + TILE, row_on ? src + a.c.plane_stride : src, row_on);
                }
            }
            put = put + 1 == a.stages ? 0 : put + 1;
            if (++half == have) peek();
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    peek();
    for (int s = 0; s < a.stages - 1; ++s) issue();

    // ---- consumer
    unsigned qf[NT][KS][2];
    float o[NT][KS][4], m[NT][2], l[NT][2], rest[NT][2];     // rest: what l is too coarse for
    int take = 0;
    bool began = false;              // the run of tiles at hand begins where its row does
    for (int n = 0; n < todo; ++n) {
        __syncwarp();                // the stage about to be filled is no longer read
        issue();
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
                l[nt][0] = l[nt][1] = rest[nt][0] = rest[nt][1] = 0.f;
            }
        }
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
        if (mask) {
            float s[NT][4], s2[NT][4];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[nt][e] = s2[nt][e] = 0.f;
            // chunk 2 ks + c of row r lies at chunk (2 ks + c) ^ (r & 7): with rows aligned to their size, one xor
            const unsigned krow = stage + (lane & 15) * ROW + ((lane >> 4 ^ lane & 7) << 4);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                unsigned k[4];
                kv_ldmatrix(k, krow ^ ks << 5);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) KvMma<T>::mma(ks & 1 ? s2[nt] : s[nt], k, qf[nt][ks][0], qf[nt][ks][1]);   // two chains
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[nt][e] += s2[nt][e];
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
                }
                pf[nt][0] = kv_movmatrix_t(KvMma<T>::pack(s[nt][0] * LIFT, s[nt][1] * LIFT));
                pf[nt][1] = kv_movmatrix_t(KvMma<T>::pack(s[nt][2] * LIFT, s[nt][3] * LIFT));
                if (__any_sync(~0u, alpha[0] != 1.f || alpha[1] != 1.f)) {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        l[nt][e] *= alpha[e];
                        rest[nt][e] *= alpha[e];
                    }
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[nt][ks][e] *= alpha[e & 1];
                }
#pragma unroll
                for (int e = 0; e < 2; ++e) {            // compensated: weights of 2^-25 of the largest would vanish one by one
                    const float x = s[nt][e] + s[nt][e + 2] + rest[nt][e], sum = l[nt][e] + x;
                    rest[nt][e] = x - (sum - l[nt][e]);
                    l[nt][e] = sum;
                }
            }
            const unsigned vrow = stage + TILE + ((lane & 7) + (lane >> 4) * 8) * ROW + ((lane >> 3 & 1 ^ lane & 7) << 4);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                unsigned v[4];
                kv_ldmatrix_t(v, vrow ^ ks << 5);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) KvMma<T>::mma(o[nt][ks], v, pf[nt][0], pf[nt][1]);
            }
        }
        else if (a.scores)           // nothing of the tile counts
            for (int e = lane; e < 16 * heads; e += 32)
                if (tile.y + e / heads < a.c.max_len)
                    a.scores[(((long long)tile.z * a.c.heads + h) * a.c.max_len + tile.y + e / heads) * a.group + g0 + e % heads] = -INFINITY;
        __syncwarp();
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
                if (a.pieces && tid == 0 && !began)
                    a.part_of[blockIdx.x] = make_int4(tile.z * rows_of_seq + tile.w, s0 - k0, KvSpan(a, tile.z).steps(a), piece);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int g = nt * 8 + (lane & 3) * 2 + e;
                        if (g >= heads) continue;
                        const int gq = h * a.group + g0 + g;
                        if (whole) {
                            const bool none = l[nt][e] == 0.f;           // the sums may be 0 * inf then
                            const float inv = none ? 0.f : 1.f / l[nt][e] * (1.f / LIFT);
                            const float lse2 = none ? -INFINITY : m[nt][e] + log2f(l[nt][e]);
                            T *to = (T *)a.out + tile.z * a.o_seq + gq * a.o_head;
#pragma unroll
                            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                                for (int b = 0; b < 2; ++b) {
                                    const int d = ks * 16 + b * 8 + (lane >> 2);
                                    if (d < a.c.dim) to[d] = kv_round<T>(none ? 0.f : o[nt][ks][2 * b + e] * inv);
                                }
                            if (lane < 4) {
                                if (a.lse) a.lse[(long long)tile.z * a.q_heads + gq] = lse2 * KV_LN2;
                                // a row without any weight has scores of -inf: less +inf they give 0
                                s_lse[hw][g] = lse2 == -INFINITY ? INFINITY : lse2;
                                if (a.pieces) a.row_lse[(long long)tile.z * a.q_heads + gq] = lse2;
                            }
                        } else {
                            float *to = a.part_o + (part * HEADS + g) * a.c.dim;
#pragma unroll
                            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                                for (int b = 0; b < 2; ++b) {
                                    const int d = ks * 16 + b * 8 + (lane >> 2);
                                    if (d < a.c.dim) to[d] = o[nt][ks][2 * b + e] * (1.f / LIFT);
                                }
                            if (lane < 4) a.part_ml[part * HEADS + g] = make_float2(m[nt][e], l[nt][e]);
                        }
                    }
            }
            // where there is no second kernel, the weights are added up here: every thread reads the scores it wrote itself
            if (a.pieces == 0 && a.scores) {
                if (a.tw > 1) __syncthreads();
                else __syncwarp();
                const KvSpan sp(a, tile.z);
                const float *from = a.scores + ((long long)tile.z * a.c.heads + h) * a.c.max_len * a.group;
                const long long w = tile.z * a.w_seq + h * a.w_head;
                for (int t = way * 32 + lane; t < sp.base; t += a.tw * 32) a.w_out[w + t] = a.w_in ? a.w_in[w + t] : 0.f;
                for (int t0 = sp.base + way * 16; t0 < sp.n; t0 += a.tw * 16) {
                    float add[2] = {0.f, 0.f};
#pragma unroll
                    for (int b = 0; b < 2; ++b)
                        if (t0 + b * 8 + (lane >> 2) < sp.n)
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                                for (int e = 0; e < 2; ++e) {
                                    const int g = nt * 8 + (lane & 3) * 2 + e;
                                    if (g < heads) add[b] += kv_exp2(from[(long long)(t0 + b * 8 + (lane >> 2)) * a.group + g] - s_lse[hw][g]);
                                }
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        add[b] += __shfl_xor_sync(~0u, add[b], 1);
                        add[b] += __shfl_xor_sync(~0u, add[b], 2);
                        const int t = t0 + b * 8 + (lane >> 2);
                        // slots of the tile that lie before the window keep their weight, even where the sum is NaN
                        if ((lane & 3) == 0 && t < sp.n) a.w_out[w + t] = (a.w_in ? a.w_in[w + t] : 0.f) + (t >= sp.first ? add[b] : 0.f);
                    }
                }
                if (a.tw > 1) __syncthreads();           // the next row's sums take the place of these
                else __syncwarp();
            }
        }
    }
}

// ---- join: what is left when rows were split.
//
// The first KV_JOIN_SHARES * pieces CTAs add up the weights, each over its equal share of the line of steps, with the sums of
// all parts of its rows.  They fit beside the first kernel and find their place in the line before it ends.  Then come
// `row_ctas` per piece that join output rows: where the piece begins inside a row, the pieces that cut that row share
// its output, in units of 32 elements of a head, among them.  What such a kernel takes is the number of loads that
// wait for one another, each close to a microsecond, times the waves of CTAs: there are three in a chain (what, the row's
// sums, the data), every load that can be in flight together is, and four CTAs per SM are all there are.
// With 2 / 3 / 4 shares 64 sequences take 91.4 / 90.0 / 89.3 us, one of 131072 slots 27.8 / 27.8 / 29.3.
constexpr int KV_JOIN_THREADS = 256, KV_JOIN_WARPS = KV_JOIN_THREADS / 32, KV_JOIN_SHARES = 3, KV_MAX_GROUP = 256;

// maximum and sum of two sets of slots together
__device__ __forceinline__ void kv_meet(float &top, float &sum, float top2, float sum2)
{
    const float t = fmaxf(top, top2), ref = kv_ref(t);
    sum = sum * kv_exp2(top - ref) + sum2 * kv_exp2(top2 - ref);
    top = t;
}

// log2 of a row's sum of exponentials for one query head, from its parts c0 .. c1: by a whole warp (`lanes` 32), or by every
// thread for itself (`lanes` 1)
template <int lanes>
__device__ __forceinline__ float kv_join_lse(const KvAttend &a, int c0, int c1, int hw, int heads_of_chunk, int g)
{
    float top = -INFINITY, sum = 0.f;
#pragma unroll 4
    for (int c = c0 + (lanes == 1 ? 0 : threadIdx.x & 31); c <= c1; c += lanes) {
        const float2 ml = a.part_ml[((c * 2 + (c == c0 ? 1 : 0)) * a.hc + hw) * heads_of_chunk + g];
        kv_meet(top, sum, ml.x, ml.y);
    }
#pragma unroll
    for (int o = lanes / 2; o; o >>= 1) kv_meet(top, sum, __shfl_xor_sync(~0u, top, o), __shfl_xor_sync(~0u, sum, o));
    return sum == 0.f ? -INFINITY : top + log2f(sum);
}

template <int n> struct KvCount { static constexpr int value = n; };

// floats of shared memory the row CTAs need: a factor for every part of every head a CTA shares in (a row of more than
// eight parts is shared by eight CTAs or more), and a float4 per thread
__host__ __device__ constexpr int kv_join_floats(int hc, int heads_of_chunk, int pieces)
{
    const int few = hc * heads_of_chunk * 8, many = (hc * heads_of_chunk / 8 + 2) * (pieces + 1);
    return (few > many ? few : many) + 4 * KV_JOIN_THREADS;
}

template <typename T>
__device__ __forceinline__ void kv_join_rows(const KvAttend &a, int heads_of_chunk, int b, int sub, int subs, float *smem)
{
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int4 of = a.part_of[b];
    if (of.z == 0) return;
    const int i = of.x / (a.head_chunks * a.group_chunks), row = of.x - i * (a.head_chunks * a.group_chunks);
    const int c0 = of.y / of.w, c1 = (of.y + of.z - 1) / of.w, parts = c1 - c0 + 1;
    const int g0 = row % a.group_chunks * heads_of_chunk, heads = min(heads_of_chunk, a.group - g0), h0 = row / a.group_chunks * a.hc;
    // units (KV head, query head, 32 elements) of this piece, one of the parts - 1 that cut the row
    const int slices = (a.c.dim + 31) / 32, all = a.hc * heads * slices, turn = (b - c0 - 1) * subs + sub, turns = (parts - 1) * subs;
    const int u0 = all * turn / turns, u1 = all * (turn + 1) / turns, p0 = u0 / slices, pairs = u1 > u0 ? (u1 - 1) / slices - p0 + 1 : 0;
    float *factor = smem + 4 * KV_JOIN_THREADS;
    const int stride = a.hc * heads_of_chunk;            // entries of a part
    auto slot = [&](int c) { return (c * 2 + (c == c0 ? 1 : 0)) * stride; };
    auto weigh = [&](int n, auto lanes) {
        constexpr int step = decltype(lanes)::value;
        const int pair = p0 + n, hw = pair / heads, g = pair - hw * heads;
        const float2 *ml = a.part_ml + hw * heads_of_chunk + g;
        const float z = kv_join_lse<step>(a, c0, c1, hw, heads_of_chunk, g);
        const int own = step == 1 ? 0 : lane;
        if (a.lse && own == 0 && pair * slices >= u0) a.lse[(long long)i * a.q_heads + (h0 + hw) * a.group + g0 + g] = z * KV_LN2;
#pragma unroll 4
        for (int c = own; c < parts; c += step) factor[n * parts + c] = z == -INFINITY ? -1.f : kv_exp2(ml[slot(c0 + c)].x - z);
    };
    if (parts <= 8)
        for (int n = tid; n < pairs; n += KV_JOIN_THREADS) weigh(n, KvCount<1>());
    else
        for (int n = warp; n < pairs; n += KV_JOIN_WARPS) weigh(n, KvCount<32>());
    __syncthreads();
    const int tasks = (u1 - u0) * 8;
    // task: elements 4 * (task % 8) .. + 3 of unit task / 8; where they lie in a part and in the output, and their factors
    struct Task {
        bool on;
        const float *from, *factor;
        T *to;
        float4 acc;
    };
    auto task = [&](int t) {
        Task x;
        const int u = u0 + t / 8, pair = u / slices, d = (u - pair * slices) * 32 + t % 8 * 4, hw = pair / heads, g = pair - hw * heads;
        x.on = t < tasks && d < a.c.dim;
        x.from = a.part_o + (hw * heads_of_chunk + g) * a.c.dim + d;
        x.factor = factor + (pair - p0) * parts;
        x.to = (T *)a.out + i * a.o_seq + ((h0 + hw) * a.group + g0 + g) * a.o_head + d;
        x.acc = make_float4(0.f, 0.f, 0.f, 0.f);
        return x;
    };
    auto add = [&](Task &x, int c) {
        const float4 v = *(const float4 *)(x.from + (long long)slot(c0 + c) * a.c.dim);
        const float f = x.factor[c];
        // a part without weight counts as 0 times what it holds, as its slots would in one sum; of a row without any (-1) nothing does
        if (!(f < 0.f)) x.acc = make_float4(x.acc.x + f * v.x, x.acc.y + f * v.y, x.acc.z + f * v.z, x.acc.w + f * v.w);
    };
    auto put = [&](const Task &x) {
        x.to[0] = kv_round<T>(x.acc.x);
        x.to[1] = kv_round<T>(x.acc.y);
        x.to[2] = kv_round<T>(x.acc.z);
        x.to[3] = kv_round<T>(x.acc.w);
    };
    if (tasks > KV_JOIN_THREADS / 2) {           // few parts: two outputs per thread at once
        for (int t = tid; t < tasks; t += 2 * KV_JOIN_THREADS) {
            Task x = task(t), y = task(t + KV_JOIN_THREADS);
#pragma unroll 2
            for (int c = 0; c < parts; ++c) {
                if (x.on) add(x, c);
                if (y.on) add(y, c);
            }
            if (x.on) put(x);
            if (y.on) put(y);
        }
    } else if (tasks > 0) {                      // many parts: several threads to an output
        int ways = 2;
        while (ways * 2 * tasks <= KV_JOIN_THREADS) ways *= 2;
        const int t = tid % tasks, way = tid / tasks;
        Task x = task(t);
        x.on = x.on && way < ways;
        float4 *box = (float4 *)smem;
        if (x.on)
#pragma unroll 8
            for (int c = way; c < parts; c += ways) add(x, c);
        box[tid] = x.acc;
        __syncthreads();
        if (way == 0 && x.on) {
            for (int w = 1; w < ways; ++w) {
                const float4 v = box[w * tasks + t];
                x.acc = make_float4(x.acc.x + v.x, x.acc.y + v.y, x.acc.z + v.z, x.acc.w + v.w);
            }
            put(x);
        }
    }
}

// `todo` steps of the line from step s on, which is step k of a row of sequence i
__device__ __forceinline__ void kv_join_weights(const KvAttend &a, int heads_of_chunk, int s, int todo, int piece, int i, int row, int k, float *lse2)
{
    const int tid = threadIdx.x, warp = tid >> 5, pairs = a.hc * a.group;
    while (todo > 0) {
        const KvSpan sp(a, i);
        const int steps = sp.steps(a), n = min(steps - k, todo), hx = row / a.group_chunks;
        if (n > 0 && row == hx * a.group_chunks) {       // the row of the KV heads' first query heads does it for all of them
            const int first = s - k;
            auto sum_of = [&](int p, auto lanes) {
                const int hw = p / a.group, g = p - hw * a.group, gc = g / heads_of_chunk, at = first + gc * steps;      // further query heads follow in the line
                const int c0 = at / piece, c1 = (at + steps - 1) / piece;
                const float z = c0 == c1 ? a.row_lse[(long long)i * a.q_heads + hx * pairs + p]
                                         : kv_join_lse<decltype(lanes)::value>(a, c0, c1, hw, heads_of_chunk, g - gc * heads_of_chunk);
                return z == -INFINITY ? INFINITY : z;    // a row without any weight has scores of -inf: less +inf they give 0
            };
            // few parts: a thread for every pair of KV and query head; many: a warp
            if (steps <= 8 * piece)
                for (int p = tid; p < pairs; p += KV_JOIN_THREADS) lse2[p] = sum_of(p, KvCount<1>());
            else
                for (int p = warp; p < pairs; p += KV_JOIN_WARPS) {
                    const float z = sum_of(p, KvCount<32>());
                    if ((tid & 31) == 0) lse2[p] = z;
                }
            __syncthreads();
            const int t0 = sp.base + k * a.tw * 16, count = min(sp.base + (k + n) * a.tw * 16, sp.n) - t0;
            const int lanes = KV_JOIN_THREADS / a.hc / 32 * 32, hw = tid / lanes;        // one warp per KV head, or several
            if (hw < a.hc) {
                const float *from = a.scores + (((long long)i * a.c.heads + hx * a.hc + hw) * a.c.max_len + t0) * a.group, *z = lse2 + hw * a.group;
                const long long w = i * a.w_seq + (hx * a.hc + hw) * a.w_head + t0;
                for (int t = tid - hw * lanes; t < count; t += 4 * lanes) {              // four slots at once
                    float v[4], add[4];
                    bool on[4];      // slots before the window keep their weight
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int u = t + e * lanes;
                        v[e] = a.w_in && u < count ? a.w_in[w + u] : 0.f;
                        on[e] = u < count && t0 + u >= sp.first;
                        add[e] = 0.f;
                    }
                    const float *at = from + (long long)t * a.group;
                    if ((a.group & 3) == 0) {
                        for (int g = 0; g < a.group; g += 4) {
                            float4 x[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                x[e] = on[e] ? *(const float4 *)(at + e * lanes * a.group + g) : make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                add[e] += (kv_exp2(x[e].x - z[g]) + kv_exp2(x[e].y - z[g + 1])) + (kv_exp2(x[e].z - z[g + 2]) + kv_exp2(x[e].w - z[g + 3]));
                        }
                    } else {
                        for (int g = 0; g < a.group; ++g) {
                            float x[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) x[e] = on[e] ? at[e * lanes * a.group + g] : -INFINITY;
#pragma unroll
                            for (int e = 0; e < 4; ++e) add[e] += kv_exp2(x[e] - z[g]);
                        }
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (t + e * lanes < count) a.w_out[w + t + e * lanes] = v[e] + (on[e] ? add[e] : 0.f);
                }
            }
            __syncthreads();         // the next row's sums take the place of these
        }
        s += n;
        todo -= n;
        k = 0;
        if (n == 0) ++i;             // a sequence without slots
        else if (++row == a.head_chunks * a.group_chunks) {
            row = 0;
            ++i;
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(KV_JOIN_THREADS, 4) kv_attend_join(const __grid_constant__ KvAttend a, int heads_of_chunk, int row_ctas)
{
    extern __shared__ __align__(16) float join_smem[];
    __shared__ int red[KV_JOIN_WARPS], at[2];
    const int shares = a.scores ? a.pieces * KV_JOIN_SHARES : 0, b = blockIdx.x - shares;
    if (b < 0) {
        const KvLine line(a, red);
        const int each = (line.total + shares - 1) / shares, s = (int)min((long long)blockIdx.x * each, (long long)line.total), n = min(line.total - s, each);
        int i = 0, row = 0, k = 0;
        if (n > 0) line.find(a, s, at, i, row, k);
        const int piece = kv_attend_piece(a, line.total);
        if (a.window > 0 && a.w_out != a.w_in) {         // slots in front of the window keep their weight: nothing to wait for
            const int rows = a.seqs * a.c.heads, split = max(1, shares / rows);
            for (int r = blockIdx.x; r < rows * split; r += shares) {
                const int j = r % rows / a.c.heads;
                const KvSpan sp(a, j);
                const long long w = j * a.w_seq + r % a.c.heads * a.w_head;
#pragma unroll 4
                for (int t = r / rows * KV_JOIN_THREADS + threadIdx.x; t < sp.base; t += split * KV_JOIN_THREADS) a.w_out[w + t] = a.w_in ? a.w_in[w + t] : 0.f;
            }
        }
        asm volatile("griddepcontrol.wait;" ::: "memory");
        kv_join_weights(a, heads_of_chunk, s, n, piece, i, row, k, join_smem);
    } else {
        asm volatile("griddepcontrol.wait;" ::: "memory");
        kv_join_rows<T>(a, heads_of_chunk, b / row_ctas, b % row_ctas, row_ctas, join_smem);
    }
}
