// Attention of one new token per sequence over a paged cache in 4 bits.  The line of steps, its pieces, the rings of the warps and
// the join are those of kv_attend.cuh; what is different is a tile, 16 slots of one KV head.
//
// Mathematics.  With element = lo + s * code, and a step s and a lowest value lo per slot and group of 32 elements,
//     q . K_t  = sum_g s_tg (sum_{d in g} q_d code_td) + sum_g lo_tg Q_g,       Q_g = sum_{d in g} q_d
//     out_d    = sum_t (p_t s_tg) code_td              + sum_t p_t lo_tg
// so codes go into the matrix instructions as they are and the steps are applied to 16 x 8 results, not to elements.  A code
// becomes a float16 number by a mask alone: four bits in the lowest places of a 16-bit word are code * 2^-24, in the next four places
// code * 2^-20, both subnormal numbers that m16n8k16 multiplies exactly.  Eight codes cost four masks and a shift.  (The powers
// of two are taken back in q, in the scale, and in the outputs.)
//   S^T[16 slots, 8 heads] = K Q^T, one group at a time.  q is scaled by a power of two so that its largest element lies in [2^8, 2^9),
//   which makes it float16 without loss down to 2^-26 of that.  The sum over lo is one more instruction in the cache's type, with Q_g
//   split into up to four parts of that type (32 bits of a bf16, 22 of an f16 Q_g).
//   O^T[dim, 8 heads] = V^T (P s)^T, again by groups; p s is rounded to float16, the only rounding besides the output's (p itself, for
//   the sum over lo and the row's sum, stays in float32).  What keeps p s in float16's range is the reference that is subtracted from the
//   scores: the running maximum plus the exponent of the largest step met so far, less 8.  Products below 2^-22 of the row's largest
//   lose bits, below 2^-32 they vanish.  The reference moves only when a score passes it by 6 or a step is larger: a
//   vote instead of a maximum over the lanes, the sums stay what they are in exact arithmetic.
// Slots: row r of a matrix instruction is slot r/2 + 4 (r%2) of the tile for r < 8, and 8 more for the others, so that the lanes' reads
// of V, two neighbouring rows of the contraction at once, fall into different banks.
//
// Masked slots (beyond the length, before the window) are loaded with their tile where their block is known: codes are numbers
// whatever they hold, scores are replaced by -inf and words by 0, so nothing of such a slot reaches a sum.
#pragma once
#include "kv_attend.cuh"

constexpr int KV_Q4_WARPS = 16, KV_Q4_STAGES = 6;
constexpr float KV_Q4_SLACK = 6.f, KV_Q4_LIFT = 8.f;
constexpr int KV_Q4_LOWEST = -80;    // exponent of a step below which it counts as this: sums of 2^31 weights stay in range

__host__ __device__ constexpr int kv_q4_threads(int groups, int tiles) { return groups * tiles <= 4 ? KV_Q4_WARPS * 32 : KV_Q4_WARPS * 16; }
__host__ __device__ constexpr int kv_q4_tile(int groups) { return 640 * groups; }
// floats of a lane that one way hands to another
__host__ __device__ constexpr int kv_q4_box(int groups, int tiles) { return tiles * (8 * groups + 4); }

template <int N> __device__ __forceinline__ void kv_lds(unsigned (&r)[N], unsigned addr)
{
    if constexpr (N == 1) asm volatile("ld.shared.b32 %0, [%1];" : "=r"(r[0]) : "r"(addr) : "memory");
    else if constexpr (N == 2) asm volatile("ld.shared.v2.b32 {%0,%1}, [%2];" : "=r"(r[0]), "=r"(r[1]) : "r"(addr) : "memory");
    else
#pragma unroll
        for (int k = 0; k < N; k += 4)
            asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(r[k]), "=r"(r[k + 1]), "=r"(r[k + 2]), "=r"(r[k + 3]) : "r"(addr + k * 4) : "memory");
}

template <typename T, int G, int NT>
__global__ void __launch_bounds__(kv_q4_threads(G, NT), 1) kv_attend_q4(const __grid_constant__ KvAttend a)
{
    constexpr int TILE = kv_q4_tile(G), KW = 256 * G, VC = 320 * G, VW = 576 * G, HEADS = 8 * NT, CHUNKS = 40 * G, LOADS = (CHUNKS + 31) / 32;
    constexpr int PARTS = G == 8 ? 2 : 1;        // matrix instructions for the sum over lo
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ int red[KV_Q4_WARPS], s_at[2];
    __shared__ int4 info[KV_Q4_WARPS][KV_Q4_STAGES];
    __shared__ float s_lse[KV_Q4_WARPS][HEADS];
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

    const unsigned ring = (unsigned)__cvta_generic_to_shared(smem) + warp * a.stages * TILE;
    const uint8_t *kbase = a.c.base + (long long)a.layer * 2 * a.c.plane_stride;
    int4 *my_info = info[warp];

    // ---- producer: block ids of two tiles of a row are read at once, lane r for row r % 16 of tile r / 16, and used one tile later.
    // A tile is 40 G pieces of 16 bytes: K's codes, K's words, V's codes, V's words.  With blocks of whole tiles these are four runs.
    int unseen = todo;               // tiles whose ids have not been read
    int id = -1, row_in = 0, ph = 0, t0 = 0, ti = 0, tch = 0, have = 0, half = 0, tk = 0, tsteps = 0;
    unsigned masks = 0, loads = 0;
    const uint8_t *headp = a.c.base;
    bool live = false, exists = false, fresh = true;   // fresh: the next tile begins this CTA's run in its row
    KvSpan span(a, pi);
    int psteps = span.steps(a);
    auto peek = [&]() {
        have = min(min(2, psteps - pk), unseen);
        half = 0;
        if (have == 0) return;
        t0 = span.base + (pk * a.tw + way) * 16;
        const int t = t0 + (lane >> 4) * a.tw * 16 + (lane & 15);
        // slots of the tile before the window are slots of the sequence: their ids are there
        exists = (lane >> 4) < have && (a.whole_tiles ? t - (lane & 15) : t) < span.n;
        live = (lane >> 4) < have && t >= span.first && t < span.n;
        if (exists) {
            const int b = t / a.c.bs;
            id = a.c.tables[pi * a.c.table_stride + b];
            row_in = t - b * a.c.bs;
        }
        ph = pch / a.group_chunks * a.hc + hw;
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
                loads = __ballot_sync(~0u, known);
                headp = known ? kbase + id * a.c.blk_stride + (long long)ph * a.c.head_stride : a.c.base;
            }
            const unsigned mask = (masks >> (half * 16)) & 0xffffu, load = (loads >> (half * 16)) & 0xffffu;
            const bool ends = tk + half == tsteps - 1;
            if (lane == 0) {
                const int flags = (fresh ? 1 << 16 : 0) | (ends || (unseen == 0 && half == have - 1) ? 1 << 17 : 0) | (tk + half == 0 ? 1 << 18 : 0) |
                                  (ends ? 1 << 19 : 0);
                my_info[put] = make_int4((int)mask | flags, t0 + half * a.tw * 16, ti, tch);
            }
            fresh = ends;
            const unsigned dst = ring + put * TILE + lane * 16;
            if (a.whole_tiles) {
                if (load & 1) {
                    const uint8_t *codes = (const uint8_t *)__shfl_sync(~0u, (unsigned long long)headp, half * 16);
                    const int row = __shfl_sync(~0u, row_in, half * 16);
                    const uint8_t *words = codes + a.c.bs * 16 * G + row * 4 * G;
                    codes += row * 16 * G;
#pragma unroll
                    for (int k = 0; k < LOADS; ++k) {
                        const int c = lane + 32 * k;
                        if (c < CHUNKS) {
                            const bool v = c >= 20 * G;
                            const int in = v ? c - 20 * G : c;
                            const uint8_t *src = (in < 16 * G ? codes + in * 16 : words + (in - 16 * G) * 16) + (v ? a.c.plane_stride : 0);
                            kv_cp16(dst + k * 512, src, true);
                        }
                    }
                }
            } else {
#pragma unroll 1
                for (int k = 0; k < LOADS; ++k) {
                    const int c = min(lane + 32 * k, CHUNKS - 1);
                    const bool v = c >= 20 * G;
                    const int in = v ? c - 20 * G : c, w = in - 16 * G;
                    // a piece of words may be of two rows: blocks are multiples of four rows, so both lie in one
                    const int r = w < 0 ? in / G : w * 4 / G;
                    const uint8_t *src = (const uint8_t *)__shfl_sync(~0u, (unsigned long long)headp, half * 16 + r);
                    const int row = __shfl_sync(~0u, row_in, half * 16 + r);
                    src += (w < 0 ? row * 16 * G + in % G * 16 : a.c.bs * 16 * G + row * 4 * G + (G == 8 ? (w & 1) * 16 : 0)) + (v ? a.c.plane_stride : 0);
                    if ((load >> r & 1) && lane + 32 * k < CHUNKS) kv_cp16(dst + k * 512, src, true);
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
    const int rho = lane >> 2, j = lane & 3, slot = (rho >> 1) + 4 * (rho & 1);
    unsigned qf[NT][G][4], ql[NT][PARTS][2];
    float fb[NT][2];
    float o[NT][G][2][4], lo[NT][G][2], m[NT][2], ref[NT][2], l[NT][2], rest[NT][2];     // rest: what l is too coarse for
    int top_step = KV_Q4_LOWEST;
    int take = 0;
    bool began = false;              // the run of tiles at hand begins where its row does
    for (int n = 0; n < todo; ++n) {
        __syncwarp();                // the stage about to be filled is no longer read
        issue();
        __syncwarp();
        const int4 tile = my_info[take];
        const unsigned mask = tile.x & 0xffff, stage = ring + take * TILE;
        const int h = tile.w / a.group_chunks * a.hc + hw, g0 = tile.w % a.group_chunks * HEADS;   // first query head in the group
        const int heads = min(HEADS, a.group - g0);
        if (tile.x & 1 << 16) {
            began = tile.x & 1 << 18;
            top_step = KV_Q4_LOWEST;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const int g = nt * 8 + rho;
                const T *q = (const T *)a.q + tile.z * a.q_seq + (long long)(h * a.group + g0 + g) * a.q_head;
                unsigned raw[G][4];
                float top = 0.f;
                bool bad = false;
#pragma unroll
                for (int b = 0; b < G; ++b) {
                    const int d = 32 * b + 8 * j;
                    raw[b][0] = raw[b][1] = raw[b][2] = raw[b][3] = 0;
                    if (g < heads && d < a.c.dim) {
                        if (a.q_vec) {
                            const uint4 v = *(const uint4 *)(q + d);
                            raw[b][0] = v.x, raw[b][1] = v.y, raw[b][2] = v.z, raw[b][3] = v.w;
                        } else
#pragma unroll
                            for (int e = 0; e < 8; ++e) raw[b][e >> 1] |= (unsigned)((const unsigned short *)q)[d + e] << (16 * (e & 1));
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float2 v = kv_unpair(raw[b][e], T());
                        top = fmaxf(top, fmaxf(fabsf(v.x), fabsf(v.y)));
                        bad |= !(fabsf(v.x) < INFINITY) || !(fabsf(v.y) < INFINITY);
                    }
                }
#pragma unroll
                for (int x = 1; x <= 2; x <<= 1) {
                    top = fmaxf(top, __shfl_xor_sync(~0u, top, x));
                    bad |= __shfl_xor_sync(~0u, (int)bad, x) != 0;
                }
                const int shift = bad || top == 0.f ? 0 : min(100, 135 - (int)(__float_as_uint(top) >> 23));
                const float by = __uint_as_float((127 + shift) << 23);
                float sum[G];
#pragma unroll
                for (int b = 0; b < G; ++b) {
                    float v[8];
                    sum[b] = 0.f;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float2 x = kv_unpair(raw[b][e], T());
                        v[2 * e] = x.x * by;
                        v[2 * e + 1] = x.y * by;
                        sum[b] += v[2 * e] + v[2 * e + 1];
                    }
                    qf[nt][b][0] = kv_pair(v[0], v[4], __half());
                    qf[nt][b][1] = kv_pair(v[1] * 0.0625f, v[5] * 0.0625f, __half());
                    qf[nt][b][2] = kv_pair(v[2], v[6], __half());
                    qf[nt][b][3] = kv_pair(v[3] * 0.0625f, v[7] * 0.0625f, __half());
                    sum[b] += __shfl_xor_sync(~0u, sum[b], 1);
                    sum[b] += __shfl_xor_sync(~0u, sum[b], 2);
                    if (bad) sum[b] = NAN;       // a query that is not finite: its row is NaN
                }
                // columns of the instruction over lo: two groups, in a part per lane (or per register, of eight groups)
                auto part = [](float x, int n) {
                    float p = kv_float(kv_round<T>(x));
                    for (int k = 0; k < n; ++k) {
                        x -= p;
                        p = kv_float(kv_round<T>(x));
                    }
                    return p;
                };
                if constexpr (G == 2) {
                    ql[nt][0][0] = kv_pair(part(sum[0], j), part(sum[1], j), T());
                    ql[nt][0][1] = 0;
                } else if constexpr (G == 4) {
                    const float x = j & 1 ? sum[2] : sum[0], y = j & 1 ? sum[3] : sum[1];
                    ql[nt][0][0] = kv_pair(part(x, j >> 1), part(y, j >> 1), T());
                    ql[nt][0][1] = kv_pair(part(x, 2 + (j >> 1)), part(y, 2 + (j >> 1)), T());
                } else {
                    const float x = j & 2 ? j & 1 ? sum[6] : sum[4] : j & 1 ? sum[2] : sum[0], y = j & 2 ? j & 1 ? sum[7] : sum[5] : j & 1 ? sum[3] : sum[1];
#pragma unroll
                    for (int p = 0; p < 2; ++p)
#pragma unroll
                        for (int b = 0; b < 2; ++b) ql[nt][p][b] = kv_pair(part(x, 2 * p + b), part(y, 2 * p + b), T());
                }
                const float scale = __uint_as_float((127 - shift) << 23) * a.scale2;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    fb[nt][e] = __shfl_sync(~0u, scale, (2 * j + e) * 4);
                    m[nt][e] = -INFINITY;
                    ref[nt][e] = (float)KV_Q4_LOWEST - KV_Q4_LIFT;
                    l[nt][e] = rest[nt][e] = 0.f;
                }
#pragma unroll
                for (int b = 0; b < G; ++b) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) o[nt][b][e >> 2][e & 3] = 0.f;
                    lo[nt][b][0] = lo[nt][b][1] = 0.f;
                }
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
            float y[NT][4];
            {
                unsigned c0[G], c1[G], w0[G], w1[G];
                kv_lds(c0, stage + (slot * 4 + j) * 4 * G);
                kv_lds(c1, stage + ((slot + 8) * 4 + j) * 4 * G);
                kv_lds(w0, stage + KW + slot * 4 * G);
                kv_lds(w1, stage + KW + (slot + 8) * 4 * G);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[nt][e] = 0.f;
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    const unsigned k0[4] = {c0[g] & 0x000f000fu, c1[g] & 0x000f000fu, c0[g] & 0x00f000f0u, c1[g] & 0x00f000f0u};
                    const unsigned h0 = c0[g] >> 8, h1 = c1[g] >> 8;
                    const unsigned k1[4] = {h0 & 0x000f000fu, h1 & 0x000f000fu, h0 & 0x00f000f0u, h1 & 0x00f000f0u};
                    const float s0 = __uint_as_float(w0[g] & 0xffff0000u), s1 = __uint_as_float(w1[g] & 0xffff0000u);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        float x[4] = {0.f, 0.f, 0.f, 0.f};
                        KvMma<__half>::mma(x, k0, qf[nt][g][0], qf[nt][g][1]);
                        KvMma<__half>::mma(x, k1, qf[nt][g][2], qf[nt][g][3]);
                        y[nt][0] = fmaf(s0, x[0], y[nt][0]);
                        y[nt][1] = fmaf(s0, x[1], y[nt][1]);
                        y[nt][2] = fmaf(s1, x[2], y[nt][2]);
                        y[nt][3] = fmaf(s1, x[3], y[nt][3]);
                    }
                }
                unsigned x0, x1, z0, z1;         // the two groups of this lane's columns
                if constexpr (G == 2) x0 = w0[0], z0 = w0[1], x1 = w1[0], z1 = w1[1];
                else if constexpr (G == 4) x0 = j & 1 ? w0[2] : w0[0], z0 = j & 1 ? w0[3] : w0[1], x1 = j & 1 ? w1[2] : w1[0], z1 = j & 1 ? w1[3] : w1[1];
                else {
                    x0 = j & 2 ? j & 1 ? w0[6] : w0[4] : j & 1 ? w0[2] : w0[0], z0 = j & 2 ? j & 1 ? w0[7] : w0[5] : j & 1 ? w0[3] : w0[1];
                    x1 = j & 2 ? j & 1 ? w1[6] : w1[4] : j & 1 ? w1[2] : w1[0], z1 = j & 2 ? j & 1 ? w1[7] : w1[5] : j & 1 ? w1[3] : w1[1];
                }
                const unsigned p0 = __byte_perm(x0, z0, 0x5410), p1 = __byte_perm(x1, z1, 0x5410), kl[4] = {p0, p1, p0, p1};
                const bool on0 = mask >> slot & 1, on1 = mask >> (slot + 8) & 1;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    float x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int p = 0; p < PARTS; ++p) KvMma<T>::mma(x, kl, ql[nt][p][0], ql[nt][p][1]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[nt][e] = (e < 2 ? on0 : on1) ? fmaf(y[nt][e], 0x1p24f, x[e]) * fb[nt][e & 1] : -INFINITY;
                    if (a.scores) {
                        const int g = nt * 8 + j * 2;
                        float *to = a.scores + (((long long)tile.z * a.c.heads + h) * a.c.max_len + tile.y + slot) * a.group + g0 + g;
#pragma unroll
                        for (int b = 0; b < 2; ++b, to += 8 * a.group) {
                            if (tile.y + slot + b * 8 >= a.c.max_len) continue;
                            if ((a.group & 1) == 0 && g < heads) *(float2 *)to = make_float2(y[nt][2 * b], y[nt][2 * b + 1]);
                            else
#pragma unroll
                                for (int e = 0; e < 2; ++e)
                                    if (g + e < heads) to[e] = y[nt][2 * b + e];
                        }
                    }
                }
            }
            unsigned w0[G], w1[G];
            kv_lds(w0, stage + VW + slot * 4 * G);
            kv_lds(w1, stage + VW + (slot + 8) * 4 * G);
            if (mask != 0xffffu) {
                const bool on0 = mask >> slot & 1, on1 = mask >> (slot + 8) & 1;
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    w0[g] = on0 ? w0[g] : 0u;
                    w1[g] = on1 ? w1[g] : 0u;
                }
            }
            // the largest step of the tile: words are in the order of their steps; those of a group that is not finite do not count
            unsigned most = 0;
#pragma unroll
            for (int g = 0; g < G; ++g) most = max(most, max(w0[g], w1[g]));
            most = __reduce_max_sync(~0u, most);
            if (most >= 0x7f800000u) {
                most = 0;
#pragma unroll
                for (int g = 0; g < G; ++g) most = max(most, max(w0[g] < 0x7f800000u ? w0[g] : 0u, w1[g] < 0x7f800000u ? w1[g] : 0u));
                most = __reduce_max_sync(~0u, most);
            }
            const int step = (int)(most >> 23) - 127;
            bool moves = step > top_step;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) moves |= fmaxf(y[nt][e], y[nt][e + 2]) > m[nt][e] + KV_Q4_SLACK;
            if (__any_sync(~0u, moves)) {
                top_step = max(top_step, step);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float x = fmaxf(y[nt][e], y[nt][e + 2]);
                        x = fmaxf(x, __shfl_xor_sync(~0u, x, 4));
                        x = fmaxf(x, __shfl_xor_sync(~0u, x, 8));
                        x = fmaxf(x, __shfl_xor_sync(~0u, x, 16));
                        x = fmaxf(x, m[nt][e]);
                        const float now = kv_ref(x) + ((float)top_step - KV_Q4_LIFT), alpha = m[nt][e] == -INFINITY ? 0.f : kv_exp2(ref[nt][e] - now);
                        m[nt][e] = x;
                        ref[nt][e] = now;
                        l[nt][e] *= alpha;
                        rest[nt][e] *= alpha;
#pragma unroll
                        for (int g = 0; g < G; ++g) {
                            lo[nt][g][e] *= alpha;
#pragma unroll
                            for (int t = 0; t < 2; ++t) {
                                o[nt][g][t][e] *= alpha;
                                o[nt][g][t][e + 2] *= alpha;
                            }
                        }
                    }
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                for (int e = 0; e < 4; ++e) y[nt][e] = kv_exp2(y[nt][e] - ref[nt][e & 1]);
#pragma unroll
                for (int e = 0; e < 2; ++e) {            // compensated: weights of 2^-25 of the largest would vanish one by one
                    const float x = y[nt][e] + y[nt][e + 2] + rest[nt][e], sum = l[nt][e] + x;
                    rest[nt][e] = x - (sum - l[nt][e]);
                    l[nt][e] = sum;
                }
            }
            unsigned v[4][G / 2];
#pragma unroll
            for (int r = 0; r < 4; ++r) kv_lds(v[r], stage + VC + (j + 4 * r) * 16 * G + rho * 2 * G);
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const unsigned r0 = __byte_perm(v[0][g >> 1], v[1][g >> 1], g & 1 ? 0x7632 : 0x5410), r1 = __byte_perm(v[2][g >> 1], v[3][g >> 1], g & 1 ? 0x7632 : 0x5410);
                const unsigned v0[4] = {r0 & 0x000f000fu, r0 & 0x00f000f0u, r1 & 0x000f000fu, r1 & 0x00f000f0u};
                const unsigned h0 = r0 >> 8, h1 = r1 >> 8;
                const unsigned v1[4] = {h0 & 0x000f000fu, h0 & 0x00f000f0u, h1 & 0x000f000fu, h1 & 0x00f000f0u};
                const float s0 = __uint_as_float(w0[g] & 0xffff0000u), s1 = __uint_as_float(w1[g] & 0xffff0000u);
                const float z0 = kv_unpair(w0[g], T()).x, z1 = kv_unpair(w1[g], T()).x;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const unsigned p0 = kv_movmatrix_t(kv_pair(y[nt][0] * s0, y[nt][1] * s0, __half())), p1 = kv_movmatrix_t(kv_pair(y[nt][2] * s1, y[nt][3] * s1, __half()));
                    KvMma<__half>::mma(o[nt][g][0], v0, p0, p1);
                    KvMma<__half>::mma(o[nt][g][1], v1, p0, p1);
#pragma unroll
                    for (int e = 0; e < 2; ++e) lo[nt][g][e] = fmaf(y[nt][e], z0, fmaf(y[nt][e + 2], z1, lo[nt][g][e]));
                }
            }
        }
        else if (a.scores)           // nothing of the tile counts
            for (int e = lane; e < 16 * heads; e += 32)
                if (tile.y + e / heads < a.c.max_len)
                    a.scores[(((long long)tile.z * a.c.heads + h) * a.c.max_len + tile.y + e / heads) * a.group + g0 + e % heads] = -INFINITY;
        __syncwarp();
        take = take + 1 == a.stages ? 0 : take + 1;

        if (tile.x & 1 << 17) {      // the CTA's last step in this row
            // element 32 g + 4 rho + 2 t + b of head 2 j + e is o[g][t][2 b + e]
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    l[nt][e] += rest[nt][e];
#pragma unroll
                    for (int x = 4; x <= 16; x <<= 1) l[nt][e] += __shfl_xor_sync(~0u, l[nt][e], x);
                    m[nt][e] = l[nt][e] == 0.f ? -INFINITY : ref[nt][e];
#pragma unroll
                    for (int g = 0; g < G; ++g) {
#pragma unroll
                        for (int x = 4; x <= 16; x <<= 1) lo[nt][g][e] += __shfl_xor_sync(~0u, lo[nt][g][e], x);
#pragma unroll
                        for (int t = 0; t < 2; ++t)
#pragma unroll
                            for (int b = 0; b < 2; ++b) o[nt][g][t][2 * b + e] = fmaf(o[nt][g][t][2 * b + e], b ? 0x1p20f : 0x1p24f, lo[nt][g][e]);
                    }
                }
            const bool whole = began && (tile.x & 1 << 19);
            if (a.tw > 1) {          // the ways of a head meet in pairs
                float *box = (float *)(smem + warps * a.stages * TILE);
                for (int st = a.tw >> 1; st >= 1; st >>= 1) {
                    if (way >= st && way < 2 * st) {
                        float *to = box + ((way - st) * a.hc + hw) * kv_q4_box(G, NT) * 32 + lane;
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                to[(nt * 4 + e) * 32] = m[nt][e];
                                to[(nt * 4 + 2 + e) * 32] = l[nt][e];
                            }
#pragma unroll
                            for (int g = 0; g < G; ++g)
#pragma unroll
                                for (int e = 0; e < 8; ++e) to[(NT * 4 + (nt * G + g) * 8 + e) * 32] = o[nt][g][e >> 2][e & 3];
                        }
                    }
                    __syncthreads();
                    if (way < st) {
                        const float *from = box + (way * a.hc + hw) * kv_q4_box(G, NT) * 32 + lane;
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            float x[2], z[2];
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const float m2 = from[(nt * 4 + e) * 32], top = fmaxf(m[nt][e], m2), r = kv_ref(top);
                                x[e] = kv_exp2(m[nt][e] - r);
                                z[e] = kv_exp2(m2 - r);
                                m[nt][e] = top;
                                l[nt][e] = l[nt][e] * x[e] + from[(nt * 4 + 2 + e) * 32] * z[e];
                            }
#pragma unroll
                            for (int g = 0; g < G; ++g)
#pragma unroll
                                for (int e = 0; e < 8; ++e)
                                    o[nt][g][e >> 2][e & 3] = o[nt][g][e >> 2][e & 3] * x[e & 1] + from[(NT * 4 + (nt * G + g) * 8 + e) * 32] * z[e & 1];
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
                        const int g = nt * 8 + j * 2 + e;
                        if (g >= heads) continue;
                        const int gq = h * a.group + g0 + g;
                        if (whole) {
                            const bool none = l[nt][e] == 0.f;
                            const float inv = none ? 0.f : 1.f / l[nt][e];
                            const float lse2 = none ? -INFINITY : m[nt][e] + log2f(l[nt][e]);
                            T *to = (T *)a.out + tile.z * a.o_seq + gq * a.o_head;
#pragma unroll
                            for (int b = 0; b < G; ++b) {
                                const int d = 32 * b + 4 * rho;
                                if (d >= a.c.dim) continue;
                                float x[4];
#pragma unroll
                                for (int k = 0; k < 4; ++k) x[k] = none ? 0.f : o[nt][b][k >> 1][2 * (k & 1) + e] * inv;
                                if (a.out_vec) *(uint2 *)(to + d) = make_uint2(kv_pair(x[0], x[1], T()), kv_pair(x[2], x[3], T()));
                                else
#pragma unroll
                                    for (int k = 0; k < 4; ++k) to[d + k] = kv_round<T>(x[k]);
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
                            for (int b = 0; b < G; ++b) {
                                const int d = 32 * b + 4 * rho;
                                if (d < a.c.dim) *(float4 *)(to + d) = make_float4(o[nt][b][0][e], o[nt][b][0][2 + e], o[nt][b][1][e], o[nt][b][1][2 + e]);
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
                for (int first = sp.base + way * 16; first < sp.n; first += a.tw * 16) {
                    float add[2] = {0.f, 0.f};
#pragma unroll
                    for (int b = 0; b < 2; ++b)
                        if (first + b * 8 + slot < sp.n)
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                                for (int e = 0; e < 2; ++e) {
                                    const int g = nt * 8 + j * 2 + e;
                                    if (g < heads) add[b] += kv_exp2(from[(long long)(first + b * 8 + slot) * a.group + g] - s_lse[hw][g]);
                                }
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        add[b] += __shfl_xor_sync(~0u, add[b], 1);
                        add[b] += __shfl_xor_sync(~0u, add[b], 2);
                        const int t = first + b * 8 + slot;
                        // slots of the tile that lie before the window keep their weight, even where the sum is NaN
                        if (j == 0 && t < sp.n) a.w_out[w + t] = (a.w_in ? a.w_in[w + t] : 0.f) + (t >= sp.first ? add[b] : 0.f);
                    }
                }
                if (a.tw > 1) __syncthreads();           // the next row's sums take the place of these
                else __syncwarp();
            }
        }
    }
}
