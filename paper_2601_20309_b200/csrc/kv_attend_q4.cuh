// Attention of one new token per sequence over a paged cache in 4 bits.  The line of steps, its pieces, the rings of the warps and
// the join are those of kv_attend.cuh; what is different is a tile, 16 slots of one KV head.
//
// Mathematics.  With element = lo + s * code, and a step s and a lowest value lo per slot and group of 32 elements,
//     q . K_t  = sum_g s_tg (sum_{d in g} q_d code_td) + sum_g lo_tg Q_g,       Q_g = sum_{d in g} q_d
//     out_d    = sum_t (p_t s_tg) code_td              + sum_t p_t lo_tg
// so codes go into the matrix instructions as they are and the steps are applied to 16 x 8 results, not to elements.  A code
// becomes a float16 number by a mask alone: four bits in the lowest places of a 16-bit word are code * 2^-24, in the next four places
// code * 2^-20, both subnormal.  Eight codes cost four masks and a shift.  (The powers of two are taken back in q, in the scale, and in
// the outputs.)
//   S^T[16 slots, 8 heads] = K Q^T, one group at a time.  q is scaled by a power of two so that its largest element lies in [2^8, 2^9), and
//   becomes float16: elements are off by 2^-33 of the largest at most, odd ones, which are taken times 2^-4 on top, by 2^-29.  The sum over
//   lo is one more instruction in the cache's type, with Q_g split into up to four parts of that type (32 bits of a bf16, 22 of an f16 Q_g).
//   O^T[dim, 8 heads] = V^T (P s)^T, again by groups; p s is rounded to float16 (p itself, for the sum over lo and the row's sum, stays in
//   float32).
//   The maximum that is subtracted from the scores is taken anew only when a step's weights add up to more than 64 in a lane: a vote instead
//   of a maximum over the lanes, the sums stay what they are in exact arithmetic.
//   What keeps p s in float16's range is a unit of the sums over codes, a power of two that follows the largest p s met so far, up where
//   a larger one comes and down as the maximum rises; the row's maximum and sum, and with them lse and weights, know nothing of V, and
//   a slot without weight sets no unit.  Products below 2^-22 of the row's largest lose bits, below 2^-33 they vanish.
// f16 outputs are fine enough to show three things more, and where the type is f16 they are taken care of.  What the rounding of p s leaves goes
// through the same product.  Codes of V are -8 to 7, and lo is lo + 8 s: the two sums would take most of each other away, but not what was
// rounded.  And codes become normal numbers by the addition that this takes anyway: products of subnormal ones lose bits at their lower end
// (they seem to be placed by their exponents, which say 7 to 10 bits more than there is).  Over 131072 slots the output is 2.06e-4 off, as with
// float32 weights, without the third 2.12e-4, without the first and the third 2.8e-4; lse of one slot 2e-7 and, with subnormal codes, 1.2e-6; 22.1,
// 21.3 and 20.6 us.  In bf16 the output is 0.00178 off and 0.00171 with float32 weights, over 2000 slots 0.00171 and 0.00165: next to the output's own
// rounding that is little for 54.5 us of the 70B shape instead of 50.7 (the first alone) or 57.3 (the first and second).  The second alone (52.3)
// would give noise of 2^-13 of a group's range to outputs that are 0.
// Slots: rows 2, 3, 6 and 7 of a matrix instruction are slots 3, 2, 7 and 6 of the tile, the others their own, 8 more for the second half, so
// that the lanes' reads of K do not collide and those of V, every other row of the contraction at once, by twos only.
//
// Masked slots (beyond the length, before the window) are loaded with their tile where their block is known: codes are numbers
// whatever they hold, scores are replaced by -inf and words by 0, so nothing of such a slot reaches a sum.
//
// Split.  Eight warps compute, a KV head each where there are eight, two tiles at once: what a step costs beside its tiles (waiting,
// the vote, the compensated sum) then counts half.  Other warps load, so that those that compute need no registers for addresses.  When
// these were compared the 70B shape took 50 us so; with one tile at once 60 (495 instead of 347 instructions per tile; now 362), with every
// warp filling its own ring by 16-byte copies 67, with the scores of one step beside the sums of the one before it 60 (registers), with
// twelve computing warps 69, with rows joined by whichever CTA comes last 71 to 88 (a row of 16384 slots has 23 parts, too much for one SM).
//
// What bounds it.  70B shape, 133 MB: 51.2 us, of which 8.5 are the join, 5 the first chain of loads (lengths, block ids, first tile), 32 the line
// of steps: 4.2 TB/s.  Without any arithmetic on the tiles the call takes 41 us.  No single part of the arithmetic shows: at 51.0 us, without
// the masks (a fifth of the instructions) 51.2, without the transpositions 50.7, without the second product 49.4.
#pragma once
#include <cfloat>
#include <type_traits>

#include "kv_attend.cuh"

constexpr int KV_Q4_WARPS = 8, KV_Q4_LOADERS = 4, KV_Q4_STAGES = 6;  // warps that compute, and that load
static_assert(2 * KV_Q4_WARPS <= 16, "a lane looks after each plane of a block, two tiles per warp, and four lanes after a tile of one per warp");
constexpr float KV_Q4_SUM = 64.f;    // what the weights of a step may add up to in a lane before the maximum is taken anew
constexpr float KV_Q4_TOP = 0x1p15f; // what a product may be in the sums' unit; a new unit makes the step's largest 2^8 or more
constexpr int KV_Q4_LIFT = 8;
constexpr int KV_Q4_LOWEST = -120;   // exponent of the smallest unit: in it weights up to 2^6 stay in range

// Where sums and queries take more than 168 registers per thread, the warps that load give theirs to those that compute.  What all
// have together has to be there at the launch: kv_q4_fits
__host__ __device__ constexpr bool kv_q4_wide(int groups, int tiles) { return groups * tiles > 4; }
constexpr int KV_Q4_REGS = 224, KV_Q4_LOADER_REGS = 40;
__host__ __device__ constexpr bool kv_q4_fits(int warps, int regs) { return warps * KV_Q4_REGS + 4 * KV_Q4_LOADER_REGS <= (warps + 4) * regs; }
// tiles of 16 slots that a warp takes at once
__host__ __device__ constexpr int kv_q4_sub(int groups, int tiles) { return groups * tiles <= 4 ? 2 : 1; }
// bytes of a tile: K's and V's codes and words
__host__ __device__ constexpr int kv_q4_tile(int groups) { return 640 * groups; }
// floats of a lane that one way hands to another
__host__ __device__ constexpr int kv_q4_box(int groups, int tiles) { return tiles * (8 * groups + 4); }

// (these and kv_transpose may change places with what stands beside them, unlike those of the other kernel)
__device__ __forceinline__ void kv_mma_f16(float (&c)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void kv_mma_f16_first(float (&c)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ void kv_mma_lo(float (&c)[4], unsigned a0, unsigned a1, unsigned b0, unsigned b1, __half) { kv_mma_f16(c, a0, a1, a0, a1, b0, b1); }
__device__ __forceinline__ void kv_mma_lo(float (&c)[4], unsigned a0, unsigned a1, unsigned b0, unsigned b1, __nv_bfloat16)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%4,%5}, {%6,%7}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(b0), "r"(b1));
}

// Codes, or codes * 16, as float16 numbers of their own size: 1024 + c has c in its lowest bits, and `less`, -1024 or below, takes that away
__device__ __forceinline__ unsigned kv_codes(unsigned masked, unsigned less)
{
    const unsigned x = masked | 0x64006400u;
    const __half2 v = __hadd2(*(const __half2 *)&x, *(const __half2 *)&less);
    return *(const unsigned *)&v;
}
// what two numbers have beyond their roundings to float16, as float16
__device__ __forceinline__ unsigned kv_left(unsigned rounded, float x, float y)
{
    float a, b;
    asm("{ .reg .b16 l, h, m; mov.b32 {l, h}, %2; mov.b16 m, 0xbc00; fma.rn.f32.f16 %0, l, m, %3; fma.rn.f32.f16 %1, h, m, %4; }" : "=f"(a), "=f"(b) : "r"(rounded), "f"(x), "f"(y));
    return kv_pair(a, b, __half());
}
__device__ __forceinline__ unsigned kv_transpose(unsigned x)
{
    unsigned y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

__device__ __forceinline__ void kv_mbar_init(unsigned bar, int count) { asm volatile("mbarrier.init.shared.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void kv_mbar_arrive(unsigned bar) { asm volatile("mbarrier.arrive.shared.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void kv_mbar_expect(unsigned bar, int bytes) { asm volatile("mbarrier.arrive.expect_tx.shared.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory"); }
__device__ __forceinline__ bool kv_mbar_try(unsigned bar, unsigned parity)
{
    unsigned ok;
    asm volatile("{ .reg .pred p; mbarrier.try_wait.parity.shared.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok;
}
__device__ __forceinline__ unsigned long long kv_now()
{
    unsigned long long t;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
    return t;
}
// Nothing here waits without a limit: `polls` looks, then looks for another `ns` (0 and 0: not one).  By a whole warp, and the same for all its
// lanes: true when the phase is over, false when the limit is reached or another warp has given up before.
__device__ __forceinline__ bool kv_mbar_wait(unsigned bar, unsigned parity, unsigned polls, unsigned long long ns, const volatile int *gave_up)
{
    bool there = polls && kv_mbar_try(bar, parity);
    if (__all_sync(~0u, there)) return true;
    unsigned long long begin = 0;
    for (unsigned n = 1;; ++n) {
        bool out = gave_up && *gave_up;
        if (n >= polls) {
            const unsigned long long now = kv_now();
            if (!begin) begin = now;
            out |= now - begin >= ns;
        }
        if (__any_sync(~0u, out)) return false;
        there = there || kv_mbar_try(bar, parity);
        if (__all_sync(~0u, there)) return true;
    }
}
__device__ __forceinline__ void kv_bulk(unsigned dst, const uint8_t *src, int bytes, unsigned bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

template <typename T, int G, int NT>
__global__ void __launch_bounds__((KV_Q4_WARPS + KV_Q4_LOADERS) * 32, 1) kv_attend_q4(const __grid_constant__ KvAttend a)
{
    constexpr int PLANE = 320 * G, WORDS = 256 * G, HEADS = 8 * NT;     // bytes of a tile's plane, and of its codes
    constexpr int PARTS = G == 8 ? 2 : 1;        // matrix instructions for the sum over lo
    constexpr int SUB = kv_q4_sub(G, NT);
    constexpr bool EXACT = std::is_same<T, __half>::value;
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ int red[KV_Q4_WARPS + KV_Q4_LOADERS], s_at[2], gave_up;
    __shared__ int4 info[KV_Q4_STAGES][KV_Q4_WARPS * SUB];
    __shared__ float s_lse[KV_Q4_WARPS][HEADS];
    __shared__ __align__(8) unsigned long long bars[2][KV_Q4_STAGES];    // filled, empty
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, ways = a.tw / SUB, warps = a.hc * ways;
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

    const unsigned filled = (unsigned)__cvta_generic_to_shared(bars[0]), empty = (unsigned)__cvta_generic_to_shared(bars[1]);
    if (tid == 0) {
        gave_up = 0;
        for (int s = 0; s < a.stages; ++s) {
            kv_mbar_init(filled + 8 * s, a.block_tiles ? 1 : 1 + 32 * KV_Q4_LOADERS);
            kv_mbar_init(empty + 8 * s, warps);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }

    // ---- this CTA's piece of the line of steps: the row and step it begins at, and how many steps it has
    int pi, pch, pk;                 // sequence, row of the sequence, step
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
    __syncthreads();                 // the barriers are there
    const int k0 = pk;
    // A wait that has run out is reported, and ends the step loops of all warps: as each of them next waits, if not before.  A stage is
    // written only after all who read it have said so, so that until then every warp finds in it what it expects.
    const auto in_time = [&](unsigned bar, unsigned parity) {
        if (kv_mbar_wait(bar, parity, a.wait_polls, a.wait_ns, &gave_up)) return true;
        if (lane == 0) {
            *(volatile int *)&gave_up = 1;
            atomicOr(a.c.status, KV_OPS_TIMEOUT);
        }
        return false;
    };

    const int loader = warp - ((int)(blockDim.x >> 5) - KV_Q4_LOADERS);
    if (loader >= 0) {
        if constexpr (kv_q4_wide(G, NT)) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(KV_Q4_LOADER_REGS));
        // ---- loading.  A stage is a step.  The block ids of the next step are read while this one is on its way.  A lane looks after
        // a tile, or, where blocks do not hold whole tiles, after the eight or four rows of one that always lie in one block (blocks
        // are multiples of four rows).
        //   Where a step is made of whole blocks, K and V of a block's heads are one bulk copy each, and the stage has what the blocks have:
        // [block][K, V][KV head][codes of its tiles, words of its tiles].  One warp does that: a bulk copy takes the SM about 100 cycles,
        // whatever its size, so 64 small ones for a step of 40 KB took 6600 cycles and four take what the memory takes.
        //   Else four warps copy 16 bytes per lane: [tile][K, V][KV head][codes, words].
        if (a.block_tiles && loader > 0) return;         // (they came for their registers)
        const int stage_bytes = a.tw * a.hc * 2 * PLANE, runs = a.whole_tiles ? 1 : a.c.bs % 8 == 0 ? 2 : 4, per = 16 / runs, roles = a.tw * runs;
        const unsigned ring = (unsigned)__cvta_generic_to_shared(smem);
        const uint8_t *kbase = a.c.base + (long long)a.layer * 2 * a.c.plane_stride;
        KvSpan span(a, pi);
        int psteps = span.steps(a), id, row, put = 0;
        bool fresh = true;           // the next step begins this CTA's run in its row
        constexpr int PIECES = (40 * G + 31) / 32;
        auto peek = [&]() {          // the lane's block id in the step the cursor is at
            const int t = span.base + pk * a.tw * 16 + lane * per;
            row = -1;                // no slot of the sequence
            id = -1;
            if (lane < roles && t < span.n) {
                const int b = t / a.c.bs;
                id = a.c.tables[pi * a.c.table_stride + b];
                row = t - b * a.c.bs;
            }
        };
        peek();
        int n = 0;
        for (; n < todo; ++n) {
            const int t0 = span.base + pk * a.tw * 16, t = t0 + lane * per, lo = max(span.first - t, 0), hi = min(span.n - t, per);
            const bool ends = pk == psteps - 1;
            const int flags = (fresh ? 1 << 16 : 0) | (ends || n == todo - 1 ? 1 << 17 : 0) | (pk == 0 ? 1 << 18 : 0) | (ends ? 1 << 19 : 0);
            fresh = ends;
            const bool known = (unsigned)id < (unsigned)a.c.nb;
            unsigned mask = row >= 0 && hi > lo ? (1u << hi) - (1u << lo) : 0u;
            if (mask && !known) {
                atomicOr(a.c.status, KV_OPS_BAD_BLOCK);
                mask = 0;
            }
            const bool load = mask != 0;
            const int r = row, tiles = a.block_tiles;
            const uint8_t *from = load ? kbase + id * a.c.blk_stride + (long long)(pch / a.group_chunks * a.hc) * a.c.head_stride : a.c.base;
            if (runs > 1) {
                mask <<= per * (lane % runs);
                mask |= __shfl_xor_sync(~0u, mask, 1);
                if (runs == 4) mask |= __shfl_xor_sync(~0u, mask, 2);
            }
            const int bytes = tiles ? __popc(__ballot_sync(~0u, load && lane % max(tiles, 1) == 0)) * tiles * 2 * a.hc * PLANE : 0;
            const int4 what = make_int4((int)mask | flags, t0 + lane / runs * 16, pi, pch);
            // the cursor moves, and the next step's ids are on their way while this one is issued
            if (++pk == psteps && n + 1 < todo) {
                pk = 0;
                if (++pch == rows_of_seq) {
                    pch = 0;
                    do span = KvSpan(a, ++pi);
                    while (span.n == 0);
                    psteps = span.steps(a);
                }
            }
            if (n + 1 < todo) peek();
            if (n >= a.stages && !in_time(empty + 8 * put, (n / a.stages - 1) & 1)) break;
            if (loader == 0 && lane < roles && lane % runs == 0) info[put][lane / runs] = what;
            __syncwarp();
            const unsigned stage = ring + put * stage_bytes, bar = filled + 8 * put;
            if (loader == 0 && lane == 0) kv_mbar_expect(bar, bytes);
            __syncwarp();
            if (tiles) {
                const int block = lane >> 1, plane = lane & 1, blocks = a.tw / tiles;
                const unsigned long long p = __shfl_sync(~0u, (unsigned long long)from, block * tiles);
                const int on = __shfl_sync(~0u, (int)load, block * tiles);
                if (block < blocks && on)
                    kv_bulk(stage + lane * tiles * a.hc * PLANE, (const uint8_t *)p + (plane ? a.c.plane_stride : 0), tiles * a.hc * PLANE, bar);
            } else {
                for (int x = loader; x < a.tw * a.hc; x += KV_Q4_LOADERS) {
                    const int tile = x / a.hc, h = x - tile * a.hc;
                    const unsigned to = stage + (tile * 2 * a.hc + h) * PLANE;
#pragma unroll
                    for (int k = 0; k < PIECES; ++k) {
                        const int c = min(lane + 32 * k, 40 * G - 1), v = c >= 20 * G, in = v ? c - 20 * G : c, w = in - 16 * G;
                        // a piece of words may be of two rows: a run has four or more, so both lie in one
                        const int of = w < 0 ? in / G : w * 4 / G, role = tile * runs + of / per, size = w < 0 ? 16 * G : 4 * G;
                        const unsigned long long p = __shfl_sync(~0u, (unsigned long long)from, role);
                        const int on = __shfl_sync(~0u, (int)load, role), first_row = __shfl_sync(~0u, r, role);
                        const uint8_t *src = (const uint8_t *)p + (v ? a.c.plane_stride : 0) + (long long)h * a.c.head_stride + (w < 0 ? 0 : a.c.bs * 16 * G) +
                                             (first_row + of % per) * size + (w < 0 ? in % G * 16 : G == 8 ? w % 2 * 16 : 0);
                        if (on && lane + 32 * k < 40 * G) kv_cp16(to + (v ? a.hc * PLANE : 0) + in * 16, src, true);
                    }
                }
                asm volatile("cp.async.mbarrier.arrive.noinc.shared.b64 [%0];" ::"r"(bar) : "memory");
            }
            put = put + 1 == a.stages ? 0 : put + 1;
        }
        // the CTA does not end before its copies: whether or not anybody still waits for them, this warp does
        if (!a.block_tiles) asm volatile("cp.async.wait_all;" ::: "memory");
        else
            for (int k = max(n - a.stages, 0); k < n; ++k)
                if (!kv_mbar_wait(filled + 8 * (k % a.stages), (k / a.stages) & 1, KV_OPS_WAIT_POLLS, KV_OPS_WAIT_NS, nullptr) && lane == 0) atomicOr(a.c.status, KV_OPS_TIMEOUT);
        return;
    }

    // ---- a computing warp
    if constexpr (kv_q4_wide(G, NT)) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(KV_Q4_REGS));
    if (warp >= warps) return;
    const int hw = warp % a.hc, way = warp / a.hc, threads = warps * 32;
    // Where a wait has run out not every warp comes to a meeting any more: nobody goes to one then, and who is there already is let go by the
    // others as they leave
    auto meet = [&]() {
        if (!__any_sync(~0u, *(volatile int *)&gave_up)) asm volatile("bar.sync 1, %0;" ::"r"(threads) : "memory");
    };
    const int rho = lane >> 2, j = lane & 3, slot = rho ^ (rho >> 1 & 1);
    // where a lane reads in a plane of a tile
    const int code_at = (slot * 4 + j) * 4 * G, word_at = slot * 4 * G, v_at = (2 * j + (j & 1)) * 16 * G + rho * 2 * G, v_odd = (j & 1 ? -16 : 16) * G;
    unsigned qf[NT][G][4], ql[NT][PARTS][2];
    float fb[NT][2];
    float o[NT][G][2][4], lo[NT][G][2], m[NT][2], per[NT][2], l[NT][2], rest[NT][2];     // per: one over the unit of o; rest: what l is too coarse for
    int take = 0;
    unsigned parity = 0;
    int h = 0, g0 = 0, heads = 0;
    bool began = false;              // the run of tiles at hand begins where its row does
    // the warp's tiles in a stage: codes of the first, from tile to tile, from codes to words, from words to words, from K to V
    const int block = max(a.block_tiles, 1), in_block = way * SUB % block, stage_bytes = a.tw * a.hc * 2 * PLANE, to_v = a.hc * block * PLANE;
    const int to_next = block == 1 ? 2 * to_v : WORDS, to_words = block * WORDS - in_block * (WORDS - 64 * G), next_words = block == 1 ? to_next : 64 * G;
    const uint8_t *own = smem + ((way * SUB / block * 2 * a.hc + hw) * block) * PLANE + in_block * WORDS;
    for (int n = 0; n < todo; ++n) {
        if (!in_time(filled + 8 * take, parity)) break;
        const int4 tile = info[take][way * SUB];
        unsigned mask[SUB], some = tile.x & 0xffff, all = some;
        mask[0] = some;
#pragma unroll
        for (int u = 1; u < SUB; ++u) {
            mask[u] = info[take][way * SUB + u].x & 0xffff;
            some |= mask[u];
            all &= mask[u];
        }
        const uint8_t *kt = own + take * stage_bytes;
        if (tile.x & 1 << 16) {
            h = tile.w / a.group_chunks * a.hc + hw;
            g0 = tile.w % a.group_chunks * HEADS;
            heads = min(HEADS, a.group - g0);
            began = tile.x & 1 << 18;
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
                const float by = a.scale2 < 0.f ? -__uint_as_float((127 + shift) << 23) : __uint_as_float((127 + shift) << 23);
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
                    if (!EXACT) sum[b] *= 0x1p-24f;      // the codes' unit; float16 has no room for that
                    if (bad) sum[b] = NAN;       // a query that is not finite: its row is NaN
                }
                // columns of the instruction over lo: two groups, in a part per lane (or per register, of eight groups)
                auto part = [](float x, int n) {
                    const float a0 = kv_float(kv_round<T>(x)), x1 = x - a0, a1 = kv_float(kv_round<T>(x1)), x2 = x1 - a1, a2 = kv_float(kv_round<T>(x2));
                    return n & 2 ? n & 1 ? x2 - a2 : a2 : n & 1 ? a1 : a0;
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
                const float scale = __uint_as_float((127 - shift) << 23) * fabsf(a.scale2) * (EXACT ? 1.f : 0x1p24f);
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    fb[nt][e] = __shfl_sync(~0u, scale, (2 * j + e) * 4);
                    m[nt][e] = -FLT_MAX;             // any score moves it, -inf does not
                    per[nt][e] = __uint_as_float((127 - KV_Q4_LOWEST) << 23);
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
        if (some) {
            float y[SUB][NT][4];
#pragma unroll
            for (int u = 0; u < SUB; ++u) {
                const uint8_t *at = kt + u * to_next;
                const auto even = [](unsigned x) { return EXACT ? kv_codes(x & 0x000f000fu, 0xe400e400u) : x & 0x000f000fu; };
                const auto odd = [](unsigned x) { return EXACT ? kv_codes(x & 0x00f000f0u, 0xe400e400u) : x & 0x00f000f0u; };
                unsigned c0[G], c1[G], w0[G], w1[G];
                kv_words(c0, at + code_at);
                kv_words(c1, at + code_at + 128 * G);
                kv_words(w0, kt + to_words + u * next_words + word_at);
                kv_words(w1, kt + to_words + u * next_words + word_at + 32 * G);
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    const unsigned h0 = c0[g] >> 8, h1 = c1[g] >> 8;
                    const float s0 = __uint_as_float(w0[g] & 0xffff0000u), s1 = __uint_as_float(w1[g] & 0xffff0000u);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        float x[4];
                        kv_mma_f16_first(x, even(c0[g]), even(c1[g]), odd(c0[g]), odd(c1[g]), qf[nt][g][0], qf[nt][g][1]);
                        kv_mma_f16(x, even(h0), even(h1), odd(h0), odd(h1), qf[nt][g][2], qf[nt][g][3]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) y[u][nt][e] = g == 0 ? (e < 2 ? s0 : s1) * x[e] : fmaf(e < 2 ? s0 : s1, x[e], y[u][nt][e]);
                    }
                }
                unsigned x0, x1, z0, z1;         // the two groups of this lane's columns
                if constexpr (G == 2) x0 = w0[0], z0 = w0[1], x1 = w1[0], z1 = w1[1];
                else if constexpr (G == 4) x0 = j & 1 ? w0[2] : w0[0], z0 = j & 1 ? w0[3] : w0[1], x1 = j & 1 ? w1[2] : w1[0], z1 = j & 1 ? w1[3] : w1[1];
                else {
                    x0 = j & 2 ? j & 1 ? w0[6] : w0[4] : j & 1 ? w0[2] : w0[0], z0 = j & 2 ? j & 1 ? w0[7] : w0[5] : j & 1 ? w0[3] : w0[1];
                    x1 = j & 2 ? j & 1 ? w1[6] : w1[4] : j & 1 ? w1[2] : w1[0], z1 = j & 2 ? j & 1 ? w1[7] : w1[5] : j & 1 ? w1[3] : w1[1];
                }
                const unsigned p0 = __byte_perm(x0, z0, 0x5410), p1 = __byte_perm(x1, z1, 0x5410);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                    for (int p = 0; p < PARTS; ++p) kv_mma_lo(y[u][nt], p0, p1, ql[nt][p][0], ql[nt][p][1], T());
                }
            }
            // the scores are rounded here, so that the largest less the maximum is 0 whatever its size.  (Masked
            // slots become -inf after that: a factor may be 0)
#pragma unroll
            for (int u = 0; u < SUB; ++u)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[u][nt][e] *= fb[nt][e & 1];
            unsigned w0[SUB][G], w1[SUB][G];
#pragma unroll
            for (int u = 0; u < SUB; ++u) {
                kv_words(w0[u], kt + to_v + to_words + u * next_words + word_at);
                kv_words(w1[u], kt + to_v + to_words + u * next_words + word_at + 32 * G);
            }
            if (all != 0xffffu)
#pragma unroll
                for (int u = 0; u < SUB; ++u) {
                    const bool on0 = mask[u] >> slot & 1, on1 = mask[u] >> (slot + 8) & 1;
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) y[u][nt][e] = (e < 2 ? on0 : on1) ? y[u][nt][e] : -INFINITY;
#pragma unroll
                    for (int g = 0; g < G; ++g) {
                        w0[u][g] = on0 ? w0[u][g] : 0u;
                        w1[u][g] = on1 ? w1[u][g] : 0u;
                    }
                }
            if (a.scores)
#pragma unroll
                for (int u = 0; u < SUB; ++u)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        const int g = nt * 8 + j * 2, t = tile.y + 16 * u + slot;
                        float *to = a.scores + (((long long)tile.z * a.c.heads + h) * a.c.max_len + t) * a.group + g0 + g;
#pragma unroll
                        for (int b = 0; b < 2; ++b, to += 8 * a.group) {
                            if (t + b * 8 >= a.c.max_len) continue;
                            if ((a.group & 1) == 0 && g < heads) *(float2 *)to = make_float2(y[u][nt][2 * b], y[u][nt][2 * b + 1]);
                            else {
                                if (g < heads) to[0] = y[u][nt][2 * b];
                                if (g + 1 < heads) to[1] = y[u][nt][2 * b + 1];
                            }
                        }
                    }
            // the largest step of each of the lane's slots (as its word, 2^-7 above it at most); groups that are not finite do not count
            float big[SUB][2], most = 0.f;
#pragma unroll
            for (int u = 0; u < SUB; ++u) {
                big[u][0] = big[u][1] = 0.f;
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    big[u][0] = fmaxf(big[u][0], __uint_as_float(w0[u][g]));
                    big[u][1] = fmaxf(big[u][1], __uint_as_float(w1[u][g]));
                }
                most = fmaxf(most, fmaxf(big[u][0], big[u][1]));
            }
            float p[SUB][NT][4], sum[NT][2];
#pragma unroll
            for (int u = 0; u < SUB; ++u)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) p[u][nt][e] = kv_exp2(y[u][nt][e] - m[nt][e & 1]);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    sum[nt][e] = p[0][nt][e] + p[0][nt][e + 2];
#pragma unroll
                    for (int u = 1; u < SUB; ++u) sum[nt][e] += p[u][nt][e] + p[u][nt][e + 2];
                }
            // no product is above the lane's sum times its largest step (each of them looked at takes the 70B shape 0.3 us more)
            bool moves = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) moves |= sum[nt][e] > KV_Q4_SUM || sum[nt][e] * per[nt][e] * most > KV_Q4_TOP;
            if (__any_sync(~0u, moves))
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float top = m[nt][e], part = 0.f;
#pragma unroll
                        for (int u = 0; u < SUB; ++u) top = fmaxf(top, fmaxf(y[u][nt][e], y[u][nt][e + 2]));
#pragma unroll
                        for (int x = 4; x <= 16; x <<= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, x));
                        top = ceilf(top);            // factors between maxima and between units are powers of two: nothing is rounded
#pragma unroll
                        for (int u = 0; u < SUB; ++u)
#pragma unroll
                            for (int b = 0; b < 2; ++b) {
                                p[u][nt][2 * b + e] = kv_exp2(y[u][nt][2 * b + e] - top);
                                part = fmaxf(part, p[u][nt][2 * b + e] * big[u][b]);
                            }
                        sum[nt][e] = p[0][nt][e] + p[0][nt][e + 2];
#pragma unroll
                        for (int u = 1; u < SUB; ++u) sum[nt][e] += p[u][nt][e] + p[u][nt][e + 2];
#pragma unroll
                        for (int x = 4; x <= 16; x <<= 1) part = fmaxf(part, __shfl_xor_sync(~0u, part, x));
                        const float rise = top - m[nt][e];
                        const int unit = 127 - (int)(__float_as_uint(per[nt][e]) >> 23),
                                  now = max(max(unit - (int)fminf(rise, 1000.f), KV_Q4_LOWEST), (int)(__float_as_uint(part) >> 23) - 127 - KV_Q4_LIFT);
                        const float alpha = kv_exp2(-rise), beta = kv_exp2((float)(unit - now) - rise);
                        m[nt][e] = top;
                        per[nt][e] = __uint_as_float((127 - now) << 23);
                        l[nt][e] *= alpha;
                        rest[nt][e] *= alpha;
#pragma unroll
                        for (int g = 0; g < G; ++g) {
                            lo[nt][g][e] *= alpha;
#pragma unroll
                            for (int t = 0; t < 2; ++t) {
                                o[nt][g][t][e] *= beta;
                                o[nt][g][t][e + 2] *= beta;
                            }
                        }
                    }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {            // compensated: weights of 2^-25 of the largest would vanish one by one
                    const float x = sum[nt][e] + rest[nt][e], total = l[nt][e] + x;
                    rest[nt][e] = x - (total - l[nt][e]);
                    l[nt][e] = total;
                }
#pragma unroll
            for (int u = 0; u < SUB; ++u) {
                const auto even = [](unsigned x) { return EXACT ? kv_codes(x & 0x000f000fu, 0xe408e408u) : x & 0x000f000fu; };     // -1032
                const auto odd = [](unsigned x) { return EXACT ? kv_codes(x & 0x00f000f0u, 0xe480e480u) : x & 0x00f000f0u; };      // -1152
                unsigned v[4][G / 2];
#pragma unroll
                for (int r = 0; r < 4; ++r) kv_words(v[r], kt + to_v + u * to_next + v_at + (r & 1 ? v_odd : 0) + r / 2 * 128 * G);
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    const unsigned r0 = __byte_perm(v[0][g >> 1], v[1][g >> 1], g & 1 ? 0x7632 : 0x5410), r1 = __byte_perm(v[2][g >> 1], v[3][g >> 1], g & 1 ? 0x7632 : 0x5410);
                    const unsigned h0 = r0 >> 8, h1 = r1 >> 8;
                    const float s0 = __uint_as_float(w0[u][g] & 0xffff0000u), s1 = __uint_as_float(w1[u][g] & 0xffff0000u);
                    float z0 = kv_unpair(w0[u][g], T()).x, z1 = kv_unpair(w1[u][g], T()).x;
                    if constexpr (EXACT) {
                        z0 = fmaf(8.f, s0, z0);
                        z1 = fmaf(8.f, s1, z1);
                    }
                    const unsigned a0 = even(r0), a1 = odd(r0), a2 = even(r1), a3 = odd(r1), b0 = even(h0), b1 = odd(h0), b2 = even(h1), b3 = odd(h1);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        const float(&q)[4] = p[u][nt];
                        const float x0 = q[0] * per[nt][0] * s0, x1 = q[1] * per[nt][1] * s0, x2 = q[2] * per[nt][0] * s1, x3 = q[3] * per[nt][1] * s1;
                        const unsigned lower = kv_pair(x0, x1, __half()), upper = kv_pair(x2, x3, __half());
                        unsigned p0 = kv_transpose(lower), p1 = kv_transpose(upper);
                        kv_mma_f16(o[nt][g][0], a0, a1, a2, a3, p0, p1);
                        kv_mma_f16(o[nt][g][1], b0, b1, b2, b3, p0, p1);
                        if constexpr (EXACT) {
                            p0 = kv_transpose(kv_left(lower, x0, x1));
                            p1 = kv_transpose(kv_left(upper, x2, x3));
                            kv_mma_f16(o[nt][g][0], a0, a1, a2, a3, p0, p1);
                            kv_mma_f16(o[nt][g][1], b0, b1, b2, b3, p0, p1);
                        }
#pragma unroll
                        for (int e = 0; e < 2; ++e) lo[nt][g][e] = fmaf(q[e], z0, fmaf(q[e + 2], z1, lo[nt][g][e]));
                    }
                }
            }
        }
        else if (a.scores)           // nothing of the tiles counts
            for (int e = lane; e < 16 * SUB * heads; e += 32)
                if (tile.y + e / heads < a.c.max_len)
                    a.scores[(((long long)tile.z * a.c.heads + h) * a.c.max_len + tile.y + e / heads) * a.group + g0 + e % heads] = -INFINITY;
        __syncwarp();
        if (lane == 0) kv_mbar_arrive(empty + 8 * take);
        if (++take == a.stages) {
            take = 0;
            parity ^= 1;
        }

        if (tile.x & 1 << 17) {      // the CTA's last step in this row
            // element 32 g + 4 rho + 2 t + b of head 2 j + e is o[g][t][2 b + e]
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    l[nt][e] += rest[nt][e];
#pragma unroll
                    for (int x = 4; x <= 16; x <<= 1) l[nt][e] += __shfl_xor_sync(~0u, l[nt][e], x);
                    if (l[nt][e] == 0.f) m[nt][e] = -INFINITY;
                    const float unit = __uint_as_float((254u << 23) - __float_as_uint(per[nt][e]));
#pragma unroll
                    for (int g = 0; g < G; ++g) {
#pragma unroll
                        for (int x = 4; x <= 16; x <<= 1) lo[nt][g][e] += __shfl_xor_sync(~0u, lo[nt][g][e], x);
#pragma unroll
                        for (int t = 0; t < 2; ++t)
#pragma unroll
                            for (int b = 0; b < 2; ++b) o[nt][g][t][2 * b + e] = fmaf(o[nt][g][t][2 * b + e] * (EXACT ? b ? 0x1p-4f : 1.f : b ? 0x1p20f : 0x1p24f), unit, lo[nt][g][e]);
                    }
                }
            const bool whole = began && (tile.x & 1 << 19);
            if (ways > 1) {          // the ways of a head meet in pairs
                float *box = (float *)(smem + a.stages * a.tw * a.hc * 2 * PLANE);
                for (int st = ways >> 1; st >= 1; st >>= 1) {
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
                    meet();
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
                    meet();
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
                if (ways > 1) meet();
                else __syncwarp();
                const KvSpan sp(a, tile.z);
                const float *from = a.scores + ((long long)tile.z * a.c.heads + h) * a.c.max_len * a.group;
                const long long w = tile.z * a.w_seq + h * a.w_head;
                for (int t = way * 32 + lane; t < sp.base; t += ways * 32) a.w_out[w + t] = a.w_in ? a.w_in[w + t] : 0.f;
                for (int base = sp.base + way * 16 * SUB; base < sp.n; base += a.tw * 16)
#pragma unroll 1
                    for (int first = base; first < base + 16 * SUB; first += 16) {
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
                if (ways > 1) meet();           // the next row's sums take the place of these
                else __syncwarp();
            }
        }
    }
    if (__any_sync(~0u, *(volatile int *)&gave_up)) asm volatile("bar.arrive 1, %0;" ::"r"(threads) : "memory");
}
