// Eviction by accumulated attention weight: `keep` slots stay, and only those at or above `keep` move, into the holes
// the evicted ones leave below it.  Sources (>= keep) and holes (< keep) never meet, so the moves need no order, and
// in a steady state (keep + d slots) at most d rows move, where closing the gaps would move nearly all.
//
// A problem is one (layer, sequence, KV head).  Weight and age of every slot are read once and become one 32-bit key.  The key
// of rank `keep` is found by digits of ten bits from above: the keys that agree so far are counted by their next digit
// in shared memory, one warp picks the digit, and as soon as at most EV_CANDS keys are left it finds the rest among
// them alone.  Ballots then number the holes and the sources in slot order, and the pairs meet through two short lists.
//   kv_evict_small    four warps per problem, keys in shared memory: many problems on an SM at once.  For short problems, and
//                     for many; next to no rows it moves itself.
//   kv_evict_select   one CTA of 256 or 1024 threads per problem, keys in registers, or a cluster of up to eight that exchange their counts
//                     through distributed shared memory.
//   kv_evict_move     the rows, spread over the GPU: 32 pairs per warp, eight 16-byte loads per lane in flight.
//
// What bounds it: the rows that move, 4*dim bytes read and written each, in pieces of 256 bytes at random places (5.3 to 6
// TB/s); beside them the instructions of the selection, which no longer depend on how many bits the weights share; for few
// short problems the chain of loads.
//
// Measured: 32 layers x 8 sequences x 8 heads of 128, 2304 -> 2048 slots, 452 MB: 110 us (selection 36, rows 70), 63 % of the
// floor; moving the rows in the selecting CTA, 256 threads each, took 125, two bits a round without digits 130, one kernel
// after the other in the first form 284.  4 x 3 x 8 heads, 16384 -> 4096: 77 us (22 + 51; counting in clusters 99).  One problem of
// 131072 slots: 34 us.  16 problems of 100 slots: 7.7 us.
#pragma once
#include "kv_ops.cuh"

struct KvEvict {
    KvView c;
    int first_layer, layers, seqs, keep, recent, sink;
    const float *w;
    const int *order;
    long long m_layer, m_seq, m_head;
    const int *seen;
    float *w_out;
    int *order_out;
    long long o_layer, o_seq, o_head;
    int *lens_out;
    int problems;
    int fused;               // kv_evict_small moves the rows itself
    int quads;               // weights and ages may be read and written four at a time
    int units_shift;         // log2 of a row's 16-byte units in K and V together, or -1
    int *count;              // [problem]: rows that move
    int *holes, *srcs;       // [problem][cap]
    int cap;
};

// weights as integers of the same order: NaN lowest, -0 equal to +0, protected slots above everything
__device__ __forceinline__ unsigned kv_evict_key(float w, bool held)
{
    if (held) return 0xFFFFFFFFu;
    if (isnan(w)) return 0u;
    const unsigned u = __float_as_uint(w + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

constexpr int EV_KEYS = 16, EV_CLUSTER = 8, EV_CANDS = 256, EV_BINS = 1024 + 32, EV_MOVE_WARPS = 8,
              EV_SMALL_THREADS = 128, EV_SMALL_SLOTS = 8192, EV_FUSED_ROWS = 64;

struct KvProblem {
    int h, i, l, n;
    long long at, to;        // first weight, first weight out
    __device__ __forceinline__ KvProblem(const KvEvict &a, int p)
    {
        h = p % a.c.heads;
        i = p / a.c.heads % a.seqs;
        l = p / a.c.heads / a.seqs;
        n = a.c.len(i);
        at = l * a.m_layer + i * a.m_seq + h * a.m_head;
        to = l * a.o_layer + i * a.o_seq + h * a.o_head;
    }
};

__device__ __forceinline__ void kv_cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}

// sums over a CTA and over its cluster; `before` = over the cluster's lower CTAs
template <int THREADS> struct KvSums {
    int (*red)[THREADS / 32];        // [2 * 2]: by turn and value
    int2 (*table)[EV_CLUSTER];       // [2]
    int rank, size, turn;
    __device__ __forceinline__ void add(int &x, int &y, int *before_x, int *before_y)
    {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, buf = turn & 1;
        ++turn;
        x = __reduce_add_sync(~0u, x);
        y = __reduce_add_sync(~0u, y);
        if (lane == 0) {
            red[buf * 2][warp] = x;
            red[buf * 2 + 1][warp] = y;
        }
        __syncthreads();
        const bool on = lane < THREADS / 32;
        x = __reduce_add_sync(~0u, on ? red[buf * 2][lane] : 0);
        y = __reduce_add_sync(~0u, on ? red[buf * 2 + 1][lane] : 0);
        *before_x = *before_y = 0;
        if (size == 1) return;
        if ((int)threadIdx.x < size) {
            const unsigned mine = (unsigned)__cvta_generic_to_shared(&table[buf][rank]);
            unsigned there;
            asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(mine), "r"(threadIdx.x));
            asm volatile("st.shared::cluster.v2.b32 [%0], {%1, %2};" ::"r"(there), "r"(x), "r"(y) : "memory");
        }
        kv_cluster_sync();
        x = y = 0;
        for (int r = 0; r < size; ++r) {
            const int2 v = table[buf][r];
            if (r < rank) {
                *before_x += v.x;
                *before_y += v.y;
            }
            x += v.x;
            y += v.y;
        }
    }
};

// Rows of up to 32 pairs, by one warp: lane q has the q-th pair (slot d < keep, slot s >= keep).
struct KvWays {
    ulonglong2 row[32];      // K of the source and of the hole, or 0
    int2 words[32];          // in 4 bits: from there to the rows' words
};

__device__ __forceinline__ void kv_evict_units(const KvEvict &a, int m, const KvWays &way)
{
    const int lane = threadIdx.x & 31, half = a.c.dim / 8, units = 2 * half;
    for (int e = lane; e < m * units; e += 32 * 8) {
        uint4 v[8];
        uint8_t *to[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const int f = e + q * 32, r = a.units_shift >= 0 ? f >> a.units_shift : f / units, u = f - r * units;
            to[q] = nullptr;
            if (f < m * units) {
                const ulonglong2 w = way.row[r];
                const long long off = u < half ? u * 16 : a.c.plane_stride + (u - half) * 16;
                if (w.x) {
                    v[q] = __ldcg((const uint4 *)(w.x + off));
                    to[q] = (uint8_t *)(w.y + off);
                }
            }
        }
#pragma unroll
        for (int q = 0; q < 8; ++q)
            if (to[q]) *(uint4 *)to[q] = v[q];
    }
}

// The same in 4 bits.  K's and V's codes and words of a row are ten units of U (twenty of 16 bytes for eight groups); a lane has the same
// unit of every third row (every row).  `box`: where the rows wait between reading and writing, so that all of them are on their way
// at once and few registers are needed (in registers 107 us for 32 layers and 8 sequences in a steady state, so 93); without
// one (few rows) three at a time
constexpr int EV_BOX = 5120;
template <typename U> __device__ __forceinline__ void kv_evict_units_q4(const KvEvict &a, int m, const KvWays &way, uint8_t *box)
{
    const int lane = threadIdx.x & 31, codes = a.c.groups * 16 / (int)sizeof(U), half = a.c.groups * 20 / (int)sizeof(U), units = 2 * half, abreast = 32 / units;
    const int r0 = lane / units, u = lane - r0 * units, in = u < half ? u : u - half;
    const long long plane = u < half ? 0 : a.c.plane_stride;
    const bool word = in >= codes;
    const int off = (word ? in - codes : in) * (int)sizeof(U);
    if (box) {
        const unsigned to = (unsigned)__cvta_generic_to_shared(box);
        const int most = EV_BOX / (units * (int)sizeof(U));
        for (int first = 0; first < m; first += most) {
            const int end = min(m, first + most);
            if (r0 < abreast)
                for (int r = first + r0; r < end; r += abreast)
                    if (way.row[r].x)
                        asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(to + ((r - first) * units + u) * (int)sizeof(U)),
                                     "l"(way.row[r].x + plane + off + (word ? way.words[r].x : 0)), "n"((int)sizeof(U))
                                     : "memory");
            asm volatile("cp.async.commit_group;\ncp.async.wait_group 0;" ::: "memory");
            if (r0 < abreast)        // every lane writes what it read itself
                for (int r = first + r0; r < end; r += abreast)
                    if (way.row[r].x) *(U *)(way.row[r].y + plane + off + (word ? way.words[r].y : 0)) = *(const U *)(box + ((r - first) * units + u) * (int)sizeof(U));
        }
        return;
    }
    for (int r = r0; r < m; r += 3 * abreast) {
        U v[3];
#pragma unroll
        for (int q = 0; q < 3; ++q)
            if (const int k = r + q * abreast; r0 < abreast && k < m && way.row[k].x) v[q] = __ldcg((const U *)(way.row[k].x + plane + off + (word ? way.words[k].x : 0)));
#pragma unroll
        for (int q = 0; q < 3; ++q)
            if (const int k = r + q * abreast; r0 < abreast && k < m && way.row[k].x) *(U *)(way.row[k].y + plane + off + (word ? way.words[k].y : 0)) = v[q];
    }
}

template <bool Q4>
__device__ __forceinline__ void kv_evict_rows(const KvEvict &a, const KvProblem &p, int m, int d, int s, KvWays &way, uint8_t *box = nullptr)
{
    const int lane = threadIdx.x & 31;
    if (lane < m) {
        const uint8_t *from = a.c.slot(p.i, s, 0), *into = a.c.slot(p.i, d, 0);
        const long long plane = (a.first_layer + p.l) * 2 * a.c.plane_stride + (long long)p.h * a.c.head_stride;
        const bool ok = from && into;            // a bad block id: the row stays where it is
        way.row[lane] = make_ulonglong2(ok ? (unsigned long long)from + plane : 0, ok ? (unsigned long long)into + plane : 0);
        if (Q4) way.words[lane] = make_int2(a.c.to_words(s), a.c.to_words(d));
        if (ok) {
            a.w_out[p.to + d] = a.w[p.at + s];
            if (a.order_out) a.order_out[p.to + d] = a.order[p.at + s];
        }
    }
    __syncwarp();
    if constexpr (!Q4) kv_evict_units(a, m, way);
    else if (a.c.groups == 2) kv_evict_units_q4<uint2>(a, m, way, box);  // words of two groups: 8 bytes
    else kv_evict_units_q4<uint4>(a, m, way, box);
    __syncwarp();
}

// Counts by digit: 32 digits per lane, each lane's shifted by one bank.
__device__ __forceinline__ int kv_evict_bin(int digit) { return digit + (digit >> 5); }

// The digit that the key of rank `want` from above has, by one warp: how many keys have a larger one, how many have it.
__device__ __forceinline__ int kv_evict_pick(const int *bins, int want, int &larger, int &equal)
{
    const int lane = threadIdx.x & 31;
    // first which 32 digits, then which of them
    int s = 0;
#pragma unroll 8
    for (int k = 0; k < 32; ++k) s += bins[lane * 33 + k];
    int x = s;                       // of this lane and those above it
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_down_sync(~0u, x, o);
        if (lane + o < 32) x += y;
    }
    const int block = __ffs(__ballot_sync(~0u, x - s < want && want <= x)) - 1, above = __shfl_sync(~0u, x - s, block);
    const int c = bins[block * 33 + lane];
    x = c;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_down_sync(~0u, x, o);
        if (lane + o < 32) x += y;
    }
    const int one = __ffs(__ballot_sync(~0u, above + x - c < want && want <= above + x)) - 1;
    larger = above + __shfl_sync(~0u, x - c, one);
    equal = __shfl_sync(~0u, c, one);
    return block * 32 + one;
}

// The key of rank `want` from above among m <= EV_CANDS keys that agree in the bits above `shift`, found by one warp; `top` has
// those bits.  Returns how many of them reach it.
__device__ __forceinline__ int kv_evict_among(const unsigned *cand, int m, int want, int shift, unsigned &top)
{
    const int lane = threadIdx.x & 31;
    unsigned key[EV_CANDS / 32];
#pragma unroll
    for (int r = 0; r < EV_CANDS / 32; ++r) key[r] = r * 32 + lane < m ? cand[r * 32 + lane] : 0u;
    int reach = m;
    for (shift -= 2; shift >= 0 && reach != want; shift -= 2) {
        unsigned packed = 0;
#pragma unroll
        for (int r = 0; r < EV_CANDS / 32; ++r) {
            packed += key[r] >= (top | 1u << shift) ? 1u : 0u;
            packed += key[r] >= (top | 2u << shift) ? 1u << 10 : 0u;
            packed += key[r] >= (top | 3u << shift) ? 1u << 20 : 0u;
        }
        packed = __reduce_add_sync(~0u, packed);         // at most EV_CANDS each: ten bits do
        const int x = packed & 1023, y = packed >> 10 & 1023, z = packed >> 20;
        if (z >= want) top |= 3u << shift, reach = z;
        else if (y >= want) top |= 2u << shift, reach = y;
        else if (x >= want) top |= 1u << shift, reach = x;
    }
    return reach;
}

template <int THREADS, bool REGS>
__global__ void __launch_bounds__(THREADS, THREADS == 256 ? 4 : 1) kv_evict_select(const __grid_constant__ KvEvict a)
{
    constexpr int WARPS = THREADS / 32;
    __shared__ int red[4][WARPS];
    __shared__ int2 table[2][EV_CLUSTER];
    __shared__ int place[EV_KEYS * WARPS];
    __shared__ unsigned cand[EV_CANDS], s_top;
    __shared__ int s_base, s_count, bins[EV_BINS], all_bins[THREADS == 1024 ? EV_BINS : 1];
    __shared__ int3 s_pick;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    unsigned rank, size;
    asm("mov.u32 %0, %cluster_ctarank;" : "=r"(rank));
    asm("mov.u32 %0, %cluster_nctaid.x;" : "=r"(size));
    KvSums<THREADS> sums{red, table, (int)rank, (int)size, 0};
    if (size > 1) kv_cluster_sync();             // every CTA of the cluster is there before anyone writes into its memory
    const int slot = blockIdx.x / size;
    const KvProblem p(a, slot);
    const bool apart = a.w_out != a.w;
    if (p.l == 0 && p.h == 0 && rank == 0 && tid == 0 && a.lens_out) a.lens_out[p.i] = min(p.n, a.keep);
    if (p.n <= a.keep) {
        if (apart)
            for (int t = rank * THREADS + tid; t < p.n; t += size * THREADS) {
                a.w_out[p.to + t] = a.w[p.at + t];
                if (a.order_out) a.order_out[p.to + t] = a.order[p.at + t];
            }
        if (rank == 0 && tid == 0) a.count[slot] = 0;
        return;
    }
    // ---- this CTA's slots: `rounds` times THREADS, side by side
    const int newest = (a.seen ? a.seen[p.i] : p.n) - a.recent;
    const int base = rank * (REGS ? EV_KEYS : (p.n + size * THREADS - 1) / (size * THREADS)) * THREADS;
    const int rounds = max(0, min(REGS ? EV_KEYS : (p.n + (int)size * THREADS - 1) / ((int)size * THREADS), (p.n - base + THREADS - 1) / THREADS));
    unsigned key[EV_KEYS];
    // the keys of rounds r0 .. r0 + 15; a slot beyond the length gets 0, which no candidate reaches
    auto load = [&](int r0, bool copy) {
        float w[EV_KEYS];
        int age[EV_KEYS];
#pragma unroll
        for (int r = 0; r < EV_KEYS; ++r) {
            const int t = base + (r0 + r) * THREADS + tid;
            const bool on = r0 + r < rounds && t < p.n;
            w[r] = on ? a.w[p.at + t] : 0.f;
            age[r] = on ? a.order ? a.order[p.at + t] : t : 0;
        }
#pragma unroll
        for (int r = 0; r < EV_KEYS; ++r) {
            const int t = base + (r0 + r) * THREADS + tid;
            const bool on = r0 + r < rounds && t < p.n;
            key[r] = on ? kv_evict_key(w[r], age[r] >= newest || age[r] < a.sink) : 0u;
            if (copy && on && t < a.keep) {  // holes are overwritten by what moves there
                a.w_out[p.to + t] = w[r];
                if (a.order_out) a.order_out[p.to + t] = age[r];
            }
        }
    };
    if (REGS) load(0, apart);
    else if (apart)
        for (int r0 = 0; r0 < rounds; r0 += EV_KEYS) load(r0, true);

    // ---- the key of rank `keep`: `top` as far as it is known, above `shift`; `over` keys are larger, `reach` at least as large
    unsigned top = 0;
    int reach = p.n, over = 0, shift = 32;
    while (shift > 0 && reach != a.keep && reach - over > EV_CANDS) {
        const int width = min(10, shift);
        for (int d = tid; d < EV_BINS; d += THREADS) bins[d] = 0;
        __syncthreads();
        for (int r0 = 0; r0 < rounds; r0 += EV_KEYS) {
            if (!REGS) load(r0, false);
#pragma unroll
            for (int r = 0; r < EV_KEYS; ++r)
                if (r0 + r < rounds) {
                    const bool in = base + (r0 + r) * THREADS + tid < p.n && (shift == 32 || (key[r] ^ top) >> shift == 0);
                    if (in) atomicAdd(&bins[kv_evict_bin(key[r] >> (shift - width) & ((1 << width) - 1))], 1);
                }
        }
        int *counts = bins;
        if (size > 1) {                      // the whole cluster's: every CTA adds all of them up for itself
            kv_cluster_sync();
            for (int d = tid; d < EV_BINS; d += THREADS) {
                int sum = 0;
                for (unsigned r = 0; r < size; ++r) {
                    unsigned there;
                    int v;
                    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"((unsigned)__cvta_generic_to_shared(&bins[d])), "r"(r));
                    asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(v) : "r"(there) : "memory");
                    sum += v;
                }
                all_bins[d] = sum;
            }
            kv_cluster_sync();               // nobody clears counts that others still read
            counts = all_bins;
        } else {
            __syncthreads();
        }
        if (warp == 0) {
            int larger, equal;
            const int digit = kv_evict_pick(counts, a.keep - over, larger, equal);
            if (lane == 0) s_pick = make_int3(digit, larger, equal);
        }
        __syncthreads();
        shift -= width;
        top |= (unsigned)s_pick.x << shift;
        over += s_pick.y;
        reach = over + s_pick.z;
    }
    if (shift > 0 && reach != a.keep) {      // few keys are left: one warp finds the rest among them alone
        if (tid == 0) s_count = 0;
        __syncthreads();
        for (int r0 = 0; r0 < rounds; r0 += EV_KEYS) {
            if (!REGS) load(r0, false);
#pragma unroll
            for (int r = 0; r < EV_KEYS; ++r)
                if (r0 + r < rounds) {
                    // a full shift only where nothing was counted yet: all keys agree
                    const bool in = base + (r0 + r) * THREADS + tid < p.n && (shift == 32 || (key[r] ^ top) >> shift == 0);
                    if (in) cand[atomicAdd(&s_count, 1)] = key[r];
                }
        }
        __syncthreads();
        const int m = reach - over;
        if (size > 1) {                      // every CTA gets the others' too
            int mine = s_count, none = 0, before, b;
            if (tid) mine = 0;
            sums.add(mine, none, &before, &b);
            const int own = s_count;
            const unsigned x = tid < own ? cand[tid] : 0u;
            kv_cluster_sync();               // all have read their own
            if (tid < own)
                for (unsigned r = 0; r < size; ++r) {
                    unsigned there;
                    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"((unsigned)__cvta_generic_to_shared(&cand[before + tid])), "r"(r));
                    asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(there), "r"(x) : "memory");
                }
            kv_cluster_sync();
        }
        if (warp == 0) {
            const int n = kv_evict_among(cand, m, a.keep - over, shift, top);
            if (lane == 0) {
                s_top = top;
                s_count = n;
            }
        }
        __syncthreads();
        top = s_top;
        reach = over + s_count;
    }
    // ---- equals of the last one: the lowest slots stay.  `spare` of them do not; equals are numbered only where some go
    const int spare = reach - a.keep;
    int ties = 0, ties_run = 0;
    if (spare > 0) {
        int none = 0, b;
        for (int r0 = 0; r0 < rounds; r0 += EV_KEYS) {
            if (!REGS) load(r0, false);
#pragma unroll
            for (int r = 0; r < EV_KEYS; ++r) ties += r0 + r < rounds && base + (r0 + r) * THREADS + tid < p.n && key[r] == top;
        }
        sums.add(ties, none, &ties_run, &b);
    }
    const int stay_ties = ties - spare;      // of the equals, in slot order
    // ---- lists, numbered in slot order: the slots of a group of 16 rounds by round, warp and lane
    // `place`: counts by round and warp become the sums in front of them; their total goes to s_base
    auto number = [&]() {
        __syncthreads();
        if (warp == 0) {
            constexpr int PER = EV_KEYS * WARPS / 32;
            int v[PER], s = 0;
#pragma unroll
            for (int q = 0; q < PER; ++q) {
                v[q] = s;
                s += place[lane * PER + q];
            }
            int x = s;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(~0u, x, o);
                if (lane >= o) x += y;
            }
#pragma unroll
            for (int q = 0; q < PER; ++q) place[lane * PER + q] = x - s + v[q];
            if (lane == 31) s_base = x;
        }
        __syncthreads();
    };
    const unsigned below = (1u << lane) - 1;
    // the equals of rounds r0 .. that do not stay, as a bit per round
    auto leavers = [&](int r0) {
        unsigned gone = 0;
        if (spare > 0) {
#pragma unroll
            for (int r = 0; r < EV_KEYS; ++r) {
                const unsigned vote = __ballot_sync(~0u, r0 + r < rounds && base + (r0 + r) * THREADS + tid < p.n && key[r] == top);
                if (lane == 0) place[r * WARPS + warp] = __popc(vote);
            }
            number();
#pragma unroll
            for (int r = 0; r < EV_KEYS; ++r) {
                const bool tie = r0 + r < rounds && base + (r0 + r) * THREADS + tid < p.n && key[r] == top;
                const unsigned vote = __ballot_sync(~0u, tie);
                if (tie && ties_run + place[r * WARPS + warp] + __popc(vote & below) >= stay_ties) gone |= 1u << r;
            }
            ties_run += s_base;
            __syncthreads();
        }
        return gone;
    };
    // whether the slot of round r is a hole or a source, as the warp's vote; its lanes below `keep` (`low`) can only be holes
    auto vote = [&](int r, int t, unsigned gone, unsigned &low) {
        const int k = a.keep - (t - lane);
        low = k >= 32 ? ~0u : k <= 0 ? 0u : (1u << k) - 1;
        const bool stays = key[r] >= top && !(gone >> r & 1);
        return __ballot_sync(~0u, t < p.n && (t < a.keep) != stays);
    };
    int holes_run = 0, srcs_run = 0, moves = 0;
    if (!REGS && size > 1) {                 // every CTA counts its own first, to know where its numbers begin
        const int ties_from = ties_run;
        int holes = 0, srcs = 0;
        for (int r0 = 0; r0 < rounds; r0 += EV_KEYS) {
            load(r0, false);
            const unsigned gone = leavers(r0);
#pragma unroll
            for (int r = 0; r < EV_KEYS; ++r)
                if (r0 + r < rounds) {
                    unsigned low;
                    const unsigned v = vote(r, base + (r0 + r) * THREADS + tid, gone, low);
                    holes += v & low & 1u << lane ? 1 : 0;
                    srcs += v & ~low & 1u << lane ? 1 : 0;
                }
        }
        sums.add(holes, srcs, &holes_run, &srcs_run);
        moves = holes;
        ties_run = ties_from;
    }
    for (int r0 = 0; r0 < rounds || (REGS && r0 == 0); r0 += EV_KEYS) {
        if (!REGS) load(r0, false);
        const unsigned gone = leavers(r0);
#pragma unroll
        for (int r = 0; r < EV_KEYS; ++r) {
            unsigned v = 0, low = 0;
            if (r0 + r < rounds) v = vote(r, base + (r0 + r) * THREADS + tid, gone, low);
            if (lane == 0) place[r * WARPS + warp] = __popc(v & low) | __popc(v & ~low) << 16;    // at most 16 * THREADS of each
        }
        number();
        if (REGS && size > 1) {
            int holes = tid == 0 ? s_base & 0xffff : 0, srcs = tid == 0 ? (int)((unsigned)s_base >> 16) : 0;
            sums.add(holes, srcs, &holes_run, &srcs_run);
            moves = holes;
        }
#pragma unroll
        for (int r = 0; r < EV_KEYS; ++r)
            if (r0 + r < rounds) {
                const int t = base + (r0 + r) * THREADS + tid;
                unsigned low;
                const unsigned v = vote(r, t, gone, low), at = place[r * WARPS + warp];
                if (v >> lane & 1) {
                    int *list = low >> lane & 1 ? a.holes + holes_run + (at & 0xffff) + __popc(v & low & below)
                                                : a.srcs + srcs_run + (at >> 16) + __popc(v & ~low & below);
                    list[(long long)slot * a.cap] = t;
                }
            }
        holes_run += s_base & 0xffff;
        srcs_run += (unsigned)s_base >> 16;
        __syncthreads();
    }
    if (size == 1) moves = holes_run;
    if (rank == 0 && tid == 0) a.count[slot] = moves;
    if (size > 1) kv_cluster_sync();             // nobody leaves while others may still write into its memory
}

template <bool Q4> __global__ void __launch_bounds__(EV_SMALL_THREADS) kv_evict_small(const __grid_constant__ KvEvict a)
{
    constexpr int THREADS = EV_SMALL_THREADS, WARPS = THREADS / 32;
    extern __shared__ __align__(16) unsigned keys[];     // [max_len rounded up to 4 * THREADS]
    __shared__ unsigned cand[EV_CANDS], s_top;
    __shared__ int bins[EV_BINS], s_count, s_ties[WARPS], s_lists[2 * EV_FUSED_ROWS];
    __shared__ int2 s_moves[WARPS];
    __shared__ int3 s_pick;
    __shared__ KvWays way[WARPS];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const KvProblem p(a, blockIdx.x);
    const bool apart = a.w_out != a.w, stay = p.n <= a.keep;
    if (tid == 0) {
        if (p.l == 0 && p.h == 0 && a.lens_out) a.lens_out[p.i] = min(p.n, a.keep);
        if (stay && !a.fused) a.count[blockIdx.x] = 0;
        s_count = 0;
    }
    const int newest = (a.seen ? a.seen[p.i] : p.n) - a.recent, padded = (p.n + 4 * THREADS - 1) / (4 * THREADS) * (4 * THREADS);
    if (stay && !apart) return;
    for (int d = tid; d < EV_BINS; d += THREADS) bins[d] = 0;
    // four slots at a time where the arrays are aligned; eight per thread in flight
    if (a.quads) {
        for (int t0 = tid * 4; t0 < padded; t0 += THREADS * 4 * 2) {
            float4 w[2];
            int4 age[2];
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int t = t0 + r * THREADS * 4;      // rows are whole quads: the last may reach past the length
                w[r] = t < p.n ? *(const float4 *)(a.w + p.at + t) : make_float4(0.f, 0.f, 0.f, 0.f);
                age[r] = t < p.n && a.order ? *(const int4 *)(a.order + p.at + t) : make_int4(t, t + 1, t + 2, t + 3);
            }
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int t = t0 + r * THREADS * 4;
                if (t >= padded) continue;
                auto key = [&](int e, float x, int y) { return t + e < p.n ? kv_evict_key(x, y >= newest || y < a.sink) : 0u; };
                *(uint4 *)(keys + t) = make_uint4(key(0, w[r].x, age[r].x), key(1, w[r].y, age[r].y), key(2, w[r].z, age[r].z), key(3, w[r].w, age[r].w));
                if (!apart) continue;
                if (t + 3 < min(p.n, a.keep)) {          // holes are overwritten by what moves there
                    *(float4 *)(a.w_out + p.to + t) = w[r];
                    if (a.order_out) *(int4 *)(a.order_out + p.to + t) = age[r];
                } else {
                    const float x[4] = {w[r].x, w[r].y, w[r].z, w[r].w};
                    const int y[4] = {age[r].x, age[r].y, age[r].z, age[r].w};
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (t + e < min(p.n, a.keep)) {
                            a.w_out[p.to + t + e] = x[e];
                            if (a.order_out) a.order_out[p.to + t + e] = y[e];
                        }
                }
            }
        }
    } else {
        for (int t0 = tid; t0 < padded; t0 += THREADS * 8) {
            float w[8];
            int age[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                const int t = t0 + r * THREADS;
                w[r] = t < p.n ? a.w[p.at + t] : 0.f;
                age[r] = t < p.n ? a.order ? a.order[p.at + t] : t : 0;
            }
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                const int t = t0 + r * THREADS;
                if (t < padded) keys[t] = t < p.n ? kv_evict_key(w[r], age[r] >= newest || age[r] < a.sink) : 0u;
                if (apart && t < min(p.n, a.keep)) {
                    a.w_out[p.to + t] = w[r];
                    if (a.order_out) a.order_out[p.to + t] = age[r];
                }
            }
        }
    }
    if (stay) return;
    __syncthreads();
    const unsigned below = (1u << lane) - 1;
    // ---- the key of rank `keep`, as kv_evict_select finds it
    unsigned top = 0;
    int reach = p.n, over = 0, shift = 32;
    while (shift > 0 && reach != a.keep && reach - over > EV_CANDS) {
        const int width = min(10, shift);
        if (shift < 32) {
            for (int d = tid; d < EV_BINS; d += THREADS) bins[d] = 0;
            __syncthreads();
        }
#pragma unroll 4
        for (int t = tid; t < padded; t += THREADS) {
            const unsigned k = keys[t];
            if (t < p.n && (shift == 32 || (k ^ top) >> shift == 0)) atomicAdd(&bins[kv_evict_bin(k >> (shift - width) & ((1 << width) - 1))], 1);
        }
        __syncthreads();
        if (warp == 0) {
            int larger, equal;
            const int digit = kv_evict_pick(bins, a.keep - over, larger, equal);
            if (lane == 0) s_pick = make_int3(digit, larger, equal);
        }
        __syncthreads();
        shift -= width;
        top |= (unsigned)s_pick.x << shift;
        over += s_pick.y;
        reach = over + s_pick.z;
    }
    if (shift > 0 && reach != a.keep) {
#pragma unroll 4
        for (int t = tid; t < padded; t += THREADS) {
            const unsigned k = keys[t];
            if (t < p.n && (shift == 32 || (k ^ top) >> shift == 0)) cand[atomicAdd(&s_count, 1)] = k;
        }
        __syncthreads();
        if (warp == 0) {
            const int n = kv_evict_among(cand, reach - over, a.keep - over, shift, top);
            if (lane == 0) {
                s_top = top;
                s_count = n;
            }
        }
        __syncthreads();
        top = s_top;
        reach = over + s_count;
    }
    // ---- lists, numbered in slot order.  Every warp has a run of slots; 32 of them vote at a time (a hole or a source, which
    // of the two goes by `keep`), and lane r keeps the vote of round r, to number and write down its slots later
    const int spare = reach - a.keep, run = padded / WARPS, from = warp * run;
    int ties = 0, stay_ties = 0;     // equals of the last key in front of this warp's run; how many of all stay
    if (spare > 0) {
        int mine = 0, all = 0;
        for (int t = from + lane; t < from + run; t += 32) mine += t < p.n && keys[t] == top;
        mine = __reduce_add_sync(~0u, mine);
        if (lane == 0) s_ties[warp] = mine;
        __syncthreads();
        for (int w = 0; w < WARPS; ++w) {
            if (w < warp) ties += s_ties[w];
            all += s_ties[w];
        }
        stay_ties = all - spare;
    }
    constexpr int GROUPS = EV_SMALL_SLOTS / WARPS / 1024;        // of 32 rounds
    unsigned votes[GROUPS];
    int2 mine = make_int2(0, 0);
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
        votes[g] = 0;
        const int rounds = min(32, run / 32 - g * 32);
#pragma unroll 4
        for (int r = 0; r < rounds; ++r) {
            const int t = from + g * 1024 + r * 32 + lane;
            const unsigned k = keys[t];
            bool stays = k >= top;
            if (spare > 0) {
                const bool tie = t < p.n && k == top;
                const unsigned v = __ballot_sync(~0u, tie);
                if (tie && ties + __popc(v & below) >= stay_ties) stays = false;
                ties += __popc(v);
            }
            const unsigned v = __ballot_sync(~0u, t < p.n && (t < a.keep) != stays);
            if (lane == r) votes[g] = v;
        }
    }
    auto low = [&](int g) {          // which of the round's slots lie below `keep`
        const int c = a.keep - (from + g * 1024 + lane * 32);
        return c >= 32 ? ~0u : c <= 0 ? 0u : (1u << c) - 1;
    };
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
        mine.x += __popc(votes[g] & low(g));
        mine.y += __popc(votes[g] & ~low(g));
    }
    mine.x = __reduce_add_sync(~0u, mine.x);
    mine.y = __reduce_add_sync(~0u, mine.y);
    if (lane == 0) s_moves[warp] = mine;
    __syncthreads();
    int holes = 0, sources = 0, moves = 0;
    for (int w = 0; w < WARPS; ++w) {
        if (w < warp) {
            holes += s_moves[w].x;
            sources += s_moves[w].y;
        }
        moves += s_moves[w].x;
    }
    int *hole_list = a.fused ? s_lists : a.holes + (long long)blockIdx.x * a.cap, *source_list = a.fused ? s_lists + EV_FUSED_ROWS : a.srcs + (long long)blockIdx.x * a.cap;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
        if (g * 1024 >= run) break;
        unsigned h = votes[g] & low(g), s = votes[g] & ~low(g);
        int x = __popc(h) | __popc(s) << 16;             // of this round and those in front of it: at most 1024 of each
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(~0u, x, o);
            if (lane >= o) x += y;
        }
        const int total = __shfl_sync(~0u, x, 31), t0 = from + g * 1024 + lane * 32;
        int *to = hole_list + holes + (x & 0xffff) - __popc(h);
        for (; h; h &= h - 1) *to++ = t0 + __ffs(h) - 1;
        to = source_list + sources + (x >> 16) - __popc(s);
        for (; s; s &= s - 1) *to++ = t0 + __ffs(s) - 1;
        holes += total & 0xffff;
        sources += total >> 16;
    }
    if (!a.fused) {
        if (tid == 0) a.count[blockIdx.x] = moves;
        return;
    }
    __syncthreads();
    for (int j = warp * 8; j < moves; j += WARPS * 8) {  // eight rows per warp: few as they are, all warps have some
        const int at = min(j + lane, moves - 1);
        kv_evict_rows<Q4>(a, p, min(moves - j, 8), s_lists[at], s_lists[EV_FUSED_ROWS + at], way[warp]);
    }
}

// rows x * 32 .. of problems y * EV_MOVE_WARPS .., a warp each: neighbouring KV heads move neighbouring slots together
template <bool Q4> __global__ void __launch_bounds__(EV_MOVE_WARPS * 32) kv_evict_move(const __grid_constant__ KvEvict a)
{
    __shared__ KvWays way[EV_MOVE_WARPS];
    __shared__ __align__(16) uint8_t box[Q4 ? EV_MOVE_WARPS : 1][Q4 ? EV_BOX : 16];
    const int warp = threadIdx.x >> 5, j = blockIdx.x * 32, lane = threadIdx.x & 31;
    for (int y = blockIdx.y * EV_MOVE_WARPS + warp; y < a.problems; y += gridDim.y * EV_MOVE_WARPS) {
        const int n = a.count[y];
        if (j >= n) continue;
        const KvProblem p(a, y);
        const int at = min(j + lane, n - 1);
        kv_evict_rows<Q4>(a, p, min(n - j, 32), a.holes[(long long)y * a.cap + at], a.srcs[(long long)y * a.cap + at], way[warp], Q4 ? box[warp] : nullptr);
    }
}
