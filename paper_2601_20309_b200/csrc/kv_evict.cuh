// Eviction by accumulated attention weight: `keep` slots stay, and only those at or above `keep` move, into the holes
// the evicted ones leave below it.  Sources (>= keep) and holes (< keep) never meet, so the moves need no order, and
// in a steady state (keep + d slots) at most d rows move, where closing the gaps would move nearly all.
//
// A problem is one (layer, sequence, KV head).  kv_evict_select reads weight and age of every slot once, as one 32-bit key
// in a register (16 per thread; a cluster of up to eight CTAs shares a long problem), and finds the key of rank `keep`
// two bits at a time: three candidates are counted per round (one packed warp reduction, one barrier; in a cluster one
// exchange through distributed shared memory), until exactly `keep` keys reach the candidate or at most EV_CANDS keys
// agree with it so far; among those one warp finds the rest.  No histogram: the keys of positive weights share their upper bits, and atomics on one bin would queue.
// Ballots then number the holes and the sources in slot order, and the pairs meet through two short lists.
//
// What bounds it: the rows that move, 4*dim bytes read and written each.  With problems for all SMs the same CTA moves its
// rows, while others select; with few, a second kernel spreads them over the GPU.
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
    int problems, slots;     // slots: how many problems' lists the workspace holds
    int fused;               // kv_evict_select moves the rows itself
    int units_shift;         // log2 of a row's 16-byte units in K and V together, or -1
    int *count;              // [slot]: rows that move
    int *holes, *srcs;       // [slot][cap]
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

constexpr int EV_KEYS = 16, EV_CLUSTER = 8, EV_CANDS = 256, EV_MOVE_THREADS = 256, EV_MOVE_ROWS = 64;

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
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// sums over a CTA and over its cluster; `before` = over the cluster's lower CTAs
template <int THREADS> struct KvSums {
    int (*red)[THREADS / 32];        // [2 * 3]: by turn and value
    int4 (*table)[EV_CLUSTER];       // [2]
    int rank, size, turn;
    // `warps`: every lane already has its warp's sums
    __device__ __forceinline__ void add(int &x, int &y, int &z, int *before_x, int *before_y, bool warps)
    {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, buf = turn & 1;
        ++turn;
        if (!warps) {
            x = __reduce_add_sync(~0u, x);
            y = __reduce_add_sync(~0u, y);
            z = __reduce_add_sync(~0u, z);
        }
        if (lane == 0) {
            red[buf * 3][warp] = x;
            red[buf * 3 + 1][warp] = y;
            red[buf * 3 + 2][warp] = z;
        }
        __syncthreads();
        const bool on = lane < THREADS / 32;
        x = __reduce_add_sync(~0u, on ? red[buf * 3][lane] : 0);
        y = __reduce_add_sync(~0u, on ? red[buf * 3 + 1][lane] : 0);
        z = __reduce_add_sync(~0u, on ? red[buf * 3 + 2][lane] : 0);
        if (before_x) *before_x = *before_y = 0;
        if (size == 1) return;
        if ((int)threadIdx.x < size) {
            const unsigned mine = (unsigned)__cvta_generic_to_shared(&table[buf][rank]);
            unsigned there;
            asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(mine), "r"(threadIdx.x));
            asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(there), "r"(x), "r"(y), "r"(z), "r"(0) : "memory");
        }
        kv_cluster_sync();
        x = y = z = 0;
        for (int r = 0; r < size; ++r) {
            const int4 v = table[buf][r];
            if (before_x && r < rank) {
                *before_x += v.x;
                *before_y += v.y;
            }
            x += v.x;
            y += v.y;
            z += v.z;
        }
    }
};

// a problem's list from row j0 on, BATCH rows and then `step` further
template <int THREADS, int BATCH>
__device__ __forceinline__ void kv_evict_rows(const KvEvict &a, const KvProblem &p, int slot, int n, int j0, int step, ulonglong2 *way)
{
    const int tid = threadIdx.x, half = a.c.dim / 8, units = 2 * half;
    const long long plane = (a.first_layer + p.l) * 2 * a.c.plane_stride + (long long)p.h * a.c.head_stride;
    auto unit = [&](int u) { return u < half ? u * 16ll : a.c.plane_stride + (u - half) * 16; };
    const long long own = unit(tid & (units - 1));       // a power of two of units: a thread always has the same
    for (int j = j0; j < n; j += step) {
        const int m = min(n - j, BATCH);
        if (tid < m) {
            const int d = a.holes[(long long)slot * a.cap + j + tid], s = a.srcs[(long long)slot * a.cap + j + tid];
            a.w_out[p.to + d] = a.w[p.at + s];
            if (a.order_out) a.order_out[p.to + d] = a.order[p.at + s];
            const uint8_t *from = a.c.slot(p.i, s, 0), *into = a.c.slot(p.i, d, 0);
            const bool ok = from && into;        // a bad block id: the row stays where it is
            way[tid] = make_ulonglong2(ok ? (unsigned long long)from + plane : 0, (unsigned long long)into + plane);
        }
        __syncthreads();
        // 16 bytes per thread and load, four loads in flight before their stores
        for (int e = tid; e < m * units; e += 4 * THREADS) {
            uint4 v[4];
            uint8_t *to[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int f = e + q * THREADS, r = a.units_shift >= 0 ? f >> a.units_shift : f / units;
                const long long off = a.units_shift >= 0 ? own : unit(f - r * units);
                to[q] = nullptr;
                if (f < m * units) {
                    const ulonglong2 w = way[r];
                    if (w.x) {
                        v[q] = __ldcs((const uint4 *)(w.x + off));
                        to[q] = (uint8_t *)(w.y + off);
                    }
                }
            }
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (to[q]) *(uint4 *)to[q] = v[q];
        }
        __syncthreads();
    }
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
    __shared__ int red[6][WARPS];
    __shared__ int4 table[2][EV_CLUSTER];
    __shared__ int place[EV_KEYS * WARPS];
    __shared__ ulonglong2 way[THREADS];
    __shared__ unsigned cand[EV_CANDS], s_top;
    __shared__ int s_base, s_count;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    unsigned rank, size;
    asm("mov.u32 %0, %cluster_ctarank;" : "=r"(rank));
    asm("mov.u32 %0, %cluster_nctaid.x;" : "=r"(size));
    KvSums<THREADS> sums{red, table, (int)rank, (int)size, 0};
    if (size > 1) kv_cluster_sync();             // every CTA of the cluster is there before anyone writes into its memory
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int slot = blockIdx.x / size;
    for (int pi = slot; pi < a.problems; pi += a.slots) {
        const KvProblem p(a, pi);
        const bool apart = a.w_out != a.w;
        if (p.l == 0 && p.h == 0 && rank == 0 && tid == 0 && a.lens_out) a.lens_out[p.i] = min(p.n, a.keep);
        if (p.n <= a.keep) {
            if (apart)
                for (int t = rank * THREADS + tid; t < p.n; t += size * THREADS) {
                    a.w_out[p.to + t] = a.w[p.at + t];
                    if (a.order_out) a.order_out[p.to + t] = a.order[p.at + t];
                }
            if (rank == 0 && tid == 0) a.count[slot] = 0;
            continue;
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

        // ---- the largest key that at least `keep` keys reach; `over` keys lie above all that agree with it so far
        unsigned top = 0;
        int reach = p.n, over = 0, shift = 32;
        while (shift > 0 && reach != a.keep && reach - over > EV_CANDS) {
            shift -= 2;
            int x = 0, y = 0, z = 0;
            for (int r0 = 0; r0 < rounds; r0 += EV_KEYS) {
                if (!REGS) load(r0, false);
                unsigned packed = 0;             // at most 16 keys a thread, 512 a warp: ten bits each
#pragma unroll
                for (int r = 0; r < EV_KEYS; ++r)
                    if (r0 + r < rounds) {
                        packed += key[r] >= (top | 1u << shift) ? 1u : 0u;
                        packed += key[r] >= (top | 2u << shift) ? 1u << 10 : 0u;
                        packed += key[r] >= (top | 3u << shift) ? 1u << 20 : 0u;
                    }
                if (REGS) packed = __reduce_add_sync(~0u, packed);
                x += packed & 1023;
                y += packed >> 10 & 1023;
                z += packed >> 20;
            }
            sums.add(x, y, z, nullptr, nullptr, REGS);
            if (z >= a.keep) top |= 3u << shift, reach = z;
            else if (y >= a.keep) top |= 2u << shift, reach = y, over = z;
            else if (x >= a.keep) top |= 1u << shift, reach = x, over = y;
            else over = x;
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
                int mine = s_count, none = 0, zero = 0, before, b;
                if (tid) mine = 0;
                sums.add(mine, none, zero, &before, &b, false);
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
            int none = 0, zero = 0, b;
            for (int r0 = 0; r0 < rounds; r0 += EV_KEYS) {
                if (!REGS) load(r0, false);
#pragma unroll
                for (int r = 0; r < EV_KEYS; ++r) ties += r0 + r < rounds && base + (r0 + r) * THREADS + tid < p.n && key[r] == top;
            }
            sums.add(ties, none, zero, &ties_run, &b, false);
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
            int holes = 0, srcs = 0, zero = 0;
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
            sums.add(holes, srcs, zero, &holes_run, &srcs_run, false);
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
                int holes = tid == 0 ? s_base & 0xffff : 0, srcs = tid == 0 ? (int)((unsigned)s_base >> 16) : 0, zero = 0;
                sums.add(holes, srcs, zero, &holes_run, &srcs_run, false);
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
        if (a.fused) {
            if (size > 1) kv_cluster_sync();     // the lists are whole
            else __syncthreads();
            kv_evict_rows<THREADS, THREADS>(a, p, slot, moves, rank * THREADS, size * THREADS, way);
            if (size > 1) kv_cluster_sync();     // and no longer read
        }
    }
    if (size > 1) kv_cluster_sync();             // nobody leaves while others may still write into its memory
}

// few problems: their rows spread over the GPU.  CTA (problem, part of its list)
__global__ void __launch_bounds__(EV_MOVE_THREADS) kv_evict_move(const __grid_constant__ KvEvict a)
{
    __shared__ ulonglong2 way[EV_MOVE_ROWS];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const KvProblem p(a, blockIdx.x);
    kv_evict_rows<EV_MOVE_THREADS, EV_MOVE_ROWS>(a, p, blockIdx.x, a.count[blockIdx.x], blockIdx.y * EV_MOVE_ROWS, gridDim.y * EV_MOVE_ROWS, way);
}
