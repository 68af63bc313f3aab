// Eviction by accumulated attention weight: `keep` slots stay, and only those at or above `keep` move, into the holes
// the evicted ones leave below it.  Sources (>= keep) and holes (< keep) never meet, so the moves need no order, and
// in a steady state (keep + d slots) at most d rows move, where closing the gaps would move nearly all.
//
// A problem is one (layer, sequence, KV head).  kv_evict_select reads weight and age of every slot once, as one 32-bit key
// in a register (16 per thread; a cluster of up to eight CTAs shares a long problem), and finds the key of rank `keep`
// two bits at a time: three candidates are counted per round (one packed warp reduction, one barrier; in a cluster one
// exchange through distributed shared memory), until exactly `keep` keys lie at or above the candidate or all bits are
// found.  No histogram: the keys of positive weights share their upper bits, and atomics on one bin would queue.
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

constexpr int EV_KEYS = 16, EV_CLUSTER = 8, EV_MOVE_THREADS = 256, EV_MOVE_ROWS = 64;

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
    __device__ __forceinline__ void add(int &x, int &y, int &z, int *before_x, int *before_y)
    {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, buf = turn & 1;
        ++turn;
        x = __reduce_add_sync(~0u, x);
        y = __reduce_add_sync(~0u, y);
        z = __reduce_add_sync(~0u, z);
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
                const int f = e + q * THREADS, r = a.units_shift >= 0 ? f >> a.units_shift : f / units, u = f - r * units;
                to[q] = nullptr;
                if (f < m * units) {
                    const ulonglong2 w = way[r];
                    const long long off = u < half ? u * 16 : a.c.plane_stride + (u - half) * 16;
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

template <int THREADS, bool REGS>
__global__ void __launch_bounds__(THREADS, THREADS == 256 ? 4 : 1) kv_evict_select(const __grid_constant__ KvEvict a)
{
    constexpr int WARPS = THREADS / 32;
    __shared__ int red[6][WARPS];
    __shared__ int4 table[2][EV_CLUSTER];
    __shared__ int place[EV_KEYS * WARPS];
    __shared__ ulonglong2 way[THREADS];
    __shared__ int s_base;
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
        const int rounds = REGS ? EV_KEYS : (p.n + size * THREADS - 1) / (size * THREADS), base = rank * rounds * THREADS;
        unsigned key[EV_KEYS];
        // the keys of rounds r0 .. r0 + 15; slots beyond the length get 0, which no candidate reaches
        auto load = [&](int r0, bool copy) {
            float w[EV_KEYS];
            int age[EV_KEYS];
#pragma unroll
            for (int r = 0; r < EV_KEYS; ++r) {
                const int t = base + (r0 + r) * THREADS + tid;
                const bool on = t < p.n && (REGS || r0 + r < rounds);
                w[r] = on ? a.w[p.at + t] : 0.f;
                age[r] = on ? a.order ? a.order[p.at + t] : t : 0;
            }
#pragma unroll
            for (int r = 0; r < EV_KEYS; ++r) {
                const int t = base + (r0 + r) * THREADS + tid;
                const bool on = t < p.n && (REGS || r0 + r < rounds);
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

        // ---- the largest key that at least `keep` keys reach
        unsigned top = 0;
        int reach = p.n;
        for (int shift = 30; shift >= 0 && reach != a.keep; shift -= 2) {
            int x = 0, y = 0, z = 0;
            for (int r0 = 0; r0 < rounds; r0 += EV_KEYS) {
                if (!REGS) load(r0, false);
                unsigned packed = 0;             // at most 16 keys a thread, 512 a warp: ten bits each
#pragma unroll
                for (int r = 0; r < EV_KEYS; ++r) {
                    packed += key[r] >= (top | 1u << shift) ? 1u : 0u;
                    packed += key[r] >= (top | 2u << shift) ? 1u << 10 : 0u;
                    packed += key[r] >= (top | 3u << shift) ? 1u << 20 : 0u;
                }
                x += packed & 1023;
                y += packed >> 10 & 1023;
                z += packed >> 20;
            }
            sums.add(x, y, z, nullptr, nullptr);
            if (z >= a.keep) top |= 3u << shift, reach = z;
            else if (y >= a.keep) top |= 2u << shift, reach = y;
            else if (x >= a.keep) top |= 1u << shift, reach = x;
        }
        // ---- equals of the last one: the lowest slots stay.  `spare` of them do not; ties are numbered only where some go
        const int spare = reach - a.keep;
        int ties = 0, ties_before = 0;
        if (spare > 0) {
            int none = 0, zero = 0, b;
            for (int r0 = 0; r0 < rounds; r0 += EV_KEYS) {
                if (!REGS) load(r0, false);
#pragma unroll
                for (int r = 0; r < EV_KEYS; ++r) ties += base + (r0 + r) * THREADS + tid < p.n && (REGS || r0 + r < rounds) && key[r] == top;
            }
            sums.add(ties, none, zero, &ties_before, &b);
        }
        const int stay_ties = ties - spare;      // of the equals, in slot order
        // ---- lists, numbered in slot order: the slots of a group of 16 rounds by round, warp and lane.  In a cluster every
        // CTA first counts its own, to know where its numbers begin
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
        int holes_run = 0, srcs_run = 0, moves = 0;
        for (int pass = size > 1 ? 0 : 1; pass < 2; ++pass) {
            int holes = 0, srcs = 0, ties_run = ties_before;
            for (int r0 = 0; r0 < rounds; r0 += EV_KEYS) {
                if (!REGS) load(r0, false);
                auto live = [&](int r) { return base + (r0 + r) * THREADS + tid < p.n && (REGS || r0 + r < rounds); };
                unsigned gone = 0;               // bit r: the slot of round r is an equal that does not stay
                if (spare > 0) {
#pragma unroll
                    for (int r = 0; r < EV_KEYS; ++r) {
                        const unsigned vote = __ballot_sync(~0u, live(r) && key[r] == top);
                        if (lane == 0) place[r * WARPS + warp] = __popc(vote);
                    }
                    number();
#pragma unroll
                    for (int r = 0; r < EV_KEYS; ++r) {
                        const bool tie = live(r) && key[r] == top;
                        const unsigned vote = __ballot_sync(~0u, tie);
                        if (tie && ties_run + place[r * WARPS + warp] + __popc(vote & below) >= stay_ties) gone |= 1u << r;
                    }
                    ties_run += s_base;
                    __syncthreads();
                }
                auto hole = [&](int r) { return live(r) && base + (r0 + r) * THREADS + tid < a.keep && (key[r] < top || (gone >> r & 1)); };
                auto source = [&](int r) { return live(r) && base + (r0 + r) * THREADS + tid >= a.keep && key[r] >= top && !(gone >> r & 1); };
                if (pass == 0) {
#pragma unroll
                    for (int r = 0; r < EV_KEYS; ++r) {
                        holes += hole(r);
                        srcs += source(r);
                    }
                    continue;
                }
#pragma unroll
                for (int r = 0; r < EV_KEYS; ++r) {
                    const unsigned h = __ballot_sync(~0u, hole(r)), s = __ballot_sync(~0u, source(r));
                    if (lane == 0) place[r * WARPS + warp] = __popc(h) | __popc(s) << 16;    // at most 16 * THREADS of each
                }
                number();
#pragma unroll
                for (int r = 0; r < EV_KEYS; ++r) {
                    const bool is_hole = hole(r), is_source = source(r);
                    const unsigned h = __ballot_sync(~0u, is_hole), s = __ballot_sync(~0u, is_source), at = place[r * WARPS + warp];
                    const int t = base + (r0 + r) * THREADS + tid;
                    if (is_hole) a.holes[(long long)slot * a.cap + holes_run + (at & 0xffff) + __popc(h & below)] = t;
                    if (is_source) a.srcs[(long long)slot * a.cap + srcs_run + (at >> 16) + __popc(s & below)] = t;
                }
                holes_run += s_base & 0xffff;
                srcs_run += (unsigned)s_base >> 16;
                __syncthreads();
            }
            if (pass == 0) {
                int zero = 0;
                sums.add(holes, srcs, zero, &holes_run, &srcs_run);
                moves = holes;
            } else if (size == 1) {
                moves = holes_run;
            }
        }
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
