// What the kernels on the device cache share: the address rule of a layer's slots, the element types, the status
// word.  Slot s of sequence i lies in row s % bs of block table[i][s / bs]; a row of one plane and KV head is head_dim
// elements at  base + block*blk_stride + (layer*2 + K|V)*plane_stride + row*row_stride + head*head_stride,
// which covers the layer-first and the block-first pool.  Offsets are 64-bit throughout.
//
// A cache in 4 bits has groups of 32 elements of a head, G of them (heads are padded to 64, 128 or 256 elements): an element is
// lo + s * code.  A plane of a block and head is bs rows of 16 G bytes of codes and then bs rows of G words, each lo (of the 16-bit
// type) in its lower and s (bf16) in its upper half, so that a tile of a head is two contiguous pieces per plane.  The codes lie as the
// attention's matrix instructions take them: K's word a G + g (a < 4) holds elements 32 g + 8 a + (0 .. 7) of the head, V's half word
// i G + g (i < 8) elements 32 g + 4 i + (0 .. 3), the lowest element in the lowest bits.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#define KV_OPS_BAD_BLOCK 1u   // a live slot's block id lies outside the pool: the slot was skipped
#define KV_OPS_TIMEOUT   4u   // a wait inside a kernel ran out: its results are not to be used
#define KV_OPS_BAD_LEN   2u   // a length outside [0, max_len]: the sequence was taken as empty

// limit of a wait inside a kernel, where the context has no other: so many looks (each may take the hardware some microseconds), then two seconds
constexpr unsigned KV_OPS_WAIT_POLLS = 64;
constexpr unsigned long long KV_OPS_WAIT_NS = 2000000000ull;

struct KvView {
    uint8_t *base;
    long long blk_stride, plane_stride;   // bytes
    int row_stride, head_stride;          // bytes; in 4 bits: of a row of codes, and of a block's rows of one head
    int bs, nb, heads, dim;
    int groups;                           // of a head in 4 bits; 0: a 16-bit cache
    const int *tables;
    long long table_stride;               // entries
    const int *lens;
    long long max_len;
    unsigned *status;

    // first byte of a sequence's slot in the given plane, for head 0; nullptr when its block id is no block of the pool
    __device__ __forceinline__ uint8_t *slot(int seq, int s, int plane) const
    {
        const int b = tables[seq * table_stride + s / bs];
        if ((unsigned)b >= (unsigned)nb) {
            atomicOr(status, KV_OPS_BAD_BLOCK);
            return nullptr;
        }
        return base + b * blk_stride + plane * plane_stride + (long long)(s % bs) * row_stride;
    }

    // from a row's codes to its words, in bytes: row r of a block has them 16 G bs + 4 G r behind the head's first byte
    __device__ __forceinline__ int to_words(int s) const { return groups * (16 * bs - 12 * (s % bs)); }

    __device__ __forceinline__ int len(int seq) const
    {
        const int n = lens[seq];
        if ((unsigned)n <= (unsigned long long)max_len) return n;
        atomicOr(status, KV_OPS_BAD_LEN);
        return 0;
    }
};

template <typename T> __device__ __forceinline__ float kv_float(T x);
template <> __device__ __forceinline__ float kv_float(__nv_bfloat16 x) { return __bfloat162float(x); }
template <> __device__ __forceinline__ float kv_float(__half x) { return __half2float(x); }
template <typename T> __device__ __forceinline__ T kv_round(float x);
template <> __device__ __forceinline__ __nv_bfloat16 kv_round(float x) { return __float2bfloat16(x); }
template <> __device__ __forceinline__ __half kv_round(float x) { return __float2half(x); }

// two elements side by side
__device__ __forceinline__ float2 kv_unpair(unsigned w, __nv_bfloat16) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
__device__ __forceinline__ float2 kv_unpair(unsigned w, __half) { return __half22float2(*(const __half2 *)&w); }
__device__ __forceinline__ unsigned kv_pair(float lo, float hi, __nv_bfloat16)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *(const unsigned *)&v;
}
__device__ __forceinline__ unsigned kv_pair(float lo, float hi, __half)
{
    const __half2 v = __floats2half2_rn(lo, hi);
    return *(const unsigned *)&v;
}

// neighbouring words, aligned to all of them or to 16 bytes
template <int N> __device__ __forceinline__ void kv_words(unsigned (&r)[N], const uint8_t *at)
{
    if constexpr (N == 1) r[0] = *(const unsigned *)at;
    else if constexpr (N == 2) {
        const uint2 v = *(const uint2 *)at;
        r[0] = v.x, r[1] = v.y;
    } else
#pragma unroll
        for (int k = 0; k < N; k += 4) {
            const uint4 v = *(const uint4 *)(at + k * 4);
            r[k] = v.x, r[k + 1] = v.y, r[k + 2] = v.z, r[k + 3] = v.w;
        }
}

// the sequence that token t belongs to: the last one that starts at or before it.  A warp looks at 32 places at once
__device__ __forceinline__ int kv_seq_of(const int *starts, int num_seqs, long long t)
{
    const int lane = threadIdx.x & 31;
    int lo = 0, n = num_seqs;        // the answer lies in [lo, lo + n)
    while (n > 1) {
        const int step = (n + 31) / 32, at = lo + lane * step;
        const unsigned v = __ballot_sync(~0u, lane * step < n && starts[at] <= t);
        const int last = v ? 31 - __clz(v) : 0;
        lo += last * step;
        n = min(step, n - last * step);
    }
    return lo;
}
