// What the kernels on the device cache share: the address rule of a layer's slots, the element types, the status
// word.  Slot s of sequence i lies in row s % bs of block table[i][s / bs]; a row of one plane and KV head is head_dim
// elements at  base + block*blk_stride + (layer*2 + K|V)*plane_stride + row*row_stride + head*head_stride,
// which covers the layer-first and the block-first pool.  Offsets are 64-bit throughout.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#define KV_OPS_BAD_BLOCK 1u   // a live slot's block id lies outside the pool: the slot was skipped
#define KV_OPS_BAD_LEN   2u   // a length outside [0, max_len]: the sequence was taken as empty

struct KvView {
    uint8_t *base;
    long long blk_stride, plane_stride;   // bytes
    int row_stride, head_stride;          // bytes
    int bs, nb, heads, dim;
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
