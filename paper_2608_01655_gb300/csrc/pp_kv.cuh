// The paged K/V cache of one worker: the handle's layout and status word, and
// what the cache's kernels share.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "pp_internal.cuh"

struct pp_kv {
    int device = 0;
    int sm_count = 0;
    int32_t blocks = 0;                 // blocks of the cache
    int32_t block_size = 0;             // tokens per block, a power of two
    int32_t block_log = 0;              // log2(block_size)
    int32_t heads = 0;                  // K/V heads
    int32_t dim = 0;                    // head dimension
    int32_t dtype = 0;
    int64_t block_stride = 0, token_stride = 0, head_stride = 0;     // elements
    int32_t *d_status = nullptr;        // device status word
    // scratch of the attention: pieces of items that several CTAs computed, their
    // maxima and sums, and arrival counts (0 between launches)
    float *d_piece = nullptr, *d_piece_stat = nullptr;
    int32_t *d_count = nullptr;
};

namespace pp {

constexpr int kKvMaxDim = 128;
constexpr int kKvMaxBlock = 512;
constexpr int32_t kKvMaxRequests = 16384;
constexpr int32_t kKvMaxBlocks = 1 << 30;
constexpr int kPieceRows = 256;                 // rows of a piece, at most

// one call of pp_paged_attention, checked
struct AttendArgs {
    int32_t requests, tokens, q_heads, group;
    const void *q;
    int64_t q_token_stride, q_head_stride;
    const void *k_cache, *v_cache;
    const int32_t *block_table;
    int32_t table_width;
    const int32_t *q_start, *length;
    int32_t max_q, window;
    float scale;
    void *out;
    int64_t out_token_stride, out_head_stride;
    float *lse;
};

// A device-side check failed; a time limit that ran out stays the status.
__device__ __forceinline__ void kv_bounds(int32_t *status)
{
    if (*(volatile int32_t *)status == PP_OK) atomicCAS(status, (int32_t)PP_OK, (int32_t)PP_EBOUNDS);
}

template <typename T> struct KvType;
template <> struct KvType<__nv_bfloat16> {
    static __device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
};
template <> struct KvType<__half> {
    static __device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
};

}  // namespace pp
