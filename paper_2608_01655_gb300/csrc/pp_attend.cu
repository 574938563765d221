// Attention of new tokens over the paged cache.
//
// Query i of a request with q new tokens and `length` tokens in all stands at
// position p = length - q + i and sees the keys j with max(0, p - window + 1)
// <= j <= p (all of them from 0 on without a window):
//   o = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m),  s_j = scale q.k_j,  m = max s_j,
//   lse = m + log sum_j exp(s_j - m);  without a visible key o = 0, lse = -inf.
#include <cudaTypedefs.h>

#include <climits>

#include "pp_attend.cuh"

namespace pp {

struct SimpleArgs {
    AttendArgs c;
    int64_t block_stride, token_stride, head_stride;
    int32_t blocks, block_log, dim;
    int32_t *status;
};

// One warp a (token, query head); the running maximum and sum stay in 32 bits.
template <typename T>
__global__ void __launch_bounds__(128) k_attend_simple(SimpleArgs a)
{
    const int lane = threadIdx.x & 31;
    const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
    if (blockIdx.x == 0)
        for (int32_t r = threadIdx.x; r <= a.c.requests; r += blockDim.x) {
            const int32_t x = a.c.q_start[r];
            if (x < 0 || x > a.c.tokens || (r ? x < a.c.q_start[r - 1] : x != 0)) kv_bounds(a.status);
        }
    const int32_t t = (int32_t)(w / a.c.q_heads), h = (int32_t)(w % a.c.q_heads);
    if (t >= a.c.tokens || t >= a.c.q_start[a.c.requests]) return;
    int32_t r = 0;
    for (int32_t len = a.c.requests; len > 1;) {
        const int32_t half = len >> 1;
        if (a.c.q_start[r + half] <= t) { r += half; len -= half; }
        else len = half;
    }
    const int32_t q_len = a.c.q_start[r + 1] - a.c.q_start[r];
    const int64_t room = (int64_t)a.c.table_width << a.block_log;
    int32_t length = a.c.length[r];
    if (length < 0 || length > room) {
        if (lane == 0) kv_bounds(a.status);
        length = (int32_t)min((int64_t)max(length, 0), room);
    }
    const int32_t pos = length - q_len + (t - a.c.q_start[r]);
    const int32_t lo = a.c.window && pos >= a.c.window ? pos - a.c.window + 1 : 0;
    const T *q = static_cast<const T *>(a.c.q) + t * a.c.q_token_stride + h * a.c.q_head_stride;
    float qv[4], o[4] = {0, 0, 0, 0}, m = -INFINITY, l = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) qv[i] = lane + 32 * i < a.dim ? KvType<T>::to_float(q[lane + 32 * i]) : 0.f;
    for (int32_t j = lo; j <= pos; ++j) {
        const int32_t id = a.c.block_table[(int64_t)r * a.c.table_width + (j >> a.block_log)];
        if (id < 0 || id >= a.blocks) {
            if (lane == 0) kv_bounds(a.status);
            continue;
        }
        const int64_t row = id * a.block_stride + (j & ((1 << a.block_log) - 1)) * a.token_stride +
                            h / a.c.group * a.head_stride;
        const T *k = static_cast<const T *>(a.c.k_cache) + row, *v = static_cast<const T *>(a.c.v_cache) + row;
        float s = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (lane + 32 * i < a.dim) s += qv[i] * KvType<T>::to_float(k[lane + 32 * i]);
#pragma unroll
        for (int x = 16; x; x >>= 1) s += __shfl_xor_sync(~0u, s, x);
        s *= a.c.scale;
        const float m2 = fmaxf(m, s), f = m2 == -INFINITY ? 1.f : expf(m - m2), p = m2 == -INFINITY ? 0.f : expf(s - m2);
        m = m2;
        l = l * f + p;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (lane + 32 * i < a.dim) o[i] = o[i] * f + p * KvType<T>::to_float(v[lane + 32 * i]);
    }
    T *out = static_cast<T *>(a.c.out) + t * a.c.out_token_stride + h * a.c.out_head_stride;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (lane + 32 * i < a.dim) out[lane + 32 * i] = KvType<T>::from_float(l == 0.f ? 0.f : o[i] / l);
    if (a.c.lse && lane == 0) a.c.lse[(int64_t)t * a.c.q_heads + h] = l == 0.f ? -INFINITY : m + logf(l);
}

AttendDev attend_dev(const pp_kv *kv, const AttendArgs &c)
{
    return {c, kv->block_stride, kv->token_stride, kv->head_stride, kv->blocks, kv->block_log, kv->dim, kv->heads,
            c.scale * 1.4426950408889634f, kv->d_status, kv->d_piece, kv->d_piece_stat, kv->d_count};
}

// The cache as (dim, token of a block, head, block), copied in boxes of 64
// elements x `rows` tokens.  Elements past `dim` and blocks past the end read
// as zeros.
pp_status cache_map(const pp_kv *kv, const void *cache, int32_t rows, CUtensorMap *map)
{
    static const auto encode = []() -> PFN_cuTensorMapEncodeTiled_v12000 {
        void *fn = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found) !=
                cudaSuccess ||
            found != cudaDriverEntryPointSuccess)
            return nullptr;
        return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(fn);
    }();
    if (!encode) return fail(PP_ECUDA, "the driver has no cuTensorMapEncodeTiled");
    const cuuint64_t size[4] = {(cuuint64_t)kv->dim, (cuuint64_t)kv->block_size, (cuuint64_t)kv->heads,
                                (cuuint64_t)kv->blocks};
    const cuuint64_t stride[3] = {2 * (cuuint64_t)kv->token_stride, 2 * (cuuint64_t)kv->head_stride,
                                  2 * (cuuint64_t)kv->block_stride};
    const cuuint32_t box[4] = {64, (cuuint32_t)rows, 1, 1}, step[4] = {1, 1, 1, 1};
    const CUresult r = encode(map, kv->dtype == PP_KV_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16,
                              4, const_cast<void *>(cache), size, stride, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return fail(PP_ECUDA, "cuTensorMapEncodeTiled failed with " + std::to_string((int)r));
    return PP_OK;
}

pp_status launch_attend(pp_kv *kv, const AttendArgs &c, cudaStream_t st)
{
    if (c.max_q == 1) return launch_attend_token(kv, c, st);
    SimpleArgs a = {c, kv->block_stride, kv->token_stride, kv->head_stride, kv->blocks, kv->block_log, kv->dim,
                    kv->d_status};
    const int64_t warps = (int64_t)c.tokens * c.q_heads;
    if ((warps + 3) / 4 > INT_MAX) return fail(PP_EINVAL, "tokens * q_heads is too large");
    const int grid = (int)((warps + 3) / 4);
    if (kv->dtype == PP_KV_BF16) k_attend_simple<__nv_bfloat16><<<grid, 128, 0, st>>>(a);
    else k_attend_simple<__half><<<grid, 128, 0, st>>>(a);
    PP_CUDA(cudaGetLastError());
    return PP_OK;
}

}  // namespace pp
