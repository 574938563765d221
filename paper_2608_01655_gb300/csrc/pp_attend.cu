// Attention of new tokens over the paged cache.
//
// Query i of a request with q new tokens and `length` tokens in all stands at
// position p = length - q + i and sees the keys j with max(0, p - window + 1)
// <= j <= p (all of them from 0 on without a window):
//   o = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m),  s_j = scale q.k_j,  m = max s_j,
//   lse = m + log sum_j exp(s_j - m);  without a visible key o = 0, lse = -inf.
#include <cudaTypedefs.h>

#include "pp_attend.cuh"

namespace pp {

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
    return c.max_q == 1 ? launch_attend_token(kv, c, st) : launch_attend_chunk(kv, c, st);
}

}  // namespace pp
