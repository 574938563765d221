// Attention of new tokens over the paged cache.
//
// Query i of a request with q new tokens and `length` tokens in all stands at
// position p = length - q + i and sees the keys j with max(0, p - window + 1)
// <= j <= p (all of them from 0 on without a window):
//   o = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m),  s_j = scale q.k_j,  m = max s_j,
//   lse = m + log sum_j exp(s_j - m);  without a visible key o = 0, lse = -inf.
#include <cudaTypedefs.h>

#include <atomic>

#include "pp_attend.cuh"

namespace pp {

static std::atomic<bool> g_lose_copies{false};

void attend_lose_copies(bool on) { g_lose_copies.store(on); }

AttendDev attend_dev(const pp_kv *kv, const AttendArgs &c)
{
    AttendDev a = {};
    a.c = c;
    a.block_stride = kv->block_stride;
    a.token_stride = kv->token_stride;
    a.head_stride = kv->head_stride;
    a.blocks = kv->blocks;
    a.block_log = kv->block_log;
    a.dim = kv->dim;
    a.kv_heads = kv->heads;
    a.scale_log2 = c.scale * 1.4426950408889634f;
    a.group_shift = 32;
    while (1 << (a.group_shift - 32) < c.group) a.group_shift++;
    a.group_mul = (((uint64_t)1 << a.group_shift) + c.group - 1) / c.group;
    a.wide_out = (reinterpret_cast<uintptr_t>(c.out) & 31) == 0 && c.out_token_stride % 16 == 0 &&
                 c.out_head_stride % 16 == 0 && kv->dim % 16 == 0;
    a.status = kv->d_status;
    a.piece = kv->d_piece;
    a.piece_stat = kv->d_piece_stat;
    a.count = kv->d_count;
    const bool lose = g_lose_copies.load(std::memory_order_relaxed);
    a.wait_limit = lose ? kAttendTestCycles : kAttendLimitCycles;
    a.lost = lose ? 16 : 0;
    return a;
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

pp_status prepare_attend()
{
    const pp_status s = prepare_attend_token();
    return s == PP_OK ? prepare_attend_chunk() : s;
}

// Rows (new tokens x heads of a group) of the longest request up to which a call
// goes to the kernel of single tokens.  That one reads K and V once for every 16
// rows and has short items to begin and to join; the chunk kernel pays for 256 rows
// whatever there are.  Kernel of single tokens against chunks', in us, 2 K/V heads
// of 128, 32 requests after 5,000 tokens / 4 after 2,000 / 1 after 50,000 (single
// passes after a flush of L2):
//   16 rows  50 : 61 / 22 : 33 / 34 : 56
//   32       64 : 61 / 21 : 31 / 36 : 56
//   64      104 : 61 / 28 : 32 / 42 : 54
// so at 64 it loses more in batches than it gains for single requests.
constexpr int64_t kFewRows = 32;

pp_status launch_attend(pp_kv *kv, const AttendArgs &c, cudaStream_t st)
{
    return (int64_t)c.max_q * c.group <= kFewRows ? launch_attend_token(kv, c, st) : launch_attend_chunk(kv, c, false, st);
}

}  // namespace pp
