// What the kernels of single tokens share, over caches of 16 and of 8 bits: items
// and their cut, instructions, and the join of an item's warps and pieces.
#pragma once

#include <cstring>
#include <type_traits>

#include "pp_attend.cuh"

namespace pp {

namespace token {
constexpr int kWarps = 8, kThreads = 32 * kWarps;
constexpr int kKeys = 16;                           // keys of a warp
constexpr int KT = kKeys * kWarps;                  // keys per tile
constexpr int kRows = 16;                           // rows of an item
constexpr int kJoinGroup = 16;                      // pieces (8 KB) joined at a time, then their groups

// Shared memory of an item's join: the rows' outputs of four warps.
template <int HALVES> struct Join {
    static constexpr int width = 64 * HALVES;
    static constexpr int pitch = width + 4;                     // floats of an output row
    static constexpr int bytes = kWarps / 2 * kRows * pitch * 4;
};
struct JoinShared {
    float stat[2][kWarps][kRows];       // maxima (log2 units) and sums
    int32_t last;
};

// Rows are (token, head of the group), token first; an item is 16 of them.
struct Shape {
    static constexpr int KT = token::KT;
    // what an item weighs beside its tiles (first rows, join): 1, 2, 3, 5 tiles take 60 requests x 4 tokens after 50 to
    // 9,000 56, 53, 48, 46 us, 300 single tokens after 50 to 3,000 85, 81, 79, 79, 256 after 100 to 8,000 -, 461, 462, 472
    static constexpr int32_t extra = 3;
    static constexpr bool many = false;
    static __device__ __forceinline__ int32_t outer(const AttendDev &a) { return a.kv_heads; }
    static __device__ __forceinline__ int32_t rows(const AttendDev &a, const Req &q) { return q.q_len * a.c.group; }
    static __device__ __forceinline__ int32_t inner(const AttendDev &a, const Req &q) { return (rows(a, q) + kRows - 1) / kRows; }
    static __device__ __forceinline__ int32_t pos(const AttendDev &a, const Req &q, int32_t row)
    {
        return q.length - q.q_len + div_group(a, row);
    }
    static __device__ __forceinline__ Keys keys(const AttendDev &a, const Req &q, int32_t i)
    {
        const int32_t r0 = i * kRows, r1 = min(r0 + kRows, rows(a, q)) - 1;
        return {first_key(a, max(pos(a, q, r0), 0)), pos(a, q, r1)};
    }
};
}  // namespace token

using namespace token;

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr));
}
__device__ __forceinline__ void ldsm4_trans(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr));
}
template <typename T>
__device__ __forceinline__ void mma16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma16<__nv_bfloat16>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
                 "{%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma16<__half>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
                 "{%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t lds32(uint32_t addr)
{
    uint32_t x;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(x) : "r"(addr));
    return x;
}

// both 16-bit halves of a register kept or cleared
__device__ __forceinline__ uint32_t keep(bool lo, bool hi) { return (lo ? 0xffffu : 0u) | (hi ? 0xffff0000u : 0u); }

// The place of row `row` of an item in [tokens][q_heads] rows.
__device__ __forceinline__ int64_t item_row(const AttendDev &a, const Cursor<Shape> &cur, int32_t row, int64_t token_stride,
                                            int64_t head_stride)
{
    const int32_t at = cur.inner * kRows + row, tok = div_group(a, at);
    return (int64_t)(cur.q.first + tok) * token_stride + (int64_t)(cur.outer * a.c.group + at - tok * a.c.group) * head_stride;
}

// The end of an item (or of a CTA's part of it): joins the warps' outputs o, maxima
// m and sums l, leaves a piece or writes the rows.  A thread's o are of rows r0 =
// lane / 4 and r0 + 8; o[n][2 x + y] of row r0 + 8 x is column 8 n + 2 (lane % 4) + y,
// with EIGHT (V rows of 8-bit numbers, which come in pairs) 16 (n / 2) + 4 (lane % 4)
// + n % 2 + 2 y.
template <typename T, int HALVES, bool EIGHT>
__device__ __forceinline__ void finish_item(const AttendDev &a, const Cursor<Shape> &cur, float (&o)[8 * HALVES][4],
                                            float (&m)[2], float (&l)[2], float *join, JoinShared &sh, int64_t total,
                                            int64_t ctas)
{
    using J = Join<HALVES>;
    constexpr int KS = 4 * HALVES;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, r0 = lane >> 2;
    const int jr = tid >> 4, jd = (tid & 15) * (4 * HALVES);          // joining: row and first column
    const int32_t row0 = cur.inner * kRows, rows = min(kRows, Shape::rows(a, cur.q) - row0);
    auto q_row = [&](int32_t row, int64_t token_stride, int64_t head_stride) { return item_row(a, cur, row, token_stride, head_stride); };

    // join the warps: the upper four hand theirs to the lower four, lane by lane,
    // then a thread has one row's 4 * HALVES columns
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        l[x] += __shfl_xor_sync(~0u, l[x], 1);
        l[x] += __shfl_xor_sync(~0u, l[x], 2);
        if ((lane & 3) == 0) {
            sh.stat[0][warp][r0 + 8 * x] = m[x];
            sh.stat[1][warp][r0 + 8 * x] = l[x];
        }
    }
    if (warp >= kWarps / 2) {
        float4 *dst = reinterpret_cast<float4 *>(join) + (warp - kWarps / 2) * 2 * KS * 32 + lane;
#pragma unroll
        for (int n = 0; n < 2 * KS; ++n) dst[32 * n] = make_float4(o[n][0], o[n][1], o[n][2], o[n][3]);
    }
    __syncthreads();
    if (warp < kWarps / 2) {
        const float4 *src = reinterpret_cast<const float4 *>(join) + warp * 2 * KS * 32 + lane;
        float f[2], g[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const float other = sh.stat[0][warp + kWarps / 2][r0 + 8 * x], up = fmaxf(m[x], other);
            const float by = up == -INFINITY ? 0.f : up;
            f[x] = exp2_approx(m[x] - by);
            g[x] = exp2_approx(other - by);
            m[x] = up;
            l[x] = f[x] * l[x] + g[x] * sh.stat[1][warp + kWarps / 2][r0 + 8 * x];
        }
#pragma unroll
        for (int n = 0; n < 2 * KS; ++n) {
            const float4 y = src[32 * n];
            o[n][0] = f[0] * o[n][0] + g[0] * y.x;
            o[n][1] = f[0] * o[n][1] + g[0] * y.y;
            o[n][2] = f[1] * o[n][2] + g[1] * y.z;
            o[n][3] = f[1] * o[n][3] + g[1] * y.w;
        }
    }
    __syncthreads();
    if (warp < kWarps / 2) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int row = r0 + 8 * x;
            if ((lane & 3) == 0) {
                sh.stat[0][warp][row] = m[x];
                sh.stat[1][warp][row] = l[x];
            }
            if (row < rows) {
                float *dst = join + (warp * kRows + row) * J::pitch;
                if constexpr (EIGHT) {
#pragma unroll
                    for (int n = 0; n < KS; ++n)
                        *reinterpret_cast<float4 *>(dst + 16 * n + 4 * (lane & 3)) =
                            make_float4(o[2 * n][2 * x], o[2 * n + 1][2 * x], o[2 * n][2 * x + 1], o[2 * n + 1][2 * x + 1]);
                } else {
#pragma unroll
                    for (int n = 0; n < 2 * KS; ++n)
                        *reinterpret_cast<float2 *>(dst + 8 * n + 2 * (lane & 3)) = make_float2(o[n][2 * x], o[n][2 * x + 1]);
                }
            }
        }
    }
    __syncthreads();
    float acc[4 * HALVES], top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int d = 0; d < 4 * HALVES; ++d) acc[d] = 0.f;
    if (jr < rows) {
#pragma unroll
        for (int w = 0; w < kWarps / 2; ++w) top = fmaxf(top, sh.stat[0][w][jr]);
        const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
        for (int w = 0; w < kWarps / 2; ++w) {
            const float f = exp2_approx(sh.stat[0][w][jr] - base);
            sum = fmaf(f, sh.stat[1][w][jr], sum);
            const float4 *src = reinterpret_cast<const float4 *>(join + (w * kRows + jr) * J::pitch + jd);
#pragma unroll
            for (int d = 0; d < HALVES; ++d) {
                const float4 y = src[d];
                acc[4 * d] = fmaf(f, y.x, acc[4 * d]);
                acc[4 * d + 1] = fmaf(f, y.y, acc[4 * d + 1]);
                acc[4 * d + 2] = fmaf(f, y.z, acc[4 * d + 2]);
                acc[4 * d + 3] = fmaf(f, y.w, acc[4 * d + 3]);
            }
        }
    }

    // an item in pieces: leave this one's, and the last to arrive joins a group's, then the groups'
    bool write = true;
    if (!cur.whole()) {
        const int64_t g0 = cur.g - cur.off;
        const int32_t cta0 = owner(g0, total, ctas), pieces = owner(g0 + cur.tiles - 1, total, ctas) - cta0 + 1;
        const int32_t mine = (int32_t)blockIdx.x - cta0;
        const int32_t groups = (pieces + kJoinGroup - 1) / kJoinGroup;
        auto put = [&](int32_t slot) {
            __syncwarp();                           // a row's 16 lanes have read what one of them writes over
            if (jr < rows) {
                float4 *dst = reinterpret_cast<float4 *>(a.piece + ((int64_t)slot * kRows + jr) * J::width + jd);
#pragma unroll
                for (int d = 0; d < HALVES; ++d)
                    dst[d] = make_float4(acc[4 * d], acc[4 * d + 1], acc[4 * d + 2], acc[4 * d + 3]);
                if (jd == 0) {
                    a.piece_stat[slot * 2 * kRows + jr] = top;
                    a.piece_stat[slot * 2 * kRows + kRows + jr] = sum;
                }
            }
        };
        // true in the CTA that arrives last of `of`
        auto arrive = [&](int32_t *count, int32_t of) {
            __threadfence();
            __syncthreads();
            if (tid == 0) {
                sh.last = atomicAdd(count, 1) == of - 1;
                if (sh.last) *count = 0;
            }
            __syncthreads();
            __threadfence();
            return sh.last != 0;
        };
        // join pieces p0, p0 + step, ...
        auto gather = [&](int32_t p0, int32_t n, int32_t step) {
            if (jr >= rows) return;
            top = -INFINITY;
            for (int32_t p = 0; p < n; ++p)
                top = fmaxf(top, __ldcg(a.piece_stat + piece_slot(cta0, p0 + p * step) * 2 * kRows + jr));
            const float base = top == -INFINITY ? 0.f : top;
            sum = 0.f;
#pragma unroll
            for (int d = 0; d < 4 * HALVES; ++d) acc[d] = 0.f;
#pragma unroll 4
            for (int32_t p = 0; p < n; ++p) {
                const int32_t slot = piece_slot(cta0, p0 + p * step);
                const float f = exp2_approx(__ldcg(a.piece_stat + slot * 2 * kRows + jr) - base);
                sum = fmaf(f, __ldcg(a.piece_stat + slot * 2 * kRows + kRows + jr), sum);
                const float4 *src =
                    reinterpret_cast<const float4 *>(a.piece + ((int64_t)slot * kRows + jr) * J::width + jd);
#pragma unroll
                for (int d = 0; d < HALVES; ++d) {
                    const float4 y = __ldcg(src + d);
                    acc[4 * d] = fmaf(f, y.x, acc[4 * d]);
                    acc[4 * d + 1] = fmaf(f, y.y, acc[4 * d + 1]);
                    acc[4 * d + 2] = fmaf(f, y.z, acc[4 * d + 2]);
                    acc[4 * d + 3] = fmaf(f, y.w, acc[4 * d + 3]);
                }
            }
        };
        put(piece_slot(cta0, mine));
        const int32_t grp = mine / kJoinGroup, p0 = grp * kJoinGroup, n = min(kJoinGroup, pieces - p0);
        write = arrive(a.count + piece_slot(cta0, p0), n);
        if (write) {
            gather(p0, n, 1);
            if (groups > 1) {
                put(piece_slot(cta0, p0));
                write = arrive(a.count + 2 * gridDim.x + piece_slot(cta0, 0), groups);
                if (write) gather(0, groups, kJoinGroup);
            }
        }
    }
    if (write && jr < rows) {
        const float inv = inverse_sum(sum, Shape::pos(a, cur.q, row0 + jr) >= 0);
        T *dst = static_cast<T *>(a.c.out) + q_row(jr, a.c.out_token_stride, a.c.out_head_stride) + jd;
        if constexpr (HALVES == 2) {
            if (jd < a.dim)
                *reinterpret_cast<uint4 *>(dst) =
                    make_uint4(Pack<T>::two(acc[0] * inv, acc[1] * inv), Pack<T>::two(acc[2] * inv, acc[3] * inv),
                               Pack<T>::two(acc[4] * inv, acc[5] * inv), Pack<T>::two(acc[6] * inv, acc[7] * inv));
        } else {
            if (jd < a.dim)
                *reinterpret_cast<uint2 *>(dst) =
                    make_uint2(Pack<T>::two(acc[0] * inv, acc[1] * inv), Pack<T>::two(acc[2] * inv, acc[3] * inv));
        }
        if (a.c.lse && jd == 0)
            a.c.lse[q_row(jr, a.c.q_heads, 1)] =
                sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
    }
    __syncthreads();                                // the join's memory is free again
}

}  // namespace pp
