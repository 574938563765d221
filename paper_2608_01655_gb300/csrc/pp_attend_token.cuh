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
constexpr int kJoinGroup = 16;                      // pieces (8 KB) joined at a time, then their groups

// Rows are (token, head of the group), token first; an item is ROWS of them, a tile KEYS keys.
// EXTRA: what an item weighs beside its tiles (first rows, join).
template <int ROWS, int KEYS, int EXTRA> struct ShapeOf {
    static constexpr int kRows = ROWS;
    static constexpr int KT = KEYS;
    static constexpr int32_t extra = EXTRA;
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

// A thread's N columns of a row: those from 4 `lane` on, four of every STEP, so that
// neighbouring threads' loads are neighbours.
template <int N, int STEP> __device__ __forceinline__ void store_columns(float *row, int lane, const float (&x)[N])
{
#pragma unroll
    for (int d = 0; d < N; d += 4)
        *reinterpret_cast<float4 *>(row + 4 * lane + d / 4 * STEP) = make_float4(x[d], x[d + 1], x[d + 2], x[d + 3]);
}
// from L2, where other CTAs left them
template <int N, int STEP> __device__ __forceinline__ void load_columns(const float *row, int lane, float (&x)[N])
{
#pragma unroll
    for (int d = 0; d < N; d += 4) {
        const float4 y = __ldcg(reinterpret_cast<const float4 *>(row + 4 * lane + d / 4 * STEP));
        x[d] = y.x;
        x[d + 1] = y.y;
        x[d + 2] = y.z;
        x[d + 3] = y.w;
    }
}

// The place of row `row` of an item in [tokens][q_heads] rows.
template <class S>
__device__ __forceinline__ int64_t item_row(const AttendDev &a, const Cursor<S> &cur, int32_t row, int64_t token_stride,
                                            int64_t head_stride)
{
    const int32_t at = cur.inner * S::kRows + row, tok = div_group(a, at);
    return (int64_t)(cur.q.first + tok) * token_stride + (int64_t)(cur.outer * a.c.group + at - tok * a.c.group) * head_stride;
}

// The end of an item, or of a CTA's part of it: leaves a piece or writes the rows.  A
// thread (tid of THREADS, which sync() is for) has PER columns of row jr (a row is within a
// warp), as in store_columns: outputs acc not yet divided, maximum and sum.
// GROUP: pieces that are joined at a time, then their groups; 0: 8, or the square root of
// the pieces if they are more.
template <typename T, class S, int PER, int THREADS, int GROUP, class SYNC>
__device__ __forceinline__ void leave_item(const AttendDev &a, const Cursor<S> &cur, int tid, float (&acc)[PER], float top,
                                           float sum, int32_t *last, int64_t total, int64_t ctas, SYNC sync)
{
    constexpr int kRows = S::kRows, kLanes = THREADS / kRows, kWidth = PER * kLanes;
    constexpr int kStep = 4 * kLanes;
    static_assert(PER % 4 == 0, "columns go four at a time");
    const int jr = tid / kLanes, lane = tid % kLanes;
    const int32_t row0 = cur.inner * kRows, rows = min(kRows, S::rows(a, cur.q) - row0);
    const uint32_t row_lanes = (uint32_t)(((uint64_t)1 << kLanes) - 1) << ((tid & 31) - lane);

    // an item in pieces: leave this one's, and the last to arrive joins a group's, then the groups'
    bool write = true;
    if (!cur.whole()) {
        const int64_t g0 = cur.g - cur.off;
        const int32_t cta0 = owner(g0, total, ctas), pieces = owner(g0 + cur.tiles - 1, total, ctas) - cta0 + 1;
        const int32_t mine = (int32_t)blockIdx.x - cta0;
        int32_t group = GROUP ? GROUP : 8;
        if (!GROUP && pieces > group)
            while (group * group < pieces) ++group;
        const int32_t groups = (pieces + group - 1) / group;
        auto put = [&](int32_t slot) {
            __syncwarp();                           // a row's lanes have read what one of them writes over
            if (jr < rows) {
                store_columns<PER, kStep>(a.piece + ((int64_t)slot * kRows + jr) * kWidth, lane, acc);
                if (lane == 0) {
                    a.piece_stat[slot * 2 * kRows + jr] = top;
                    a.piece_stat[slot * 2 * kRows + kRows + jr] = sum;
                }
            }
        };
        // true in the CTA that arrives last of `of`
        auto arrive = [&](int32_t *count, int32_t of) {
            __threadfence();
            sync();
            if (tid == 0) {
                *last = atomicAdd(count, 1) == of - 1;
                if (*last) *count = 0;
            }
            sync();
            __threadfence();
            return *last != 0;
        };
        // join pieces p0, p0 + step, ...
        auto gather = [&](int32_t p0, int32_t n, int32_t step) {
            if (jr >= rows) return;
            if constexpr (GROUP != 0) {
                top = -INFINITY;
                for (int32_t p = 0; p < n; ++p)
                    top = fmaxf(top, __ldcg(a.piece_stat + piece_slot(cta0, p0 + p * step) * 2 * kRows + jr));
            }
            auto stat = [&](int32_t p) { return a.piece_stat + piece_slot(cta0, p0 + p * step) * 2 * kRows + jr; };
            constexpr int kOwn = GROUP ? 1 : (20 + kLanes - 1) / kLanes;    // a lane's pieces (20 * 20 are more than CTAs)
            float own[kOwn];
            if constexpr (GROUP == 0) {
                // the statistics, a piece a lane, on their way together
#pragma unroll
                for (int x = 0; x < kOwn; ++x) own[x] = lane + x * kLanes < n ? __ldcg(stat(lane + x * kLanes)) : -INFINITY;
                top = own[0];
#pragma unroll
                for (int x = 1; x < kOwn; ++x) top = fmaxf(top, own[x]);
#pragma unroll
                for (int o = kLanes / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(row_lanes, top, o));
            }
            const float base = top == -INFINITY ? 0.f : top;
            sum = 0.f;
#pragma unroll
            for (int d = 0; d < PER; ++d) acc[d] = 0.f;
#pragma unroll 4
            for (int32_t p = 0; p < n; ++p) {
                const int32_t slot = piece_slot(cta0, p0 + p * step);
                const float f = exp2_approx(__ldcg(stat(p)) - base);
                sum = fmaf(f, __ldcg(stat(p) + kRows), sum);
                float y[PER];
                load_columns<PER, kStep>(a.piece + ((int64_t)slot * kRows + jr) * kWidth, lane, y);
#pragma unroll
                for (int d = 0; d < PER; ++d) acc[d] = fmaf(f, y[d], acc[d]);
            }
        };
        put(piece_slot(cta0, mine));
        const int32_t grp = mine / group, p0 = grp * group, n = min(group, pieces - p0);
        write = arrive(a.count + piece_slot(cta0, p0), n);
        if (write) {
            gather(p0, n, 1);
            if (groups > 1) {
                put(piece_slot(cta0, p0));
                write = arrive(a.count + 2 * gridDim.x + piece_slot(cta0, 0), groups);
                if (write) gather(0, groups, group);
            }
        }
    }
    if (write && jr < rows) {
        const float inv = inverse_sum(sum, S::pos(a, cur.q, row0 + jr) >= 0);
        T *dst = static_cast<T *>(a.c.out) + item_row(a, cur, jr, a.c.out_token_stride, a.c.out_head_stride) + 4 * lane;
#pragma unroll
        for (int d = 0; d < PER; d += 4) {
            if (4 * lane + d / 4 * kStep >= a.dim) continue;
            *reinterpret_cast<uint2 *>(dst + d / 4 * kStep) =
                make_uint2(Pack<T>::two(acc[d] * inv, acc[d + 1] * inv), Pack<T>::two(acc[d + 2] * inv, acc[d + 3] * inv));
        }
        if (a.c.lse && lane == 0)
            a.c.lse[item_row(a, cur, jr, a.c.q_heads, 1)] =
                sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
    }
}

}  // namespace pp
