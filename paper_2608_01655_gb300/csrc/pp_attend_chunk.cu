// Attention of chunks of new tokens over the paged cache, on tcgen05.
//
// The queries of a K/V head are rows (token, head of the group), token first,
// so 128 rows are a few neighbouring tokens whatever the group is, and only
// tiles on the diagonal need masks.  An item is 256 rows: two stages of 128 that
// share every K and V tile (128 keys).  Per stage and tile
//   S = Q K^T      operands in shared memory, accumulator in tensor memory,
//   P = exp2(scale S - m) by one warpgroup, a row a thread, written over S,
//   O += P V       P from tensor memory, V as it lies in the cache.
// The stages take turns: while one warpgroup works on its S, the tensor cores
// run the other stage's products.  m is a maximum that was found once and moves
// only when a tile's weights add up to more than 2^12, so O is rescaled (in tensor
// memory) hardly ever, and no tile waits for its maximum; weights are at most
// 2^12 then, which both 16-bit types hold as precisely as 1.
//
// Warps: 0-3 and 4-7 the stages' softmax, 8-11 the outputs of both, 12 and 13 the
// stages' products, 14 and 15 the copies of K and V.  V tiles that not every row
// sees in full are looked over by the softmax warps: an infinity or a NaN there
// would pass through a weight of 0, so it is replaced by 0 and added in the
// epilogue to the rows that do see it.
//
// What bounds it: at width 128 a tile of both stages is 2,048 cycles of products
// (57% tensor cycles in a 2,048-token chunk after 4,096), 1,100 to 1,300 cycles of
// softmax a stage (128 exponentials a thread at 5 cycles, two warps a scheduler)
// and 1,000 cycles of hand-over; at width 64 the products are half and the
// exponentials bound it.  256 rows an item is what tensor memory holds (two S and
// two O of 128 columns).
// Measured, single passes after a pause: 8,192 new tokens after 24,576 (28 heads on 4,
// width 128) 1.90 ms, 1,770 TFLOP/s or 95% of the measured library product (in a row,
// under the power limit, 2.07 ms and 1,630, of a library product's 1,722 there); 8,192
// tokens of 16 heads from nothing 217 us, 1,270 TFLOP/s; the same at width 64 166 us,
// 830 TFLOP/s.
#include <algorithm>
#include <new>
#include <type_traits>

#include "pp_attend.cuh"

namespace pp {

namespace chunk {
constexpr int KT = 128;                             // keys per tile
constexpr int kRows = 128;                          // rows of a stage
constexpr int kThreads = 512;
constexpr int kAlone = 4;                           // pieces of an item that one CTA joins
constexpr int kBad = 16;                            // marks of items, the stages are fewer apart
constexpr float kMaxSum = 4096.f;                   // of the weights of a row and tile, before m moves

template <int HALVES> struct Layout {
    static constexpr int half = KT * 128;                       // bytes of 64 columns of a tile
    static constexpr int tile = half * HALVES;
    static constexpr int k_slots = HALVES == 2 ? 3 : 5, v_slots = HALVES == 2 ? 2 : 5;     // tiles in flight
    static constexpr int width = 64 * HALVES;
    static constexpr int tiles = (2 + k_slots + v_slots) * tile;
};

struct Shape {
    static constexpr int KT = chunk::KT;
    // what an item weighs beside its tiles (queries, first maximum, outputs): 2, 3, 4 tiles take 8,192 tokens of 16 heads
    // from nothing 236, 218, 215 us, 60 requests x 40 to 90 after 50 to 9,000 182, 174, 171, 24 x 1 to 2,000 with a window
    // 251, 251, 254, 16 x 16 after 3,000 42, 43, 43
    static constexpr int32_t extra = 3;
    static constexpr bool many = true;
    static __device__ __forceinline__ int32_t outer(const AttendDev &a) { return a.kv_heads; }
    static __device__ __forceinline__ int32_t rows(const AttendDev &a, const Req &q) { return q.q_len * a.c.group; }
    static __device__ __forceinline__ int32_t inner(const AttendDev &a, const Req &q)
    {
        return (rows(a, q) + 2 * kRows - 1) / (2 * kRows);
    }
    static __device__ __forceinline__ int32_t pos(const AttendDev &a, const Req &q, int32_t row)
    {
        return q.length - q.q_len + div_group(a, row);
    }
    static __device__ __forceinline__ Keys keys(const AttendDev &a, const Req &q, int32_t i)
    {
        const int32_t r0 = i * 2 * kRows, r1 = min(r0 + 2 * kRows, rows(a, q)) - 1;
        return {first_key(a, max(pos(a, q, r0), 0)), pos(a, q, r1)};
    }
};

// what rows [r0, r1] of a request all see
struct Common {
    int32_t lo, hi;
    __device__ __forceinline__ Common(const AttendDev &a, const Req &q, int32_t r0, int32_t r1)
        : lo(first_key(a, Shape::pos(a, q, r1))), hi(Shape::pos(a, q, r0))
    {
    }
    __device__ __forceinline__ bool covers(int32_t j0) const { return j0 >= lo && j0 + KT - 1 <= hi; }
};
}  // namespace chunk

using namespace chunk;

// ---------------------------------------------------------------------------
// tcgen05
// ---------------------------------------------------------------------------
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// Columns of this warp's 32 lanes, loaded and landed: in one statement, for nothing
// else tells the compiler that the registers are not to be read before.
__device__ __forceinline__ void tc_ld64(uint32_t *r, uint32_t addr)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%64];\n"
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%32, %33, %34, %35, %36, %37, %38, %39, %40, %41, %42, %43, %44, %45, %46, %47, "
        "%48, %49, %50, %51, %52, %53, %54, %55, %56, %57, %58, %59, %60, %61, %62, %63}, [%65];\n"
        "tcgen05.wait::ld.sync.aligned;\n"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
          "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
          "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31]),
          "=r"(r[32]), "=r"(r[33]), "=r"(r[34]), "=r"(r[35]), "=r"(r[36]), "=r"(r[37]), "=r"(r[38]), "=r"(r[39]),
          "=r"(r[40]), "=r"(r[41]), "=r"(r[42]), "=r"(r[43]), "=r"(r[44]), "=r"(r[45]), "=r"(r[46]), "=r"(r[47]),
          "=r"(r[48]), "=r"(r[49]), "=r"(r[50]), "=r"(r[51]), "=r"(r[52]), "=r"(r[53]), "=r"(r[54]), "=r"(r[55]),
          "=r"(r[56]), "=r"(r[57]), "=r"(r[58]), "=r"(r[59]), "=r"(r[60]), "=r"(r[61]), "=r"(r[62]), "=r"(r[63])
        : "r"(addr), "r"(addr + 32)
        : "memory");
}
__device__ __forceinline__ void tc_ld32(uint32_t *r, uint32_t addr)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n"
        "tcgen05.wait::ld.sync.aligned;\n"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
          "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
          "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr)
        : "memory");
}
__device__ __forceinline__ void tc_ld8(uint32_t *r, uint32_t addr)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];\n"
        "tcgen05.wait::ld.sync.aligned;\n"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
        : "r"(addr)
        : "memory");
}
__device__ __forceinline__ void tc_st32(uint32_t addr, const uint32_t *r)
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};" ::"r"(r[0]),
        "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]),
        "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]),
        "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(addr)
        : "memory");
}

__device__ __forceinline__ void tc_st8(uint32_t addr, const uint32_t *r)
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};" ::"r"(r[0]), "r"(r[1]),
                 "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(addr)
                 : "memory");
}

// Shared-memory operand: rows of 128 bytes swizzled by 128 bytes, groups of 8
// rows `group` bytes apart; for an operand whose long side is contiguous
// (V), `next` is the distance of its 64-element halves.
__device__ __forceinline__ uint64_t smem_operand(uint32_t addr, uint32_t next, uint32_t group)
{
    return (uint64_t)((addr & 0x3ffff) >> 4) | (uint64_t)(next >> 4) << 16 | (uint64_t)(group >> 4) << 32 |
           (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
// 32-bit sums of 16-bit products, 128 rows; `transposed`: B's rows run along the summed index
template <typename T> __device__ __forceinline__ uint32_t mma_kind(int n, bool transposed)
{
    const uint32_t type = std::is_same<T, __nv_bfloat16>::value ? 1 : 0;
    return 1u << 4 | type << 7 | type << 10 | (transposed ? 1u << 16 : 0) | (uint32_t)(n / 8) << 17 | (128u / 16) << 24;
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t kind, bool add)
{
    asm volatile(
        "{\n"
        ".reg .pred p;\n"
        "setp.ne.b32 p, %4, 0;\n"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n"
        "}\n" ::"r"(d),
        "l"(a), "l"(b), "r"(kind), "r"((uint32_t)add)
        : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t kind, bool add)
{
    asm volatile(
        "{\n"
        ".reg .pred p;\n"
        "setp.ne.b32 p, %4, 0;\n"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n"
        "}\n" ::"r"(d),
        "r"(a), "l"(b), "r"(kind), "r"((uint32_t)add)
        : "memory");
}

__device__ __forceinline__ float max3(float a, float b, float c)
{
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
__device__ __forceinline__ uint64_t pair(float lo, float hi)
{
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ float2 unpair(uint64_t x)
{
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(x));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b)
{
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}

// one lane of the warp, always the same.  The products are issued under it and
// not under a comparison of the lane's number: the compiler knows then that a
// single thread holds their operands (an instruction took 90 cycles otherwise, 64 now).
__device__ __forceinline__ bool elected()
{
    uint32_t yes;
    asm volatile(
        "{\n"
        ".reg .pred p;\n"
        "elect.sync _|p, 0xffffffff;\n"
        "selp.u32 %0, 1, 0, p;\n"
        "}\n"
        : "=r"(yes));
    return yes != 0;
}

// x * 0 + acc: stays 0 unless x has an infinity or a NaN
template <typename T> __device__ __forceinline__ uint32_t taint(uint32_t x, uint32_t acc)
{
    uint32_t r;
    if constexpr (std::is_same<T, __nv_bfloat16>::value)
        asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(x), "r"(0u), "r"(acc));
    else
        asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(x), "r"(0u), "r"(acc));
    return r;
}
// 16-bit value without a finite number
template <typename T> __device__ __forceinline__ bool not_finite(uint32_t bits)
{
    const uint32_t e = std::is_same<T, __nv_bfloat16>::value ? 0x7f80u : 0x7c00u;
    return (bits & e) == e;
}

// ---------------------------------------------------------------------------
// The roles
// ---------------------------------------------------------------------------
struct Bars {
    uint32_t k_full, k_empty, v_full, v_empty, q_full, s_full, p_full, o_done, o_free, fin, pass, stat_full, stat_free;     // shared addresses
};

// Shared memory: the stages' queries, K tiles, V tiles.
template <int HALVES> __device__ __forceinline__ uint32_t k_at(uint32_t base, uint32_t slot)
{
    return base + (2 + slot) * Layout<HALVES>::tile;
}
template <int HALVES> __device__ __forceinline__ uint32_t v_at(uint32_t base, uint32_t slot)
{
    return base + (2 + Layout<HALVES>::k_slots + slot) * Layout<HALVES>::tile;
}
__device__ __forceinline__ void to_tensor_cores() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// The tiles of the stretch, of K (which = 0) or V (1), a box a lane: lanes are
// (half, box).
template <int HALVES>
__device__ __forceinline__ void copy_role(const AttendDev &a, const SchedShared &sched, int which, const CUtensorMap *map,
                                          uint32_t base, const Bars &b, volatile int32_t *dead)
{
    using L = Layout<HALVES>;
    const int lane = threadIdx.x & 31;
    const int box_log = min(a.block_log, 7), boxes = KT >> box_log;        // 16 at most
    const int box = lane % boxes, half = lane / boxes;
    const bool asks = half < HALVES;
    const uint32_t dst = (which ? v_at<HALVES>(base, 0) : k_at<HALVES>(base, 0)) + half * L::half + (box << box_log) * 128;
    const uint32_t full = which ? b.v_full : b.k_full, empty = which ? b.v_empty : b.k_empty;
    const uint32_t slots = which ? L::v_slots : L::k_slots;
    const int32_t in_block = (1 << a.block_log) - 1;

    Cursor<Shape> cur(a, sched);
    const uint32_t lost = which ? 0 : a.lost;
    uint32_t slot = 0, turn = 0, used = 0;
    bool stop = false;
    do {
        const int32_t *row = a.c.block_table + (int64_t)cur.r * a.c.table_width;
        const int32_t t0 = cur.k.lo / KT + cur.off;
        auto block = [&](int32_t t) {
            return asks ? key_block(a, row, cur.k, t * KT + (box << box_log), 1 << box_log) : -1;
        };
        int32_t id = block(t0);
        for (int32_t i = 0; i < cur.len; ++i) {
            const int32_t after = i + 1 < cur.len ? block(t0 + i + 1) : -1;
            if (used == slots) mbar_wait(empty + 8 * slot, turn ^ 1, dead, a);
            stop = __any_sync(~0u, *dead);              // all lanes go on, or none
            if (stop) break;
            if (lane == 0) mbar_expect(full + 8 * slot, L::tile + lost);
            __syncwarp();
            if (asks)
                box_rows(dst + slot * L::tile, map, full + 8 * slot, half * 64, ((t0 + i) * KT + (box << box_log)) & in_block,
                         cur.outer, id < 0 ? a.blocks : id);
            id = after;
            if (used < slots) ++used;
            if (++slot == slots) {
                slot = 0;
                turn ^= 1;
            }
        }
    } while (!stop && cur.next(a));
    // copies in flight land before the CTA ends, which may not wait for them any more
    int32_t none = 0;
    for (uint32_t x = 0; x < used; ++x) {
        if (slot == 0) turn ^= 1;
        slot = slot ? slot - 1 : slots - 1;
        mbar_wait(full + 8 * slot, turn, &none, a);
    }
}

// Tensor memory: S (and P over it) of stage s at column 128 s, O at 256 + 128 s.
// A warp issues one stage's products: issue waits for the tensor cores, so the
// time that one warp spends on barriers and bookkeeping is the other's products'.
// They pass each other the turn after every O and S: left alone the stages fall
// into step, both at their products, then both at their softmax.
template <typename T, int HALVES>
__device__ __forceinline__ void mma_role(const AttendDev &a, const SchedShared &sched, int s, uint32_t base,
                                         uint32_t tmem, const Bars &b, volatile int32_t *dead)
{
    using L = Layout<HALVES>;
    const uint32_t kind_s = mma_kind<T>(KT, false), kind_o = mma_kind<T>(L::width, true);
    const uint32_t t_s = tmem + 128 * s, t_o = tmem + 256 + 128 * s;
    const uint64_t q_op = smem_operand(base + s * L::tile, 16, 1024);
    Cursor<Shape> cur(a, sched);
    uint32_t ks = 0, k_turn = 0, vs = 0, v_turn = 0, q_turn = 0, p_turn = 0, pass = 0;
    auto step = [](uint32_t &slot, uint32_t &turn, uint32_t slots) {
        if (++slot == slots) {
            slot = 0;
            turn ^= 1;
        }
    };
    auto issue_s = [&]() {                              // K has been waited for
        const uint64_t k_op = smem_operand(k_at<HALVES>(base, ks), 16, 1024);
        if (elected()) {
#pragma unroll
            for (int h = 0; h < HALVES; ++h)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    constexpr int half = L::half >> 4;
                    mma_ss(t_s, q_op + h * half + 2 * k, k_op + h * half + 2 * k, kind_s, h + k > 0);
                }
            tc_commit(b.s_full + 8 * s);
            tc_commit(b.k_empty + 8 * ks);
        }
        step(ks, k_turn, L::k_slots);
    };
    do {
        if (s * kRows >= Shape::rows(a, cur.q) - cur.inner * 2 * kRows) {        // no rows in this stage
            for (int32_t i = 0; i < cur.len; ++i) {
                mbar_wait(b.k_full + 8 * ks, k_turn, dead, a);
                mbar_wait(b.v_full + 8 * vs, v_turn, dead, a);
                if (elected()) {
                    mbar_arrive(b.k_empty + 8 * ks);
                    mbar_arrive(b.v_empty + 8 * vs);
                }
                step(ks, k_turn, L::k_slots);
                step(vs, v_turn, L::v_slots);
            }
            continue;
        }
        const bool both = Shape::rows(a, cur.q) - cur.inner * 2 * kRows > kRows;
        mbar_wait(b.q_full + 8 * s, q_turn & 1, dead, a);
        mbar_wait(b.k_full + 8 * ks, k_turn, dead, a);
        tc_after();
        issue_s();
        // O is free when its last item's output has been read
        if (q_turn) mbar_wait(b.o_free + 8 * s, (q_turn - 1) & 1, dead, a);
        for (int32_t i = 0; i < cur.len; ++i) {
            // what is likely there already first: a wait costs 85 cycles even then
            mbar_wait(b.v_full + 8 * vs, v_turn, dead, a);
            if (i + 1 < cur.len) mbar_wait(b.k_full + 8 * ks, k_turn, dead, a);
            if (both) {
                if (s == 1 || pass) mbar_wait(b.pass + 8 * s, (pass + s + 1) & 1, dead, a);
                ++pass;
            }
            const uint64_t v_op = smem_operand(v_at<HALVES>(base, vs), L::half, 1024);
            mbar_wait(b.p_full + 8 * s, p_turn++ & 1, dead, a);
            tc_after();
            if (elected()) {
#pragma unroll
                for (int k = 0; k < KT / 16; ++k)
                    mma_ts(t_o, t_s + 8 * k, v_op + 128 * k, kind_o, i > 0 || k > 0);
                tc_commit(b.v_empty + 8 * vs);
                if (i == cur.len - 1) tc_commit(b.o_done + 8 * s);
            }
            step(vs, v_turn, L::v_slots);
            if (i + 1 < cur.len) issue_s();
            if (both && elected()) mbar_arrive(b.pass + 8 * (1 - s));
        }
        ++q_turn;
    } while (cur.next(a));
    // every product has ended before the tensor memory is given back
    if (elected()) tc_commit(b.fin + 8 * s);
    int32_t none = 0;
    mbar_wait(b.fin + 8 * s, 0, &none, a);
}

// A warpgroup replaces what is not finite in a V tile by 0.  Where that is in a
// row from key lo to hi, `mark` says so first: the other stage's warpgroup does
// the same beside this one and may find the zeros already.
template <typename T, int HALVES>
__device__ __forceinline__ void clean_tile(uint4 *v, int t, int32_t j0, int32_t lo, int32_t hi, volatile int32_t *mark,
                                           int32_t tag)
{
    using L = Layout<HALVES>;
    uint32_t any = 0;
#pragma unroll 8
    for (int x = t; x < L::tile / 16; x += kRows) {
        const uint4 y = v[x];
        any = taint<T>(y.x, taint<T>(y.y, taint<T>(y.z, taint<T>(y.w, any))));
    }
    if ((any & 0x7fff7fffu) != 0) {
#pragma unroll 1
        for (int x = t; x < L::tile / 16; x += kRows) {
            const uint4 y = v[x];
            uint32_t e[4] = {y.x, y.y, y.z, y.w};
            bool hit = false;
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                if (not_finite<T>(e[n])) { e[n] &= 0xffff0000u; hit = true; }
                if (not_finite<T>(e[n] >> 16)) { e[n] &= 0xffffu; hit = true; }
            }
            if (!hit) continue;
            const int32_t j = j0 + (int32_t)(x * 16 % L::half / 128);
            if (j >= lo && j <= hi) *mark = tag;
            __threadfence_block();
            v[x] = make_uint4(e[0], e[1], e[2], e[3]);
        }
    }
    to_tensor_cores();
}

// The stages' rows of an item.
__device__ __forceinline__ int32_t stage_row(const Cursor<Shape> &c, int s) { return c.inner * 2 * kRows + s * kRows; }

// What the roles share beside the tiles; a stage's softmax hands its rows' m and l
// to the output.
template <int HALVES> struct Shared {
    SchedShared sched;
    float m[2][kRows], l[2][kRows];
    uint64_t bar[2 * (Layout<HALVES>::k_slots + Layout<HALVES>::v_slots) + 18];
    int32_t dead, last, more[2], bad[kBad];
    uint32_t tmem;
    alignas(8) uint8_t walk[2][sizeof(Cursor<Shape>)];  // the softmax's, kept out of its registers
};

// One stage: queries to shared memory, softmax of its S.
template <typename T, int HALVES>
__device__ __forceinline__ void softmax_role(const AttendDev &a, const SchedShared &sched, int s, uint8_t *mem, uint32_t base,
                                             uint32_t tmem, const Bars &b, volatile float *m_out, volatile float *l_out,
                                             volatile int32_t *bad, volatile int32_t *dead, Cursor<Shape> *walk,
                                             volatile int32_t *more)
{
    using L = Layout<HALVES>;
    const int t = threadIdx.x & 127;
    const uint32_t t_s = tmem + ((uint32_t)(t & ~31) << 16) + 128 * s, t_o = t_s + 256;

    // asks for the stage's queries, a fixed 16-byte piece of every 16th or 8th row a thread
    auto ask_q = [&](const Cursor<Shape> &c) {
        constexpr int per = 8 * HALVES, step = kRows / per;
        const int piece = t % per, first = t / per;
        const int32_t rows = Shape::rows(a, c.q), r0 = stage_row(c, s);
        const bool in = piece * 8 < a.dim;
        const char *q = reinterpret_cast<const char *>(static_cast<const T *>(a.c.q) + (int64_t)c.q.first * a.c.q_token_stride +
                                                       (int64_t)c.outer * a.c.group * a.c.q_head_stride + (in ? piece * 8 : 0));
        const uint32_t dst = base + s * L::tile + (piece >> 3) * L::half + first * 128;
#pragma unroll 4
        for (int i = 0; i < kRows / step; ++i) {
            const int32_t row = min(r0 + first + i * step, rows - 1), tok = div_group(a, row), g = row - tok * a.c.group;
            copy16(dst + i * step * 128 + (((piece ^ (first + i * step)) & 7) << 4),
                   q + 2 * (tok * a.c.q_token_stride + g * a.c.q_head_stride), in && r0 + first + i * step < rows ? 16 : 0);
        }
    };
    auto have_q = [&]() {
        copies_wait();
        to_tensor_cores();
        mbar_arrive(b.q_full + 8 * s);
    };

    // one thread walks, all read
    Cursor<Shape> &cur = *walk;
    if (t == 0) new (walk) Cursor<Shape>(a, sched);
    named_sync(2 + s, kRows);
    auto walk_on = [&]() {
        named_sync(2 + s, kRows);
        if (t == 0) *more = cur.next(a);
        named_sync(2 + s, kRows);
        return *more != 0;
    };
    uint32_t s_turn = 0, k = 0, given = 0;              // k: tile of the stretch
    int32_t item = 0;
    bool asked = false;
    for (bool go = true; go; ++item) {
        const int32_t rows = Shape::rows(a, cur.q), r0 = stage_row(cur, s), row = r0 + t;
        if (r0 >= rows) {                               // this item has one stage only
            k += cur.len;
            go = walk_on();
            continue;
        }
        if (!asked) {
            ask_q(cur);
            have_q();
        }
        asked = false;
        const bool live = row < rows;
        const int32_t pos = live ? Shape::pos(a, cur.q, row) : -1, lo = pos < 0 ? 0 : first_key(a, pos);
        const Common all(a, cur.q, r0, min(r0 + kRows, rows) - 1);
        const Common item_sees(a, cur.q, r0 - s * kRows, min(r0 - s * kRows + 2 * kRows, rows) - 1);
        const int32_t t0 = cur.k.lo / KT + cur.off, len = cur.len;
        const Keys keys = cur.k;
        float m = live ? -INFINITY : 0.f, l = 0.f;

        for (int32_t i = 0; i < len; ++i, ++k) {
            mbar_wait(b.s_full + 8 * s, s_turn++ & 1, dead, a);
            tc_after();
            if (i == len - 1) {
                // the last S is there, so the queries' place is free: the next item's are asked for
                go = walk_on();
                asked = go && stage_row(cur, s) < Shape::rows(a, cur.q);
                if (asked) ask_q(cur);
            }
            const int32_t j0 = (t0 + i) * KT;
            const bool late = j0 + KT - 1 > all.hi, early = j0 < all.lo;
            const int32_t from = lo - j0, to = pos - j0;
            // 64 columns of S; keys that the row does not see are -infinity
            auto load = [&](uint32_t (&x)[64], int h) {
                tc_ld64(x, t_s + 64 * h);
                if (late) {
#pragma unroll
                    for (int c = 0; c < 64; ++c)
                        if (c > to - 64 * h) x[c] = 0xff800000u;
                }
                if (early) {
#pragma unroll
                    for (int c = 0; c < 64; ++c)
                        if (c < from - 64 * h) x[c] = 0xff800000u;
                }
            };
            uint32_t p[64];
            // The weights are computed from the m at hand, without a look at the
            // maximum: their sum shows whether m is still good (no weight is above
            // it).  If not, as in the first tile with a key to see, the maximum is
            // found, m moves and they are computed once more.  A warp does that
            // together, but a row whose m is good keeps it: its bits do not depend
            // on the rows beside it, which may see keys that it does not.
            float total = INFINITY;
            for (bool sure = i == 0;;) {
                if (sure) {
                    float up = m;
#pragma unroll 1
                    for (int h = 0; h < 2; ++h) {
                        uint32_t x[64];
                        load(x, h);
                        float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                        for (int c = 0; c < 64; c += 2)
                            top[(c >> 1) & 3] = max3(top[(c >> 1) & 3], __uint_as_float(x[c]), __uint_as_float(x[c + 1]));
                        up = fmaxf(up, fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * a.scale_log2);
                    }
                    if (total <= kMaxSum && m != -INFINITY) up = m;
                    if (i > 0) {
                        // every product on O that was issued before this S has ended with it
                        const float f = up == m ? 1.f : exp2_approx(m - up);
                        l *= f;
#pragma unroll 1
                        for (int c = 0; c < L::width; c += 8) {
                            uint32_t o[8];
                            tc_ld8(o, t_o + c);
#pragma unroll
                            for (int y = 0; y < 8; ++y) o[y] = __float_as_uint(__uint_as_float(o[y]) * f);
                            tc_st8(t_o + c, o);
                        }
                    }
                    m = up;
                }
                const float at = m == -INFINITY ? 0.f : m;
                const uint64_t mul = pair(a.scale_log2, a.scale_log2), sub = pair(-at, -at);
                uint64_t sum[2] = {0, 0};
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t x[64];
                    load(x, h);
#pragma unroll
                    for (int c = 0; c < 64; c += 2) {
                        const float2 e = unpair(fma2(pair(__uint_as_float(x[c]), __uint_as_float(x[c + 1])), mul, sub));
                        const float p0 = exp2_approx(e.x), p1 = exp2_approx(e.y);
                        sum[(c >> 1) & 1] = add2(sum[(c >> 1) & 1], pair(p0, p1));
                        p[32 * h + c / 2] = Pack<T>::two(p0, p1);
                    }
                }
                const float2 both = unpair(add2(sum[0], sum[1]));
                total = both.x + both.y;
                if (sure || !__any_sync(~0u, !(total <= kMaxSum) || m == -INFINITY)) break;
                sure = true;
            }
            tc_st32(t_s, p);
            tc_st32(t_s + 32, p + 32);
            if (!item_sees.covers(j0)) {
                const uint32_t slot = k % L::v_slots;
                mbar_wait(b.v_full + 8 * slot, (k / L::v_slots) & 1, dead, a);
                clean_tile<T, HALVES>(reinterpret_cast<uint4 *>(mem + v_at<HALVES>(0, slot)), t, j0, keys.lo, keys.hi,
                                      bad + item % kBad, item + 1);
            }
            l += total;
            tc_wait_st();
            tc_before();
            mbar_arrive(b.p_full + 8 * s);
        }
        if (asked) have_q();
        if (given) mbar_wait(b.stat_free + 8 * s, (given - 1) & 1, dead, a);
        ++given;
        m_out[t] = m;
        l_out[t] = l;
        mbar_arrive(b.stat_full + 8 * s);
    }
}

// A row of the output: where it goes.
template <typename T> struct OutRow {
    const AttendDev &a;
    T *out;
    float *lse;
    bool live, sees;                                    // a row of the request; one with a key to see
    __device__ __forceinline__ OutRow(const AttendDev &a_, const Cursor<Shape> &c, int32_t row)
        : a(a_), live(row < Shape::rows(a_, c.q))
    {
        const int32_t in = div_group(a, row), tok = c.q.first + in, head = c.outer * a.c.group + row - in * a.c.group;
        out = static_cast<T *>(a.c.out) + (int64_t)tok * a.c.out_token_stride + (int64_t)head * a.c.out_head_stride;
        lse = a.c.lse ? a.c.lse + (int64_t)tok * a.c.q_heads + head : nullptr;
        sees = c.q.length - c.q.q_len + in >= 0;
    }
    __device__ __forceinline__ float inverse(float sum) const { return inverse_sum(sum, sees); }
    // 16 columns
    __device__ __forceinline__ void put(const float *o, int c, float inv) const
    {
        uint32_t w[8];
#pragma unroll
        for (int y = 0; y < 8; ++y) w[y] = Pack<T>::two(o[2 * y] * inv, o[2 * y + 1] * inv);
        if (!live) return;
        if (a.wide_out) {                               // whole sectors
            if (c < a.dim)
                asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(out + c), "r"(w[0]), "r"(w[1]),
                             "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                             : "memory");
        } else {
#pragma unroll
            for (int y = 0; y < 8; y += 4)
                if (c + 2 * y < a.dim)
                    *reinterpret_cast<uint4 *>(out + c + 2 * y) = make_uint4(w[y], w[y + 1], w[y + 2], w[y + 3]);
        }
    }
    __device__ __forceinline__ void put_lse(float top, float sum) const
    {
        if (live && lse) *lse = sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
    }
};

// The pieces of an item, from the CTA that has its first tile on.
template <int HALVES> struct Pieces {
    static constexpr int width = Layout<HALVES>::width;
    const AttendDev &a;
    int32_t cta0;
    __device__ __forceinline__ float *stat(int32_t p, int s, int t) const
    {
        return a.piece_stat + (piece_slot(cta0, p) * 2 + s) * 2 * kRows + t;
    }
    __device__ __forceinline__ float4 *at(int32_t p, int s, int c, int t) const
    {
        return reinterpret_cast<float4 *>(a.piece) + ((int64_t)(piece_slot(cta0, p) * 2 + s) * (width / 4) + c / 4) * kRows + t;
    }
    // joins a stage's n <= kAlone pieces; the statistics' loads are on their way together
    template <typename T> __device__ __forceinline__ void join(int s, int t, int32_t n, const OutRow<T> &out) const
    {
        if (!out.live) return;
        float f[kAlone], part[kAlone], top = -INFINITY, sum = 0.f;
#pragma unroll
        for (int p = 0; p < kAlone; ++p) {
            f[p] = __ldcg(stat(min(p, n - 1), s, t));
            part[p] = __ldcg(stat(min(p, n - 1), s, t) + kRows);
        }
#pragma unroll
        for (int p = 0; p < kAlone; ++p) top = fmaxf(top, f[p]);
        const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
        for (int p = 0; p < kAlone; ++p) {
            f[p] = exp2_approx(f[p] - base);
            if (p < n) sum = fmaf(f[p], part[p], sum);
        }
        const float scale = out.inverse(sum);
#pragma unroll 1
        for (int c = 0; c < width; c += 32) {
            float o[32];
#pragma unroll
            for (int y = 0; y < 32; ++y) o[y] = 0.f;
#pragma unroll
            for (int p = 0; p < kAlone; ++p)
                if (p < n) add<32>(o, f[p], at(p, s, c, t));
            out.put(o, c, scale);
            out.put(o + 16, c + 16, scale);
        }
        out.put_lse(top, sum);
    }
    // 16 columns of a stage's n pieces
    template <typename T>
    __device__ __forceinline__ void join_share(int s, int t, int32_t n, const OutRow<T> &out, int c, float top) const
    {
        if (!out.live) return;
        const float base = top == -INFINITY ? 0.f : top;
        float sum = 0.f, o[16];
#pragma unroll
        for (int y = 0; y < 16; ++y) o[y] = 0.f;
#pragma unroll 2
        for (int32_t p = 0; p < n; ++p) {
            const float f = exp2_approx(__ldcg(stat(p, s, t)) - base);
            sum = fmaf(f, __ldcg(stat(p, s, t) + kRows), sum);
            add<16>(o, f, at(p, s, c, t));
        }
        out.put(o, c, out.inverse(sum));
        if (c == 0) out.put_lse(top, sum);
    }
    __device__ __forceinline__ float highest(int s, int t, int32_t n) const
    {
        float top = -INFINITY;
#pragma unroll 4
        for (int32_t p = 0; p < n; ++p) top = fmaxf(top, __ldcg(stat(p, s, t)));
        return top;
    }

private:
    template <int N> static __device__ __forceinline__ void add(float *o, float f, const float4 *src)
    {
#pragma unroll
        for (int y = 0; y < N; y += 4) {
            const float4 z = __ldcg(src + y / 4 * kRows);
            o[y] = fmaf(f, z.x, o[y]);
            o[y + 1] = fmaf(f, z.y, o[y + 1]);
            o[y + 2] = fmaf(f, z.z, o[y + 2]);
            o[y + 3] = fmaf(f, z.w, o[y + 3]);
        }
    }
};

// The join of an item, in its counters: the first counts the CTAs that have left
// their piece (low half) and, of many pieces, those that are through with the join
// (high half), the second the shares taken. Up to kAlone pieces are joined by the
// CTA that is last to leave one, beside its next tiles. More would take it long (a
// piece is up to 128 KB, and a join's rate is one SM's), so the join is cut into
// shares of 16 columns of a stage, which the last CTA and those that are at their
// end take one by one; those wait for it a little while, and nothing depends on it
// that they do.  100 new tokens after 50,000 (16 heads on 2, 19 pieces an item): 61
// us, 83 where one CTA joins; 30 after 8,000, 4 requests: 42 against 64.  Shares
// from 3 pieces on cost more than they give (8 x 60-700 tokens after 512-8,192: 101
// against 95 us), from 9 on less (500 tokens after 20,000: 91 against 87).
template <typename T, int HALVES> struct Joiner {
    static constexpr int64_t kPatience = 40000;         // cycles
    const AttendDev &a;
    const Cursor<Shape> &cur;
    const Pieces<HALVES> ps;
    const int32_t pieces;
    volatile int32_t *word;                             // shared memory
    __device__ __forceinline__ Joiner(const AttendDev &a_, const Cursor<Shape> &c, int64_t line, int64_t ctas, volatile int32_t *w)
        : a(a_), cur(c), ps{a_, owner(c.g - c.off, line, ctas)},
          pieces(owner(c.g - c.off + c.tiles - 1, line, ctas) - ps.cta0 + 1), word(w)
    {
    }
    __device__ __forceinline__ int32_t mine() const { return (int32_t)blockIdx.x - ps.cta0; }
    __device__ __forceinline__ int stages() const { return Shape::rows(a, cur.q) - stage_row(cur, 0) > kRows ? 2 : 1; }
    __device__ __forceinline__ int32_t *count() const { return a.count + piece_slot(ps.cta0, 0); }
    __device__ __forceinline__ int32_t *taken() const { return count() + 2 * gridDim.x; }
    // what thread 0 says
    template <class F> __device__ __forceinline__ int32_t agree(F say) const
    {
        named_sync(1, kRows);
        if ((threadIdx.x & 127) == 0) *word = say();
        named_sync(1, kRows);
        return *word;
    }
    // after this CTA's piece; true: help() is to follow
    __device__ __forceinline__ bool arrive() const
    {
        __threadfence();
        const bool last = agree([&] { return (atomicAdd(count(), 1) & 0xffff) == pieces - 1; }) != 0;
        if (!last) return pieces > kAlone;
        __threadfence();
        if (pieces > kAlone) {
            take();
        } else {
            const int t = threadIdx.x & 127;
            if (t == 0) *count() = 0;
#pragma unroll 1
            for (int s = 0; s < stages(); ++s) ps.template join<T>(s, t, pieces, OutRow<T>(a, cur, stage_row(cur, s) + t));
        }
        return false;
    }
    // at the CTA's end, if it was not the last
    __device__ __forceinline__ void help() const
    {
        const bool all = agree([&] {
            const int64_t start = clock64();
            int32_t n;
            do {
                asm volatile("ld.acquire.gpu.global.b32 %0, [%1];" : "=r"(n) : "l"(count()) : "memory");
            } while ((n & 0xffff) != pieces && clock64() - start < kPatience);
            return (n & 0xffff) == pieces;
        }) != 0;
        __threadfence();
        take(all);
    }

private:
    // shares while there are any; the last CTA to be through leaves the counters at 0
    __device__ __forceinline__ void take(bool any = true) const
    {
        constexpr int32_t per_stage = Layout<HALVES>::width / 16;
        const int t = threadIdx.x & 127;
        const int32_t shares = stages() * per_stage;
        int at = -1;
        float top = 0.f;
#pragma unroll 1
        while (any) {
            const int32_t x = agree([&] { return atomicAdd(taken(), 1); });
            if (x >= shares) break;
            const int s = x / per_stage;
            if (s != at) top = ps.highest(s, t, pieces);
            at = s;
            ps.template join_share<T>(s, t, pieces, OutRow<T>(a, cur, stage_row(cur, s) + t), x % per_stage * 16, top);
        }
        if (t == 0 && atomicAdd(count(), 1 << 16) >> 16 == pieces - 1) {
            *taken() = 0;
            *count() = 0;
        }
    }
};

// Outputs, and the join of items in pieces, of both stages in turn, while the
// other warps are at the next item.
template <typename T, int HALVES>
__device__ __forceinline__ void output_role(const AttendDev &a, const SchedShared &sched, uint32_t tmem, const Bars &b,
                                            const volatile float *m_in, const volatile float *l_in,
                                            volatile int32_t *bad, volatile int32_t *dead, volatile int32_t *last)
{
    using L = Layout<HALVES>;
    const int t = threadIdx.x & 127;
    const int64_t line = sched.total, ctas = sched.ctas;
    Cursor<Shape> cur(a, sched);
    uint32_t turn[2] = {0, 0};
    int32_t item = 0;
    uint32_t waits = 0;                                 // this CTA's pieces (bits) whose join it is to help with
    do {
        const int32_t rows = Shape::rows(a, cur.q), t0 = cur.k.lo / KT + cur.off;
        const int stages = rows - stage_row(cur, 0) > kRows ? 2 : 1;
        const bool whole = cur.whole();
        const int64_t g0 = cur.g - cur.off;
        const Pieces<HALVES> ps = {a, owner(g0, line, ctas)};
        const int32_t mine = (int32_t)blockIdx.x - ps.cta0;
#pragma unroll 1
        for (int s = 0; s < stages; ++s) {
            const int32_t row = stage_row(cur, s) + t;
            const OutRow<T> out(a, cur, row);
            const uint32_t t_o = tmem + ((uint32_t)(t & ~31) << 16) + 256 + 128 * s;
            const uint32_t now = s ? turn[1]++ & 1 : turn[0]++ & 1;
            mbar_wait(b.stat_full + 8 * s, now, dead, a);
            const float m = m_in[kRows * s + t], l = l_in[kRows * s + t];
            mbar_arrive(b.stat_free + 8 * s);
            mbar_wait(b.o_done + 8 * s, now, dead, a);
            tc_after();
            const float inv = out.inverse(l);
            const bool fix = bad[item % kBad] == item + 1;
#pragma unroll 1
            for (int c = 0; c < L::width; c += 32) {
                uint32_t x[32];
                float o[32];
                tc_ld32(x, t_o + c);
#pragma unroll
                for (int y = 0; y < 32; ++y) o[y] = __uint_as_float(x[y]);
                if (fix) {
                    const int32_t pos = out.live ? Shape::pos(a, cur.q, row) : -1, r0 = stage_row(cur, 0);
                    const Common item_sees(a, cur.q, r0, min(r0 + 2 * kRows, rows) - 1);
#pragma unroll 1
                    for (int32_t j = max(pos < 0 ? 0 : first_key(a, pos), t0 * KT); j <= min(pos, (t0 + cur.len) * KT - 1); ++j) {
                        if (item_sees.covers(j / KT * KT)) continue;
                        const int32_t id = a.c.block_table[(int64_t)cur.r * a.c.table_width + (j >> a.block_log)];
                        if (id < 0 || id >= a.blocks) continue;
                        const T *v = static_cast<const T *>(a.c.v_cache) + id * a.block_stride +
                                     (j & ((1 << a.block_log) - 1)) * a.token_stride + cur.outer * a.head_stride + c;
#pragma unroll
                        for (int y = 0; y < 32; ++y)
                            if (c + y < a.dim) {
                                const float z = KvType<T>::to_float(v[y]);
                                if (!(fabsf(z) < INFINITY)) o[y] += z;
                            }
                    }
                }
                if (whole) {
                    out.put(o, c, inv);
                    out.put(o + 16, c + 16, inv);
                } else if (out.live) {
#pragma unroll
                    for (int y = 0; y < 32; y += 4)
                        ps.at(mine, s, c, t)[y / 4 * kRows] = make_float4(o[y], o[y + 1], o[y + 2], o[y + 3]);
                }
            }
            tc_before();
            mbar_arrive(b.o_free + 8 * s);
            if (whole) {
                out.put_lse(m, l);
            } else {
                *ps.stat(mine, s, t) = m;
                ps.stat(mine, s, t)[kRows] = l;
            }
        }
        if (!whole && Joiner<T, HALVES>(a, cur, line, ctas, last).arrive()) waits |= 1u << item;
        ++item;
    } while (cur.next(a));
    // a CTA's pieces are of its first two items at most
    if (!waits) return;
    Cursor<Shape> again(a, sched);
    do {
        if (waits & 1) Joiner<T, HALVES>(a, again, line, ctas, last).help();
        waits >>= 1;
    } while (waits && again.next(a));
}

template <typename T, int HALVES>
__global__ void __launch_bounds__(kThreads, 1) k_attend_chunk(const __grid_constant__ AttendDev a,
                                                              const __grid_constant__ CUtensorMap km,
                                                              const __grid_constant__ CUtensorMap vm)
{
    using L = Layout<HALVES>;
    extern __shared__ __align__(1024) uint8_t raw[];
    Shared<HALVES> &sh = *reinterpret_cast<Shared<HALVES> *>(raw + L::tiles);
    const int tid = threadIdx.x, warp = tid >> 5;
    const uint32_t base = smem_u32(raw);
    if (base & 1023) {                                  // the swizzle counts from multiples of 1,024 bytes
        if (tid == 0) atomicExch(a.status, (int32_t)PP_ECUDA);
        return;
    }
    Bars b;
    b.k_full = smem_u32(sh.bar);
    b.k_empty = b.k_full + 8 * L::k_slots;
    b.v_full = b.k_empty + 8 * L::k_slots;
    b.v_empty = b.v_full + 8 * L::v_slots;
    b.q_full = b.v_empty + 8 * L::v_slots;
    b.s_full = b.q_full + 16;
    b.p_full = b.s_full + 16;
    b.o_done = b.p_full + 16;
    b.o_free = b.o_done + 16;
    b.fin = b.o_free + 16;
    b.pass = b.fin + 16;
    b.stat_full = b.pass + 16;
    b.stat_free = b.stat_full + 16;
    if (tid == 0) {
        sh.dead = 0;
        for (int i = 0; i < L::k_slots; ++i) {
            mbar_init(b.k_full + 8 * i, 1);
            mbar_init(b.k_empty + 8 * i, 2);
        }
        for (int i = 0; i < L::v_slots; ++i) {
            mbar_init(b.v_full + 8 * i, 1);
            mbar_init(b.v_empty + 8 * i, 2);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(b.q_full + 8 * s, kRows);
            mbar_init(b.s_full + 8 * s, 1);
            mbar_init(b.p_full + 8 * s, kRows);
            mbar_init(b.o_done + 8 * s, 1);
            mbar_init(b.o_free + 8 * s, kRows);
            mbar_init(b.fin + 8 * s, 1);
            mbar_init(b.pass + 8 * s, 1);
            mbar_init(b.stat_full + 8 * s, kRows);
            mbar_init(b.stat_free + 8 * s, kRows);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (tid < kBad) sh.bad[tid] = 0;
    // What comes from the kernel before, where this one was launched beside its end (pp_kv8.cu): table and rows.  All
    // CTAs wait for it, so that this kernel's end is its end too.
    auto wait_for_rows = [] { asm volatile("griddepcontrol.wait;" ::: "memory"); };
    if (!schedule<Shape>(a, sh.sched)) {
        wait_for_rows();
        return;
    }
    if (warp == 12) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&sh.tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
        tc_before();
    }
    __syncthreads();
    tc_after();
    const uint32_t tmem = sh.tmem;

    wait_for_rows();

    // 512 threads x 128 registers = 128 x (2 for softmax + for output + for the others)
    constexpr int kSoftmax = HALVES == 2 ? 144 : 128, kOutput = HALVES == 2 ? 144 : 160, kOthers = 512 - 2 * kSoftmax - kOutput;
    if (warp < 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmax));
        softmax_role<T, HALVES>(a, sh.sched, warp >> 2, raw, base, tmem, b, sh.m[warp >> 2], sh.l[warp >> 2], sh.bad, &sh.dead,
                                reinterpret_cast<Cursor<Shape> *>(sh.walk[warp >> 2]), &sh.more[warp >> 2]);
    } else if (warp < 12) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kOutput));
        output_role<T, HALVES>(a, sh.sched, tmem, b, sh.m[0], sh.l[0], sh.bad, &sh.dead, &sh.last);
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOthers));
        if (warp < 14) mma_role<T, HALVES>(a, sh.sched, warp - 12, base, tmem, b, &sh.dead);
        else copy_role<HALVES>(a, sh.sched, warp - 14, warp == 14 ? &km : &vm, base, b, &sh.dead);
    }
    tc_before();
    __syncthreads();
    if (warp == 12) {
        tc_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
    }
}

template <int HALVES> constexpr int shared_bytes()
{
    constexpr int bytes = Layout<HALVES>::tiles + sizeof(Shared<HALVES>);
    static_assert(bytes <= 232448, "shared memory of a CTA");
    return bytes;
}

template <typename T, int HALVES> static cudaError_t prepare_t()
{
    return cudaFuncSetAttribute(k_attend_chunk<T, HALVES>, cudaFuncAttributeMaxDynamicSharedMemorySize, shared_bytes<HALVES>());
}

template <typename T, int HALVES>
static pp_status launch_t(pp_kv *kv, const AttendArgs &c, bool beside, cudaStream_t st)
{
    AttendDev a = attend_dev(kv, c);
    a.few_pieces = beside;
    CUtensorMap km, vm;
    const int32_t rows = std::min(kv->block_size, KT);
    pp_status s = cache_map(kv, c.k_cache, rows, &km);
    if (s == PP_OK) s = cache_map(kv, c.v_cache, rows, &vm);
    if (s != PP_OK) return s;
    if (!beside) {
        k_attend_chunk<T, HALVES><<<kv->sm_count, kThreads, shared_bytes<HALVES>(), st>>>(a, km, vm);
        PP_CUDA(cudaGetLastError());
        return PP_OK;
    }
    cudaLaunchAttribute early = {};
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t config = {};
    config.gridDim = dim3(kv->sm_count);
    config.blockDim = dim3(kThreads);
    config.dynamicSmemBytes = shared_bytes<HALVES>();
    config.stream = st;
    config.attrs = &early;
    config.numAttrs = 1;
    PP_CUDA(cudaLaunchKernelEx(&config, k_attend_chunk<T, HALVES>, a, km, vm));
    return PP_OK;
}

pp_status prepare_attend_chunk()
{
    PP_CUDA((prepare_t<__nv_bfloat16, 1>()));
    PP_CUDA((prepare_t<__nv_bfloat16, 2>()));
    PP_CUDA((prepare_t<__half, 1>()));
    PP_CUDA((prepare_t<__half, 2>()));
    return PP_OK;
}

// beside: the kernel before lets this one start while it ends; only its last CTAs' results are waited for.
pp_status launch_attend_chunk(pp_kv *kv, const AttendArgs &c, bool beside, cudaStream_t st)
{
    if (kv->dtype == PP_KV_BF16)
        return kv->dim > 64 ? launch_t<__nv_bfloat16, 2>(kv, c, beside, st) : launch_t<__nv_bfloat16, 1>(kv, c, beside, st);
    return kv->dim > 64 ? launch_t<__half, 2>(kv, c, beside, st) : launch_t<__half, 1>(kv, c, beside, st);
}

}  // namespace pp
