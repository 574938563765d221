// Attention of single new tokens, or of a few, over a paged cache of 8-bit numbers.
//
// With codes c (e4m3) and exponents e of the blocks and heads, k = c 2^ke, v = c 2^ve:
//   s_j = scale q.k_j = (scale 2^ke) q.c_j,
//   o = sum_j exp(s_j) 2^ve c_j / sum_j exp(s_j).
// Codes become 16-bit floating numbers exactly, and stay without their scales: K's
// multiplies the score, V's is added to it in log2 units.  So a weight is
//   w_j = exp2(s_j log2(e) + ve - m),  m = max over j of s_j log2(e) + ve - 15,
// at most 2^15 whatever the blocks' sizes are, and the sum below is of w_j 2^-ve.  (ve is
// from -40 to 40: a weight that is lost below 2^-126 is less than 2^-61 of that sum.)
// Queries become 16-bit numbers of 11 bits with a power of two for each row, its
// largest value near 2^14: bf16's 8 bits fit, and what falls below 2^-24 is 2^-38 of
// the row's largest.  Weights are rounded to 16-bit numbers for their product, the sum is
// of unrounded ones: 11 bits down to 2^-29 of the largest, below that off by 2^-40 of it.
// So 2^20 keys lose 2^-11 of the scale of the largest one's block at most (448 of them
// 2^-40 each), about e4m3's own last step at that scale, 2^-10.  With weights up to 1
// instead of 2^15, many small ones beside a large one were part of the sum alone.
//
// An item is 8 or 16 rows (new token, query head) of one K/V head.  The products are
// transposed, keys and the head's elements outside, the rows inside: S^T = K Q^T, O^T =
// V^T P^T.  So 8 rows fill an instruction (m16n8k16), and the codes, which have to be
// widened, are its larger operand.  P^T's operand is S^T's accumulator with its 8 x 8
// squares transposed, one instruction each.  The products' summed index may be taken in
// any order: a lane takes 16 or 32 neighbouring codes of a K row by 16-byte loads, and
// Q's operand is laid out to match.  V's codes come in pairs of columns from a
// transposing load of 16-bit units; a permutation of bytes puts two keys' codes
// together, and an operand's rows are the even columns, then the odd ones.
// The cut of the work and the ring of copies are those of the 16-bit kernel; a warp's 16
// keys are 4 KB here.
//
// Bound by memory, half the 16-bit kernel's bytes, with little room for instructions: a
// code is widened, two to an instruction, on the pipe that the softmax uses too (57% of
// its cycles; all 55% of the issue slots, matrix instructions 16%).  12 warps at the
// products and four that join and store beside them: 128 tokens after 200 to 16,000, 28
// heads on 4 of 128, take 130 us (763 MB, 5.8 TB/s; 112 at the rate of a copy), where
// rows as the larger operand, 16 of them, took 172, and transposed products without
// warps for the outputs 150.  2 after 131,000 and 200,000: 41 us a call in a graph (26 at
// the rate of a copy; 5.5 before the first products, 26 of tiles, 8 to 10 of joins), 4
// after 36 to 900: 11.
#include "pp_attend_token.cuh"

namespace pp {

namespace token {
// ROWS of an item, 64 * HALVES columns
template <int ROWS, int HALVES> struct Layout8 {
    static constexpr int warps = ROWS == 8 ? 12 : 8;            // at the products; four more at the outputs
    static constexpr int threads = 32 * (warps + 4);
    static constexpr int rows = kKeys * 64 * HALVES;            // bytes of a warp's K or V
    static constexpr int stages = (ROWS == 8 ? 3 : 4) * (HALVES == 2 ? 1 : 2);
    static constexpr int ring = warps * stages * 2 * rows;
    static constexpr int width = 64 * HALVES;
    static constexpr int pitch = width + 4;                     // floats of an output row in shared memory
    static constexpr int join = warps * ROWS * pitch * 4;
    static constexpr int bytes = 128 + ring + join;
    static_assert(bytes < 225 * 1024, "shared memory of a CTA");
    // of a thread: the launch's 128 (168 for 12 warps), shared out
    static constexpr int output_registers = ROWS == 8 ? 80 : 88, registers = ROWS == 8 ? 144 : 208;
    static_assert(128 * output_registers + 32 * warps * registers <= threads * (ROWS == 8 ? 128 : 168), "registers of a CTA");
    // an item's weight: 8 rows 2, 3, 5 tiles: 128 tokens after 200 to 16,000 133, 128, 132 us, 300 after 50 to 3,000 48, 47,
    // 50; 16 rows 3, 6, 9: 60 requests x 4 after 50 to 9,000 84, 68, 68, 20 x 3 after 100 to 5,000 26, 27, 45
    using Shape = ShapeOf<ROWS, kKeys * warps, ROWS == 8 ? 3 : 6>;
};
}  // namespace token

// Byte offset of the 16-byte piece `piece` of key `row`.  Lines of 128 bytes (a row, or
// two of 64) are swizzled so that neither 8 rows' pieces of one number nor two rows'
// pieces that a K load takes together share a bank.
template <int HALVES> __device__ __forceinline__ uint32_t piece_at(int row, int piece)
{
    if (HALVES == 2) return row * 128 + (((piece ^ row) & 7) << 4);
    return (row >> 1) * 128 + ((((row & 1) * 4 + piece) ^ (row >> 1 & 3)) << 4);
}

// two codes (the register's low or high half) as 16-bit floating numbers
template <int HIGH> __device__ __forceinline__ uint32_t widen(uint32_t codes)
{
    uint32_t r;
    if (HIGH)
        asm("{\n.reg .b16 lo, hi;\nmov.b32 {lo, hi}, %1;\ncvt.rn.f16x2.e4m3x2 %0, hi;\n}" : "=r"(r) : "r"(codes));
    else
        asm("{\n.reg .b16 lo, hi;\nmov.b32 {lo, hi}, %1;\ncvt.rn.f16x2.e4m3x2 %0, lo;\n}" : "=r"(r) : "r"(codes));
    return r;
}
__device__ __forceinline__ uint4 lds128(uint32_t addr)
{
    uint4 x;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "r"(addr));
    return x;
}
// the transposed 8 x 8 square of 16-bit numbers
__device__ __forceinline__ uint32_t transpose8(uint32_t x)
{
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
__device__ __forceinline__ float power_of_two(int e) { return __int_as_float((e + 127) << 23); }    // -126 <= e <= 127

// 0xff in the bytes that hold NaN
__device__ __forceinline__ uint32_t nan_bytes(uint32_t x)
{
    const uint32_t top = ((x & 0x7f7f7f7fu) + 0x01010101u & 0x80808080u) >> 7;
    return top * 0xffu;
}

// A warp's copies of its keys, tile after tile along the stretch.  Lane l keeps, of the
// warp's keys in the l-th of the next 32 tiles, where they begin in the cache and the
// exponents of their two groups of 8 (K's and V's, a byte each), which go beside the
// tile's keys.
template <class L, int HALVES> struct Feed8 {
    using Shape = typename L::Shape;
    static constexpr int KT = Shape::KT, per_row = 4 * HALVES, step = 32 / per_row;     // pieces of a row, rows at a time
    const AttendDev &a;
    Cursor<Shape> cur;
    const char *from;                   // this lane's piece of a step's rows, where the cache's first key is
    int64_t v_from_k, stride;           // bytes; of `step` rows
    uint32_t ring, slot = 0, dst, bytes;
    uint32_t *exps;                     // shared memory, [stages]
    int32_t i = 0, j0;                  // tile of the part, its first key of this warp
    int64_t at0, at1;                   // keys 0 - 7 and 8 - 15, -1: not in the cache
    uint32_t scales;
    bool more, wide;                    // wide: rows have all their pieces
    __device__ __forceinline__ Feed8(const AttendDev &a_, const SchedShared &sched, uint32_t ring_, uint32_t *exps_)
        : a(a_), cur(a_, sched), stride(step * a_.token_stride), ring(ring_), exps(exps_), more(true), wide(a_.dim == 64 * HALVES)
    {
        const int lane = threadIdx.x & 31, sub = lane / per_row, piece = lane % per_row;
        dst = piece_at<HALVES>(sub, piece);
        bytes = piece * 16 < a.dim ? 16 : 0;
        from = static_cast<const char *>(a.c.k_cache) + sub * a.token_stride + (bytes ? piece * 16 : 0);
        v_from_k = static_cast<const char *>(a.c.v_cache) - static_cast<const char *>(a.c.k_cache);
        enter();
    }
    // a part's first tile
    __device__ __forceinline__ void enter()
    {
        i = 0;
        j0 = (cur.k.lo / KT + cur.off) * KT + (int32_t)(threadIdx.x >> 5) * kKeys;
        if (threadIdx.x < 32) {         // the item's queries, which are read when this tile's turn comes
            const int32_t row = threadIdx.x % Shape::kRows, rows = Shape::rows(a, cur.q) - cur.inner * Shape::kRows;
            const char *q = static_cast<const char *>(a.c.q) + 2 * item_row(a, cur, min(row, rows - 1), a.c.q_token_stride, a.c.q_head_stride);
            const int32_t at = threadIdx.x / Shape::kRows * 128;
            if (row < rows && at < 2 * a.dim) asm volatile("prefetch.global.L2 [%0];" ::"l"(q + at));
        }
        look();
    }
    __device__ __forceinline__ uint32_t scale_of(int32_t block) const
    {
        if (block < 0) return 0;
        const int64_t at = (int64_t)block * a.kv_heads + cur.outer;
        const int ke = min(max((int)a.c.k_exp[at], kLeastExp), kMostExp), ve = min(max((int)a.c.v_exp[at], kLeastExp), kMostExp);
        return (ke & 0xff) | (ve & 0xff) << 8;
    }
    __device__ __forceinline__ void look()
    {
        const int32_t *row = a.c.block_table + (int64_t)cur.r * a.c.table_width;
        const int32_t ahead = threadIdx.x & 31, j = j0 + ahead * KT, in_block = (1 << a.block_log) - 1;
        const bool in = i + ahead < cur.len;
        const int32_t lower = in ? key_block(a, row, cur.k, j, 8) : -1;
        const int32_t upper =
            !in ? -1 : a.block_log > 3 && lower >= 0 && j + 8 <= cur.k.hi ? lower : key_block(a, row, cur.k, j + 8, 8);
        const int64_t head = cur.outer * a.head_stride;
        at0 = lower < 0 ? -1 : head + lower * a.block_stride + (j & in_block) * a.token_stride;
        at1 = upper < 0 ? -1 : head + upper * a.block_stride + ((j + 8) & in_block) * a.token_stride;
        scales = scale_of(lower);
        scales |= (upper == lower ? scales : scale_of(upper)) << 16;
    }
    // 8 rows of K and of V, from row `row` of the tile on
    template <bool ALL> __device__ __forceinline__ void rows8(uint32_t to, int row, int64_t at) const
    {
        const uint32_t some = ALL || at >= 0 ? bytes : 0;
        const char *k = from + (ALL || at >= 0 ? at : 0);
#pragma unroll
        for (int x = 0; x < 8; x += step) {
            // row & 7 = x + sub, x = 0 or 4, so the swizzle of a line of 128 bytes changes by 4 pieces
            const uint32_t d = to + (row + x) * 64 * HALVES + (dst ^ (x << 4));
            if constexpr (ALL) {
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(d), "l"(k) : "memory");
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(d + L::rows), "l"(k + v_from_k) : "memory");
            } else {
                copy16(d, k, some);
                copy16(d + L::rows, k + v_from_k, some);
            }
            k += stride;
        }
    }
    // asks for the next tile, into the ring's next place
    __device__ __forceinline__ void ask()
    {
        if (more) {
            const int64_t b0 = __shfl_sync(~0u, at0, i & 31), b1 = __shfl_sync(~0u, at1, i & 31);
            if (j0 <= cur.k.hi && j0 + kKeys - 1 >= cur.k.lo) {
                const uint32_t to = ring + slot * 2 * L::rows;
                if (wide && b0 >= 0 && b1 >= 0) {
                    rows8<true>(to, 0, b0);
                    rows8<true>(to, 8, b1);
                } else {
                    rows8<false>(to, 0, b0);
                    rows8<false>(to, 8, b1);
                }
                // after the copies, which need not wait for them
                const uint32_t e = __shfl_sync(~0u, scales, i & 31);
                if ((threadIdx.x & 31) == 0) exps[slot] = e;
            }
            j0 += KT;
            if (++i == cur.len) {
                more = cur.next(a);
                if (more) enter();
            } else if ((i & 31) == 0) {
                look();
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        if (++slot == L::stages) slot = 0;
    }
};

// A row's 8 * HALVES pairs of elements of a lane, as operands; what the row is to be
// multiplied with after the product is returned.
template <int HALVES>
__device__ __forceinline__ float query_row(const __half *, const uint4 (&x)[2 * HALVES], uint32_t (&to)[8 * HALVES])
{
#pragma unroll
    for (int n = 0; n < 2 * HALVES; ++n) {
        to[4 * n] = x[n].x;
        to[4 * n + 1] = x[n].y;
        to[4 * n + 2] = x[n].z;
        to[4 * n + 3] = x[n].w;
    }
    return 1.f;
}
template <int HALVES>
__device__ __forceinline__ float query_row(const __nv_bfloat16 *, const uint4 (&x)[2 * HALVES], uint32_t (&to)[8 * HALVES])
{
    uint32_t top = 0;                                   // exponent of the largest finite element
#pragma unroll
    for (int n = 0; n < 2 * HALVES; ++n) {
        const uint32_t w[4] = {x[n].x, x[n].y, x[n].z, x[n].w};
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            to[4 * n + y] = w[y];
            const uint32_t lo = w[y] >> 7 & 0xff, hi = w[y] >> 23 & 0xff;
            top = max(top, max(lo == 255 ? 0 : lo, hi == 255 ? 0 : hi));
        }
    }
    top = max(top, __shfl_xor_sync(~0u, top, 1));       // a row is four lanes'
    top = max(top, __shfl_xor_sync(~0u, top, 2));
    const int up = min(14 + 127 - (int)top, 126);
    const float f = power_of_two(up);
#pragma unroll
    for (int n = 0; n < 8 * HALVES; ++n)
        to[n] = Pack<__half>::two(__uint_as_float(to[n] << 16) * f, __uint_as_float(to[n] & 0xffff0000u) * f);
    return power_of_two(-up);
}

// A warp's part of a row's statistics; the join's place is handed over by barriers.
template <int ROWS, int HALVES> struct Shared8 {
    using L = Layout8<ROWS, HALVES>;
    SchedShared sched;
    float stat[2][L::warps][ROWS];
    uint32_t exps[L::warps][L::stages];
    int32_t last;
};
constexpr int kJoinFull = 1, kJoinFree = 2, kOutput = 3;        // named barriers
// What is subtracted from a row's scores, from their maximum: the largest weight is 2^15 (f16 ends at 2^16).  Rounded
// up, so that it is not more where scores are so large that 15 is not a number of their steps.
__device__ __forceinline__ float below(float top) { return __fsub_ru(top, 15.f); }

// The products of a warp's keys, item after item.
template <typename T, int ROWS, int HALVES>
__device__ __forceinline__ void product_role(const AttendDev &a, Shared8<ROWS, HALVES> &sh, uint8_t *raw, uint32_t base, float *join)
{
    using L = Layout8<ROWS, HALVES>;
    using Shape = typename L::Shape;
    constexpr int NB = ROWS / 8;                        // 8 rows each
    constexpr int KS = 4 * HALVES;                      // 16-wide steps of the head dimension
    constexpr int KT = Shape::KT;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    // accumulators: keys or columns g and g + 8, rows 2 c and 2 c + 1 of 8
    const int g = lane >> 2, c = lane & 3;
    const int dim0 = 16 * HALVES * c;                   // this lane's elements of a K row and of Q
    // ldmatrix rows of V: 8 keys and the next 8, then the same of the next piece
    const int vrow = ((lane >> 3) & 1) * 8 + (lane & 7), vpiece = lane >> 4;

    const uint32_t ring = base + warp * L::stages * 2 * L::rows;
    Feed8<L, HALVES> feed(a, sh.sched, ring, sh.exps[warp]);
#pragma unroll 1
    for (int x = 0; x < L::stages; ++x) feed.ask();
    Cursor<Shape> cur(a, sh.sched);
    uint32_t slot = 0;
    bool again = false;
    do {
        const int32_t row0 = cur.inner * ROWS, rows = min(ROWS, Shape::rows(a, cur.q) - row0);
        uint32_t qf[NB][KS][2];
        float q_by[NB][2];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const bool in = 8 * b + g < rows;
            const T *qp = static_cast<const T *>(a.c.q) +
                          (in ? item_row(a, cur, 8 * b + g, a.c.q_token_stride, a.c.q_head_stride) : 0) + dim0;
            uint4 raw_q[2 * HALVES];
            uint32_t two[2 * KS];
#pragma unroll
            for (int n = 0; n < 2 * HALVES; ++n)
                raw_q[n] = in && dim0 + 8 * n < a.dim ? __ldg(reinterpret_cast<const uint4 *>(qp) + n) : make_uint4(0, 0, 0, 0);
            const float by = query_row<HALVES>(qp, raw_q, two) * a.scale_log2;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                qf[b][k][0] = two[2 * k];
                qf[b][k][1] = two[2 * k + 1];
            }
            q_by[b][0] = __shfl_sync(~0u, by, 8 * c);
            q_by[b][1] = __shfl_sync(~0u, by, 8 * c + 4);
        }
        // keys that all rows see; the rows of one token see the same
        const int32_t pos0 = Shape::pos(a, cur.q, row0), pos1 = cur.k.hi;
        const int32_t all_lo = first_key(a, pos1), all_hi = pos0;
        // last key and first key of row 8 b + 2 c + y (none: -1, 0)
        auto row_pos = [&](int b, int y) { return 8 * b + 2 * c + y < rows ? Shape::pos(a, cur.q, row0 + 8 * b + 2 * c + y) : -1; };
        float o[KS][NB][4], m[NB][2], l[NB][2];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            m[b][0] = m[b][1] = -INFINITY;
            l[b][0] = l[b][1] = 0.f;
#pragma unroll
            for (int n = 0; n < KS; ++n)
#pragma unroll
                for (int x = 0; x < 4; ++x) o[n][b][x] = 0.f;
        }

        const int32_t t0 = cur.k.lo / KT + cur.off;
#pragma unroll 1
        for (int32_t i = 0; i < cur.len; ++i) {
            const uint32_t kt = ring + slot * 2 * L::rows, vt = kt + L::rows;
            const uint32_t *const e_at = &sh.exps[warp][slot];
            if (++slot == L::stages) slot = 0;
            const int32_t j0 = (t0 + i) * KT + warp * kKeys;        // this warp's first key
            asm volatile("cp.async.wait_group %0;" ::"n"(L::stages - 1) : "memory");
            __syncwarp();
            if (j0 <= cur.k.hi && j0 + kKeys - 1 >= cur.k.lo) {
                const uint32_t e = *reinterpret_cast<const volatile uint32_t *>(e_at);
                float sc[NB][4];
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int x = 0; x < 4; ++x) sc[b][x] = 0.f;
#pragma unroll
                for (int h = 0; h < HALVES; ++h) {
                    const uint4 x = lds128(kt + piece_at<HALVES>(g, HALVES * c + h));
                    const uint4 y = lds128(kt + piece_at<HALVES>(8 + g, HALVES * c + h));
                    const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const uint32_t f[4] = {widen<0>(xs[k]), widen<0>(ys[k]), widen<1>(xs[k]), widen<1>(ys[k])};
#pragma unroll
                        for (int b = 0; b < NB; ++b) mma16<__half>(sc[b], f, qf[b][4 * h + k][0], qf[b][4 * h + k][1]);
                    }
                }
                const bool edge = j0 < all_lo || j0 + kKeys - 1 > all_hi;
                uint32_t vk0 = ~0u, vk1 = ~0u;                      // V rows that some row sees, as the operand holds them
                float v_down[2];
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    const int ke = (int8_t)(e >> 16 * n), ve = (int8_t)(e >> (16 * n + 8));
                    const float by = power_of_two(ke);
                    v_down[n] = power_of_two(-ve);
#pragma unroll
                    for (int b = 0; b < NB; ++b)
#pragma unroll
                        for (int y = 0; y < 2; ++y) sc[b][2 * n + y] = fmaf(sc[b][2 * n + y] * by, q_by[b][y], (float)ve);
                }
                if (edge) {
#pragma unroll
                    for (int b = 0; b < NB; ++b)
#pragma unroll
                        for (int y = 0; y < 2; ++y) {
                            const int32_t pos = row_pos(b, y), lo = pos < 0 ? 0 : first_key(a, pos);
#pragma unroll
                            for (int n = 0; n < 2; ++n) {
                                const int32_t j = j0 + g + 8 * n;
                                if (j < lo || j > pos) sc[b][2 * n + y] = -INFINITY;
                            }
                        }
                    bool in[4];
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const int32_t j = j0 + 2 * c + (x & 1) + 8 * (x >> 1);
                        in[x] = j >= cur.k.lo && j <= cur.k.hi;
                    }
                    vk0 = keep(in[0], in[1]);
                    vk1 = keep(in[2], in[3]);
                }
                bool higher = false;
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int y = 0; y < 2; ++y) higher |= fmaxf(sc[b][y], sc[b][2 + y]) > m[b][y];
                if (__any_sync(~0u, higher)) {
#pragma unroll
                    for (int b = 0; b < NB; ++b) {
#pragma unroll
                        for (int y = 0; y < 2; ++y) {
                            float up = fmaxf(sc[b][y], sc[b][2 + y]);
                            up = fmaxf(up, __shfl_xor_sync(~0u, up, 4));
                            up = fmaxf(up, __shfl_xor_sync(~0u, up, 8));
                            up = fmaxf(m[b][y], fmaxf(up, __shfl_xor_sync(~0u, up, 16)));
                            const float f = up == -INFINITY ? 1.f : exp2_approx(below(m[b][y]) - below(up));
                            m[b][y] = up;
                            l[b][y] *= f;
#pragma unroll
                            for (int n = 0; n < KS; ++n) {
                                o[n][b][y] *= f;
                                o[n][b][2 + y] *= f;
                            }
                        }
                    }
                }
                if (edge && pos0 != pos1) {
                    // some rows see keys that others do not: a NaN is added to those who do, then cleared
                    bool strange = false;
                    uint4 *const v = reinterpret_cast<uint4 *>(raw + (vt - smem_u32(raw))) + lane;
#pragma unroll
                    for (int x = 0; x < L::rows / 512; ++x) {
                        const uint4 y = v[32 * x];
                        strange |= (nan_bytes(y.x) | nan_bytes(y.y) | nan_bytes(y.z) | nan_bytes(y.w)) != 0;
                    }
                    if (__any_sync(~0u, strange)) {
#pragma unroll
                        for (int b = 0; b < NB; ++b)
#pragma unroll
                            for (int y = 0; y < 2; ++y) {
                                const int32_t pos = row_pos(b, y), lo = pos < 0 ? 0 : first_key(a, pos);
#pragma unroll 1
                                for (int32_t j = max(j0, lo); j <= min(j0 + kKeys - 1, pos); ++j) {
#pragma unroll
                                    for (int n = 0; n < KS; ++n) {
                                        const uint32_t at = vt + piece_at<HALVES>(j - j0, n) + 2 * g;
                                        const uint32_t odd = nan_bytes(lds32(at & ~3u)) >> 8 * (at & 2);
                                        if (odd & 0xffu) o[n][b][y] = NAN;
                                        if (odd & 0xff00u) o[n][b][2 + y] = NAN;
                                    }
                                }
                            }
                        __syncwarp();
#pragma unroll 1
                        for (int x = 0; x < L::rows / 512; ++x) {
                            const uint4 y = v[32 * x];
                            v[32 * x] = make_uint4(y.x & ~nan_bytes(y.x), y.y & ~nan_bytes(y.y), y.z & ~nan_bytes(y.z), y.w & ~nan_bytes(y.w));
                        }
                        __syncwarp();
                    }
                }
                uint32_t pf[NB][2];
#pragma unroll
                for (int b = 0; b < NB; ++b) {
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        const float at = m[b][y] == -INFINITY ? 0.f : below(m[b][y]);
#pragma unroll
                        for (int n = 0; n < 2; ++n) {
                            sc[b][2 * n + y] = exp2_approx(sc[b][2 * n + y] - at);
                            l[b][y] = fmaf(sc[b][2 * n + y], v_down[n], l[b][y]);
                        }
                    }
#pragma unroll
                    for (int n = 0; n < 2; ++n) pf[b][n] = transpose8(Pack<__half>::two(sc[b][2 * n], sc[b][2 * n + 1]));
                }
#pragma unroll
                for (int n = 0; n < KS; n += 2) {
                    uint32_t w[4];
                    ldsm4_trans(w, vt + piece_at<HALVES>(vrow, n + vpiece));
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        // codes of columns d, d + 1 of two keys: to both keys' of d, both keys' of d + 1
                        const uint32_t lo = __byte_perm(w[2 * x], 0, 0x3120), hi = __byte_perm(w[2 * x + 1], 0, 0x3120);
                        uint32_t f[4] = {widen<0>(lo), widen<1>(lo), widen<0>(hi), widen<1>(hi)};
                        if (edge) {
                            f[0] &= vk0;
                            f[1] &= vk0;
                            f[2] &= vk1;
                            f[3] &= vk1;
                        }
#pragma unroll
                        for (int b = 0; b < NB; ++b) mma16<__half>(o[n + x][b], f, pf[b][0], pf[b][1]);
                    }
                }
            }
            __syncwarp();
            feed.ask();                                             // into the place just read
        }

        // hand over, once the last item's place has been read
        if (again) named_sync(kJoinFree, L::threads);
        again = true;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                const int row = 8 * b + 2 * c + y;
                l[b][y] += __shfl_xor_sync(~0u, l[b][y], 4);
                l[b][y] += __shfl_xor_sync(~0u, l[b][y], 8);
                l[b][y] += __shfl_xor_sync(~0u, l[b][y], 16);
                if (g == 0) {
                    sh.stat[0][warp][row] = below(m[b][y]);
                    sh.stat[1][warp][row] = l[b][y];
                }
                float *dst = join + (warp * ROWS + row) * L::pitch + 2 * g;
#pragma unroll
                for (int n = 0; n < KS; ++n) *reinterpret_cast<float2 *>(dst + 16 * n) = make_float2(o[n][b][y], o[n][b][2 + y]);
            }
        }
        named_arrive(kJoinFull, L::threads);
    } while (cur.next(a));
    named_sync(kJoinFree, L::threads);
}

// Joins the warps' parts of the items, and the pieces of items that other CTAs have
// parts of, while the other warps are at the next item.
template <typename T, int ROWS, int HALVES>
__device__ __forceinline__ void output_role(const AttendDev &a, Shared8<ROWS, HALVES> &sh, const float *join)
{
    using L = Layout8<ROWS, HALVES>;
    using Shape = typename L::Shape;
    constexpr int per = L::width * ROWS / 128;
    const int t = threadIdx.x & 127, jr = t / (128 / ROWS), lane = t % (128 / ROWS);
    const int64_t total = sh.sched.total, ctas = min((int64_t)gridDim.x, total);
    Cursor<Shape> cur(a, sh.sched);
    do {
        float acc[per], top = -INFINITY, sum = 0.f;
#pragma unroll
        for (int d = 0; d < per; ++d) acc[d] = 0.f;
        named_sync(kJoinFull, L::threads);
#pragma unroll
        for (int w = 0; w < L::warps; ++w) top = fmaxf(top, sh.stat[0][w][jr]);
        const float at = top == -INFINITY ? 0.f : top;
#pragma unroll 4
        for (int w = 0; w < L::warps; ++w) {
            const float f = exp2_approx(sh.stat[0][w][jr] - at);
            sum = fmaf(f, sh.stat[1][w][jr], sum);
            const float4 *src = reinterpret_cast<const float4 *>(join + (w * ROWS + jr) * L::pitch) + lane;
#pragma unroll
            for (int d = 0; d < per; d += 4) {
                const float4 y = src[d / 4 * (128 / ROWS)];
                acc[d] = fmaf(f, y.x, acc[d]);
                acc[d + 1] = fmaf(f, y.y, acc[d + 1]);
                acc[d + 2] = fmaf(f, y.z, acc[d + 2]);
                acc[d + 3] = fmaf(f, y.w, acc[d + 3]);
            }
        }
        named_arrive(kJoinFree, L::threads);
        leave_item<T, Shape, per, 128, 0>(a, cur, t, acc, top, sum, &sh.last, total, ctas, [] { named_sync(kOutput, 128); });
    } while (cur.next(a));
}

template <typename T, int ROWS, int HALVES>
__global__ void __launch_bounds__(Layout8<ROWS, HALVES>::threads, 1) k_attend_token8(const __grid_constant__ AttendDev a)
{
    using L = Layout8<ROWS, HALVES>;
    extern __shared__ uint8_t raw[];
    __shared__ Shared8<ROWS, HALVES> shared;
    const uint32_t base = (smem_u32(raw) + 127) & ~127u;
    float *join = reinterpret_cast<float *>(raw + (base - smem_u32(raw)) + L::ring);
    if (!schedule<typename L::Shape>(a, shared.sched)) return;
    if (threadIdx.x < 32 * L::warps) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(L::registers));
        product_role<T, ROWS, HALVES>(a, shared, raw, base, join);
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(L::output_registers));
        output_role<T, ROWS, HALVES>(a, shared, join);
    }
}

template <typename T, int ROWS, int HALVES> static cudaError_t prepare_t()
{
    return cudaFuncSetAttribute(k_attend_token8<T, ROWS, HALVES>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                Layout8<ROWS, HALVES>::bytes);
}
template <typename T> static cudaError_t prepare_all()
{
    for (const cudaError_t e : {prepare_t<T, 8, 1>(), prepare_t<T, 8, 2>(), prepare_t<T, 16, 1>(), prepare_t<T, 16, 2>()})
        if (e != cudaSuccess) return e;
    return cudaSuccess;
}

template <typename T, int ROWS, int HALVES>
static pp_status launch_t(pp_kv *kv, const AttendArgs &c, cudaStream_t st)
{
    using L = Layout8<ROWS, HALVES>;
    const AttendDev a = attend_dev(kv, c);
    k_attend_token8<T, ROWS, HALVES><<<kv->sm_count, L::threads, L::bytes, st>>>(a);
    PP_CUDA(cudaGetLastError());
    return PP_OK;
}
template <typename T> static pp_status launch_rows(pp_kv *kv, const AttendArgs &c, cudaStream_t st)
{
    // 8 rows an item where that is all that a request has
    if ((int64_t)c.max_q * c.group <= 8) return kv->dim > 64 ? launch_t<T, 8, 2>(kv, c, st) : launch_t<T, 8, 1>(kv, c, st);
    return kv->dim > 64 ? launch_t<T, 16, 2>(kv, c, st) : launch_t<T, 16, 1>(kv, c, st);
}

pp_status prepare_attend_token8()
{
    PP_CUDA(prepare_all<__nv_bfloat16>());
    PP_CUDA(prepare_all<__half>());
    return PP_OK;
}

pp_status launch_attend_token8(pp_kv *kv, const AttendArgs &c, cudaStream_t st)
{
    return kv->dtype == PP_KV_BF16 ? launch_rows<__nv_bfloat16>(kv, c, st) : launch_rows<__half>(kv, c, st);
}

}  // namespace pp
