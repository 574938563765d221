// Attention of single new tokens, or of a few, over a paged cache of 8-bit numbers.
//
// With codes c (e4m3) and exponents e of the blocks and heads, k = c 2^ke, v = c 2^ve:
//   s_j = scale q.k_j = (scale 2^ke) q.c_j,
//   o = sum_j exp(s_j) 2^ve c_j / sum_j exp(s_j).
// Codes become 16-bit floating numbers exactly, and stay without their scales: K's
// multiplies the score, V's is added to it in log2 units.  So a weight is
//   w_j = exp2(s_j log2(e) + ve - m),  m = max over j of s_j log2(e) + ve,
// at most 1 whatever the blocks' sizes are, and the sum below is of w_j 2^-ve.  (ve is
// from -40 to 40: a weight that is lost below 2^-126 is less than 2^-46 of that sum.)
// Queries become 16-bit numbers of 11 bits with a power of two for each row, its
// largest value near 2^14: bf16's 8 bits fit, and what falls below 2^-24 is 2^-38 of
// the row's largest.  Weights are rounded to 11 bits for their product.
//
// Items, tiles, the cut of the work and the joins are those of the 16-bit kernel; a
// warp's 16 keys are 4 KB here.  The products' summed index may be taken in any
// order: a lane takes 16 or 32 neighbouring codes of a K row by 16-byte loads, and Q's
// operand is laid out to match.  V's codes come in pairs of columns from a
// transposing load of 16-bit units; two keys' codes are put together by a permutation
// of bytes, which leaves an output tile the even columns and the next the odd ones.
#include "pp_attend_token.cuh"

namespace pp {

namespace token {
template <int HALVES> struct Layout8 {
    static constexpr int rows = kKeys * 64 * HALVES;            // bytes of a warp's K or V
    static constexpr int stages = HALVES == 2 ? 5 : 10;
    static constexpr int ring = kWarps * stages * 2 * rows;
    static constexpr int bytes = 128 + ring + Join<HALVES>::bytes;
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
__device__ __forceinline__ float power_of_two(int e) { return __int_as_float((e + 127) << 23); }    // -126 <= e <= 127

// 0xff in the bytes that hold NaN
__device__ __forceinline__ uint32_t nan_bytes(uint32_t x)
{
    const uint32_t top = ((x & 0x7f7f7f7fu) + 0x01010101u & 0x80808080u) >> 7;
    return top * 0xffu;
}

// A warp's copies of its keys, as in the 16-bit kernel; beside a tile's keys go the
// exponents of their two groups of 8 (K's and V's, a byte each).
template <int HALVES> struct Feed8 {
    using L = Layout8<HALVES>;
    static constexpr int per_row = 4 * HALVES, step = 32 / per_row;     // pieces of a row, rows at a time
    const AttendDev &a;
    Cursor<Shape> cur;
    uint32_t ring, slot = 0, bytes;
    int64_t src;
    uint32_t *exps;                     // shared memory, [stages]
    int32_t i = 0, lower, upper;
    uint32_t scales;
    bool more;
    __device__ __forceinline__ Feed8(const AttendDev &a_, const SchedShared &sched, uint32_t ring_, uint32_t *exps_)
        : a(a_), cur(a_, sched), ring(ring_), exps(exps_), more(true)
    {
        const int lane = threadIdx.x & 31, sub = lane / per_row, piece = lane % per_row;
        bytes = piece * 16 < a.dim ? 16 : 0;
        src = sub * a.token_stride + (bytes ? piece * 16 : 0);
        look();
    }
    __device__ __forceinline__ int32_t first(int32_t tile) const
    {
        return (cur.k.lo / KT + cur.off + tile) * KT + (int32_t)(threadIdx.x >> 5) * kKeys;
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
        const int32_t tile = i + (threadIdx.x & 31), j = first(tile);
        lower = tile < cur.len ? key_block(a, row, cur.k, j, 8) : -1;
        upper = tile >= cur.len ? -1 : a.block_log > 3 && lower >= 0 && j + 8 <= cur.k.hi ? lower : key_block(a, row, cur.k, j + 8, 8);
        scales = scale_of(lower);
        scales |= (upper == lower ? scales : scale_of(upper)) << 16;
    }
    // 8 rows
    __device__ __forceinline__ void rows8(uint32_t to, int row, const char *from, bool some) const
    {
        const int lane = threadIdx.x & 31, sub = lane / per_row, piece = lane % per_row;
#pragma unroll
        for (int x = 0; x < 8; x += step)
            copy16(to + piece_at<HALVES>(row + x + sub, piece), from + src + x * a.token_stride, some ? bytes : 0);
    }
    // asks for the next tile, into the ring's next place
    __device__ __forceinline__ void ask()
    {
        if (more) {
            const int32_t j0 = first(i), in_block = (1 << a.block_log) - 1;
            const int32_t b0 = __shfl_sync(~0u, lower, i & 31), b1 = __shfl_sync(~0u, upper, i & 31);
            const uint32_t e = __shfl_sync(~0u, scales, i & 31);
            if (j0 <= cur.k.hi && j0 + kKeys - 1 >= cur.k.lo) {
                if ((threadIdx.x & 31) == 0) exps[slot] = e;
                const int64_t head = cur.outer * a.head_stride;
                const int64_t at0 = head + max(b0, 0) * a.block_stride + (j0 & in_block) * a.token_stride;
                const int64_t at1 = head + max(b1, 0) * a.block_stride + ((j0 + 8) & in_block) * a.token_stride;
                const char *k = static_cast<const char *>(a.c.k_cache), *v = static_cast<const char *>(a.c.v_cache);
                const uint32_t to = ring + slot * 2 * L::rows;
                rows8(to, 0, k + at0, b0 >= 0);
                rows8(to, 8, k + at1, b1 >= 0);
                rows8(to + L::rows, 0, v + at0, b0 >= 0);
                rows8(to + L::rows, 8, v + at1, b1 >= 0);
            }
            if (++i == cur.len) {
                i = 0;
                more = cur.next(a);
                if (more) look();
            } else if ((i & 31) == 0) {
                look();
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        if (++slot == L::stages) slot = 0;
    }
};

// A row's 8 * HALVES elements of a lane, as operands; `by` is what the row is to be
// multiplied with after the product.
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

template <typename T, int HALVES>
__global__ void __launch_bounds__(kThreads, 1) k_attend_token8(const __grid_constant__ AttendDev a)
{
    using L = Layout8<HALVES>;
    constexpr int KS = 4 * HALVES;                      // 16-wide steps of the head dimension
    extern __shared__ uint8_t raw[];
    __shared__ SchedShared sched;
    __shared__ JoinShared shared;
    __shared__ uint32_t exps[kWarps][L::stages];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t base = (smem_u32(raw) + 127) & ~127u;
    float *join = reinterpret_cast<float *>(raw + (base - smem_u32(raw)) + L::ring);
    if (!schedule<Shape>(a, sched)) return;
    const int64_t total = sched.total, ctas = min((int64_t)gridDim.x, total);

    const int r0 = lane >> 2, c0 = 2 * (lane & 3);      // this thread's rows r0, r0 + 8; its keys in an operand
    const int dim0 = 16 * HALVES * (lane & 3);          // its elements of a K row and of Q
    // ldmatrix rows of V: 8 keys and the next 8, then the same of the next piece
    const int vrow = ((lane >> 3) & 1) * 8 + (lane & 7), vpiece = lane >> 4;

    const uint32_t ring = base + warp * L::stages * 2 * L::rows;
    Feed8<HALVES> feed(a, sched, ring, exps[warp]);
#pragma unroll 1
    for (int x = 0; x < L::stages; ++x) feed.ask();
    Cursor<Shape> cur(a, sched);
    uint32_t slot = 0;
    do {
        const int32_t row0 = cur.inner * kRows, rows = min(kRows, Shape::rows(a, cur.q) - row0);
        uint32_t qf[KS][4];
        float q_by[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const bool in = r0 + 8 * x < rows;
            const T *qp = static_cast<const T *>(a.c.q) +
                          (in ? item_row(a, cur, r0 + 8 * x, a.c.q_token_stride, a.c.q_head_stride) : 0) + dim0;
            uint4 raw_q[2 * HALVES];
            uint32_t two[2 * KS];
#pragma unroll
            for (int n = 0; n < 2 * HALVES; ++n)
                raw_q[n] = in && dim0 + 8 * n < a.dim ? __ldg(reinterpret_cast<const uint4 *>(qp) + n) : make_uint4(0, 0, 0, 0);
            q_by[x] = query_row<HALVES>(qp, raw_q, two);
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                qf[k][x] = two[2 * k];
                qf[k][x + 2] = two[2 * k + 1];
            }
        }
        // keys that all rows see; the rows of one token see the same
        const int32_t pos0 = Shape::pos(a, cur.q, row0), pos1 = cur.k.hi;
        const int32_t all_lo = first_key(a, pos1), all_hi = pos0;
        float o[2 * KS][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
        for (int n = 0; n < 2 * KS; ++n)
#pragma unroll
            for (int x = 0; x < 4; ++x) o[n][x] = 0.f;

        const int32_t t0 = cur.k.lo / KT + cur.off;
#pragma unroll 1
        for (int32_t i = 0; i < cur.len; ++i) {
            const uint32_t kt = ring + slot * 2 * L::rows, vt = kt + L::rows;
            const uint32_t *const e_at = &exps[warp][slot];
            if (++slot == L::stages) slot = 0;
            const int32_t j0 = (t0 + i) * KT + warp * kKeys;        // this warp's first key
            asm volatile("cp.async.wait_group %0;" ::"n"(L::stages - 1) : "memory");
            __syncwarp();
            if (j0 <= cur.k.hi && j0 + kKeys - 1 >= cur.k.lo) {
                const uint32_t e = *reinterpret_cast<const volatile uint32_t *>(e_at);
                float sc[2][4];
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int x = 0; x < 4; ++x) sc[n][x] = 0.f;
#pragma unroll
                for (int h = 0; h < HALVES; ++h) {
#pragma unroll
                    for (int n = 0; n < 2; ++n) {
                        const uint4 c = lds128(kt + piece_at<HALVES>(8 * n + r0, HALVES * (lane & 3) + h));
                        mma16<__half>(sc[n], qf[4 * h], widen<0>(c.x), widen<1>(c.x));
                        mma16<__half>(sc[n], qf[4 * h + 1], widen<0>(c.y), widen<1>(c.y));
                        mma16<__half>(sc[n], qf[4 * h + 2], widen<0>(c.z), widen<1>(c.z));
                        mma16<__half>(sc[n], qf[4 * h + 3], widen<0>(c.w), widen<1>(c.w));
                    }
                }
                const bool edge = j0 < all_lo || j0 + kKeys - 1 > all_hi;
                uint32_t vk0 = ~0u, vk1 = ~0u;                      // V rows that some row sees, as the operand holds them
                float v_up[2], v_down[2];
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    const int ke = (int8_t)(e >> 16 * n), ve = (int8_t)(e >> (16 * n + 8));
                    const float by = a.scale_log2 * power_of_two(ke);
                    v_up[n] = (float)ve;
                    v_down[n] = power_of_two(-ve);
#pragma unroll
                    for (int x = 0; x < 4; ++x) sc[n][x] = fmaf(sc[n][x] * by, q_by[x >> 1], v_up[n]);
                }
                if (edge) {
                    bool in[4];
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        const int32_t pos = r0 + 8 * y < rows ? Shape::pos(a, cur.q, row0 + r0 + 8 * y) : -1;
                        const int32_t lo = pos < 0 ? 0 : first_key(a, pos);
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            const int32_t j = j0 + c0 + (x & 1) + 8 * (x >> 1);
                            in[x] = j >= cur.k.lo && j <= cur.k.hi;
                            if (j < lo || j > pos) sc[x >> 1][2 * y + (x & 1)] = -INFINITY;
                        }
                    }
                    vk0 = keep(in[0], in[1]);
                    vk1 = keep(in[2], in[3]);
                }
                float top[2], at[2];
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    top[x] = fmaxf(fmaxf(sc[0][2 * x], sc[0][2 * x + 1]), fmaxf(sc[1][2 * x], sc[1][2 * x + 1]));
                    top[x] = fmaxf(top[x], __shfl_xor_sync(~0u, top[x], 1));
                    top[x] = fmaxf(top[x], __shfl_xor_sync(~0u, top[x], 2));
                }
                if (__any_sync(~0u, top[0] > m[0] || top[1] > m[1])) {
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const float up = fmaxf(m[x], top[x]);
                        const float f = up == -INFINITY ? 1.f : exp2_approx(m[x] - up);
                        m[x] = up;
                        l[x] *= f;
#pragma unroll
                        for (int n = 0; n < 2 * KS; ++n) {
                            o[n][2 * x] *= f;
                            o[n][2 * x + 1] *= f;
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
                        for (int y = 0; y < 2; ++y) {
                            const int32_t pos = r0 + 8 * y < rows ? Shape::pos(a, cur.q, row0 + r0 + 8 * y) : -1;
                            const int32_t lo = pos < 0 ? 0 : first_key(a, pos);
#pragma unroll 1
                            for (int32_t j = max(j0, lo); j <= min(j0 + kKeys - 1, pos); ++j) {
#pragma unroll
                                for (int n = 0; n < KS; ++n) {
                                    const uint32_t odd = nan_bytes(lds32(vt + piece_at<HALVES>(j - j0, n) + 2 * c0));
                                    if (odd & 0xffu) o[2 * n][2 * y] = NAN;
                                    if (odd & 0xff00u) o[2 * n + 1][2 * y] = NAN;
                                    if (odd & 0xff0000u) o[2 * n][2 * y + 1] = NAN;
                                    if (odd & 0xff000000u) o[2 * n + 1][2 * y + 1] = NAN;
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
                uint32_t pf[4];
#pragma unroll
                for (int x = 0; x < 2; ++x) at[x] = m[x] == -INFINITY ? 0.f : m[x];
#pragma unroll
                for (int n = 0; n < 2; ++n) {
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        sc[n][x] = exp2_approx(sc[n][x] - at[x >> 1]);
                        l[x >> 1] = fmaf(sc[n][x], v_down[n], l[x >> 1]);
                    }
                    pf[2 * n] = Pack<__half>::two(sc[n][0], sc[n][1]);
                    pf[2 * n + 1] = Pack<__half>::two(sc[n][2], sc[n][3]);
                }
#pragma unroll
                for (int n = 0; n < KS; n += 2) {
                    uint32_t b[4];
                    ldsm4_trans(b, vt + piece_at<HALVES>(vrow, n + vpiece));
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        // codes of columns d, d + 1 of two keys: to both keys' of d, both keys' of d + 1
                        const uint32_t lo = __byte_perm(b[2 * x], 0, 0x3120), hi = __byte_perm(b[2 * x + 1], 0, 0x3120);
                        uint32_t f[4] = {widen<0>(lo), widen<0>(hi), widen<1>(lo), widen<1>(hi)};
                        if (edge) {
                            f[0] &= vk0;
                            f[1] &= vk1;
                            f[2] &= vk0;
                            f[3] &= vk1;
                        }
                        mma16<__half>(o[2 * (n + x)], pf, f[0], f[1]);
                        mma16<__half>(o[2 * (n + x) + 1], pf, f[2], f[3]);
                    }
                }
            }
            __syncwarp();
            feed.ask();                                             // into the place just read
        }
        finish_item<T, HALVES, true>(a, cur, o, m, l, join, shared, total, ctas);
    } while (cur.next(a));
}

template <typename T, int HALVES> static cudaError_t prepare_t()
{
    return cudaFuncSetAttribute(k_attend_token8<T, HALVES>, cudaFuncAttributeMaxDynamicSharedMemorySize, Layout8<HALVES>::bytes);
}

template <typename T, int HALVES>
static pp_status launch_t(pp_kv *kv, const AttendArgs &c, cudaStream_t st)
{
    const AttendDev a = attend_dev(kv, c);
    k_attend_token8<T, HALVES><<<kv->sm_count, kThreads, Layout8<HALVES>::bytes, st>>>(a);
    PP_CUDA(cudaGetLastError());
    return PP_OK;
}

pp_status prepare_attend_token8()
{
    PP_CUDA((prepare_t<__nv_bfloat16, 1>()));
    PP_CUDA((prepare_t<__nv_bfloat16, 2>()));
    PP_CUDA((prepare_t<__half, 1>()));
    PP_CUDA((prepare_t<__half, 2>()));
    return PP_OK;
}

pp_status launch_attend_token8(pp_kv *kv, const AttendArgs &c, cudaStream_t st)
{
    if (kv->dtype == PP_KV_BF16)
        return kv->dim > 64 ? launch_t<__nv_bfloat16, 2>(kv, c, st) : launch_t<__nv_bfloat16, 1>(kv, c, st);
    return kv->dim > 64 ? launch_t<__half, 2>(kv, c, st) : launch_t<__half, 1>(kv, c, st);
}

}  // namespace pp
