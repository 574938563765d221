// Attention of single new tokens, or of a few, over the paged cache.
//
// An item is 16 rows (new token, query head) of one K/V head, token first: they
// see the same keys, or all but a few, so each K and V row is read once for them.
// What bounds it is the read of K and V: an operation a byte for each row that
// shares it, 1 (a single token of a head of its own) to 16, and 32 where a second
// item's read comes from L2.  The products run on m16n8k16 tensor instructions with those 16 rows (padded), which
// keeps scores, weights and sums in registers: the score's accumulators are the
// next product's operand as they stand (a 128-row product would have 120 rows of
// padding and pass its weights through tensor memory).  A tile is 128 keys, 16 a
// warp.  Every warp copies its own rows, into a ring of its own (three tiles of
// 64 KB an SM are on their way), and has its own running maximum, sum and output,
// joined once an item: between items no warp waits for another.  Keys that not
// every row sees are masked row by row; an infinite or NaN V row among them is
// replaced by zeros and added to the rows that see it.
// Measured, single passes after a flush of L2: 128 requests of 200 to 16,000 tokens
// (28 heads on 4, width 128, blocks of 16, 1.52 GB) 253 us, 6.0 TB/s or 89% of the
// measured copy rate (among other passes 237, 6.4); two contexts of 131,000 and
// 200,000 tokens 85 us, 4.1 TB/s (67, 5.2): 10 us of it are the launch, the cut
// of the line and the first rows' latency, 5 the joins of 38 pieces an item; 32
// requests of 4 tokens after 5,000 (16 rows on each of 2 heads, 164 MB) 50 us.
// DRAM 75% of its cycles and 17% of the tensor instructions' in the former's half.
#include "pp_attend_token.cuh"

namespace pp {

namespace token {
constexpr int kRows = 16;                           // rows of an item
// an item's weight of 1, 2, 3, 5 tiles: 60 requests x 4 tokens after 50 to 9,000 56, 53, 48, 46 us, 300 single tokens
// after 50 to 3,000 85, 81, 79, 79, 256 after 100 to 8,000 -, 461, 462, 472
using Shape = ShapeOf<kRows, KT, 3>;

template <int HALVES> struct Layout {
    static constexpr int half = kKeys * 128;                    // bytes of 64 columns of a warp's keys
    static constexpr int rows = half * HALVES;                  // of its K or V
    static constexpr int stages = HALVES == 2 ? 3 : 6;
    static constexpr int ring = kWarps * stages * 2 * rows;
    static constexpr int width = 64 * HALVES;
    static constexpr int pitch = width + 4;                     // floats of an output row in shared memory
    static constexpr int join = kWarps / 2 * kRows * pitch * 4;
    static constexpr int bytes = 128 + ring + join;
};

}  // namespace token

// byte offset of element (row, 8 * piece) of a warp's K or V
__device__ __forceinline__ uint32_t row_at(int row, int piece)
{
    return (piece >> 3) * (kKeys * 128) + row * 128 + (((piece ^ row) & 7) << 4);
}

// 16-bit halves that are infinite or NaN become 0
template <typename T> __device__ __forceinline__ uint32_t finite_only(uint32_t x)
{
    constexpr uint32_t e = std::is_same<T, __nv_bfloat16>::value ? 0x7f80u : 0x7c00u;
    if ((x & e) == e) x &= 0xffff0000u;
    if ((x & e << 16) == e << 16) x &= 0xffffu;
    return x;
}
template <typename T> __device__ __forceinline__ float half_value(uint32_t bits)
{
    const uint16_t h = (uint16_t)bits;
    T v;
    memcpy(&v, &h, 2);
    return KvType<T>::to_float(v);
}

// A warp's copies of its keys, tile after tile along the stretch.  Lane l keeps
// the block of the warp's keys in the l-th of the next 32 tiles (two blocks of 8
// tokens: the second's in `upper`), so that a tile waits for no table entry.
template <int HALVES> struct Feed {
    using L = Layout<HALVES>;
    const AttendDev &a;
    Cursor<Shape> cur;
    RowLane<HALVES> rl;
    uint32_t ring, slot = 0;
    int32_t i = 0, lower, upper;
    bool more;
    __device__ __forceinline__ Feed(const AttendDev &a_, const SchedShared &sched, uint32_t ring_)
        : a(a_), cur(a_, sched), rl(a_, L::half), ring(ring_), more(true)
    {
        look();
    }
    __device__ __forceinline__ int32_t first(int32_t tile) const
    {
        return (cur.k.lo / KT + cur.off + tile) * KT + (int32_t)(threadIdx.x >> 5) * kKeys;
    }
    __device__ __forceinline__ void look()
    {
        const int32_t *row = a.c.block_table + (int64_t)cur.r * a.c.table_width;
        const int32_t tile = i + (threadIdx.x & 31), j = first(tile);
        lower = tile < cur.len ? key_block(a, row, cur.k, j, 8) : -1;
        upper = tile >= cur.len ? -1 : a.block_log > 3 && lower >= 0 && j + 8 <= cur.k.hi ? lower : key_block(a, row, cur.k, j + 8, 8);
    }
    // asks for the next tile, into the ring's next place
    __device__ __forceinline__ void ask()
    {
        if (more) {
            const int32_t j0 = first(i), in_block = (1 << a.block_log) - 1;
            const int32_t b0 = __shfl_sync(~0u, lower, i & 31), b1 = __shfl_sync(~0u, upper, i & 31);
            if (j0 <= cur.k.hi && j0 + kKeys - 1 >= cur.k.lo) {
                const int64_t token_bytes = 2 * a.token_stride, head = 2 * cur.outer * a.head_stride;
                const int64_t at0 = head + max(b0, 0) * 2 * a.block_stride + (j0 & in_block) * token_bytes;
                const int64_t at1 = head + max(b1, 0) * 2 * a.block_stride + ((j0 + 8) & in_block) * token_bytes;
                const char *k = static_cast<const char *>(a.c.k_cache), *v = static_cast<const char *>(a.c.v_cache);
                const uint32_t to = ring + slot * 2 * L::rows;
                rl.rows8(to, k + at0, token_bytes, b0 >= 0);
                rl.rows8(to + 1024, k + at1, token_bytes, b1 >= 0);
                rl.rows8(to + L::rows, v + at0, token_bytes, b0 >= 0);
                rl.rows8(to + L::rows + 1024, v + at1, token_bytes, b1 >= 0);
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

template <typename T, int HALVES>
__global__ void __launch_bounds__(kThreads, 1) k_attend_token(const __grid_constant__ AttendDev a)
{
    using L = Layout<HALVES>;
    constexpr int KS = 4 * HALVES;                      // 16-wide steps of the head dimension
    extern __shared__ uint8_t raw[];
    __shared__ SchedShared sched;
    __shared__ float stat[2][kWarps][kRows];
    __shared__ int32_t last;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t base = (smem_u32(raw) + 127) & ~127u;
    float *join = reinterpret_cast<float *>(raw + (base - smem_u32(raw)) + L::ring);
    if (!schedule<Shape>(a, sched)) return;
    const int64_t total = sched.total, ctas = min((int64_t)gridDim.x, total);

    const int r0 = lane >> 2, c0 = 2 * (lane & 3);      // this thread's rows r0, r0 + 8; its columns
    // ldmatrix rows: K (keys outside, dims inside a group of four matrices), V (the other way round)
    const int krow = (lane >> 4) * 8 + (lane & 7), kpiece = (lane >> 3) & 1;
    const int vrow = ((lane >> 3) & 1) * 8 + (lane & 7), vpiece = lane >> 4;
    const int jr = tid >> 4, jd = (tid & 15) * 4;       // joining: row and first columns, 64 apart

    const uint32_t ring = base + warp * L::stages * 2 * L::rows;
    Feed<HALVES> feed(a, sched, ring);
#pragma unroll 1
    for (int x = 0; x < L::stages; ++x) feed.ask();
    Cursor<Shape> cur(a, sched);
    uint32_t slot = 0;
    do {
        const int32_t row0 = cur.inner * kRows, rows = min(kRows, Shape::rows(a, cur.q) - row0);
        uint32_t qf[KS][4];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const bool in = r0 + 8 * x < rows;
            const T *qp = static_cast<const T *>(a.c.q) + (in ? item_row(a, cur, r0 + 8 * x, a.c.q_token_stride, a.c.q_head_stride) : 0);
#pragma unroll
            for (int k = 0; k < KS; ++k) {
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const int d = 16 * k + c0 + 8 * y;
                    qf[k][x + 2 * y] = in && d < a.dim ? __ldg(reinterpret_cast<const uint32_t *>(qp + d)) : 0u;
                }
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
            if (++slot == L::stages) slot = 0;
            const int32_t j0 = (t0 + i) * KT + warp * kKeys;        // this warp's first key
            asm volatile("cp.async.wait_group %0;" ::"n"(L::stages - 1) : "memory");
            __syncwarp();
            if (j0 <= cur.k.hi && j0 + kKeys - 1 >= cur.k.lo) {
                float sc[2][4];
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int x = 0; x < 4; ++x) sc[n][x] = 0.f;
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    uint32_t b[4];
                    ldsm4(b, kt + row_at(krow, 2 * k + kpiece));
                    mma16<T>(sc[0], qf[k], b[0], b[1]);
                    mma16<T>(sc[1], qf[k], b[2], b[3]);
                }
                const bool edge = j0 < all_lo || j0 + kKeys - 1 > all_hi;
                uint32_t vk0 = ~0u, vk1 = ~0u;                      // V rows that some row sees, as the operand holds them
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
                float top[2], base[2];
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    top[x] = fmaxf(fmaxf(sc[0][2 * x], sc[0][2 * x + 1]), fmaxf(sc[1][2 * x], sc[1][2 * x + 1]));
                    top[x] = fmaxf(top[x], __shfl_xor_sync(~0u, top[x], 1));
                    top[x] = fmaxf(top[x], __shfl_xor_sync(~0u, top[x], 2)) * a.scale_log2;
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
                    // some rows see keys that others do not: what is not finite is added to those who do, then cleared
                    bool strange = false;
                    uint4 *const v = reinterpret_cast<uint4 *>(raw + (vt - smem_u32(raw))) + lane;
#pragma unroll
                    for (int x = 0; x < L::rows / 512; ++x) {
                        const int32_t j = j0 + ((4 * x + (lane >> 3)) & (kKeys - 1));   // 128 bytes a key, in each half
                        const uint4 y = v[32 * x];
                        const bool odd = finite_only<T>(y.x) != y.x || finite_only<T>(y.y) != y.y || finite_only<T>(y.z) != y.z ||
                                         finite_only<T>(y.w) != y.w;
                        strange |= odd && j >= cur.k.lo && j <= cur.k.hi;
                    }
                    if (__any_sync(~0u, strange)) {
#pragma unroll
                        for (int y = 0; y < 2; ++y) {
                            const int32_t pos = r0 + 8 * y < rows ? Shape::pos(a, cur.q, row0 + r0 + 8 * y) : -1;
                            const int32_t lo = pos < 0 ? 0 : first_key(a, pos);
#pragma unroll 1
                            for (int32_t j = max(j0, lo); j <= min(j0 + kKeys - 1, pos); ++j) {
#pragma unroll
                                for (int n = 0; n < 2 * KS; ++n) {
                                    const uint32_t two = lds32(vt + row_at(j - j0, n) + 2 * c0);
                                    const uint32_t odd = two ^ finite_only<T>(two);     // only what is not finite is left
                                    if (odd & 0xffffu) o[n][2 * y] += half_value<T>(two);
                                    if (odd >> 16) o[n][2 * y + 1] += half_value<T>(two >> 16);
                                }
                            }
                        }
                        __syncwarp();
#pragma unroll 1
                        for (int x = 0; x < L::rows / 512; ++x) {
                            const uint4 y = v[32 * x];
                            v[32 * x] = make_uint4(finite_only<T>(y.x), finite_only<T>(y.y), finite_only<T>(y.z), finite_only<T>(y.w));
                        }
                        __syncwarp();
                    }
                }
                uint32_t pf[4];
#pragma unroll
                for (int x = 0; x < 2; ++x) base[x] = m[x] == -INFINITY ? 0.f : m[x];
#pragma unroll
                for (int n = 0; n < 2; ++n) {
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        sc[n][x] = exp2_approx(fmaf(sc[n][x], a.scale_log2, -base[x >> 1]));
                        l[x >> 1] += sc[n][x];
                    }
                    pf[2 * n] = Pack<T>::two(sc[n][0], sc[n][1]);
                    pf[2 * n + 1] = Pack<T>::two(sc[n][2], sc[n][3]);
                }
#pragma unroll
                for (int n = 0; n < KS; ++n) {
                    uint32_t b[4];
                    ldsm4_trans(b, vt + row_at(vrow, 2 * n + vpiece));
                    if (edge) {
                        b[0] &= vk0;
                        b[1] &= vk1;
                        b[2] &= vk0;
                        b[3] &= vk1;
                    }
                    mma16<T>(o[2 * n], pf, b[0], b[1]);
                    mma16<T>(o[2 * n + 1], pf, b[2], b[3]);
                }
            }
            __syncwarp();
            feed.ask();                                             // into the place just read
        }

        // join the warps: the upper four hand theirs to the lower four, lane by lane,
        // then a thread has one row's 4 * HALVES columns
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            l[x] += __shfl_xor_sync(~0u, l[x], 1);
            l[x] += __shfl_xor_sync(~0u, l[x], 2);
            if ((lane & 3) == 0) {
                stat[0][warp][r0 + 8 * x] = m[x];
                stat[1][warp][r0 + 8 * x] = l[x];
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
                const float other = stat[0][warp + kWarps / 2][r0 + 8 * x], up = fmaxf(m[x], other);
                const float by = up == -INFINITY ? 0.f : up;
                f[x] = exp2_approx(m[x] - by);
                g[x] = exp2_approx(other - by);
                m[x] = up;
                l[x] = f[x] * l[x] + g[x] * stat[1][warp + kWarps / 2][r0 + 8 * x];
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
                    stat[0][warp][row] = m[x];
                    stat[1][warp][row] = l[x];
                }
                if (row < rows) {
                    float *dst = join + (warp * kRows + row) * L::pitch + c0;
#pragma unroll
                    for (int n = 0; n < 2 * KS; ++n)
                        *reinterpret_cast<float2 *>(dst + 8 * n) = make_float2(o[n][2 * x], o[n][2 * x + 1]);
                }
            }
        }
        __syncthreads();
        float acc[4 * HALVES], top = -INFINITY, sum = 0.f;
#pragma unroll
        for (int d = 0; d < 4 * HALVES; ++d) acc[d] = 0.f;
        if (jr < rows) {
#pragma unroll
            for (int w = 0; w < kWarps / 2; ++w) top = fmaxf(top, stat[0][w][jr]);
            const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
            for (int w = 0; w < kWarps / 2; ++w) {
                const float f = exp2_approx(stat[0][w][jr] - base);
                sum = fmaf(f, stat[1][w][jr], sum);
                const float4 *src = reinterpret_cast<const float4 *>(join + (w * kRows + jr) * L::pitch + jd);
#pragma unroll
                for (int d = 0; d < HALVES; ++d) {
                    const float4 y = src[16 * d];
                    acc[4 * d] = fmaf(f, y.x, acc[4 * d]);
                    acc[4 * d + 1] = fmaf(f, y.y, acc[4 * d + 1]);
                    acc[4 * d + 2] = fmaf(f, y.z, acc[4 * d + 2]);
                    acc[4 * d + 3] = fmaf(f, y.w, acc[4 * d + 3]);
                }
            }
        }

        leave_item<T, Shape, 4 * HALVES, kThreads, kJoinGroup>(a, cur, tid, acc, top, sum, &last, total, ctas, [] { __syncthreads(); });
        __syncthreads();                                // the join's memory is free again
    } while (cur.next(a));
}

template <typename T, int HALVES> static cudaError_t prepare_t()
{
    return cudaFuncSetAttribute(k_attend_token<T, HALVES>, cudaFuncAttributeMaxDynamicSharedMemorySize, Layout<HALVES>::bytes);
}

template <typename T, int HALVES>
static pp_status launch_t(pp_kv *kv, const AttendArgs &c, cudaStream_t st)
{
    const AttendDev a = attend_dev(kv, c);
    k_attend_token<T, HALVES><<<kv->sm_count, kThreads, Layout<HALVES>::bytes, st>>>(a);
    PP_CUDA(cudaGetLastError());
    return PP_OK;
}

pp_status prepare_attend_token()
{
    PP_CUDA((prepare_t<__nv_bfloat16, 1>()));
    PP_CUDA((prepare_t<__nv_bfloat16, 2>()));
    PP_CUDA((prepare_t<__half, 1>()));
    PP_CUDA((prepare_t<__half, 2>()));
    return PP_OK;
}

pp_status launch_attend_token(pp_kv *kv, const AttendArgs &c, cudaStream_t st)
{
    if (kv->dtype == PP_KV_BF16)
        return kv->dim > 64 ? launch_t<__nv_bfloat16, 2>(kv, c, st) : launch_t<__nv_bfloat16, 1>(kv, c, st);
    return kv->dim > 64 ? launch_t<__half, 2>(kv, c, st) : launch_t<__half, 1>(kv, c, st);
}

}  // namespace pp
