// Attention of single new tokens over the paged cache.
//
// An item is one new token and up to 16 query heads of one K/V head: they see
// the same keys, so each K and V row is read once for them.  What bounds it is
// the read of K and V (4 to 32 operations a byte); the products run on
// m16n8k16 tensor instructions with the heads as the 16 rows (padded), which
// keeps scores, weights and sums in registers: the score's accumulators are the
// next product's operand as they stand.  A tile is 64 keys; four warps take 16
// keys each, two groups of warps take turns at the tiles, and every warp has its
// own running maximum, sum and output, joined once an item.
#include <algorithm>
#include <climits>

#include "pp_attend.cuh"

namespace pp {

namespace token {
constexpr int KT = 64;                              // keys per tile
constexpr int kWarps = 8, kGroups = 2;
constexpr int kThreads = 32 * (kWarps + 1);         // and one warp that copies
constexpr int kRows = 16;                           // query heads of an item

template <int HALVES> struct Layout {
    static constexpr int tile = KT * 128 * HALVES;              // bytes of K or of V
    static constexpr int stages = HALVES == 2 ? 4 : 8;
    static constexpr int width = 64 * HALVES;
    static constexpr int pitch = width + 4;                     // floats of an output row in shared memory
    static constexpr int join = kWarps * kRows * pitch * 4;
    static constexpr int bytes = 1024 + stages * 2 * tile + join;
};

struct Shape {
    static constexpr int KT = token::KT;
    static __device__ __forceinline__ int32_t row_tiles(const AttendDev &a) { return (a.c.group + kRows - 1) / kRows; }
    static __device__ __forceinline__ int32_t outer(const AttendDev &a) { return a.kv_heads * row_tiles(a); }
    static __device__ __forceinline__ int32_t inner(const AttendDev &, const Req &q) { return q.q_len; }
    static __device__ __forceinline__ Keys keys(const AttendDev &a, const Req &q, int32_t i)
    {
        const int32_t pos = q.length - q.q_len + i;
        return {pos < 0 ? 0 : first_key(a, pos), pos};
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

// byte offset of element (row, 8 * chunk) of a tile: halves of 64 elements, rows of 128 bytes
__device__ __forceinline__ uint32_t tile_at(int row, int chunk)
{
    return (chunk >> 3) * (KT * 128) + row * 128 + (((chunk ^ row) & 7) << 4);
}

// both 16-bit halves of a register kept or cleared
__device__ __forceinline__ uint32_t keep(bool lo, bool hi) { return (lo ? 0xffffu : 0u) | (hi ? 0xffff0000u : 0u); }

// Copies the stretch's tiles, one box a lane: lanes are (K or V, half, box).
template <int HALVES>
__device__ __forceinline__ void copy_tiles(const AttendDev &a, const SchedShared &sched, const CUtensorMap *km,
                                           const CUtensorMap *vm, uint32_t stage0, uint32_t full, uint32_t empty,
                                           volatile int32_t *dead)
{
    using L = Layout<HALVES>;
    const int lane = threadIdx.x & 31;
    const int box_log = min(a.block_log, 6), boxes = KT >> box_log;        // 8 at most
    const int box = lane % boxes, which = lane / boxes;                    // (half, K or V)
    const bool active = which < 2 * HALVES;
    const int half = which % HALVES;
    const bool is_v = which >= HALVES;
    const uint32_t dst = (is_v ? L::tile : 0) + half * (KT * 128) + (box << box_log) * 128;
    const CUtensorMap *map = is_v ? vm : km;

    Cursor<Shape> cur(a, sched);
    uint32_t seq = 0;
    do {
        const int32_t *row = a.c.block_table + (int64_t)cur.r * a.c.table_width;
        const int32_t head = cur.outer / Shape::row_tiles(a);
        const int32_t t0 = cur.k.lo / KT + cur.off;
        auto entry = [&](int32_t t) {                   // block of this lane's box of tile t
            const int32_t j = t * KT + (box << box_log);
            if (!active || j > cur.k.hi || j + (1 << box_log) <= cur.k.lo) return a.blocks;
            int32_t id = row[j >> a.block_log];
            if (id < 0 || id >= a.blocks) {
                kv_bounds(a.status);
                id = a.blocks;
            }
            return id;
        };
        int32_t id = entry(t0);
        for (int32_t i = 0; i < cur.len; ++i, ++seq) {
            const int32_t after = i + 1 < cur.len ? entry(t0 + i + 1) : 0;
            const uint32_t s = seq % L::stages, turn = seq / L::stages;
            if (turn) mbar_wait(empty + 8 * s, (turn - 1) & 1, dead, a.status);
            if (*dead) break;
            if (lane == 0) mbar_expect(full + 8 * s, 2 * L::tile);
            __syncwarp();
            const int32_t j = (t0 + i) * KT + (box << box_log);
            if (active)
                tma_rows(stage0 + s * 2 * L::tile + dst, map, full + 8 * s, half * 64, j & ((1 << a.block_log) - 1),
                         head, id);
            id = after;
        }
    } while (!*dead && cur.next(a));
    if (*dead) {
        // copies in flight land before the CTA ends (the limit is the same, without a flag)
        int32_t none = 0;
        for (uint32_t x = seq > L::stages ? seq - L::stages : 0; x < seq; ++x)
            mbar_wait(full + 8 * (x % L::stages), (x / L::stages) & 1, &none, a.status);
    }
}

template <typename T, int HALVES>
__global__ void __launch_bounds__(kThreads) k_attend_token(const __grid_constant__ AttendDev a,
                                                           const __grid_constant__ CUtensorMap km,
                                                           const __grid_constant__ CUtensorMap vm)
{
    using L = Layout<HALVES>;
    constexpr int KS = 4 * HALVES;                      // 16-wide steps of the head dimension
    extern __shared__ uint8_t raw[];
    __shared__ SchedShared sched;
    __shared__ alignas(8) uint64_t bars[2 * L::stages];
    __shared__ float stat[2][kWarps][kRows];
    __shared__ int32_t dead, last;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t stage0 = (smem_u32(raw) + 1023) & ~1023u;
    float *join = reinterpret_cast<float *>(raw + (stage0 - smem_u32(raw)) + L::stages * 2 * L::tile);
    const uint32_t full = smem_u32(bars), empty = full + 8 * L::stages;
    if (tid == 0) {
        dead = 0;
        for (int s = 0; s < L::stages; ++s) {
            mbar_init(full + 8 * s, 1);
            mbar_init(empty + 8 * s, kWarps / kGroups);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (!schedule<Shape>(a, sched)) return;             // its barriers order the set-up too
    const int64_t total = sched.total, ctas = min((int64_t)gridDim.x, total);
    if (warp == kWarps) {
        copy_tiles<HALVES>(a, sched, &km, &vm, stage0, full, empty, &dead);
        return;
    }

    const int group = warp / (kWarps / kGroups), sub = warp % (kWarps / kGroups);
    const int r0 = lane >> 2, c0 = 2 * (lane & 3);      // this thread's rows r0, r0 + 8; its columns
    // ldmatrix rows: K (keys outside, dims inside a group of four matrices), V (the other way round)
    const int krow = sub * 16 + (lane >> 4) * 8 + (lane & 7), kchunk = (lane >> 3) & 1;
    const int vrow = sub * 16 + ((lane >> 3) & 1) * 8 + (lane & 7), vchunk = lane >> 4;
    const int jr = tid >> 4, jd = (tid & 15) * (4 * HALVES);          // joining: row and first column

    Cursor<Shape> cur(a, sched);
    uint32_t seq = 0;
    do {
        const int32_t tiles_of = Shape::row_tiles(a), head = cur.outer / tiles_of;
        const int32_t row0 = cur.outer % tiles_of * kRows, rows = min(kRows, a.c.group - row0);
        const int32_t tok = cur.q.first + cur.inner;
        const T *qp = static_cast<const T *>(a.c.q) + (int64_t)tok * a.c.q_token_stride +
                      (int64_t)(head * a.c.group + row0) * a.c.q_head_stride;
        uint32_t qf[KS][4];
#pragma unroll
        for (int k = 0; k < KS; ++k) {
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int row = r0 + 8 * (x & 1), d = 16 * k + c0 + 8 * (x >> 1);
                qf[k][x] = row < rows && d < a.dim
                               ? __ldg(reinterpret_cast<const uint32_t *>(qp + row * a.c.q_head_stride + d))
                               : 0u;
            }
        }
        float o[2 * KS][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
        for (int n = 0; n < 2 * KS; ++n)
#pragma unroll
            for (int x = 0; x < 4; ++x) o[n][x] = 0.f;

        const int32_t t0 = cur.k.lo / KT + cur.off;
        for (int32_t i = 0; i < cur.len; ++i, ++seq) {
            if ((int)(seq & (kGroups - 1)) != group) continue;
            const uint32_t s = seq % L::stages;
            const uint32_t kt = stage0 + s * 2 * L::tile, vt = kt + L::tile;
            const int32_t j0 = (t0 + i) * KT + sub * 16;            // this warp's first key
            mbar_wait(full + 8 * s, (seq / L::stages) & 1, &dead, a.status);
            if (j0 <= cur.k.hi && j0 + 15 >= cur.k.lo) {
                float sc[2][4];
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int x = 0; x < 4; ++x) sc[n][x] = 0.f;
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    uint32_t b[4];
                    ldsm4(b, kt + tile_at(krow, 2 * k + kchunk));
                    mma16<T>(sc[0], qf[k], b[0], b[1]);
                    mma16<T>(sc[1], qf[k], b[2], b[3]);
                }
                const bool edge = j0 < cur.k.lo || j0 + 15 > cur.k.hi;
                uint32_t vk0 = ~0u, vk1 = ~0u;                      // V rows that count, as the operand holds them
                if (edge) {
                    bool in[4];
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const int32_t j = j0 + c0 + (x & 1) + 8 * (x >> 1);
                        in[x] = j >= cur.k.lo && j <= cur.k.hi;
                        if (!in[x]) sc[x >> 1][x & 1] = sc[x >> 1][2 + (x & 1)] = -INFINITY;
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
                    ldsm4_trans(b, vt + tile_at(vrow, 2 * n + vchunk));
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
            if (lane == 0) mbar_arrive(empty + 8 * s);
        }

        // join the warps: a thread has one row's 4 * HALVES columns
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            l[x] += __shfl_xor_sync(~0u, l[x], 1);
            l[x] += __shfl_xor_sync(~0u, l[x], 2);
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
        named_sync(1, 32 * kWarps);
        float acc[4 * HALVES], top = -INFINITY, sum = 0.f;
#pragma unroll
        for (int d = 0; d < 4 * HALVES; ++d) acc[d] = 0.f;
        if (jr < rows) {
#pragma unroll
            for (int w = 0; w < kWarps; ++w) top = fmaxf(top, stat[0][w][jr]);
            const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float f = exp2_approx(stat[0][w][jr] - base);
                sum = fmaf(f, stat[1][w][jr], sum);
                const float4 *src = reinterpret_cast<const float4 *>(join + (w * kRows + jr) * L::pitch + jd);
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
                if (jr < rows) {
                    float4 *dst = reinterpret_cast<float4 *>(a.piece + ((int64_t)slot * kRows + jr) * L::width + jd);
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
                named_sync(1, 32 * kWarps);
                if (tid == 0) {
                    last = atomicAdd(count, 1) == of - 1;
                    if (last) *count = 0;
                }
                named_sync(1, 32 * kWarps);
                __threadfence();
                return last != 0;
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
                        reinterpret_cast<const float4 *>(a.piece + ((int64_t)slot * kRows + jr) * L::width + jd);
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
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
            const int32_t x = head * a.c.group + row0 + jr;
            T *dst = static_cast<T *>(a.c.out) + (int64_t)tok * a.c.out_token_stride + x * a.c.out_head_stride + jd;
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
                a.c.lse[(int64_t)tok * a.c.q_heads + x] =
                    sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
        }
        named_sync(1, 32 * kWarps);                     // the join's memory is free again
    } while (cur.next(a));
}

template <typename T, int HALVES>
static pp_status launch_t(pp_kv *kv, const AttendArgs &c, cudaStream_t st)
{
    const AttendDev a = attend_dev(kv, c);
    CUtensorMap km, vm;
    const int32_t rows = std::min(kv->block_size, KT);
    pp_status s = cache_map(kv, c.k_cache, rows, &km);
    if (s == PP_OK) s = cache_map(kv, c.v_cache, rows, &vm);
    if (s != PP_OK) return s;
    PP_CUDA(cudaFuncSetAttribute(k_attend_token<T, HALVES>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 Layout<HALVES>::bytes));
    k_attend_token<T, HALVES><<<kv->sm_count, kThreads, Layout<HALVES>::bytes, st>>>(a, km, vm);
    PP_CUDA(cudaGetLastError());
    return PP_OK;
}

pp_status launch_attend_token(pp_kv *kv, const AttendArgs &c, cudaStream_t st)
{
    if (kv->dtype == PP_KV_BF16)
        return kv->dim > 64 ? launch_t<__nv_bfloat16, 2>(kv, c, st) : launch_t<__nv_bfloat16, 1>(kv, c, st);
    return kv->dim > 64 ? launch_t<__half, 2>(kv, c, st) : launch_t<__half, 1>(kv, c, st);
}

}  // namespace pp
