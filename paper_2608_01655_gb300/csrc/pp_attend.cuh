// What the attention kernels share: the split of the work over CTAs, the
// asynchronous copies of cache tiles, bounded waits, and the join of the
// pieces of an item that several CTAs computed.
//
// An item is what one pass over keys serves (queries that share a K/V head and
// lie together); its keys are cut into tiles.  The tiles of all items, in a
// fixed order, are one line that is cut into equal stretches, one per CTA, so
// that the load is even whatever the lengths are.  Every CTA works the cut
// out by itself from q_start and length.  A stretch that covers an item only
// in part gives a piece (output not yet divided, maximum, sum).  The last CTA
// to leave a piece of an item sees to their join, in a fixed order and, of chunks,
// with the help of those that are at their end; no CTA has to wait for another.
// Equal stretches cost two joins a CTA at most, 10 to 20 thousand cycles that
// mostly run beside other tiles; whole items only would leave SMs idle (8 requests of 60 to 700 new tokens
// after up to 8,192: 144 items of up to 70 tiles on 152 SMs, 39 tiles a stretch).
#pragma once

#include <cuda.h>

#include "pp_kv.cuh"

namespace pp {

struct AttendDev {
    AttendArgs c;
    int64_t block_stride, token_stride, head_stride;
    int32_t blocks, block_log, dim, kv_heads;
    float scale_log2;                   // scale * log2(e)
    int32_t group_shift;                // x / group = x * group_mul >> group_shift for 0 <= x < 2^30
    uint64_t group_mul;
    int32_t wide_out;                   // rows of out start at 32-byte boundaries
    int32_t *status;
    float *piece;                       // pieces' outputs, [slot][...]
    float *piece_stat;                  // their maxima (log2 units) and sums
    int32_t *count;                     // [2][slots] state of the joins, left at 0 by every launch
    int32_t few_pieces;                 // stretches are long enough that a join takes no longer than they do
    int64_t wait_limit;                 // cycles after which one wait gives up
    uint32_t lost;                      // bytes of a K tile that are waited for and never come (tests)
};

// With few_pieces: what a piece costs its item's join, in tiles.  Of an item of T tiles in stretches of s the
// last ends after s + kPieceTiles T / s tiles, least with s = sqrt(kPieceTiles T).  Stretches of less than two tiles
// are left alone.  2 requests of 85 tokens after 9,300 and 11,200 (2 heads on 1), one tile a stretch 60 us and more, with
// 0.15, 0.42, 1.2 32, 40, 44; 34 after 20,000 (8 on 2) 52, 40, 41, 49; 100 after 50,000 (16 on 2) 68, 67, 67, 69.
constexpr float kPieceTiles = 0.15f;
constexpr int64_t kAttendLimitCycles = 4000ll * 1000 * 1000;  // about 2 s
constexpr int64_t kAttendTestCycles = 4ll * 1000 * 1000;      // about 2 ms, while pp_test_inject has copies lost

// ---------------------------------------------------------------------------
// Requests and their items
// ---------------------------------------------------------------------------
struct Req {
    int32_t first, q_len, length;       // first query row, queries, tokens
};

__device__ __forceinline__ Req load_req(const AttendDev &a, int32_t r, bool report)
{
    const int32_t x = a.c.q_start[r], y = a.c.q_start[r + 1], n = a.c.length[r];
    const int64_t room = (int64_t)a.c.table_width << a.block_log;
    Req q;
    q.first = min(max(x, 0), a.c.tokens);
    q.q_len = min(max(y, q.first), a.c.tokens) - q.first;
    q.length = (int32_t)min((int64_t)max(n, 0), room);
    if (report && (q.first != x || q.first + q.q_len != y || q.length != n)) kv_bounds(a.status);
    return q;
}

// The multiplier is 2^shift / group rounded up, shift = 32 + ceil(log2 group):
// it is less than 2^(shift - 32) / group too large, x times that less than 1 / group.
__device__ __forceinline__ int32_t div_group(const AttendDev &a, int32_t x)
{
    return (int32_t)((uint64_t)x * a.group_mul >> a.group_shift);
}

// keys that a query at `pos` sees: [lo, pos]
__device__ __forceinline__ int32_t first_key(const AttendDev &a, int32_t pos)
{
    return a.c.window && pos >= a.c.window ? pos - a.c.window + 1 : 0;
}

struct Keys {
    int32_t lo, hi;                     // first and last key of the item (hi < lo: none)
};

// An item with nothing to see still has a tile, so that its rows are written.
template <int KT> __device__ __forceinline__ int32_t key_tiles(Keys k) { return k.hi < k.lo ? 1 : k.hi / KT - k.lo / KT + 1; }

// Shape: static constants KT (keys per tile), extra (below) and many (requests
// may have many items) and, for a request, inner(a, q) items for each of outer(a)
// (heads), keys(a, q, i) of inner item i.
struct Place {
    int32_t r, outer, inner, off;       // an item and a tile of it
};
struct SchedShared {
    int64_t warp_sum[32];
    int64_t total, begin, ctas;
    int32_t count, extra;
    Place first, end;                   // where the stretch begins; the tile after it
};

// for sums below 2^57
__device__ __forceinline__ int64_t warp_sum64(int64_t x)
{
    const uint32_t low = (uint32_t)(x & 0x3ffffff), high = (uint32_t)(x >> 26);
    return (int64_t)__reduce_add_sync(~0u, low) + ((int64_t)__reduce_add_sync(~0u, high) << 26);
}
__device__ __forceinline__ Req shfl_req(const Req &q, int src)
{
    return {__shfl_sync(~0u, q.first, src), __shfl_sync(~0u, q.q_len, src), __shfl_sync(~0u, q.length, src)};
}

// Tiles of each lane's request, over its inner items; requests with more than a
// few items are summed by the whole warp, one after another.
template <class S> __device__ __forceinline__ int64_t request_tiles(const AttendDev &a, const Req &q)
{
    const int lane = threadIdx.x & 31;
    const int32_t n = S::inner(a, q);
    const bool big = n > 4;
    int64_t mine = 0;
    if (!big)
        for (int32_t i = 0; i < n; ++i) mine += key_tiles<S::KT>(S::keys(a, q, i));
    for (uint32_t left = __ballot_sync(~0u, big); left; left &= left - 1) {
        const int src = __ffs(left) - 1;
        const Req x = shfl_req(q, src);
        int64_t sum = 0;
        for (int32_t i = lane, m = S::inner(a, x); i < m; i += 32) sum += key_tiles<S::KT>(S::keys(a, x, i));
        sum = warp_sum64(sum);
        if (lane == src) mine = sum;
    }
    return mine;
}

// Sum over the warp (few: every warp has the same values) or the CTA, and the sum
// before this thread.
__device__ __forceinline__ int64_t scan64(int64_t v, int64_t *excl, int64_t *warp_total, bool few)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    int64_t x = v;                                      // inclusive within the warp
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(~0u, x, o);
        if (lane >= o) x += y;
    }
    if (few) {
        *excl = x - v;
        return __shfl_sync(~0u, x, 31);
    }
    __syncthreads();
    if (lane == 31) warp_total[warp] = x;
    __syncthreads();
    int64_t before = 0, total = 0;
    for (int w = 0; w < warps; ++w) {
        const int64_t y = warp_total[w];
        if (w < warp) before += y;
        total += y;
    }
    *excl = before + x - v;
    return total;
}

// x / y for 0 <= x, 0 < y: most are small, and a 64-bit division takes three times as long
__device__ __forceinline__ int64_t quotient(int64_t x, int64_t y)
{
    return ((x | y) >> 32) == 0 ? (int64_t)((uint32_t)x / (uint32_t)y) : x / y;
}

// The CTA's stretch: false if it has none.  All threads of the CTA call it.
template <class S> __device__ __forceinline__ bool schedule(const AttendDev &a, SchedShared &sm)
{
    // up to 32 requests every warp works all of it out, which takes one barrier in all
    const bool few = a.c.requests <= 32;
    const int lane = threadIdx.x & 31, me = few ? lane : threadIdx.x;
    const int32_t R = a.c.requests, T = few ? 32 : blockDim.x, outer = S::outer(a);
    const bool report = blockIdx.x == 0;
    if (report && threadIdx.x == 0 && a.c.q_start[0] != 0) kv_bounds(a.status);
    Req q;
    int64_t mine, tiles = 0, items = 0, excl, excl_items = 0, before = 0;   // of one head: this lane's request, all of its requests
    if (S::many && few) {
        // requests of many items: a warp sums up one after another, lanes taking items
        for (int32_t r = threadIdx.x >> 5; r < R; r += blockDim.x >> 5) {
            q = load_req(a, r, report);
            int64_t sum = 0;
            for (int32_t i = lane, n = S::inner(a, q); i < n; i += 32) sum += key_tiles<S::KT>(S::keys(a, q, i));
            sum = warp_sum64(sum);
            if (lane == 0) sm.warp_sum[r] = sum;
        }
        __syncthreads();
        q = Req{0, 0, 0};
        if (lane < R) q = load_req(a, lane, false);
        tiles = mine = lane < R ? sm.warp_sum[lane] : 0;
        items = S::inner(a, q);
    } else {
        for (int32_t base = 0; base < R; base += T) {
            const int32_t r = base + me;
            q = Req{0, 0, 0};
            if (r < R) q = load_req(a, r, report);
            tiles += mine = request_tiles<S>(a, q);
            items += S::inner(a, q);
        }
    }
    tiles = scan64(tiles, &excl, sm.warp_sum, few) * outer;
    if (tiles == 0) return false;
    // with few tiles a CTA, every tile to a CTA of its own counts more than an even load; every stretch has a tile
    const int32_t extra = tiles >= (S::extra < 4 ? 4 : S::extra + 1) * (int64_t)gridDim.x ? S::extra : 0;
    const int64_t all_items = extra || a.few_pieces ? scan64(items, &excl_items, sm.warp_sum, few) * outer : 0;
    const int64_t total = tiles + all_items * extra;
    excl += excl_items * extra;
    int64_t ctas = min((int64_t)gridDim.x, total);
    if (a.few_pieces) {
        const float least = sqrtf(kPieceTiles * (float)tiles / (float)all_items);
        if (least >= 2.f) ctas = min(ctas, max((int64_t)((float)total / least), (int64_t)1));
    }
    if (blockIdx.x >= ctas) return false;
    const int64_t begin = quotient(total * blockIdx.x, ctas), end = quotient(total * (blockIdx.x + 1), ctas);
    for (int32_t base = 0; base < R; base += T) {
        const int32_t r = base + me;
        if (R > T) {
            q = Req{0, 0, 0};
            if (r < R) q = load_req(a, r, false);
            mine = request_tiles<S>(a, q);
        }
        mine += (int64_t)S::inner(a, q) * extra;
        if (R > T) {
            const int64_t here = scan64(mine, &excl, sm.warp_sum, few);
            excl += before;
            before += here;
        }
        // the warp that has the request of the stretch's first tile, or of the one after it, looks for the item
#pragma unroll 1
        for (int which = 0; which < 2; ++which) {
            const int64_t tile = which ? end : begin;
            const uint32_t who =
                __ballot_sync(~0u, mine > 0 && excl * outer <= tile && tile < (excl + mine) * outer);
            if (!who) continue;
            const int src = __ffs(who) - 1;
            const Req x = shfl_req(q, src);
            const int64_t per = __shfl_sync(~0u, mine, src), off = tile - __shfl_sync(~0u, excl, src) * outer;
            const int32_t head = (int32_t)quotient(off, per), count = S::inner(a, x);
            int64_t rem = off - head * per;
            if (count == 1) {
                if (lane == 0) (which ? sm.end : sm.first) = Place{r - lane + src, head, 0, (int32_t)rem};
                continue;
            }
            for (int32_t i0 = 0; i0 < count; i0 += 32) {
                const int64_t n = i0 + lane < count ? key_tiles<S::KT>(S::keys(a, x, i0 + lane)) + extra : 0;
                int64_t incl = n;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int64_t y = __shfl_up_sync(~0u, incl, o);
                    if (lane >= o) incl += y;
                }
                const uint32_t past = __ballot_sync(~0u, rem < incl);
                if (past) {
                    if (lane == __ffs(past) - 1)
                        (which ? sm.end : sm.first) = Place{r - lane + src, head, i0 + lane, (int32_t)(rem - (incl - n))};
                    break;
                }
                rem -= __shfl_sync(~0u, incl, 31);
            }
        }
    }
    if (threadIdx.x == 0) {
        if (end == total) sm.end = Place{0, 0, 0, 0};   // nothing goes on after the last tile
        sm.count = (int32_t)(end - begin);
        sm.extra = extra;
        sm.begin = begin;
        sm.total = total;
        sm.ctas = ctas;
    }
    __syncthreads();
    return true;
}

// Walks the CTA's stretch item by item; every role of a CTA has its own.  The
// parts of items that other CTAs have the rest of come first, so that the joins
// of their pieces run beside the whole items' tiles.
template <class S> struct Cursor {
    int32_t r, outer, inner, off;       // the item and the first tile of it
    int32_t tiles, len;                 // of the item; of this CTA's part [off, off + len), 0: nothing in the stretch
    int64_t g;                          // that tile's number on the line
    Req q;
    Keys k;
    int32_t left, tail;                 // of the line: whole items to come, the part that ends the stretch
    Place after;                        // the next whole item
    int64_t after_g;
    const SchedShared *sched;

    __device__ __forceinline__ Cursor(const AttendDev &a, const SchedShared &sm) : after(sm.first), after_g(sm.begin), sched(&sm)
    {
        // the end's part, unless that is in the first item
        tail = sm.end.off > 0 && sm.end.off < sm.count ? sm.end.off : 0;
        left = sm.count - tail;
        go(a, sm.first, sm.begin);
        len = max(0, min(tiles - off, sm.count));
        if (whole() && tail) {
            to_tail(a);
        } else {
            taken(a, min(tiles + sm.extra - off, left));
            if (len == 0) next(a);      // all of the first item was before the stretch
        }
    }
    __device__ __forceinline__ void go(const AttendDev &a, const Place &p, int64_t at)
    {
        r = p.r;
        outer = p.outer;
        inner = p.inner;
        off = p.off;
        g = at;
        q = load_req(a, r, false);
        k = S::keys(a, q, inner);
        tiles = key_tiles<S::KT>(k);
    }
    __device__ __forceinline__ void to_tail(const AttendDev &a)
    {
        go(a, Place{sched->end.r, sched->end.outer, sched->end.inner, 0}, sched->begin + sched->count - tail);
        len = min(tail, tiles);
        tail = 0;
    }
    // `after` moves past the current item, to a request that may have none
    __device__ __forceinline__ void taken(const AttendDev &a, int32_t of_line)
    {
        after_g += of_line;
        left -= of_line;
        after = Place{r, outer, inner + 1, 0};
        if (after.inner >= S::inner(a, q)) {
            after.inner = 0;
            if (++after.outer >= S::outer(a)) {
                after.outer = 0;
                ++after.r;
            }
        }
    }
    __device__ __forceinline__ bool next(const AttendDev &a)
    {
        if (tail) {
            to_tail(a);
            return true;
        }
        if (left <= 0) return false;
        if (after.inner == 0 && after.outer == 0)       // a new request: the next one with items
            while (S::inner(a, load_req(a, after.r, false)) == 0) ++after.r;
        go(a, after, after_g);
        len = tiles;
        taken(a, tiles + sched->extra);
        return true;
    }
    __device__ __forceinline__ bool whole() const { return off == 0 && len == tiles; }
};

// ---------------------------------------------------------------------------
// Barriers and copies
// ---------------------------------------------------------------------------
__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile(
        "{\n"
        ".reg .pred p;\n"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n"
        "selp.u32 %0, 1, 0, p;\n"
        "}\n"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}
// Bounded wait.  When one runs out, `dead` (of the CTA) is set and no later
// wait of the CTA waits: its loops run to their end over whatever is there, the
// status says PP_ETIMEOUT, and the launch ends.  (Inlined: a call would keep
// registers from code that runs on a share of its own.)
__device__ __forceinline__ void mbar_wait(uint32_t bar, uint32_t parity, volatile int32_t *dead, const AttendDev &a)
{
    int64_t t0 = 0;
    for (uint32_t it = 0; !mbar_try(bar, parity); ++it) {
        if ((it & 127) != 127) continue;
        if (*dead) return;
        const int64_t now = clock64();
        if (t0 == 0) {
            t0 = now;
        } else if (now - t0 > a.wait_limit) {
            *dead = 1;
            atomicExch(a.status, (int32_t)PP_ETIMEOUT);
            return;
        }
    }
}

// ---------------------------------------------------------------------------
// Cache rows to shared memory
// ---------------------------------------------------------------------------
// Rows of K or V lie in halves of 64 elements, 128 bytes a row, whose 16-byte
// pieces are swizzled by the row (piece ^ row % 8): the layout that ldmatrix
// reads without conflicts and the tensor cores' operands take.  Two ways get
// them there.  A tensor-map box costs one lane an instruction but ends with its
// block, and measured on this GPU machines of 128-byte rows take 52 cycles and 5.3 a
// row, from L2 as from HBM: over all SMs 3.2 TB/s with 8 rows, 4.4 with 16, 6.2
// with 64.  16-byte copies, a warp's 32 at a time, reach 9 TB/s (one warp an SM)
// to 21 (eight) from L2, but each costs the warp some five instructions, and
// operands of the tensor cores need a fence after them.  Single tokens take the
// second way with eight warps (128 requests, 1.52 GB in blocks of 16: 256 us against
// 297); chunks, whose warps have the softmax to do, the first (8,192 tokens after
// 24,576: 1.97 ms against 2.31 with V by copies).  Both pairs were measured on the
// kernels as they were then; these calls take 253 us and 1.90 ms now.
__device__ __forceinline__ void copy16(uint32_t dst, const char *src, uint32_t bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// A lane's share of copies of whole rows: `step` rows of 16-byte pieces at a time.
template <int HALVES> struct RowLane {
    static constexpr int per_row = 8 * HALVES, step = 32 / per_row;
    uint32_t dst, bytes;                // in a group of 8 rows; 0: past the head dimension, zeros are written
    int64_t src;
    __device__ __forceinline__ RowLane(const AttendDev &a, uint32_t half_bytes)
    {
        const int lane = threadIdx.x & 31, sub = lane / per_row, piece = lane % per_row;
        dst = (piece >> 3) * half_bytes + sub * 128 + (((piece ^ sub) & 7) << 4);
        bytes = piece * 8 < a.dim ? 16 : 0;
        src = 2 * sub * a.token_stride + (bytes ? piece * 16 : 0);
    }
    // 8 rows; `from` is the first row's head, `to` at a multiple of 1,024 bytes
    __device__ __forceinline__ void rows8(uint32_t to, const char *from, int64_t token_bytes, bool some) const
    {
#pragma unroll
        for (int x = 0; x < 8; x += step) copy16(to + x * 128 + (dst ^ (x << 4)), from + src + x * token_bytes, some ? bytes : 0);
    }
};

// box of tokens x 64 elements of one block and head, rows swizzled as above; a
// block number out of range gives zeros
__device__ __forceinline__ void box_rows(uint32_t dst, const CUtensorMap *map, uint32_t bar, int32_t x, int32_t token,
                                         int32_t head, int32_t block)
{
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(token), "r"(head), "r"(block), "r"(bar)
        : "memory");
}
__device__ __forceinline__ void mbar_expect(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}

// block that holds key j of the request, -1 if the item sees none of keys j .. j + n - 1
__device__ __forceinline__ int32_t key_block(const AttendDev &a, const int32_t *row, Keys k, int32_t j, int32_t n)
{
    if (j > k.hi || j + n - 1 < k.lo) return -1;
    const int32_t id = row[j >> a.block_log];
    if (id >= 0 && id < a.blocks) return id;
    kv_bounds(a.status);
    return -1;
}

__device__ __forceinline__ void named_sync(int id, int threads)
{
    asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}

__device__ __forceinline__ void named_arrive(int id, int threads)
{
    asm volatile("bar.arrive %0, %1;" ::"r"(id), "r"(threads) : "memory");
}

__device__ __forceinline__ float exp2_approx(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// What a row's output is multiplied with.  No weight is above 0 where the row sees no
// key (zeros), or only scores of -infinity: 0 / 0 then, as the formula has it.
__device__ __forceinline__ float inverse_sum(float sum, bool sees)
{
    return sum == 0.f ? (sees ? NAN : 0.f) : 1.f / sum;
}

template <typename T> struct Pack;
template <> struct Pack<__nv_bfloat16> {
    static __device__ __forceinline__ uint32_t two(float lo, float hi)
    {
        uint32_t r;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
        return r;
    }
};
template <> struct Pack<__half> {
    static __device__ __forceinline__ uint32_t two(float lo, float hi)
    {
        uint32_t r;
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
        return r;
    }
};

// ---------------------------------------------------------------------------
// Pieces of an item
// ---------------------------------------------------------------------------
// CTA whose stretch holds tile g of the line
__device__ __forceinline__ int32_t owner(int64_t g, int64_t total, int64_t ctas)
{
    return (int32_t)quotient((g + 1) * ctas - 1, total);
}
// a CTA has at most two pieces: one that goes on an item begun before it (0)
// and one of an item that goes on after it (1)
__device__ __forceinline__ int32_t piece_slot(int32_t cta0, int32_t p) { return p == 0 ? 2 * cta0 + 1 : 2 * (cta0 + p); }

// Host (pp_attend.cu)
pp_status cache_map(const pp_kv *kv, const void *cache, int32_t rows, CUtensorMap *map);
AttendDev attend_dev(const pp_kv *kv, const AttendArgs &c);

pp_status prepare_attend_token();
pp_status prepare_attend_chunk();
pp_status launch_attend_token(pp_kv *kv, const AttendArgs &c, cudaStream_t st);
pp_status prepare_attend_token8();
pp_status launch_attend_token8(pp_kv *kv, const AttendArgs &c, cudaStream_t st);
pp_status launch_attend_chunk(pp_kv *kv, const AttendArgs &c, bool beside, cudaStream_t st);

}  // namespace pp
