// A paged cache of 8-bit numbers: the write of new K and V rows, and attention over it.
//
// An element is code * 2^e: an e4m3 number and an exponent of its block and head.
// Scales are powers of two, so that codes go to another scale, or to 16-bit floating
// numbers, without a rounding but where they fall below e4m3's normal range.
#include <algorithm>
#include <climits>
#include <cstring>
#include <type_traits>

#include "pp_attend.cuh"

namespace pp {

__device__ __forceinline__ float scale_of(int e) { return __int_as_float((e + 127) << 23); }     // 2^e

// ---------------------------------------------------------------------------
// Write.
// ---------------------------------------------------------------------------
struct Write8Args {
    int32_t tokens, heads, per_head, window;            // vectors of 8 elements a head; tokens of a CTA
    const uint4 *k, *v;
    int64_t k_token, k_head, v_token, v_head;           // strides in vectors
    const int64_t *slot;
    uint8_t *kc, *vc;
    int8_t *ke, *ve;
    int64_t block_stride, token_stride, head_stride;    // bytes
    int64_t slots;
    int32_t block_log;
    int32_t *status;
    int32_t *claim;                                     // of each block, the first token of its last run, of any call
};

constexpr int kWrite8Warps = 8, kWrite8Threads = 32 * kWrite8Warps;
constexpr int kWrite8Ctas = 3;                          // of an SM
constexpr int kWrite8Held = 8;                          // vectors that a lane has on their way

// bits of a 16-bit infinity
template <typename T> constexpr uint32_t kInfinity = std::is_same<T, __nv_bfloat16>::value ? 0x7f80u : 0x7c00u;

// the larger of `top` and |x| of 8 numbers, even and odd ones apart; infinities and NaN as they are
__device__ __forceinline__ uint32_t largest(uint32_t top, const uint4 &x)
{
    return __vimax3_u16x2(__vimax3_u16x2(top, x.x & 0x7fff7fffu, x.y & 0x7fff7fffu), x.z & 0x7fff7fffu, x.w & 0x7fff7fffu);
}
// |x| of two 16-bit numbers; where x is infinite or NaN it becomes NaN and 0 is returned
template <typename T> __device__ __forceinline__ uint32_t sizes(uint32_t &x)
{
    constexpr uint32_t e = kInfinity<T>;
    uint32_t m = x & 0x7fff7fffu;
    if ((m & 0xffffu) >= e) {
        x |= 0x7fffu;
        m &= 0xffff0000u;
    }
    if (m >= e << 16) {
        x |= 0x7fff0000u;
        m &= 0xffffu;
    }
    return m;
}
template <typename T> __device__ __forceinline__ uint32_t sizes8(uint4 &x)
{
    const uint32_t a = sizes<T>(x.x), b = sizes<T>(x.y), c = sizes<T>(x.z), d = sizes<T>(x.w);
    return __vmaxu2(__vmaxu2(a, b), __vmaxu2(c, d));
}
template <typename T> __device__ __forceinline__ float low_value(uint32_t x);
template <> __device__ __forceinline__ float low_value<__nv_bfloat16>(uint32_t x) { return __uint_as_float(x << 16); }
template <> __device__ __forceinline__ float low_value<__half>(uint32_t x)
{
    return __half2float(__ushort_as_half((unsigned short)(x & 0xffffu)));
}
template <typename T> __device__ __forceinline__ float high_value(uint32_t x);
template <> __device__ __forceinline__ float high_value<__nv_bfloat16>(uint32_t x) { return __uint_as_float(x & 0xffff0000u); }
template <> __device__ __forceinline__ float high_value<__half>(uint32_t x) { return low_value<__half>(x >> 16); }
// two numbers to codes, to the nearest, beyond 448 to that, NaN to NaN
__device__ __forceinline__ uint32_t codes2(float lo, float hi)
{
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
template <typename T> __device__ __forceinline__ uint2 codes8(const uint4 &x, float by)
{
    auto four = [&](uint32_t a, uint32_t b) {
        return codes2(low_value<T>(a) * by, high_value<T>(a) * by) | codes2(low_value<T>(b) * by, high_value<T>(b) * by) << 16;
    };
    return make_uint2(four(x.x, x.y), four(x.z, x.w));
}
// four codes times `by`
__device__ __forceinline__ uint32_t rescale4(uint32_t x, float by)
{
    uint32_t h[2];
    asm("{\n.reg .b16 lo, hi;\nmov.b32 {lo, hi}, %2;\ncvt.rn.f16x2.e4m3x2 %0, lo;\ncvt.rn.f16x2.e4m3x2 %1, hi;\n}"
        : "=r"(h[0]), "=r"(h[1])
        : "r"(x));
    return codes2(low_value<__half>(h[0] & 0xffffu) * by, low_value<__half>(h[0] >> 16) * by) |
           codes2(low_value<__half>(h[1] & 0xffffu) * by, low_value<__half>(h[1] >> 16) * by) << 16;
}
// the least e, kLeastExp <= e <= kMostExp, with x <= 448 * 2^e (448 = 1.75 * 2^8)
__device__ __forceinline__ int least_exponent(float x)
{
    const uint32_t b = __float_as_uint(x);
    const int e = (int)(b >> 23) - 127 - 8 + ((b & 0x7fffffu) > 0x600000u);
    return min(max(e, kLeastExp), kMostExp);
}

struct Run8 {
    int32_t first, count, block;                        // first token, tokens to the last one, block
};
// Shared memory of a CTA: a place for every vector that a lane has on its way, and what the
// warps of a team tell each other.
struct Write8Shared {
    uint4 held[kWrite8Warps][kWrite8Held][32];
    uint32_t top[kWrite8Warps];
    int32_t begins[kWrite8Warps];
    uint8_t list[kWrite8Warps][32];                     // tokens that are runs
};

// What becomes of the exponents, from the size of the largest finite new element.
__device__ __forceinline__ int next_exponent(float top, bool begins, int old)
{
    const int need = least_exponent(top);
    return begins ? need : max(old, need);
}
// Some lanes' (of `lanes`, me among them) share of a block's rows of one head to a new scale.
__device__ __forceinline__ void rescale_rows(const Write8Args &a, uint8_t *rows, float by, int me, int lanes)
{
    const int32_t pieces = a.per_head / 2;              // of 16 codes
    for (int32_t l = me; l < pieces << a.block_log; l += lanes) {
        uint4 *p = reinterpret_cast<uint4 *>(rows + l / pieces * a.token_stride) + l % pieces;
        const uint4 x = *p;
        *p = make_uint4(rescale4(x.x, by), rescale4(x.y, by), rescale4(x.z, by), rescale4(x.w, by));
    }
}

// A head of K or V (unit = 2 h + is_v) of a run by a team of TEAM warps: the largest size,
// the exponent, the block's other rows if that grows, the codes.  A lane has vector `col`
// of a row of every step's `some` rows a warp; those of kWrite8Held steps are read once.
template <typename T, int TEAM>
__device__ __forceinline__ void write_unit(const Write8Args &a, const Run8 &run, int32_t unit, Write8Shared &sh)
{
    constexpr int kThreads = 32 * TEAM;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, of_team = warp % TEAM, me = 32 * of_team + lane;
    auto sync = [&]() {                                 // a barrier of its own for every team of every size
        if (TEAM == 1) __syncwarp();
        else named_sync((TEAM == 2 ? 1 : TEAM == 4 ? 5 : 7) + warp / TEAM, kThreads);
    };
    const bool is_v = unit & 1;
    const int32_t h = unit >> 1;
    const int some = 32 / a.per_head, sub = lane / a.per_head, col = lane - sub * a.per_head;
    const int32_t step = TEAM * some, ahead = of_team * some + sub, past = sub < some ? run.count : 0;  // past: no row from here on
    const int64_t token = is_v ? a.v_token : a.k_token;
    const uint4 *src = (is_v ? a.v + h * a.v_head : a.k + h * a.k_head) + run.first * token + col;
    uint8_t *dst = (is_v ? a.vc : a.kc) + run.block * a.block_stride + h * a.head_stride;
    int8_t *exponent = (is_v ? a.ve : a.ke) + (int64_t)run.block * a.heads + h;
    // place in the block of token n of the run (-1: left out)
    auto place = [&](int32_t n) {
        const int64_t s = a.slot[run.first + n];
        return s >= 0 && s < a.slots ? (int32_t)(s & ((1 << a.block_log) - 1)) : -1;
    };
    // rows that are left out are loaded and not used, so that no load waits for a slot
    uint4(*held)[32] = sh.held[warp];
    int32_t row[kWrite8Held];
#pragma unroll
    for (int y = 0; y < kWrite8Held; ++y) {
        const int32_t n = ahead + y * step;
        if (n < past) copy16(smem_u32(&held[y][lane]), reinterpret_cast<const char *>(src + n * token), 16);
        row[y] = n < past ? place(n) : -1;
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    const int old = min(max((int)*exponent, kLeastExp), kMostExp);
    const int32_t rest = ahead + kWrite8Held * step;    // rows that are read again
    uint32_t top = 0;
    bool begins = false;
#pragma unroll 4
    for (int32_t n = rest; n < past; n += step) {
        const int32_t at = place(n);
        begins |= at == 0;
        const uint4 x = __ldg(src + n * token);
        if (at >= 0) top = largest(top, x);
    }
    copies_wait();                                      // a lane reads what it copied itself
#pragma unroll
    for (int y = 0; y < kWrite8Held; ++y) {
        begins |= row[y] == 0;
        if (row[y] >= 0) top = largest(top, held[y][lane]);
    }
    begins = __any_sync(~0u, begins);
    if (TEAM > 1 && lane == 0) sh.begins[warp] = begins;
    // the largest of the team's
    auto all_of = [&](uint32_t mine) {
        mine = __reduce_max_sync(~0u, max(mine & 0xffffu, mine >> 16));
        if (TEAM > 1) {
            if (lane == 0) sh.top[warp] = mine;
            sync();
#pragma unroll
            for (int w = 0; w < TEAM; ++w) mine = max(mine, sh.top[warp - of_team + w]);
        }
        return mine;
    };
    top = all_of(top);
    if (TEAM > 1)
#pragma unroll
        for (int w = 0; w < TEAM; ++w) begins |= sh.begins[warp - of_team + w] != 0;
    const bool strange = top >= kInfinity<T>;           // the same in all the team
    if (strange) {                                      // the largest finite one; the others become NaN
        sync();                                         // all have read the first ones
        top = 0;
        for (int32_t n = ahead; n < past; n += step) {
            uint4 x = __ldg(src + n * token);
            if (place(n) >= 0) top = __vmaxu2(top, sizes8<T>(x));
        }
        top = all_of(top);
    }
    const int e = next_exponent(low_value<T>(top), begins, old);
    // the rows that the block has go to the new scale; those of this call are written over them
    if (!begins && e > old) rescale_rows(a, dst, scale_of(old - e), me, kThreads);
    sync();                                             // all have read the exponent, and old rows are done
    if (me == 0) *exponent = (int8_t)e;
    const float by = scale_of(-e);
    dst += 8 * col;
    auto put = [&](int32_t at, uint4 x) {
        if (strange) sizes8<T>(x);
        *reinterpret_cast<uint2 *>(dst + at * a.token_stride) = codes8<T>(x, by);
    };
#pragma unroll
    for (int y = 0; y < kWrite8Held; ++y)
        if (row[y] >= 0) put(row[y], held[y][lane]);
#pragma unroll 4
    for (int32_t n = rest; n < past; n += step) {
        const int32_t at = place(n);
        const uint4 x = __ldg(src + n * token);
        if (at >= 0) put(at, x);
    }
    if (TEAM > 1) sync();                               // the team's shared memory is free again
}

// Runs of one token among the 32 from t0 on, whose lanes `list` names: units first .. past
// - 1 of theirs, counted run after run, side by side.  block: of each lane's token.  (Two or
// four times as many together cost a step of 64 tokens 0.4 and 1.1 us more, in code, and
// save 30,011 tokens nothing.)
template <typename T>
__device__ __forceinline__ void write_singles(const Write8Args &a, int32_t t0, int32_t block, const uint8_t *list, int32_t first, int32_t past)
{
    const int lane = threadIdx.x & 31, some = 32 / a.per_head, sub = lane / a.per_head, col = lane - sub * a.per_head, all = 2 * a.heads;
    const int32_t n = first + sub, r = n / all, u = n - r * all, h = u >> 1;
    const bool live = sub < some && n < past;
    const int from = live ? list[r] : 0;
    const int32_t b = __shfl_sync(~0u, block, from), t = t0 + from;
    uint8_t *const rows = (u & 1 ? a.vc : a.kc) + b * a.block_stride + h * a.head_stride;       // the block's, of the head
    int8_t *const exponent = (u & 1 ? a.ve : a.ke) + (int64_t)b * a.heads + h;
    uint4 x = make_uint4(0, 0, 0, 0);
    int32_t at = 0;
    int old = 0;
    if (live) {
        x = __ldg(u & 1 ? a.v + t * a.v_token + h * a.v_head + col : a.k + t * a.k_token + h * a.k_head + col);
        at = (int32_t)(a.slot[t] & ((1 << a.block_log) - 1));
        old = min(max((int)*exponent, kLeastExp), kMostExp);
    }
    uint32_t top = largest(0, x), mine = 0;
    if (__any_sync(~0u, (top & 0xffffu) >= kInfinity<T> || top >> 16 >= kInfinity<T>)) top = sizes8<T>(x);
    top = max(top & 0xffffu, top >> 16);
    for (int s = 0; s < some; ++s) {
        const uint32_t of_unit = __reduce_max_sync(~0u, sub == s ? top : 0);
        if (sub == s) mine = of_unit;
    }
    const int e = next_exponent(low_value<T>(mine), at == 0, old);
    // units whose scale grows, one after another
    for (uint32_t grow = __ballot_sync(~0u, live && col == 0 && at != 0 && e > old); grow; grow &= grow - 1) {
        const int src = __ffs(grow) - 1;
        const uint64_t where = __shfl_sync(~0u, (uint64_t)rows, src);
        rescale_rows(a, reinterpret_cast<uint8_t *>(where), scale_of(__shfl_sync(~0u, old - e, src)), lane, 32);
    }
    __syncwarp();                                       // all have read the exponents, and old rows are done
    if (!live) return;
    if (col == 0) *exponent = (int8_t)e;
    *reinterpret_cast<uint2 *>(rows + at * a.token_stride + 8 * col) = codes8<T>(x, scale_of(-e));
}

// claimed, of a warp whose lanes' tokens t0 on lead runs of blocks `here` where it is not -1: first tokens of runs of
// those blocks, of this call or another.  Out of line, since calls with the same map as the last one do not come here.
static __device__ __noinline__ void find_apart(const int64_t *slot, int32_t tokens, int64_t slots, int32_t block_log, int32_t *status,
                                               int32_t here, int32_t claimed, int32_t t0)
{
    const int lane = threadIdx.x & 31;
    auto block_of = [&](int32_t t) {
        const int64_t s = t >= 0 && t < tokens ? slot[t] : -1;
        return s >= 0 && s < slots ? (int32_t)(s >> block_log) : -1;
    };
    const bool other = claimed >= 0 && claimed != t0 + lane && block_of(claimed) == here;
    for (uint32_t apart = __ballot_sync(~0u, other); apart; apart &= apart - 1) {
        const int src = __ffs(apart) - 1;
        const int32_t block = __shfl_sync(~0u, here, src), x = block_of(__shfl_sync(~0u, claimed, src) - 32 + lane);
        const uint32_t not_left_out = __ballot_sync(~0u, x >= 0);
        const int32_t block_before = __shfl_sync(~0u, x, (31 - __clz(not_left_out)) & 31);
        if (lane == 0 && (not_left_out == 0 || block_before != block)) kv_bounds(status);
    }
}

// A run is the tokens of one block, which stand next to one another but for fewer than
// 32 that are left out between two; its first token leads it.  Every warp of a CTA finds
// the leaders among `window` tokens by itself, 32 at a time, from their slots and those of
// 32 tokens to either side.  Every leader leaves its number in its block's claim.  If it
// finds another one there that leads a run of that block in this call's map, the block's
// tokens lie apart.  So a call need not clear the claims, and no map that keeps to the rule
// is reported, whatever earlier calls left.  (64 single tokens 2.62 us a call in a graph,
// 2.54 without; 30,011 20.3 and 20.0; with the search below in line 2.70 and 20.7.)
// A run's rows of one head and of K or V are a team's, a warp for every kWrite8Held steps
// of them, TEAMS warps at most; those of runs of one token go several to a warp.
// Three bytes an element, all read and written once where a run fits kWrite8Held steps; a
// run's chain of slots, rows, largest size and codes is what takes the time: 30,011 tokens
// of 4 heads of 128 take 23 us from cold caches (14 at the rate of a copy, 60% of the issue
// slots), with blocks of 32 28, of 64 29, of 512 52; as 30,011 runs of one token (2 heads)
// 35.  64 single tokens of 2 heads: 2.7 us a call in a graph.  K and V of a head by one
// warp together: 25 us for 30,011 tokens, 3.7 for 64.
template <typename T, int TEAMS>
__global__ void __launch_bounds__(kWrite8Threads, kWrite8Ctas) k_kv_write8(const __grid_constant__ Write8Args a)
{
    __shared__ Write8Shared sh;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    // block of token t, -1 if it is left out or no token
    auto block_of = [&](int32_t t) {
        const int64_t s = t >= 0 && t < a.tokens ? a.slot[t] : -1;
        return s >= 0 && s < a.slots ? (int32_t)(s >> a.block_log) : -1;
    };
    // the warps of this CTA, and of those of the same tokens, share the units of all runs out
    const int32_t all = 2 * a.heads, workers = gridDim.y * kWrite8Warps, some = 32 / a.per_head;
    int32_t next = blockIdx.y * kWrite8Warps + warp;    // this warp's next task, counted from the run's first
    const int32_t begin = blockIdx.x * a.window, end = min(begin + a.window, a.tokens);
    int32_t before = block_of(begin - 32 + lane), here = block_of(begin + lane), after = block_of(begin + 32 + lane);
    for (int32_t t0 = begin; t0 < end; t0 += 32) {
        const int32_t t1 = min(t0 + 32, end), later_on = t1 < end ? block_of(t0 + 64 + lane) : -1;
        if (warp == 0 && blockIdx.y == 0 && t0 + lane < t1 && a.slot[t0 + lane] >= a.slots) kv_bounds(a.status);
        // tokens that are not left out: 64 from t0 - 32 on, and 64 from t0 on
        const uint32_t known_before = __ballot_sync(~0u, before >= 0), known = __ballot_sync(~0u, here >= 0);
        const uint32_t known_after = __ballot_sync(~0u, after >= 0);
        // the nearest of the 32 before this lane's token, and its block
        const uint64_t back = (((uint64_t)known << 32 | known_before) >> lane) & 0xffffffffu;     // bit 31: the one before
        const int nearest = 31 - __clz((uint32_t)back) + lane;                                  // counted from t0 - 32
        const int32_t block_before = __shfl_sync(~0u, before, nearest & 31), block_here = __shfl_sync(~0u, here, nearest & 31);
        const bool leads = here >= 0 && ((uint32_t)back == 0 || (nearest < 32 ? block_before : block_here) != here);
        const uint32_t leaders = __ballot_sync(~0u, leads), later = leaders & ~1u << lane;
        // a run that another one follows here ends with the last token before that
        const int32_t counted = later ? 31 - __clz(known & (later & -later) - 1) - lane + 1 : 0;

        // the tokens of the run that lane f's token leads, counted from that: all before one of another block, or before 32 left out
        auto run_of = [&](int f, int32_t block) {
            const uint64_t same = (uint64_t)__ballot_sync(~0u, after == block) << 32 | __ballot_sync(~0u, here == block);
            const uint64_t valid = (uint64_t)known_after << 32 | known, from = ~0ull << f;
            uint64_t none = ~valid & from;                  // then: bits that begin 32 left out
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) none &= none >> o;
            const uint64_t ends = (valid & ~same & from) | none;
            const uint64_t mine = same & from & (ends ? (ends & -ends) - 1 : ~0ull);
            int32_t last = 63 - __clzll(mine);
            if (!ends && t0 + 64 < a.tokens) {              // it may go on: 128 tokens at a time
                last += t0;
                for (bool more = true; more;) {
                    int32_t b[4];
                    const int32_t at = last + 1;
#pragma unroll
                    for (int y = 0; y < 4; ++y) b[y] = block_of(at + 32 * y + lane);
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        if (!more) continue;
                        uint32_t good = __ballot_sync(~0u, b[y] == block);
                        const uint32_t other = __ballot_sync(~0u, b[y] >= 0 && b[y] != block);
                        if (other) good &= (other & -other) - 1;
                        if (good) last = at + 32 * y + 31 - __clz(good);
                        // 32 left out, or more to come than this can tell: the next look is from `last` on
                        if (other || !good) more = false;
                        else if (good != ~0u) break;
                    }
                }
                last -= t0;
            }
            return last - f + 1;
        };
        uint32_t left = leaders & (uint32_t)((1ull << (t1 - t0)) - 1);
        int32_t claimed = -1;                               // looked at when this warp is done with the tokens
        if (warp == 0 && blockIdx.y == 0 && (left >> lane & 1)) claimed = atomicExch(a.claim + here, t0 + lane);
        const uint32_t singles = __ballot_sync(~0u, counted == 1) & left;
        if (singles) {
            if (singles >> lane & 1) sh.list[warp][__popc(singles & ((1u << lane) - 1))] = (uint8_t)lane;
            __syncwarp();
            const int32_t units = __popc(singles) * all, tasks = (units + some - 1) / some;
            for (; next < tasks; next += workers) write_singles<T>(a, t0, here, sh.list[warp], next * some, units);
            next -= tasks;
            __syncwarp();                               // the list is free again
        }
        for (left &= ~singles; left; left &= left - 1) {
            const int lead = __ffs(left) - 1;
            const int32_t block = __shfl_sync(~0u, here, lead), count = __shfl_sync(~0u, counted, lead);
            const Run8 run = {t0 + lead, count ? count : run_of(lead, block), block};
            const int32_t warps = (run.count + kWrite8Held * some - 1) / (kWrite8Held * some);     // with rows
            if (TEAMS == 1 || warps == 1) {
                for (; next < all; next += workers) write_unit<T, 1>(a, run, next, sh);
                next -= all;
                continue;
            }
            auto by_teams = [&](auto size) {
                constexpr int TEAM = decltype(size)::value;
                constexpr int kTeams = kWrite8Warps / TEAM;
                for (int32_t u = blockIdx.y * kTeams + warp / TEAM; u < all; u += gridDim.y * kTeams) write_unit<T, TEAM>(a, run, u, sh);
            };
            if (TEAMS == 2 || warps == 2) by_teams(std::integral_constant<int, 2>());
            else if (TEAMS == 4 || warps <= 4) by_teams(std::integral_constant<int, TEAMS < 4 ? TEAMS : 4>());
            else by_teams(std::integral_constant<int, TEAMS>());
        }
        if (__any_sync(~0u, claimed >= 0 && claimed != t0 + lane)) find_apart(a.slot, a.tokens, a.slots, a.block_log, a.status, here, claimed, t0);
        before = here;
        here = after;
        after = later_on;
    }
}

// ---------------------------------------------------------------------------
// Attention of chunks: the visible blocks as 16-bit rows in the caller's workspace
// (exact in bf16), then the kernel of 16-bit caches over them.
// ---------------------------------------------------------------------------
struct Unpack8Args {
    AttendDev a;
    uint4 *k, *v;                                       // [capacity][heads][block_size][dim]
    int32_t *table;                                     // [requests][table_width]
    int32_t capacity;
};

constexpr int kUnpackThreads = 512;

// two codes (the low half) times `by`, as two 16-bit numbers
template <typename T> __device__ __forceinline__ uint32_t wide2(uint32_t codes, float by)
{
    uint32_t h, r;
    asm("{\n.reg .b16 lo, hi;\nmov.b32 {lo, hi}, %1;\ncvt.rn.f16x2.e4m3x2 %0, lo;\n}" : "=r"(h) : "r"(codes));
    r = Pack<T>::two(low_value<__half>(h) * by, high_value<__half>(h) * by);
    if constexpr (std::is_same<T, __half>::value) {     // what f16 does not reach becomes its largest
        __half2 x;
        memcpy(&x, &r, 4);
        const __half2 most = __half2half2(__ushort_as_half(0x7bff));
        x = __hmax2_nan(__hmin2_nan(x, most), __hneg2(most));
        memcpy(&r, &x, 4);
    }
    return r;
}
template <typename T> __device__ __forceinline__ void unpack16(uint4 *to, const uint4 &x, float by)
{
    // a whole sector
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(wide2<T>(x.x, by)),
                 "r"(wide2<T>(x.x >> 16, by)), "r"(wide2<T>(x.y, by)), "r"(wide2<T>(x.y >> 16, by)), "r"(wide2<T>(x.z, by)),
                 "r"(wide2<T>(x.z >> 16, by)), "r"(wide2<T>(x.w, by)), "r"(wide2<T>(x.w >> 16, by))
                 : "memory");
}

// Blocks that a request's queries see: [lo, hi], none if hi < lo.
__device__ __forceinline__ Keys seen_blocks(const AttendDev &a, const Req &q)
{
    if (q.q_len == 0 || q.length == 0) return {0, -1};
    return {first_key(a, max(q.length - q.q_len, 0)) >> a.block_log, (q.length - 1) >> a.block_log};
}

// Every CTA sums up the requests' visible blocks (8 bytes a request, from L2 after the
// first) and a warp takes up to 16 rows of a block and head at a time, numbered through
// all requests; a lane has one piece of 16 codes of every few rows.  A block that several
// requests see is unpacked for each.  A byte read and two written, which the attention
// then reads, mostly from L2: 20 us for 32,768 tokens of 4 heads of 128 (100 MB, 5 TB/s),
// 13 for 8 requests of up to 8,900 tokens and 2 heads, 43 for 24 of up to 8,000 with 16
// heads of 64.  The short ones wait for the requests' sums and for three loads in a row
// (table, exponents, codes); the attention's launch and its cut of the work go beside them.
template <typename T> __global__ void __launch_bounds__(kUnpackThreads, 2) k_unpack8(const __grid_constant__ Unpack8Args u)
{
    extern __shared__ int32_t pre[];                    // blocks before request r, then its first
    __shared__ int64_t warp_sum[32];
    const AttendDev &a = u.a;
    const int tid = threadIdx.x, lane = tid & 31;
    int32_t *const low = pre + a.c.requests;
    // the attention's launch and its cut of the work, which need nothing from here, go beside this kernel's end
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int32_t R = a.c.requests, per = (R + kUnpackThreads - 1) / kUnpackThreads;
    const int32_t first = min(tid * per, R), past = min(first + per, R);
    int64_t mine = 0, excl;
    for (int32_t r = first; r < past; ++r) {
        const Keys k = seen_blocks(a, load_req(a, r, false));
        mine += k.hi - k.lo + 1;
    }
    const int64_t all = scan64(mine, &excl, warp_sum, false);
    const int32_t total = (int32_t)min(all, (int64_t)u.capacity);
    if (all > u.capacity && blockIdx.x == 0 && tid == 0) kv_bounds(a.status);
    for (int32_t r = first; r < past; ++r) {
        const Keys k = seen_blocks(a, load_req(a, r, false));
        pre[r] = (int32_t)min(excl, (int64_t)INT_MAX);
        low[r] = k.lo;
        excl += k.hi - k.lo + 1;
    }
    __syncthreads();

    const int32_t warps = gridDim.x * (kUnpackThreads / 32), rows_log = min(a.block_log, 4);
    const int32_t parts_log = a.block_log - rows_log;   // of a block
    const int32_t pieces = a.dim / 16, some = 32 / pieces;              // a row's, rows at a time
    const int32_t sub = lane / pieces, piece = lane - sub * pieces;
    const int64_t units = (int64_t)total * a.kv_heads << parts_log;
    for (int64_t n = blockIdx.x * (kUnpackThreads / 32) + (tid >> 5); n < units; n += warps) {
        const int64_t of_block = n >> parts_log;
        const int32_t x = (int32_t)quotient(of_block, a.kv_heads), h = (int32_t)(of_block - (int64_t)x * a.kv_heads);
        const int32_t row0 = (int32_t)(n & ((1 << parts_log) - 1)) << rows_log;
        int32_t r = 0;                                  // the last request that begins at x or before
        for (int32_t len = R; len > 1;) {
            const int32_t half = len >> 1;
            if (pre[r + half] <= x) {
                r += half;
                len -= half;
            } else {
                len = half;
            }
        }
        const int32_t j = low[r] + x - pre[r];
        const int64_t entry = (int64_t)r * a.c.table_width + j;
        const int32_t id = a.c.block_table[entry];
        const bool ok = id >= 0 && id < a.blocks;
        if (h == 0 && row0 == 0 && lane == 0) u.table[entry] = ok ? x : -1;
        if (!ok) continue;
        const int64_t from = id * a.block_stride + h * a.head_stride + piece * 16, at = (int64_t)id * a.kv_heads + h;
        const uint8_t *k = static_cast<const uint8_t *>(a.c.k_cache) + from, *v = static_cast<const uint8_t *>(a.c.v_cache) + from;
        const float kb = scale_of(min(max((int)a.c.k_exp[at], kLeastExp), kMostExp));
        const float vb = scale_of(min(max((int)a.c.v_exp[at], kLeastExp), kMostExp));
        const int64_t to = (of_block << a.block_log) * (2 * pieces) + 2 * piece;
        uint4 y[4], z[4];                               // 16 rows of 8 pieces are four steps
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int32_t row = i * some + sub;
            if (sub < some && row < 1 << rows_log) {
                y[i] = *reinterpret_cast<const uint4 *>(k + (row0 + row) * a.token_stride);
                z[i] = *reinterpret_cast<const uint4 *>(v + (row0 + row) * a.token_stride);
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int32_t row = i * some + sub;
            if (sub < some && row < 1 << rows_log) {
                unpack16<T>(u.k + to + (row0 + row) * (2 * pieces), y[i], kb);
                unpack16<T>(u.v + to + (row0 + row) * (2 * pieces), z[i], vb);
            }
        }
    }
    // blocks that have no place
    if (all > u.capacity)
        for (int32_t r = blockIdx.x; r < R; r += gridDim.x) {
            const Keys k = seen_blocks(a, load_req(a, r, false));
            for (int32_t j = k.lo + tid; j <= k.hi; j += kUnpackThreads)
                if ((int64_t)pre[r] + j - k.lo >= total) u.table[(int64_t)r * a.c.table_width + j] = -1;
        }
}

pp_status prepare_kv8()
{
    const int most = 2 * (int)sizeof(int32_t) * kKvMaxRequests;
    PP_CUDA(cudaFuncSetAttribute(k_unpack8<__nv_bfloat16>, cudaFuncAttributeMaxDynamicSharedMemorySize, most));
    PP_CUDA(cudaFuncSetAttribute(k_unpack8<__half>, cudaFuncAttributeMaxDynamicSharedMemorySize, most));
    return prepare_attend_token8();
}

// A workspace: the table, then K's rows, then V's.
static int64_t table_bytes(int32_t requests, int32_t width) { return ((int64_t)requests * width * 4 + 255) / 256 * 256; }
static int64_t block_bytes(const pp_kv *kv) { return (int64_t)2 * kv->heads * kv->block_size * kv->dim; }

// Rows (new tokens x heads of a group) of the longest request up to which a call goes
// to the kernel of single tokens.  That one reads codes once for every 16 rows; chunks'
// are unpacked, which costs 15 us and more, and take 256 rows whatever there are.  In us,
// 2 K/V heads of 128, single passes after a flush of L2, 32 requests after 5,000 tokens /
// 4 after 2,000 / 1 after 50,000 (64 rows here by items of 16):
//   32 rows   68 : 104 / 25 : 37 / 35 : 70
//   64       123 : 104 / 23 : 37 / 47 : 70
// In between the batch's times meet at some 52.
constexpr int64_t kFewRows8 = 48;

static pp_status launch_attend8(pp_kv *kv, AttendArgs c, void *workspace, int64_t bytes, cudaStream_t st)
{
    if ((int64_t)c.max_q * c.group <= kFewRows8) return launch_attend_token8(kv, c, st);
    if (!workspace) return fail(PP_EINVAL, "chunks need a workspace of pp_kv_workspace bytes");
    if (reinterpret_cast<uintptr_t>(workspace) & 31) return fail(PP_EINVAL, "workspace must be aligned to 32 bytes");
    const int64_t head = table_bytes(c.requests, c.table_width);
    const int64_t capacity = std::min<int64_t>((bytes - head) / (2 * block_bytes(kv)), kKvMaxBlocks);
    if (bytes < head || capacity < 1) return fail(PP_EINVAL, "the workspace is too small: see pp_kv_workspace");
    Unpack8Args u = {};
    u.a = attend_dev(kv, c);
    char *const at = static_cast<char *>(workspace);
    u.table = reinterpret_cast<int32_t *>(at);
    u.k = reinterpret_cast<uint4 *>(at + head);
    u.v = reinterpret_cast<uint4 *>(at + head + capacity * block_bytes(kv));
    u.capacity = (int32_t)capacity;
    const size_t shared = 2 * sizeof(int32_t) * c.requests;
    if (kv->dtype == PP_KV_BF16) k_unpack8<__nv_bfloat16><<<2 * kv->sm_count, kUnpackThreads, shared, st>>>(u);
    else k_unpack8<__half><<<2 * kv->sm_count, kUnpackThreads, shared, st>>>(u);
    PP_CUDA(cudaGetLastError());
    pp_kv wide = *kv;
    wide.eight = false;
    wide.blocks = u.capacity;
    wide.token_stride = kv->dim;
    wide.head_stride = (int64_t)kv->dim * kv->block_size;
    wide.block_stride = wide.head_stride * kv->heads;
    c.k_cache = u.k;
    c.v_cache = u.v;
    c.block_table = u.table;
    return launch_attend_chunk(&wide, c, true, st);
}

static pp_status check_exps(const void *k_exp, const void *v_exp)
{
    if (!k_exp || !v_exp) return fail(PP_EINVAL, "null exponents");
    if (k_exp == v_exp) return fail(PP_EINVAL, "K and V have exponents of their own");
    return PP_OK;
}

}  // namespace pp

using namespace pp;

extern "C" pp_status pp_kv_write8(pp_kv *kv, int32_t tokens, const void *k, int64_t k_token_stride, int64_t k_head_stride,
                                  const void *v, int64_t v_token_stride, int64_t v_head_stride, const int64_t *slot_map,
                                  void *k_cache, int8_t *k_exp, void *v_cache, int8_t *v_exp, void *stream)
{
    if (!kv) return fail(PP_EINVAL, "null cache handle");
    if (!kv->eight) return fail(PP_EINVAL, "the cache holds 16-bit numbers: pp_kv_write writes them");
    if (tokens < 0 || tokens > 1 << 30) return fail(PP_EINVAL, "tokens must be between 0 and 2^30");
    if (tokens == 0) return PP_OK;
    if (!k || !v || !slot_map || !k_cache || !v_cache) return fail(PP_EINVAL, "null pointer");
    pp_status s = check_exps(k_exp, v_exp);
    if (s != PP_OK) return s;
    const void *const buffers[4] = {k_cache, v_cache, k_exp, v_exp};
    for (int i = 1; i < 4; ++i)
        for (int j = 0; j < i; ++j)
            if (buffers[i] == buffers[j]) return fail(PP_EINVAL, "caches and exponents must be four different buffers");
    if (!aligned16(k) || !aligned16(v) || !aligned16(k_cache) || !aligned16(v_cache))
        return fail(PP_EINVAL, "k, v and the caches must be aligned to 16 bytes");
    if (!stride_ok(k_token_stride) || !stride_ok(k_head_stride) || !stride_ok(v_token_stride) || !stride_ok(v_head_stride))
        return fail(PP_EINVAL, "strides must be positive multiples of 8 elements below 2^38");
    s = check_device(kv);
    if (s != PP_OK) return s;
    Write8Args a = {};
    a.tokens = tokens;
    a.heads = kv->heads;
    a.per_head = kv->dim / 8;
    a.k = static_cast<const uint4 *>(k);
    a.v = static_cast<const uint4 *>(v);
    a.k_token = k_token_stride / 8;
    a.k_head = k_head_stride / 8;
    a.v_token = v_token_stride / 8;
    a.v_head = v_head_stride / 8;
    a.slot = slot_map;
    a.kc = static_cast<uint8_t *>(k_cache);
    a.vc = static_cast<uint8_t *>(v_cache);
    a.ke = k_exp;
    a.ve = v_exp;
    a.block_stride = kv->block_stride;
    a.token_stride = kv->token_stride;
    a.head_stride = kv->head_stride;
    a.slots = (int64_t)kv->blocks << kv->block_log;
    a.block_log = kv->block_log;
    a.status = kv->d_status;
    a.claim = kv->d_claim;
    // CTAs for one round of the SMs, or fewer where blocks are larger than that and a CTA would have no run's first
    // token; more CTAs share its heads out, as far as its warps would not take them in one go.
    const int32_t ctas = kWrite8Ctas * kv->sm_count, held = kWrite8Held * (32 / a.per_head);
    const int32_t warps = std::min((kv->block_size + held - 1) / held, kWrite8Warps);      // of a whole block's rows
    const int32_t teams = warps <= 1 ? 1 : warps <= 2 ? 2 : warps <= 4 ? 4 : 8;
    const int32_t even = (tokens - 1) / ctas + 1;
    a.window = kv->block_size > 32 ? std::max(even, std::min(kv->block_size, 4 * even)) : even;
    const int32_t windows = (tokens - 1) / a.window + 1;
    const int32_t rounds = (2 * kv->heads * teams + kWrite8Warps - 1) / kWrite8Warps;
    const dim3 grid(windows, std::min(std::max(2 * ctas / windows, 1), rounds));
    const cudaStream_t st = (cudaStream_t)stream;
    auto launch = [&](auto *of1, auto *of2, auto *of4, auto *of8) {
        (teams == 1 ? of1 : teams == 2 ? of2 : teams == 4 ? of4 : of8)<<<grid, kWrite8Threads, 0, st>>>(a);
    };
    if (kv->dtype == PP_KV_BF16)
        launch(k_kv_write8<__nv_bfloat16, 1>, k_kv_write8<__nv_bfloat16, 2>, k_kv_write8<__nv_bfloat16, 4>, k_kv_write8<__nv_bfloat16, 8>);
    else
        launch(k_kv_write8<__half, 1>, k_kv_write8<__half, 2>, k_kv_write8<__half, 4>, k_kv_write8<__half, 8>);
    PP_CUDA(cudaGetLastError());
    return PP_OK;
}

extern "C" pp_status pp_kv_workspace(const pp_kv *kv, int32_t requests, int32_t table_width, int32_t blocks, size_t *bytes)
{
    if (!kv) return fail(PP_EINVAL, "null cache handle");
    if (!bytes) return fail(PP_EINVAL, "null pointer");
    *bytes = 0;
    if (!kv->eight) return fail(PP_EINVAL, "a cache of 16-bit numbers needs no workspace");
    if (requests < 0 || requests > kKvMaxRequests) return fail(PP_EINVAL, "requests must be between 0 and 16384");
    if (table_width < 1 || blocks < 0 || blocks > kKvMaxBlocks)
        return fail(PP_EINVAL, "table_width must be >= 1, blocks between 0 and 2^30");
    *bytes = (size_t)table_bytes(requests, table_width) + (size_t)std::max(blocks, 1) * 2 * (size_t)block_bytes(kv);
    return PP_OK;
}

extern "C" pp_status pp_paged_attention8(pp_kv *kv, int32_t requests, int32_t tokens, int32_t q_heads, const void *q,
                                         int64_t q_token_stride, int64_t q_head_stride, const void *k_cache,
                                         const int8_t *k_exp, const void *v_cache, const int8_t *v_exp,
                                         int32_t table_width, const int32_t *block_table, const int32_t *q_start,
                                         const int32_t *length, int32_t max_q, int32_t window, float scale, void *out,
                                         int64_t out_token_stride, int64_t out_head_stride, float *lse, void *workspace,
                                         size_t workspace_bytes, void *stream)
{
    if (!kv) return fail(PP_EINVAL, "null cache handle");
    if (!kv->eight) return fail(PP_EINVAL, "the cache holds 16-bit numbers: pp_paged_attention reads it");
    const AttendArgs a = {requests, tokens, q_heads, q_heads / kv->heads, q, q_token_stride, q_head_stride, k_cache,
                          v_cache, block_table, table_width, q_start, length, max_q, window, scale, out,
                          out_token_stride, out_head_stride, lse, k_exp, v_exp};
    bool nothing = false;
    pp_status s = check_attend(kv, a, &nothing);
    if (s != PP_OK || nothing) return s;
    s = check_exps(k_exp, v_exp);
    if (s != PP_OK) return s;
    return launch_attend8(kv, a, workspace, (int64_t)std::min<size_t>(workspace_bytes, (size_t)1 << 62), (cudaStream_t)stream);
}
