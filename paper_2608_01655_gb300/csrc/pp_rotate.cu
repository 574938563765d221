// Norms of query and key heads and the rotation to their positions, in one pass, with
// the keys and values into the paged cache or the keys to rows.
//
// A row x of D elements at position p, R of them rotated, frequencies f_i, amplitude A:
//   y = x, or with a weight y = x w / sqrt(mean(x^2) + eps);
//   (y_a, y_b) -> A (y_a cos t - y_b sin t, y_b cos t + y_a sin t),  t = p f_i, i < R / 2,
// where pair i is (i, i + R/2) or, interleaved, (2 i, 2 i + 1); the rest is y.
#include <algorithm>
#include <climits>
#include <cmath>
#include <type_traits>

#include "pp_attend.cuh"
#include "pp_rotate_lanes.h"

namespace pp {

struct RotateRows {
    const uint4 *in;
    uint4 *out;
    int64_t in_token, in_head, out_token, out_head;     // vectors
    const uint4 *weight;                                // vectors of a row, or null
};
struct RotateArgs {
    int32_t tokens, heads[2], per_head, rotated;        // heads of q and of k; vectors a head; elements
    int32_t split;                                      // groups of lanes that share a token's rows
    RotateRows rows[2];                                 // of q and of k (out: null where k goes to the cache only)
    const int32_t *position;
    const uint64_t *turns;
    float eps, amplitude, inverse_dim;
    const uint4 *v;
    int64_t v_token, v_head;
    const int64_t *slot;                                // null: no cache
    uint4 *kc, *vc;
    int64_t block_stride, token_stride, head_stride;    // vectors
    int64_t slots;
    int32_t block_log;
    int32_t *status;
};

// kHalf: R / 2 is a multiple of 8, so that whole vectors are pairs.  Otherwise (kHalfOdd) a pair's other element is at
// any place of another lane's vectors and read from there by itself: 30,011 tokens of 16 + 4 heads of 128, into the
// cache, with 120 of them rotated 152 us from cold caches, with norms 214, where 128 take 64 and 81; of 80 with 40
// rotated 99 and 142, with 32 54 and 68.  64 tokens 4.7 to 6.6 us in a graph, 3.4 to 4.2.
enum { kHalf = 0, kInterleaved = 1, kHalfOdd = 2 };

constexpr int kRotateThreads = 128;
constexpr int kRotateAhead = 4;                         // rows of a group on their way
constexpr int kRotateCtas = 4;                          // of an SM

template <typename T> __device__ __forceinline__ float2 floats(uint32_t x);
template <> __device__ __forceinline__ float2 floats<__nv_bfloat16>(uint32_t x)
{
    return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
}
template <> __device__ __forceinline__ float2 floats<__half>(uint32_t x)
{
    return make_float2(__half2float(__ushort_as_half((unsigned short)(x & 0xffff))),
                       __half2float(__ushort_as_half((unsigned short)(x >> 16))));
}
template <typename T> __device__ __forceinline__ void floats8(const uint4 &x, float *to)
{
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 y = floats<T>(w[i]);
        to[2 * i] = y.x;
        to[2 * i + 1] = y.y;
    }
}
// two 32-bit numbers in a register pair
__device__ __forceinline__ uint64_t pack2(float lo, float hi)
{
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ float2 unpack2(uint64_t x)
{
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(x));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b)
{
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
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
template <typename T> __device__ __forceinline__ void twos(const uint4 &x, uint64_t (&to)[4])
{
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 y = floats<T>(w[i]);
        to[i] = pack2(y.x, y.y);
    }
}
template <typename T> __device__ __forceinline__ uint4 pack8(const uint64_t (&x)[4])
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 y = unpack2(x[i]);
        w[i] = Pack<T>::two(y.x, y.y);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// cos and sin of position * frequency.  `turns` is the frequency as a 64-bit fraction of
// a turn: the product modulo 2^64 is exact, and its high half a signed fraction (cut to
// 2^-29.3 rad, then rounded to 24 bits: 2^-23.3 rad).
__device__ __forceinline__ void angle(int32_t position, uint64_t turns, float amplitude, float &cos, float &sin)
{
    const int32_t part = (int32_t)((uint64_t)(int64_t)position * turns >> 32);
    sincospif((float)part * 0x1p-31f, &sin, &cos);
    cos *= amplitude;
    sin *= amplitude;
}

// A group of LANES lanes takes a token, or with `split` a share of its rows; a lane two
// vectors of 8 elements of each row, in half layout those of 8 pairs, so that a pair is
// one lane's and a lane's angles serve all its rows.  The norm's weights are multiplied
// into them once a token, and a row by its norm in the end:
//   y_a' = n (x_a (w_a cos) - x_b (w_b sin)),  y_b' = n (x_b (w_b cos) + x_a (w_a sin)).
// Bound by memory, 4 bytes an element: each lane copies its vectors of the next rows to
// places of its own in shared memory, so that many are on their way without registers.
// 30,011 tokens of 28 + 4 heads of 128 with norms, into the cache: 100 us from cold
// caches, 5.5 TB/s (82 us at the rate of a copy); without norms 85.  The norms' sums and
// products are a third of the instructions, which take 60% of the issue slots.  3 or 6
// rows ahead and 5 or 6 CTAs an SM were no faster than 4 and 4.  64 tokens of 16 + 2
// heads: 3.7 us a call in a graph.
template <typename T, int LAYOUT, int LANES, bool NORM>
__global__ void __launch_bounds__(kRotateThreads, kRotateCtas) k_kv_rotate(const __grid_constant__ RotateArgs a)
{
    __shared__ uint4 ahead[kRotateAhead][2][kRotateThreads];
    constexpr int kGroups = 32 / LANES;                 // of a warp
    const int32_t turned = LAYOUT == kHalf ? a.rotated / 16 : -1;       // lanes with vectors of pairs
    const RotateLane vectors = rotate_lane(threadIdx.x, LANES, a.per_head, turned);
    const int lane = vectors.lane, of_warp = vectors.of_warp;
    const int64_t group = ((int64_t)blockIdx.x * (kRotateThreads / 32) + threadIdx.x / 32) * kGroups + of_warp;
    const int32_t t = (int32_t)min(group / a.split, (int64_t)a.tokens - 1), share = (int32_t)(group % a.split);
    const bool in = of_warp < kGroups && group < (int64_t)a.tokens * a.split;
    const bool first_half = LAYOUT == kHalf && vectors.at[0] < turned;
    const int32_t at[2] = {vectors.at[0], vectors.at[1]};     // this lane's vectors, from per_head on: none
    const bool has[2] = {at[0] < a.per_head, at[1] < a.per_head};

    int64_t cache = -1;                                 // the token's place in the caches
    if (a.slot && in) {
        const int64_t s = a.slot[t];
        if (s >= a.slots) {
            if (share == 0 && lane == 0) kv_bounds(a.status);
        } else if (s >= 0) {
            cache = (s >> a.block_log) * a.block_stride + (s & ((1 << a.block_log) - 1)) * a.token_stride;
        }
    }

    // The rows: share, share + split, ... of those of q (kind 0), then of k (1), then of v (2).  Every group of a warp
    // takes the same number of steps.
    const int32_t nq = a.heads[0], nk = a.heads[1], all = nq + nk * (a.slot ? 2 : 1);
    auto first_of = [&](int kind) { return kind == 0 ? 0 : kind == 1 ? nq : nq + nk; };
    auto past = [&](int kind) { return kind == 0 ? nq : kind == 1 ? nq + nk : all; };
    const uint4 *ask_at = nullptr;                      // the next row, and from one to the next
    int64_t ask_step = 0;
    int32_t ask_row = share, ask_past = 0;              // its number, and where that of the next kind begins
    int ask_place = 0;
    auto ask = [&]() {
        if (in && ask_row < all) {
            if (ask_row >= ask_past) {
                const int kind = ask_row < nq ? 0 : ask_row < nq + nk ? 1 : 2;
                const RotateRows &r = a.rows[min(kind, 1)];
                const int64_t head = kind == 2 ? a.v_head : r.in_head;
                ask_at = (kind == 2 ? a.v + t * a.v_token : r.in + t * r.in_token) + (ask_row - first_of(kind)) * head;
                ask_step = a.split * head;
                ask_past = past(kind);
                if (kind == 2 && cache < 0) ask_row = all;
            }
            if (ask_row < all)
#pragma unroll
                for (int x = 0; x < 2; ++x)
                    if (has[x])
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(&ahead[ask_place][x][threadIdx.x])),
                                     "l"(ask_at + at[x])
                                     : "memory");
            ask_at += ask_step;
            ask_row += a.split;
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        if (++ask_place == kRotateAhead) ask_place = 0;
    };
#pragma unroll
    for (int x = 0; x < 2; ++x)                         // vectors that a row does not have count as zeros
        if (!has[x])
#pragma unroll
            for (int y = 0; y < kRotateAhead; ++y) ahead[y][x][threadIdx.x] = make_uint4(0, 0, 0, 0);
#pragma unroll 1
    for (int x = 0; x < kRotateAhead; ++x) ask();

    // cos and sin: of pair i in half layout, of vector i / 4's pair i % 4 interleaved, of element i otherwise
    constexpr int kAngles = LAYOUT == kHalfOdd ? 16 : 8;
    float cos[kAngles], sin[kAngles];
    const int32_t position = a.position[t], pairs = a.rotated / 2;
#pragma unroll
    for (int i = 0; i < kAngles; ++i) {
        int32_t pair;
        if (LAYOUT == kHalf) {
            pair = first_half ? 8 * lane + i : pairs;
        } else if (LAYOUT == kInterleaved) {
            pair = 4 * at[i / 4] + i % 4;
        } else {
            pair = 8 * at[i / 8] + i % 8;
            if (pair >= pairs) pair = pair < a.rotated ? pair - pairs : pairs;
        }
        cos[i] = 1.f;
        sin[i] = 0.f;
        if (pair < pairs) angle(position, a.turns[pair], a.amplitude, cos[i], sin[i]);
    }

    // Of a lane's 8 pairs: what x_a and x_b count for in y_a', and in y_b', two pairs each.  Where a pair does not turn
    // cos is 1.
    uint64_t aa[4], ab[4], bb[4], ba[4];
    float w[LAYOUT == kHalfOdd ? 16 : 1];
    const uint4 *weight = nullptr;                      // of the rows at hand
    uint4 *out = nullptr, *stored = nullptr;            // where the next one goes
    int64_t out_step = 0, stored_step = 0;
    int32_t row = share, row_past = 0;
    bool is_v = false;
    auto enter = [&]() {                                // rows of another kind
        const int kind = row < nq ? 0 : row < nq + nk ? 1 : 2;
        const RotateRows &r = a.rows[min(kind, 1)];
        const int32_t h = row - first_of(kind);
        row_past = past(kind);
        is_v = kind == 2;
        out = is_v || !r.out ? nullptr : r.out + t * r.out_token + h * r.out_head;
        stored = kind == 0 || cache < 0 ? nullptr : (is_v ? a.vc : a.kc) + cache + h * a.head_stride;
        out_step = a.split * r.out_head;
        stored_step = a.split * a.head_stride;
        if (is_v) return;
        weight = NORM ? r.weight : nullptr;
        float u[16];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            if (NORM && weight && has[x]) floats8<T>(__ldg(weight + at[x]), u + 8 * x);
            else
#pragma unroll
                for (int i = 0; i < 8; ++i) u[8 * x + i] = 1.f;
        }
        if constexpr (LAYOUT == kHalfOdd) {
#pragma unroll
            for (int i = 0; i < 16; ++i) w[i] = u[i];
        } else {
            float f[4][8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int lo = LAYOUT == kHalf ? i : 2 * i, hi = LAYOUT == kHalf ? i + 8 : 2 * i + 1;
                f[0][i] = NORM ? u[lo] * cos[i] : cos[i];
                f[1][i] = NORM ? u[hi] * -sin[i] : -sin[i];
                f[2][i] = NORM ? u[hi] * cos[i] : cos[i];
                f[3][i] = NORM ? u[lo] * sin[i] : sin[i];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                aa[i] = pack2(f[0][2 * i], f[0][2 * i + 1]);
                ab[i] = pack2(f[1][2 * i], f[1][2 * i + 1]);
                bb[i] = pack2(f[2][2 * i], f[2][2 * i + 1]);
                ba[i] = pack2(f[3][2 * i], f[3][2 * i + 1]);
            }
        }
    };
    int place = 0;
#pragma unroll 1
    for (int32_t steps = (all + a.split - 1) / a.split; steps > 0; --steps, row += a.split) {
        const bool live = in && row < all;
        if (live && row >= row_past) enter();
        asm volatile("cp.async.wait_group %0;" ::"n"(kRotateAhead - 1) : "memory");
        if (LAYOUT == kHalfOdd) __syncwarp();           // the others' vectors are read too
        const uint4 raw[2] = {ahead[place][0][threadIdx.x], ahead[place][1][threadIdx.x]};
        uint4 packed[2] = {raw[0], raw[1]};
        uint64_t e[2][4];                               // two elements each
        twos<T>(raw[0], e[0]);
        twos<T>(raw[1], e[1]);
        const bool norm = NORM && weight;
        float by = 1.f;
        if (NORM) {
            uint64_t sum[2] = {0, 0};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                sum[0] = fma2(e[0][i], e[0][i], sum[0]);
                sum[1] = fma2(e[1][i], e[1][i], sum[1]);
            }
            const float2 two = unpack2(add2(sum[0], sum[1]));
            const float mine = two.x + two.y;
            float total = mine;
            if constexpr ((LANES & (LANES - 1)) == 0) {
#pragma unroll
                for (int o = LANES / 2; o > 0; o >>= 1) total += __shfl_xor_sync(~0u, total, o);
            } else {
                // in the same order for all lanes
                total = 0.f;
#pragma unroll
                for (int o = 0; o < LANES; ++o) total += __shfl_sync(~0u, mine, min(of_warp * LANES + o, 31));
            }
            if (norm) by = rsqrtf(fmaf(total, a.inverse_dim, a.eps));
        }
        const uint64_t by2 = pack2(by, by);
        if (!is_v) {
            bool changed = true;                        // else the row's bits stay
            if (LAYOUT == kHalf) {
                if (first_half) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint64_t lo = e[0][i], hi = e[1][i];
                        e[0][i] = fma2(lo, aa[i], mul2(hi, ab[i]));
                        e[1][i] = fma2(hi, bb[i], mul2(lo, ba[i]));
                        if (NORM) {
                            e[0][i] = mul2(e[0][i], by2);
                            e[1][i] = mul2(e[1][i], by2);
                        }
                    }
                } else if (norm) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        e[0][i] = mul2(mul2(e[0][i], aa[i]), by2);
                        e[1][i] = mul2(mul2(e[1][i], bb[i]), by2);
                    }
                } else {
                    changed = false;
                }
            } else if (LAYOUT == kInterleaved) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float2 x = unpack2(e[i / 4][i % 4]), fa = unpack2(aa[i / 2]), fb = unpack2(ab[i / 2]);
                    const float2 ga = unpack2(bb[i / 2]), gb = unpack2(ba[i / 2]);
                    const float a0 = i % 2 ? fa.y : fa.x, b0 = i % 2 ? fb.y : fb.x, a1 = i % 2 ? ga.y : ga.x, b1 = i % 2 ? gb.y : gb.x;
                    const bool turns = 4 * at[i / 4] + i % 4 < pairs;
                    const float lo = turns ? x.x * a0 + x.y * b0 : x.x * a0, hi = turns ? x.y * a1 + x.x * b1 : x.y * a1;
                    e[i / 4][i % 4] = NORM ? mul2(pack2(lo, hi), by2) : pack2(lo, hi);
                }
            } else if constexpr (LAYOUT == kHalfOdd) {
#pragma unroll
                for (int i = 0; i < 16; i += 2) {
                    const float2 x = unpack2(e[i / 8][i % 8 / 2]);
                    float y[2] = {x.x, x.y};
#pragma unroll
                    for (int z = 0; z < 2; ++z) {
                        const int32_t d = 8 * at[i / 8] + i % 8 + z, p = d < pairs ? d + pairs : d - pairs;
                        if (norm) y[z] = by * (y[z] * w[i + z]);
                        if (has[i / 8] && d < a.rotated) {
                            const T *from = reinterpret_cast<const T *>(
                                &ahead[place][rotate_which(LANES, p / 8)][rotate_holder(threadIdx.x, LANES, p / 8)]);
                            float other = KvType<T>::to_float(from[p % 8]);
                            if (norm) other = by * (other * KvType<T>::to_float(reinterpret_cast<const T *>(weight)[p]));
                            y[z] = y[z] * cos[i + z] + (d < pairs ? -other : other) * sin[i + z];
                        }
                    }
                    e[i / 8][i % 8 / 2] = pack2(y[0], y[1]);
                }
            }
            if (changed) {
                packed[0] = pack8<T>(e[0]);
                packed[1] = pack8<T>(e[1]);
            }
        }
        if (LAYOUT == kHalfOdd) __syncwarp();           // all have read what the next copies overwrite
        if (++place == kRotateAhead) place = 0;
        ask();
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            if (!live || !has[x]) continue;
            if (out) out[at[x]] = packed[x];
            if (stored) stored[at[x]] = packed[x];
        }
        if (out) out += out_step;
        if (stored) stored += stored_step;
    }
}

}  // namespace pp

using namespace pp;

extern "C" pp_status pp_rotary_frequencies(int32_t pairs, double base, double factor, double original, double slow,
                                           double fast, double *frequency)
{
    if (pairs < 0 || pairs > kKvMaxDim / 2) return fail(PP_EINVAL, "pairs must be between 0 and 64");
    if (pairs > 0 && !frequency) return fail(PP_EINVAL, "null pointer");
    if (!(base > 0) || !std::isfinite(base)) return fail(PP_EINVAL, "base must be positive and finite");
    if (!(factor > 0) || !std::isfinite(factor)) return fail(PP_EINVAL, "factor must be positive and finite");
    if (!(original >= 0) || !std::isfinite(original)) return fail(PP_EINVAL, "original must be >= 0 and finite");
    if (original > 0 && (!(slow < fast) || !std::isfinite(slow) || !std::isfinite(fast)))
        return fail(PP_EINVAL, "slow must be below fast, and both finite");
    const double turn = 6.283185307179586;
    double out[kKvMaxDim / 2];
    for (int32_t i = 0; i < pairs; ++i) {
        const double f = std::pow(base, -(double)i / pairs);
        const double keep = original > 0 ? std::min(std::max((original * f / turn - slow) / (fast - slow), 0.0), 1.0) : 0.0;
        out[i] = f * (keep + (1.0 - keep) / factor);
        if (!std::isfinite(out[i])) return fail(PP_EINVAL, "base and factor give a frequency that is not finite");
    }
    std::copy_n(out, pairs, frequency);
    return PP_OK;
}

extern "C" pp_status pp_rotary_turns(int32_t pairs, const double *frequency, uint64_t *turns)
{
    if (pairs < 0 || pairs > kKvMaxDim / 2) return fail(PP_EINVAL, "pairs must be between 0 and 64");
    if (pairs > 0 && (!frequency || !turns)) return fail(PP_EINVAL, "null pointer");
    for (int32_t i = 0; i < pairs; ++i)
        if (!std::isfinite(frequency[i])) return fail(PP_EINVAL, "frequencies must be finite");
    for (int32_t i = 0; i < pairs; ++i) {
        // of the size, so that what is below a whole turn keeps its bits whatever the sign is
        const double t = std::fabs(frequency[i]) / 6.283185307179586;
        const uint64_t part = (uint64_t)std::rint(std::ldexp(t - std::floor(t), 64));
        turns[i] = frequency[i] < 0 ? 0 - part : part;
    }
    return PP_OK;
}

extern "C" pp_status pp_kv_rotate(pp_kv *kv, int32_t tokens, int32_t q_heads, const void *q, int64_t q_token_stride,
                                  int64_t q_head_stride, const void *k, int64_t k_token_stride, int64_t k_head_stride,
                                  const void *q_weight, const void *k_weight, float eps, const int32_t *position,
                                  int32_t rotated, int32_t interleaved, const uint64_t *turns, float amplitude,
                                  void *q_out, int64_t q_out_token_stride, int64_t q_out_head_stride, void *k_out,
                                  int64_t k_out_token_stride, int64_t k_out_head_stride, const void *v,
                                  int64_t v_token_stride, int64_t v_head_stride, const int64_t *slot_map, void *k_cache,
                                  void *v_cache, void *stream)
{
    if (!kv) return fail(PP_EINVAL, "null cache handle");
    if (tokens < 0 || tokens > 1 << 30) return fail(PP_EINVAL, "tokens must be between 0 and 2^30");
    if (q_heads < 0 || q_heads > 1 << 20) return fail(PP_EINVAL, "q_heads must be between 0 and 2^20");
    if (rotated < 0 || rotated > kv->dim || rotated % 2)
        return fail(PP_EINVAL, "rotated must be even, between 0 and head_dim");
    if (!(eps >= 0) || !(eps < INFINITY)) return fail(PP_EINVAL, "eps must be >= 0 and finite");
    if (!std::isfinite(amplitude)) return fail(PP_EINVAL, "amplitude must be finite");
    if (tokens == 0) return PP_OK;
    const bool caches = slot_map || k_cache || v_cache || v;
    if (caches && kv->eight) return fail(PP_EINVAL, "the cache holds 8-bit numbers: rows go to k_out, then to pp_kv_write8");
    if (caches && (!slot_map || !k_cache || !v_cache || !v))
        return fail(PP_EINVAL, "v, slot_map, k_cache and v_cache go together");
    if (!caches && !k_out) return fail(PP_EINVAL, "k goes to k_out or to the cache");
    if (!k || !position || (q_heads > 0 && (!q || !q_out)) || (rotated > 0 && !turns)) return fail(PP_EINVAL, "null pointer");
    for (const void *p : {q, k, (const void *)q_out, (const void *)k_out, v, (const void *)k_cache, (const void *)v_cache,
                          q_weight, k_weight})
        if (!aligned16(p)) return fail(PP_EINVAL, "rows, weights and caches must be aligned to 16 bytes");
    if (reinterpret_cast<uintptr_t>(turns) & 7) return fail(PP_EINVAL, "turns must be aligned to 8 bytes");
    if (!stride_ok(k_token_stride) || !stride_ok(k_head_stride) ||
        (q_heads > 0 && (!stride_ok(q_token_stride) || !stride_ok(q_head_stride) || !stride_ok(q_out_token_stride) ||
                         !stride_ok(q_out_head_stride))) ||
        (k_out && (!stride_ok(k_out_token_stride) || !stride_ok(k_out_head_stride))) ||
        (caches && (!stride_ok(v_token_stride) || !stride_ok(v_head_stride))))
        return fail(PP_EINVAL, "strides must be positive multiples of 8 elements below 2^38");
    if (q_heads > 0 && rows_overlap(kv->dim, {{q_out_token_stride, tokens}, {q_out_head_stride, q_heads}}))
        return fail(PP_EINVAL, "rows of q_out would overlap with these strides");
    if (k_out && rows_overlap(kv->dim, {{k_out_token_stride, tokens}, {k_out_head_stride, kv->heads}}))
        return fail(PP_EINVAL, "rows of k_out would overlap with these strides");
    // buffers that begin at one place share a row, which two groups would write, or one while another reads it
    const void *const outs[4] = {q_heads > 0 ? q_out : nullptr, k_out, k_cache, v_cache};
    const void *const ins[3] = {q_heads > 0 ? q : nullptr, k, v};
    for (int i = 0; i < 4; ++i) {
        for (int j = 0; outs[i] && j < 4; ++j)
            if (j != i && outs[j] == outs[i]) return fail(PP_EINVAL, "q_out, k_out and the caches must be different buffers");
        for (int j = 0; outs[i] && j < 3; ++j)
            if ((j != i || j == 2) && ins[j] == outs[i])
                return fail(PP_EINVAL, "an output over another one's input: only q_out may be q and k_out k");
    }
    // in place a row is read before it is written; other rows over it would be a race
    if ((q_heads > 0 && q_out == q && tokens * (int64_t)q_heads > 1 &&
         ((tokens > 1 && q_out_token_stride != q_token_stride) || (q_heads > 1 && q_out_head_stride != q_head_stride))) ||
        (k_out && k_out == k && tokens * (int64_t)kv->heads > 1 &&
         ((tokens > 1 && k_out_token_stride != k_token_stride) || (kv->heads > 1 && k_out_head_stride != k_head_stride))))
        return fail(PP_EINVAL, "rows in place keep their strides");
    pp_status s = check_device(kv);
    if (s != PP_OK) return s;
    RotateArgs a = {};
    a.tokens = tokens;
    a.heads[0] = q_heads;
    a.heads[1] = kv->heads;
    a.per_head = kv->dim / 8;
    a.rotated = rotated;
    a.rows[0] = {static_cast<const uint4 *>(q), static_cast<uint4 *>(q_out), q_token_stride / 8, q_head_stride / 8,
                 q_out_token_stride / 8, q_out_head_stride / 8, static_cast<const uint4 *>(q_weight)};
    a.rows[1] = {static_cast<const uint4 *>(k), static_cast<uint4 *>(k_out), k_token_stride / 8, k_head_stride / 8,
                 k_out_token_stride / 8, k_out_head_stride / 8, static_cast<const uint4 *>(k_weight)};
    a.position = position;
    a.turns = turns;
    a.eps = eps;
    a.amplitude = amplitude;
    a.inverse_dim = 1.f / (float)kv->dim;
    if (caches) {
        a.v = static_cast<const uint4 *>(v);
        a.v_token = v_token_stride / 8;
        a.v_head = v_head_stride / 8;
        a.slot = slot_map;
        a.kc = static_cast<uint4 *>(k_cache);
        a.vc = static_cast<uint4 *>(v_cache);
        a.block_stride = kv->block_stride / 8;
        a.token_stride = kv->token_stride / 8;
        a.head_stride = kv->head_stride / 8;
        a.slots = (int64_t)kv->blocks << kv->block_log;
        a.block_log = kv->block_log;
    }
    a.status = kv->d_status;
    const int layout = interleaved ? kInterleaved : rotated % 16 == 0 ? kHalf : kHalfOdd;
    const int lanes = rotate_lanes(kv->dim);
    const int32_t rows = q_heads + kv->heads * (caches ? 2 : 1);
    // How many groups share a token's rows: all groups take rounds of as many as the SMs hold, of rows and of the
    // token's angles, which take as long as some kAngleRows rows.  30,011 tokens of 36 rows: 3.1 rounds of whole
    // tokens, which are 4 of 39 rows, or 6.2 of halves, 7 of 21.
    constexpr int kAngleRows = 3;
    const int64_t per_cta = kRotateThreads / 32 * (32 / lanes), held = (int64_t)kv->sm_count * kRotateCtas * per_cta;
    int64_t least = INT64_MAX;
    for (int32_t split = 1, share; split <= 64; split = (rows + share - 2) / (share - 1)) {    // the least for each share
        share = (rows + split - 1) / split;
        const int64_t rounds = ((int64_t)tokens * split + held - 1) / held, cost = rounds * (share + kAngleRows);
        if (cost < least) {
            least = cost;
            a.split = split;
        }
        if (share == 1) break;
    }
    const int64_t grid = ((int64_t)tokens * a.split + per_cta - 1) / per_cta;
    if (grid > INT_MAX) return fail(PP_EINVAL, "too many tokens");
    const cudaStream_t st = (cudaStream_t)stream;
    auto launch = [&](auto type) {
        using T = decltype(type);
        auto of = [&](auto l, auto n) {
            constexpr int LAYOUT = decltype(l)::value;
            constexpr bool NORM = decltype(n)::value;
            switch (lanes) {
            case 1: k_kv_rotate<T, LAYOUT, 1, NORM><<<(int)grid, kRotateThreads, 0, st>>>(a); break;
            case 2: k_kv_rotate<T, LAYOUT, 2, NORM><<<(int)grid, kRotateThreads, 0, st>>>(a); break;
            case 4: k_kv_rotate<T, LAYOUT, 4, NORM><<<(int)grid, kRotateThreads, 0, st>>>(a); break;
            case 5: k_kv_rotate<T, LAYOUT, 5, NORM><<<(int)grid, kRotateThreads, 0, st>>>(a); break;
            case 6: k_kv_rotate<T, LAYOUT, 6, NORM><<<(int)grid, kRotateThreads, 0, st>>>(a); break;
            default: k_kv_rotate<T, LAYOUT, 8, NORM><<<(int)grid, kRotateThreads, 0, st>>>(a);
            }
        };
        auto with = [&](auto l) {
            if (q_weight || k_weight) of(l, std::true_type());
            else of(l, std::false_type());
        };
        if (layout == kHalf) with(std::integral_constant<int, kHalf>());
        else if (layout == kInterleaved) with(std::integral_constant<int, kInterleaved>());
        else with(std::integral_constant<int, kHalfOdd>());
    };
    if (kv->dtype == PP_KV_BF16) launch(__nv_bfloat16());
    else launch(__half());
    PP_CUDA(cudaGetLastError());
    return PP_OK;
}
