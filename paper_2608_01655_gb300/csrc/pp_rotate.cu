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

enum { kHalf = 0, kInterleaved = 1, kHalfOdd = 2 };     // kHalf: R / 2 is a multiple of 8

constexpr int kRotateThreads = 256;
constexpr int kRotateRows = 2;                          // rows of a group on their way

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
template <typename T> __device__ __forceinline__ uint4 pack8(const float *x)
{
    return make_uint4(Pack<T>::two(x[0], x[1]), Pack<T>::two(x[2], x[3]), Pack<T>::two(x[4], x[5]), Pack<T>::two(x[6], x[7]));
}

// cos and sin of position * frequency.  `turns` is the frequency as a 64-bit fraction of
// a turn: the product modulo 2^64 is exact, and its high half a signed fraction.
__device__ __forceinline__ void angle(int32_t position, uint64_t turns, float amplitude, float &cos, float &sin)
{
    const int32_t part = (int32_t)((uint64_t)(int64_t)position * turns >> 32);
    sincospif((float)part * 0x1p-31f, &sin, &cos);
    cos *= amplitude;
    sin *= amplitude;
}

// A group of LANES lanes takes a token, or with `split` a share of its rows; a lane two
// vectors of 8 elements of each row, in half layout those of 8 pairs, so that a pair is
// one lane's and a lane's angles serve all its rows.  Bound by memory: 4 bytes an
// element.
template <typename T, int LAYOUT, int LANES>
__global__ void __launch_bounds__(kRotateThreads) k_kv_rotate(const __grid_constant__ RotateArgs a)
{
    const int lane = threadIdx.x % LANES;
    const int64_t group = (int64_t)blockIdx.x * (kRotateThreads / LANES) + threadIdx.x / LANES;
    const int32_t t = (int32_t)min(group / a.split, (int64_t)a.tokens - 1), share = (int32_t)(group % a.split);
    const bool in = group < (int64_t)a.tokens * a.split;

    // this lane's vectors, per_head: none
    const int32_t turned = LAYOUT == kHalf ? a.rotated / 16 : 0;        // lanes with vectors of pairs
    int32_t at[2];
    if (LAYOUT == kHalf && lane < turned) {
        at[0] = lane;
        at[1] = lane + turned;
    } else if (LAYOUT == kHalf) {
        at[0] = 2 * turned + 2 * (lane - turned);
        at[1] = at[0] + 1;
    } else {
        at[0] = lane;
        at[1] = lane + LANES;
    }
    const bool has[2] = {at[0] < a.per_head, at[1] < a.per_head};

    // the angles: of pair i in half layout, of vector x's pair i - 4 x interleaved, of
    // element i otherwise
    constexpr int kAngles = LAYOUT == kHalfOdd ? 16 : 8;
    float cos[kAngles], sin[kAngles];
    const int32_t position = a.position[t], pairs = a.rotated / 2;
#pragma unroll
    for (int i = 0; i < kAngles; ++i) {
        int32_t pair;
        if (LAYOUT == kHalf) {
            pair = lane < turned ? 8 * lane + i : pairs;
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

    const int32_t nq = a.heads[0], nk = a.heads[1], all = nq + nk + (a.slot ? nk : 0);
    int64_t cache = -1;                                 // the token's place in the caches
    if (a.slot && in) {
        const int64_t s = a.slot[t];
        if (s >= a.slots) {
            if (share == 0 && lane == 0) kv_bounds(a.status);
        } else if (s >= 0) {
            cache = (s >> a.block_log) * a.block_stride + (s & ((1 << a.block_log) - 1)) * a.token_stride;
        }
    }
    uint4 weight[2][2];
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int x = 0; x < 2; ++x)
            weight[n][x] = a.rows[n].weight && has[x] ? __ldg(a.rows[n].weight + at[x]) : make_uint4(0, 0, 0, 0);

    // every group of a warp takes the same number of steps, with rows or without
    const int32_t steps = (all + a.split - 1) / a.split;
#pragma unroll 1
    for (int32_t step = 0; step < steps; step += kRotateRows) {
        uint4 raw[kRotateRows][2];
        bool live[kRotateRows];
#pragma unroll
        for (int y = 0; y < kRotateRows; ++y) {
            const int32_t row = (step + y) * a.split + share;
            live[y] = in && step + y < steps && row < all;
            const bool is_v = row >= nq + nk, is_k = row >= nq;
            const RotateRows &r = a.rows[is_k];
            const int32_t h = row - (is_v ? nq + nk : is_k ? nq : 0);
            const uint4 *src = is_v ? a.v + t * a.v_token + h * a.v_head : r.in + t * r.in_token + h * r.in_head;
#pragma unroll
            for (int x = 0; x < 2; ++x) raw[y][x] = live[y] && has[x] && !(is_v && cache < 0) ? src[at[x]] : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int y = 0; y < kRotateRows; ++y) {
            const int32_t row = (step + y) * a.split + share;
            const bool is_v = row >= nq + nk, is_k = row >= nq;
            const RotateRows &r = a.rows[is_k];
            const int32_t h = row - (is_v ? nq + nk : is_k ? nq : 0);
            float e[16];
            floats8<T>(raw[y][0], e);
            floats8<T>(raw[y][1], e + 8);
            float other[16];                            // kHalfOdd: the pairs' other elements
            float w_other[16];
            if (LAYOUT == kHalfOdd && live[y] && !is_v) {
                const T *base = reinterpret_cast<const T *>(r.in + t * r.in_token + h * r.in_head);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int32_t d = 8 * at[i / 8] + i % 8, p = d < pairs ? d + pairs : d - pairs;
                    const bool some = has[i / 8] && d < a.rotated;
                    other[i] = some ? KvType<T>::to_float(base[p]) : 0.f;
                    w_other[i] = some && r.weight ? KvType<T>::to_float(reinterpret_cast<const T *>(r.weight)[p]) : 1.f;
                }
            }
            if (a.rows[0].weight || a.rows[1].weight) { // the lanes of a warp may have rows of both
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < 16; ++i) sum = fmaf(e[i], e[i], sum);
#pragma unroll
                for (int o = LANES / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
                const float by = rsqrtf(fmaf(sum, a.inverse_dim, a.eps));
                if (!is_v && r.weight) {
                    float w[16];
                    floats8<T>(weight[is_k][0], w);
                    floats8<T>(weight[is_k][1], w + 8);
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        e[i] = e[i] * by * w[i];
                        if (LAYOUT == kHalfOdd) other[i] = other[i] * by * w_other[i];
                    }
                }
            }
            if (!is_v) {
                if (LAYOUT == kHalf) {
                    if (lane < turned) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float lo = e[i], hi = e[8 + i];
                            e[i] = lo * cos[i] - hi * sin[i];
                            e[8 + i] = hi * cos[i] + lo * sin[i];
                        }
                    }
                } else if (LAYOUT == kInterleaved) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        if (4 * at[i / 4] + i % 4 >= pairs) continue;
                        const float lo = e[2 * i], hi = e[2 * i + 1];
                        e[2 * i] = lo * cos[i] - hi * sin[i];
                        e[2 * i + 1] = hi * cos[i] + lo * sin[i];
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int32_t d = 8 * at[i / 8] + i % 8;
                        if (d < a.rotated) e[i] = e[i] * cos[i] + (d < pairs ? -other[i] : other[i]) * sin[i];
                    }
                }
            }
            __syncwarp();                               // all have read a row that may be written in place
            if (!live[y]) continue;
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                if (!has[x]) continue;
                const uint4 packed = is_v ? raw[y][x] : pack8<T>(e + 8 * x);
                if (!is_v && r.out) r.out[t * r.out_token + h * r.out_head + at[x]] = packed;
                if (is_k && cache >= 0) (is_v ? a.vc : a.kc)[cache + h * a.head_stride + at[x]] = packed;
            }
        }
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
    if (original > 0 && !(slow < fast)) return fail(PP_EINVAL, "slow must be below fast");
    const double turn = 6.283185307179586;
    for (int32_t i = 0; i < pairs; ++i) {
        const double f = std::pow(base, -(double)i / pairs);
        const double keep = original > 0 ? std::min(std::max((original * f / turn - slow) / (fast - slow), 0.0), 1.0) : 0.0;
        frequency[i] = f * (keep + (1.0 - keep) / factor);
    }
    return PP_OK;
}

extern "C" pp_status pp_rotary_turns(int32_t pairs, const double *frequency, uint64_t *turns)
{
    if (pairs < 0 || pairs > kKvMaxDim / 2) return fail(PP_EINVAL, "pairs must be between 0 and 64");
    if (pairs > 0 && (!frequency || !turns)) return fail(PP_EINVAL, "null pointer");
    for (int32_t i = 0; i < pairs; ++i)
        if (!std::isfinite(frequency[i])) return fail(PP_EINVAL, "frequencies must be finite");
    for (int32_t i = 0; i < pairs; ++i) {
        const double t = frequency[i] / 6.283185307179586, part = t - std::floor(t);
        turns[i] = part < 1.0 ? (uint64_t)std::ldexp(part, 64) : 0;     // a tiny negative frequency rounds to a whole turn
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
    const int lanes = kv->dim > 64 ? 8 : kv->dim > 32 ? 4 : kv->dim > 16 ? 2 : 1;
    const int32_t rows = q_heads + kv->heads * (caches ? 2 : 1);
    // with few tokens several groups share a token's rows, so that there is a warp for every scheduler or so
    const int64_t want = (int64_t)kv->sm_count * 8 * (32 / lanes);
    a.split = (int32_t)std::min<int64_t>(std::max<int64_t>(want / tokens, 1), rows);
    const int64_t groups = (int64_t)tokens * a.split, per_cta = kRotateThreads / lanes;
    const int64_t grid = (groups + per_cta - 1) / per_cta;
    if (grid > INT_MAX) return fail(PP_EINVAL, "too many tokens");
    const cudaStream_t st = (cudaStream_t)stream;
    auto launch = [&](auto type) {
        using T = decltype(type);
        auto of = [&](auto l) {
            constexpr int LAYOUT = decltype(l)::value;
            switch (lanes) {
            case 1: k_kv_rotate<T, LAYOUT, 1><<<(int)grid, kRotateThreads, 0, st>>>(a); break;
            case 2: k_kv_rotate<T, LAYOUT, 2><<<(int)grid, kRotateThreads, 0, st>>>(a); break;
            case 4: k_kv_rotate<T, LAYOUT, 4><<<(int)grid, kRotateThreads, 0, st>>>(a); break;
            default: k_kv_rotate<T, LAYOUT, 8><<<(int)grid, kRotateThreads, 0, st>>>(a);
            }
        };
        if (layout == kHalf) of(std::integral_constant<int, kHalf>());
        else if (layout == kInterleaved) of(std::integral_constant<int, kInterleaved>());
        else of(std::integral_constant<int, kHalfOdd>());
    };
    if (kv->dtype == PP_KV_BF16) launch(__nv_bfloat16());
    else launch(__half());
    PP_CUDA(cudaGetLastError());
    return PP_OK;
}
