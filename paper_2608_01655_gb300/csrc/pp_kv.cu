// A worker's paged K/V cache: the handle, the resident chunks' block map, a
// step's block tables and slot map, and the write of new K and V rows.
#include <algorithm>
#include <climits>
#include <cstdlib>
#include <exception>
#include <initializer_list>
#include <new>
#include <vector>

#include "pp_kv.cuh"

namespace pp {

// ---------------------------------------------------------------------------
// Chunk map (host).  A resident set is closed under parents, so it is a forest.
// A run of chunks each of which is the heavy child of the one before (the child
// with the most resident chunks below it) gets consecutive blocks and is one
// segment: a request's path crosses at most log2(n) + 1 of them, and the block
// tables' kernel reads one record a segment instead of one a chunk.
// ---------------------------------------------------------------------------
static pp_status chunk_map(int32_t n, const int32_t *parent, const int32_t *weight, const uint8_t *resident,
                           int32_t blocks_per_slot, int32_t *map, int32_t *blocks)
{
    for (int32_t v = 0; v < n; ++v) {
        if (parent[v] < -1 || parent[v] >= n || parent[v] == v)
            return fail(PP_ENOTTREE, "parent id out of range or self-parent at node " + std::to_string(v));
        if (weight[v] < 1) return fail(PP_EINVAL, "chunk weight must be >= 1");
    }
    // order: every parent before its children
    std::vector<int32_t> kids(n, 0), order;
    std::vector<int64_t> first((size_t)n + 1, 0);
    for (int32_t v = 0; v < n; ++v)
        if (parent[v] >= 0) kids[parent[v]]++;
    for (int32_t v = 0; v < n; ++v) first[v + 1] = first[v] + kids[v];
    std::vector<int32_t> child(n);
    std::vector<int64_t> at(first.begin(), first.end() - 1);
    order.reserve(n);
    for (int32_t v = 0; v < n; ++v) {
        if (parent[v] < 0) order.push_back(v);
        else child[at[parent[v]]++] = v;
    }
    for (size_t i = 0; i < order.size(); ++i)
        for (int64_t c = first[order[i]]; c < first[order[i] + 1]; ++c) order.push_back(child[c]);
    if ((int32_t)order.size() != n) return fail(PP_ENOTTREE, "parent array contains a cycle");

    int64_t total = 0;
    for (int32_t v = 0; v < n; ++v) {
        if (!resident[v]) continue;
        if (parent[v] >= 0 && !resident[parent[v]])
            return fail(PP_EINVAL, "the resident set is not closed under parents at node " + std::to_string(v));
        total += (int64_t)weight[v] * blocks_per_slot;
        if (total > kKvMaxBlocks) return fail(PP_EOVERFLOW, "the resident chunks need more than 2^30 blocks");
    }
    std::vector<int32_t> size(n, 1), heavy(n, -1);
    for (int32_t i = n - 1; i >= 0; --i) {
        const int32_t v = order[i], p = parent[v];
        if (p >= 0 && resident[v]) size[p] += size[v];
    }
    for (int32_t v = 0; v < n; ++v) {
        const int32_t p = parent[v];
        if (p >= 0 && resident[v] && (heavy[p] < 0 || size[v] > size[heavy[p]])) heavy[p] = v;
    }
    int32_t used = 0;
    for (int32_t v : order) {
        const int32_t p = parent[v];
        int32_t *rec = map + 4 * (int64_t)v;
        if (!resident[v]) {
            rec[0] = p < 0 ? -1 : resident[p] ? p : map[4 * (int64_t)p];
            rec[1] = -1;
            rec[2] = rec[3] = 0;
        } else if (p < 0 || heavy[p] != v) {             // a segment's first chunk: lay out the run
            const int32_t begin = p < 0 ? 0 : map[4 * (int64_t)p + 3], base = used;
            int32_t end = begin;
            for (int32_t b = v; b >= 0; b = heavy[b]) {
                const int32_t w = weight[b] * blocks_per_slot;
                end += w;
                used += w;
                int32_t *r = map + 4 * (int64_t)b;
                r[0] = p;
                r[1] = base;
                r[2] = begin;
                r[3] = end;
            }
        }
    }
    *blocks = used;
    return PP_OK;
}

// ---------------------------------------------------------------------------
// Block tables.
// ---------------------------------------------------------------------------
struct TablesArgs {
    int32_t requests, n_chunks, free_count, table_width, max_tokens, blocks, block_log;
    const int32_t *length, *cached, *node;
    const int4 *map;
    const int32_t *free_blocks, *free_head;
    int32_t *free_head_out, *table, *position, *q_start;
    int64_t *slot;
    int32_t *status;
    int32_t wide;                       // slot and position start at 16-byte boundaries
};

constexpr int kTabThreads = 1024;

// A request's counts from its length, its node and its cached tokens.
// `up` is the deepest resident chunk of an admitted request's path, else -1.
struct TabRow {
    int32_t length, cached, up;
};

__device__ __forceinline__ TabRow tab_row(const TablesArgs &a, int32_t r, bool report)
{
    TabRow w;
    bool bad = false;
    const int64_t room = (int64_t)a.table_width << a.block_log;
    w.length = a.length[r];
    if (w.length < 0) { bad = true; w.length = 0; }
    if (w.length > room) { bad = true; w.length = (int32_t)room; }
    int32_t node = a.node ? a.node[r] : -1;
    if (node < -1 || node >= a.n_chunks) { bad = true; node = -1; }
    w.up = -1;
    if (node >= 0) {
        int4 rec = a.map[node];
        w.up = node;
        if (rec.y < 0) {
            w.up = rec.x;
            if (w.up >= a.n_chunks) { bad = true; w.up = -1; }
            if (w.up >= 0) rec = a.map[w.up];
        }
        // whole blocks, and never all of the request: its last token is computed
        const int64_t have = w.up >= 0 ? (int64_t)max(rec.w, 0) << a.block_log : 0;
        const int32_t whole = max(w.length - 1, 0) >> a.block_log << a.block_log;
        w.cached = (int32_t)min(have, (int64_t)whole);
    } else {
        w.cached = a.cached[r];
        if (w.cached < 0 || w.cached > w.length) { bad = true; w.cached = min(max(w.cached, 0), w.length); }
    }
    if (bad && report) kv_bounds(a.status);
    return w;
}

// the last i in [0, n) with pre[i] <= x (pre ascending, pre[0] <= x)
__device__ __forceinline__ int32_t tab_find(const int32_t *pre, int32_t n, int32_t x)
{
    int32_t lo = 0;
    for (int32_t len = n; len > 1;) {
        const int32_t half = len >> 1;
        if (pre[lo + half] <= x) { lo += half; len -= half; }
        else len = half;
    }
    return lo;
}

// Every CTA scans all requests' counts (12 bytes a request and two chunk records
// of an admitted one, from L2 after the first) and keeps the prefix sums in shared
// memory, so one launch without any exchange between CTAs does it.  Then a
// quarter of the warps walks the admitted requests' paths, a chain of dependent
// loads a segment, and fills in the new blocks, while the others write the tokens'
// slots and positions, four a thread.  Latency bounds it up to some hundred
// thousand new tokens, then the 12 bytes a token.  Measured: 16 requests of a
// token each 5 us, 192 admitted with 58,000 new tokens 7 us, 2,048 requests with 2.3
// million 16 us (1.7 TB/s; 4 us at the copy rate: the scan is 4 us, each of five
// passes over the tokens a search in the prefix sums and a table look-up).
constexpr int kTabWalkers = kTabThreads / 4;
constexpr int kTabRun = 4;                          // tokens of a thread
constexpr int kTabPass = kTabRun * (kTabThreads - kTabWalkers);    // tokens that a CTA writes at once

__global__ void __launch_bounds__(kTabThreads) k_block_tables(TablesArgs a)
{
    extern __shared__ int32_t sm[];
    int32_t *tok = sm, *nbk = tok + a.requests + 1, *held = nbk + a.requests + 1;
    __shared__ int64_t wsum[2][32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int32_t bs = 1 << a.block_log;

    // each thread takes neighbouring requests: new tokens and new blocks, summed up
    const int32_t per = (a.requests + kTabThreads - 1) / kTabThreads;
    const int32_t first = min(tid * per, a.requests), past = min(first + per, a.requests);
    int64_t my_t = 0, my_b = 0;
#pragma unroll 2
    for (int32_t r = first; r < past; ++r) {
        const TabRow w = tab_row(a, r, blockIdx.x == 0);
        const int32_t t = w.length - w.cached;
        const int32_t b = (int32_t)(((w.length + (int64_t)bs - 1) >> a.block_log) - ((w.cached + (int64_t)bs - 1) >> a.block_log));
        tok[r] = t;
        nbk[r] = b;
        held[r] = w.cached;
        my_t += t;
        my_b += b;
    }
    int64_t st = my_t, sb = my_b;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t x = __shfl_up_sync(~0u, st, o), y = __shfl_up_sync(~0u, sb, o);
        if (lane >= o) { st += x; sb += y; }
    }
    if (lane == 31) { wsum[0][warp] = st; wsum[1][warp] = sb; }
    __syncthreads();
    int64_t tot_t = wsum[0][lane], tot_b = wsum[1][lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t u = __shfl_up_sync(~0u, tot_t, o), v = __shfl_up_sync(~0u, tot_b, o);
        if (lane >= o) { tot_t += u; tot_b += v; }
    }
    const int64_t before_t = __shfl_sync(~0u, tot_t, warp ? warp - 1 : 0), before_b = __shfl_sync(~0u, tot_b, warp ? warp - 1 : 0);
    tot_t = __shfl_sync(~0u, tot_t, 31);
    tot_b = __shfl_sync(~0u, tot_b, 31);
    st += (warp ? before_t : 0) - my_t;
    sb += (warp ? before_b : 0) - my_b;
    for (int32_t r = first; r < past; ++r) {
        const int32_t t = tok[r], b = nbk[r];
        tok[r] = (int32_t)min(st, (int64_t)INT_MAX);
        nbk[r] = (int32_t)min(sb, (int64_t)INT_MAX);
        st += t;
        sb += b;
    }
    const int32_t tokens = (int32_t)min(tot_t, (int64_t)a.max_tokens);
    const int32_t fresh_blocks = (int32_t)min(tot_b, (int64_t)INT_MAX);
    int32_t head = a.free_head[0];
    const bool bad_head = head < 0 || head > a.free_count;
    head = min(max(head, 0), a.free_count);
    const int32_t spare = a.free_count - head;
    if (tid == 0) {
        tok[a.requests] = (int32_t)min(tot_t, (int64_t)INT_MAX);
        nbk[a.requests] = fresh_blocks;
        if (blockIdx.x == 0) {
            if (bad_head || tot_t > a.max_tokens || tot_b > spare) kv_bounds(a.status);
            a.free_head_out[0] = head + min(fresh_blocks, spare);
        }
    }
    __syncthreads();

    // blocks held by a request before the step
    auto have_of = [&](int32_t r) { return (int32_t)(((int64_t)held[r] + bs - 1) >> a.block_log); };

    if (tid < kTabWalkers) {
        const int32_t gtid = blockIdx.x * kTabWalkers + tid, gthreads = gridDim.x * kTabWalkers;
        for (int32_t r = gtid; r <= a.requests; r += gthreads) a.q_start[r] = tok[r];
        // admitted requests' shared blocks: a warp a request walks the segments of its path upwards
        if (a.node) {
            for (int32_t r = warp * gridDim.x + blockIdx.x; r < a.requests; r += gridDim.x * (kTabWalkers / 32)) {
                if (a.node[r] < 0) continue;
                int32_t cur = tab_row(a, r, false).up, top = held[r] >> a.block_log, last = INT_MAX;
                int32_t *row = a.table + (int64_t)r * a.table_width;
                while (cur >= 0 && top > 0) {
                    const int4 seg = a.map[cur];
                    // a map of pp_chunk_map only goes down, to a segment that begins at 0
                    bool bad = seg.x >= a.n_chunks || seg.y < 0 || seg.z < 0 || seg.z >= seg.w || seg.z >= last;
                    if (!bad) {
                        for (int32_t j = seg.z + lane; j < min(seg.w, top); j += 32) {
                            const int64_t id = (int64_t)seg.y + (j - seg.z);
                            if (id >= a.blocks) bad = true;
                            row[j] = id < a.blocks ? (int32_t)id : -1;
                        }
                    }
                    if (__any_sync(~0u, bad)) {
                        if (lane == 0) kv_bounds(a.status);
                        break;
                    }
                    top = min(top, seg.z);
                    last = seg.z;
                    cur = seg.x;
                }
            }
        }
        // new blocks
        for (int64_t x = gtid; x < fresh_blocks; x += gthreads) {
            const int32_t i = (int32_t)x, r = tab_find(nbk, a.requests, i);
            int32_t id = i < spare ? a.free_blocks[head + i] : -1;
            if (id >= a.blocks || (id < 0 && i < spare)) { kv_bounds(a.status); id = -1; }
            a.table[(int64_t)r * a.table_width + have_of(r) + (i - nbk[r])] = id;
        }
        return;
    }

    // tokens; a running request's last partly filled block is the only old entry read
    constexpr int kRun = kTabRun;
    const int64_t runs = ((int64_t)a.max_tokens + kRun - 1) / kRun;
    const int64_t step = (int64_t)gridDim.x * (kTabThreads - kTabWalkers);
    for (int64_t x = (int64_t)blockIdx.x * (kTabThreads - kTabWalkers) + tid - kTabWalkers; x < runs; x += step) {
        const int32_t i0 = (int32_t)(kRun * x), n = min(kRun, a.max_tokens - i0);
        int64_t slot[kRun];
        int32_t pos[kRun];
        int32_t r = i0 < tokens ? tab_find(tok, a.requests, i0) : 0, block = -1, id = -1;
#pragma unroll
        for (int y = 0; y < kRun; ++y) {
            const int32_t i = i0 + y;
            slot[y] = -1;
            pos[y] = 0;
            if (i >= tokens || y >= n) continue;
            if (i >= tok[r + 1]) {                      // the next request with new tokens
                do ++r;
                while (i >= tok[r + 1]);
                block = -1;
            }
            pos[y] = held[r] + (i - tok[r]);
            const int32_t j = pos[y] >> a.block_log;
            if (j != block) {
                block = j;
                const int32_t have = have_of(r);
                if (j < have) {
                    id = a.table[(int64_t)r * a.table_width + j];
                    if (id < 0 || id >= a.blocks) kv_bounds(a.status);
                } else {
                    const int64_t k = (int64_t)nbk[r] + (j - have);
                    id = k < spare ? a.free_blocks[head + k] : -1;
                }
            }
            if (id >= 0 && id < a.blocks) slot[y] = ((int64_t)id << a.block_log) + (pos[y] & (bs - 1));
        }
        if (n == kRun && a.wide) {
#pragma unroll
            for (int y = 0; y < kRun; y += 2)
                *reinterpret_cast<longlong2 *>(a.slot + i0 + y) = make_longlong2(slot[y], slot[y + 1]);
#pragma unroll
            for (int y = 0; y < kRun; y += 4)
                *reinterpret_cast<int4 *>(a.position + i0 + y) = make_int4(pos[y], pos[y + 1], pos[y + 2], pos[y + 3]);
        } else {
#pragma unroll
            for (int y = 0; y < kRun; ++y)
                if (y < n) {
                    a.slot[i0 + y] = slot[y];
                    a.position[i0 + y] = pos[y];
                }
        }
    }
}

// ---------------------------------------------------------------------------
// Write of new rows: 16 bytes of K and of V a thread and step, a CTA some whole
// tokens.  Bound by memory: 30,011 tokens of 4 heads of 128 (123 MB) 18.4 us,
// 6.7 TB/s; 64 tokens 4 us, a launch.
// ---------------------------------------------------------------------------
struct WriteArgs {
    int32_t tokens, per_token, per_head, tokens_per_cta;     // vectors per token and per head
    const uint4 *k, *v;
    int64_t k_token, k_head, v_token, v_head;                // strides in vectors
    const int64_t *slot;
    uint4 *kc, *vc;
    int64_t block_stride, token_stride, head_stride;
    int64_t slots;
    int32_t block_log;
    int32_t *status;
};

constexpr int kWriteThreads = 256;

__global__ void __launch_bounds__(kWriteThreads) k_kv_write(WriteArgs a)
{
    const int32_t t0 = blockIdx.x * a.tokens_per_cta;
    const int32_t count = min(a.tokens_per_cta, a.tokens - t0) * a.per_token;
    for (int32_t l = threadIdx.x; l < count; l += kWriteThreads) {
        const int32_t t = t0 + l / a.per_token, x = l % a.per_token;
        const int32_t h = x / a.per_head, d = x % a.per_head;
        const int64_t slot = a.slot[t];
        if (slot < 0) continue;
        if (slot >= a.slots) {
            kv_bounds(a.status);
            continue;
        }
        const int64_t dst = (slot >> a.block_log) * a.block_stride +
                            (slot & ((1 << a.block_log) - 1)) * a.token_stride + h * a.head_stride + d;
        const uint4 kv = a.k[t * a.k_token + h * a.k_head + d], vv = a.v[t * a.v_token + h * a.v_head + d];
        a.kc[dst] = kv;
        a.vc[dst] = vv;
    }
}

// bytes between two rows of 16-bit elements that a 16-byte copy can start at
static bool stride_ok(int64_t s) { return s > 0 && s % 8 == 0 && s < (int64_t)1 << 38; }
static bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// Whether rows of `dim` elements at sums of d * stride (0 <= d < extent) share an
// element.  Where each stride passes all that lies within the smaller ones, as in every
// order of dimensions with any padding, they do not.  Other layouts are searched: for
// each difference along two dimensions the nearest ones of the third, the longest.
struct Extent {
    int64_t stride, count;
};
static bool rows_overlap(int64_t dim, std::initializer_list<Extent> all)
{
    Extent e[3] = {{0, 1}, {0, 1}, {0, 1}};
    int n = 0;
    for (const Extent &x : all)
        if (x.count > 1) e[n++] = x;
    std::sort(e, e + n, [](const Extent &x, const Extent &y) { return x.stride < y.stride; });
    __int128 span = dim;
    bool nested = true;
    for (int i = 0; i < n; ++i) {
        nested = nested && e[i].stride >= span;
        span += (__int128)(e[i].count - 1) * e[i].stride;
    }
    if (nested) return false;
    std::sort(e, e + n, [](const Extent &x, const Extent &y) { return x.count > y.count; });
    for (int64_t x = 0; x < e[1].count; ++x)
        for (int64_t y = x ? 1 - e[2].count : 0; y < e[2].count; ++y) {
            const int64_t at = x * e[1].stride + y * e[2].stride;
            const int64_t down = (at >= 0 ? at : at - e[0].stride + 1) / e[0].stride;
            for (int64_t z = down; z <= down + 1; ++z) {
                if (x == 0 && y == 0 && z == 0) continue;
                if (std::abs(z) < e[0].count && std::abs(at - z * e[0].stride) < dim) return true;
            }
        }
    return false;
}

static pp_status check_device(const pp_kv *kv)
{
    int dev = 0;
    PP_CUDA(cudaGetDevice(&dev));
    if (dev != kv->device) return fail(PP_EINVAL, "the cache's device must be the current device");
    return PP_OK;
}

pp_status launch_attend(pp_kv *kv, const AttendArgs &a, cudaStream_t st);
pp_status prepare_attend();            // kernel attributes on the current device

}  // namespace pp

using namespace pp;

extern "C" pp_status pp_chunk_map(int32_t n, const int32_t *parent, const int32_t *weight, const uint8_t *resident,
                                  int32_t blocks_per_slot, int32_t *map, int32_t *blocks)
{
    if (n < 0) return fail(PP_EINVAL, "n must be >= 0");
    if (!blocks || (n > 0 && (!parent || !weight || !resident || !map))) return fail(PP_EINVAL, "null pointer");
    if (blocks_per_slot < 1 || blocks_per_slot > kKvMaxBlocks)
        return fail(PP_EINVAL, "blocks_per_slot must be between 1 and 2^30");
    try {
        return chunk_map(n, parent, weight, resident, blocks_per_slot, map, blocks);
    } catch (const std::exception &) {
        return fail(PP_ENOMEM, "host allocation failed");
    }
}

extern "C" pp_status pp_kv_create(int32_t blocks, int32_t block_size, int32_t kv_heads, int32_t head_dim,
                                  int32_t dtype, int64_t block_stride, int64_t token_stride, int64_t head_stride,
                                  void *stream, pp_kv **out)
{
    if (!out) return fail(PP_EINVAL, "out is null");
    *out = nullptr;
    if (blocks < 1 || blocks > kKvMaxBlocks) return fail(PP_EINVAL, "blocks must be between 1 and 2^30");
    if (block_size < 8 || block_size > kKvMaxBlock || (block_size & (block_size - 1)))
        return fail(PP_EINVAL, "block_size must be a power of two from 8 to 512");
    if (kv_heads < 1 || kv_heads > 65535) return fail(PP_EINVAL, "kv_heads must be between 1 and 65535");
    if (head_dim < 8 || head_dim > kKvMaxDim || head_dim % 8)
        return fail(PP_EINVAL, "head_dim must be a multiple of 8 from 8 to 128");
    if (dtype != PP_KV_BF16 && dtype != PP_KV_F16) return fail(PP_EINVAL, "unknown dtype");
    if (block_stride == 0 && token_stride == 0 && head_stride == 0) {
        head_stride = head_dim;
        token_stride = (int64_t)kv_heads * head_dim;
        block_stride = token_stride * block_size;
    }
    if (!stride_ok(block_stride) || !stride_ok(token_stride) || !stride_ok(head_stride))
        return fail(PP_EINVAL, "strides must be positive multiples of 8 elements below 2^38");
    if (token_stride < head_dim || head_stride < head_dim || block_stride < head_dim)
        return fail(PP_EINVAL, "strides must be at least head_dim: rows would overlap");
    if (rows_overlap(head_dim, {{block_stride, blocks}, {token_stride, block_size}, {head_stride, kv_heads}}))
        return fail(PP_EINVAL, "rows of the cache would overlap with these strides");
    pp_kv *kv = new (std::nothrow) pp_kv();
    if (!kv) return fail(PP_ENOMEM, "host allocation failed");
    kv->blocks = blocks;
    kv->block_size = block_size;
    while ((1 << kv->block_log) < block_size) kv->block_log++;
    kv->heads = kv_heads;
    kv->dim = head_dim;
    kv->dtype = dtype;
    kv->block_stride = block_stride;
    kv->token_stride = token_stride;
    kv->head_stride = head_stride;
    auto device_part = [&]() -> pp_status {
        PP_CUDA(cudaGetDevice(&kv->device));
        PP_CUDA(cudaDeviceGetAttribute(&kv->sm_count, cudaDevAttrMultiProcessorCount, kv->device));
        PP_CUDA(cudaMalloc(&kv->d_status, sizeof(int32_t)));
        PP_CUDA(cudaMemsetAsync(kv->d_status, 0, sizeof(int32_t), (cudaStream_t)stream));
        PP_CUDA(cudaFuncSetAttribute(k_block_tables, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                     (int)(sizeof(int32_t) * (3 * (size_t)kKvMaxRequests + 2))));
        pp_status s = prepare_attend();
        if (s != PP_OK) return s;
        // two pieces a CTA, one CTA an SM
        const size_t slots = 2 * (size_t)kv->sm_count;
        PP_CUDA(cudaMalloc(&kv->d_piece, slots * kPieceRows * kKvMaxDim * sizeof(float)));
        PP_CUDA(cudaMalloc(&kv->d_piece_stat, slots * kPieceRows * 2 * sizeof(float)));
        const size_t count_bytes = 4 * slots * sizeof(int32_t);
        PP_CUDA(cudaMalloc(&kv->d_count, count_bytes));
        PP_CUDA(cudaMemsetAsync(kv->d_count, 0, count_bytes, (cudaStream_t)stream));
        PP_CUDA(cudaStreamSynchronize((cudaStream_t)stream));
        return PP_OK;
    };
    const pp_status s = device_part();
    if (s != PP_OK) {
        pp_kv_destroy(kv);
        return s;
    }
    *out = kv;
    return PP_OK;
}

extern "C" pp_status pp_kv_destroy(pp_kv *kv)
{
    if (!kv) return PP_OK;
    if (kv->d_status) {
        int cur = 0;
        cudaGetDevice(&cur);
        cudaSetDevice(kv->device);
        cudaFree(kv->d_status);
        cudaFree(kv->d_piece);
        cudaFree(kv->d_piece_stat);
        cudaFree(kv->d_count);
        cudaSetDevice(cur);
    }
    delete kv;
    return PP_OK;
}

extern "C" pp_status pp_kv_sync(pp_kv *kv, void *stream)
{
    if (!kv) return fail(PP_EINVAL, "null cache handle");
    // on `stream` itself: the legacy stream would wait for other work, and clear the word after later
    // calls on streams that do not wait for it.  A launch that gave up has no arrivals left to clear:
    // its CTAs still leave their pieces, and the joins put their counters back to 0.
    const cudaStream_t st = (cudaStream_t)stream;
    int32_t v = 0;
    PP_CUDA(cudaMemcpyAsync(&v, kv->d_status, sizeof(v), cudaMemcpyDeviceToHost, st));
    PP_CUDA(cudaStreamSynchronize(st));
    if (v == PP_OK) return PP_OK;
    PP_CUDA(cudaMemsetAsync(kv->d_status, 0, sizeof(int32_t), st));
    PP_CUDA(cudaStreamSynchronize(st));
    if (v == PP_ETIMEOUT) return fail(PP_ETIMEOUT, "a bounded device wait ran out");
    if (v == PP_EBOUNDS)
        return fail(PP_EBOUNDS, "device bounds check failed (a length, block, slot, chunk or token count)");
    return fail(PP_ECUDA, "unknown device status " + std::to_string(v));
}

extern "C" pp_status pp_block_tables(pp_kv *kv, int32_t requests, const int32_t *length, const int32_t *cached,
                                     const int32_t *node, int32_t n_chunks, const int32_t *chunk_map,
                                     int32_t free_count, const int32_t *free_blocks, const int32_t *free_head,
                                     int32_t *free_head_out, int32_t table_width, int32_t *block_table,
                                     int32_t max_tokens, int64_t *slot_map, int32_t *position, int32_t *q_start,
                                     void *stream)
{
    if (!kv) return fail(PP_EINVAL, "null cache handle");
    if (requests < 0 || requests > kKvMaxRequests) return fail(PP_EINVAL, "requests must be between 0 and 16384");
    if (table_width < 1 || max_tokens < 0 || free_count < 0 || n_chunks < 0)
        return fail(PP_EINVAL, "table_width must be >= 1, max_tokens, free_count and n_chunks >= 0");
    if (!q_start || !free_head || !free_head_out) return fail(PP_EINVAL, "null pointer");
    if (requests > 0 && (!length || !cached || !block_table)) return fail(PP_EINVAL, "null pointer");
    if (max_tokens > 0 && (!slot_map || !position)) return fail(PP_EINVAL, "null slot_map or position");
    if (free_count > 0 && !free_blocks) return fail(PP_EINVAL, "null free_blocks");
    if (node && n_chunks > 0 && !chunk_map) return fail(PP_EINVAL, "node is given without chunk_map");
    if (free_head == free_head_out) return fail(PP_EINVAL, "free_head and free_head_out must be different words");
    if (node && !aligned16(chunk_map)) return fail(PP_EINVAL, "chunk_map must be aligned to 16 bytes");
    pp_status s = check_device(kv);
    if (s != PP_OK) return s;
    TablesArgs a = {requests, n_chunks, free_count, table_width, max_tokens, kv->blocks, kv->block_log,
                    length, cached, node, reinterpret_cast<const int4 *>(chunk_map), free_blocks, free_head,
                    free_head_out, block_table, position, q_start, slot_map, kv->d_status,
                    aligned16(slot_map) && aligned16(position)};
    // a CTA for every kTabPass tokens (one pass of its warps) or 8 table rows (a warp's walk each), as many as
    // there are SMs at most
    const int64_t want = std::max<int64_t>(((int64_t)max_tokens + kTabPass - 1) / kTabPass, (requests + 7) / 8);
    const int grid = (int)std::min<int64_t>(std::max<int64_t>(want, 1), kv->sm_count);
    const size_t smem = sizeof(int32_t) * (3 * (size_t)requests + 2);
    k_block_tables<<<grid, kTabThreads, smem, (cudaStream_t)stream>>>(a);
    PP_CUDA(cudaGetLastError());
    return PP_OK;
}

extern "C" pp_status pp_kv_write(pp_kv *kv, int32_t tokens, const void *k, int64_t k_token_stride,
                                 int64_t k_head_stride, const void *v, int64_t v_token_stride, int64_t v_head_stride,
                                 const int64_t *slot_map, void *k_cache, void *v_cache, void *stream)
{
    if (!kv) return fail(PP_EINVAL, "null cache handle");
    if (tokens < 0 || tokens > 1 << 30) return fail(PP_EINVAL, "tokens must be between 0 and 2^30");
    if (tokens == 0) return PP_OK;
    if (!k || !v || !slot_map || !k_cache || !v_cache) return fail(PP_EINVAL, "null pointer");
    if (!aligned16(k) || !aligned16(v) || !aligned16(k_cache) || !aligned16(v_cache))
        return fail(PP_EINVAL, "k, v and the caches must be aligned to 16 bytes");
    if (!stride_ok(k_token_stride) || !stride_ok(k_head_stride) || !stride_ok(v_token_stride) ||
        !stride_ok(v_head_stride))
        return fail(PP_EINVAL, "strides must be positive multiples of 8 elements below 2^38");
    pp_status s = check_device(kv);
    if (s != PP_OK) return s;
    WriteArgs a = {};
    a.tokens = tokens;
    a.per_head = kv->dim / 8;
    a.per_token = kv->heads * a.per_head;
    a.tokens_per_cta = std::max(1, 4 * kWriteThreads / a.per_token);
    a.k = static_cast<const uint4 *>(k);
    a.v = static_cast<const uint4 *>(v);
    a.k_token = k_token_stride / 8;
    a.k_head = k_head_stride / 8;
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
    a.status = kv->d_status;
    const int grid = (tokens - 1) / a.tokens_per_cta + 1;
    k_kv_write<<<grid, kWriteThreads, 0, (cudaStream_t)stream>>>(a);
    PP_CUDA(cudaGetLastError());
    return PP_OK;
}

extern "C" pp_status pp_paged_attention(pp_kv *kv, int32_t requests, int32_t tokens, int32_t q_heads, const void *q,
                                        int64_t q_token_stride, int64_t q_head_stride, const void *k_cache,
                                        const void *v_cache, int32_t table_width, const int32_t *block_table,
                                        const int32_t *q_start, const int32_t *length, int32_t max_q, int32_t window,
                                        float scale, void *out, int64_t out_token_stride, int64_t out_head_stride,
                                        float *lse, void *stream)
{
    if (!kv) return fail(PP_EINVAL, "null cache handle");
    if (requests < 0 || requests > kKvMaxRequests) return fail(PP_EINVAL, "requests must be between 0 and 16384");
    if (tokens < 0 || max_q < 0 || window < 0 || table_width < 1)
        return fail(PP_EINVAL, "tokens, max_q and window must be >= 0, table_width >= 1");
    if (q_heads < 1 || q_heads % kv->heads || q_heads > 1 << 20)
        return fail(PP_EINVAL, "q_heads must be a positive multiple of kv_heads, at most 2^20");
    if ((int64_t)tokens * (q_heads / kv->heads) > 1 << 30)
        return fail(PP_EINVAL, "tokens * q_heads / kv_heads must be at most 2^30");
    if (!(scale > 0) || scale > 1e30f) return fail(PP_EINVAL, "scale must be positive and finite");
    if (requests == 0 || tokens == 0) return PP_OK;
    if (!q || !k_cache || !v_cache || !block_table || !q_start || !length || !out)
        return fail(PP_EINVAL, "null pointer");
    if (!aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(out))
        return fail(PP_EINVAL, "q, out and the caches must be aligned to 16 bytes");
    if (!stride_ok(q_token_stride) || !stride_ok(q_head_stride) || !stride_ok(out_token_stride) ||
        !stride_ok(out_head_stride))
        return fail(PP_EINVAL, "strides must be positive multiples of 8 elements below 2^38");
    if (rows_overlap(kv->dim, {{out_token_stride, tokens}, {out_head_stride, q_heads}}))
        return fail(PP_EINVAL, "rows of out would overlap with these strides");
    pp_status s = check_device(kv);
    if (s != PP_OK) return s;
    const AttendArgs a = {requests, tokens, q_heads, q_heads / kv->heads, q, q_token_stride, q_head_stride, k_cache,
                          v_cache, block_table, table_width, q_start, length, max_q, window, scale, out,
                          out_token_stride, out_head_stride, lse};
    return launch_attend(kv, a, (cudaStream_t)stream);
}
