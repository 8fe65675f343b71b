// Trees of drafted tokens over the paged cache: masks of ancestors and positions, and the accepted rows moved into place.
#include "mx_cache.h"

namespace mx {
namespace {

// ---- mx_tree_plan ---------------------------------------------------------------------------------------
// mask(i) = {i} or mask(parent(i)), depth(i) = depth(parent(i)) + 1.  Integers only, twelve bytes a node and word: bound by the
// latency of one launch and of the chain of parents (4 requests of 5 nodes 2.1 us in the kernel, 200 of up to 180 nodes, three words,
// 3.1; 5 with the call).  Deep trees of several words are the slow ones: 0.23 us a step of a chain, 240 us for 1024 nodes in a row.
struct TreeArgs {
    const int32_t* parents;
    const int32_t* q_start;
    const int32_t* ctx;
    uint64_t* masks;
    int32_t* positions;
    int64_t tokens;
    int32_t requests, words;
};

constexpr int kTreeThreads = 256;

__device__ __forceinline__ int tokens_of(const int32_t* q_start, int64_t tokens, int b, int64_t* first) {
    const int64_t lo = q_start[b], hi = q_start[b + 1];
    const int64_t t0 = lo < 0 ? 0 : lo > tokens ? tokens : lo, t1 = hi > tokens ? tokens : hi;
    *first = t0;
    return (int)(t1 > t0 ? t1 - t0 : 0);
}

__device__ __forceinline__ void put_position(const TreeArgs& a, int64_t t, int64_t ctx, int depth) {
    if (a.positions == nullptr) return;
    const int64_t p = (ctx > 0 ? ctx : 0) + depth;
    a.positions[t] = (int32_t)(p < INT32_MAX ? p : INT32_MAX);
}

// What belongs to no tree: a mask without bits, no position.
__device__ __forceinline__ void put_nothing(const TreeArgs& a, int64_t t) {
    for (int w = 0; w < a.words; ++w) a.masks[t * a.words + w] = 0;
    if (a.positions != nullptr) a.positions[t] = -1;
}

__device__ __forceinline__ void tree_padding(const TreeArgs& a) {
    const int64_t first = a.requests ? a.q_start[0] : 0, end = a.requests ? a.q_start[a.requests] : 0;
    const int64_t lead = first < 0 ? 0 : first > a.tokens ? a.tokens : first, tail = end < lead ? lead : end > a.tokens ? a.tokens : end;
    const int64_t n = lead + a.tokens - tail;
    for (int64_t t = (int64_t)blockIdx.x * kTreeThreads + threadIdx.x; t < n; t += (int64_t)gridDim.x * kTreeThreads)
        put_nothing(a, t < lead ? t : tail + t - lead);
}

// One word a node: a wave a request, a lane a node.  A lane holds its nearest ancestors' mask and the next one above them, and takes over
// that one's, which doubles their number: six exchanges.
__global__ __launch_bounds__(kTreeThreads) void tree_word_kernel(TreeArgs a) {
    const int lane = threadIdx.x & 63, b = blockIdx.x * (kTreeThreads / 64) + (threadIdx.x >> 6);
    if (b < a.requests) {
        int64_t t0;
        const int n = tokens_of(a.q_start, a.tokens, b, &t0);
        const int64_t ctx = a.ctx[b];
        int up = lane < n ? a.parents[t0 + lane] : -1;
        up = up >= 0 && up < lane ? up : -1;
        uint32_t lo = lane < 32 ? 1u << lane : 0, hi = lane < 32 ? 0 : 1u << (lane - 32);
        int depth = up >= 0;
#pragma unroll
        for (int s = 0; s < 6; ++s) {
            const int from = up < 0 ? 0 : up;
            const uint32_t l = __shfl(lo, from), h = __shfl(hi, from);
            const int d = __shfl(depth, from), u = __shfl(up, from);
            if (up >= 0) {
                lo |= l;
                hi |= h;
                depth += d;
                up = u;
            }
        }
        if (lane < n) {
            a.masks[t0 + lane] = (uint64_t)hi << 32 | lo;
            put_position(a, t0 + lane, ctx, depth);
        }
        for (int64_t i = 64 + lane; i < n; i += 64) put_nothing(a, t0 + i);
    }
    tree_padding(a);
}

// Several words: a workgroup a request, its parents in LDS, a thread a node that follows them up.  They have falling numbers, so the words
// are finished one after another.
__global__ __launch_bounds__(kTreeThreads) void tree_words_kernel(TreeArgs a) {
    __shared__ int16_t parent[MX_TREE_MAX_NODES];
    const int b = blockIdx.x;
    if (b < a.requests) {
        int64_t t0;
        const int n = tokens_of(a.q_start, a.tokens, b, &t0), nodes = min(n, 64 * a.words);
        const int64_t ctx = a.ctx[b];
        for (int i = threadIdx.x; i < nodes; i += kTreeThreads) {
            const int p = a.parents[t0 + i];
            parent[i] = (int16_t)(p >= 0 && p < i ? p : -1);
        }
        __syncthreads();
        for (int64_t i = threadIdx.x; i < n; i += kTreeThreads) {
            if (i >= nodes) {
                put_nothing(a, t0 + i);
                continue;
            }
            uint64_t* to = a.masks + (t0 + i) * a.words;
            uint64_t bits = 0;
            int depth = -1, word = a.words - 1;
            for (int node = (int)i; node >= 0; node = parent[node]) {
                for (; word > node >> 6; --word) {
                    to[word] = bits;
                    bits = 0;
                }
                bits |= 1ull << (node & 63);
                ++depth;
            }
            for (; word >= 0; --word) {
                to[word] = bits;
                bits = 0;
            }
            put_position(a, t0 + i, ctx, depth);
        }
    }
    tree_padding(a);
}

// ---- mx_cache_move --------------------------------------------------------------------------------------
// Row path[i] of a request's new tokens goes to place i, path[i] >= i and rising, so a run of rows may be written once all of it has been
// read: what later runs read lies past it.  A wave takes a request, a head and one of the two tensors, 16 bytes a lane, as many rows
// at once as it holds (four of 128 bfloat16 elements, eight of 128 MXInt ones).  A few kilobytes a request: bound by the chain of
// loads lengths, path, table, row, each of which waits for the one before (one request 3.4 us in the kernel, 96 requests of 8 heads 5.5).
struct MoveArgs {
    uint8_t* data[2];
    uint8_t* exps[2];
    const int32_t* table;
    const int32_t* ctx;
    const int32_t* path;
    const int32_t* kept;
    int64_t width, path_width;
    int64_t max_keys;          // width * page
    uint32_t pages;
    int32_t requests, heads;
    int32_t pieces, row_exps;  // of a row: 16-byte pieces, exponent bytes (no more than pieces)
    int32_t page_log2;
};

__global__ __launch_bounds__(256) void cache_move_kernel(MoveArgs a) {
    const int lane = threadIdx.x & 63;
    const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int which = (int)(unit & 1);
    const int64_t rest = unit >> 1;
    const int b = (int)(rest / a.heads), h = (int)(rest - (int64_t)b * a.heads);
    if (b >= a.requests) return;
    const int64_t ctx = a.ctx[b];
    const int64_t kept = min((int64_t)a.kept[b], a.path_width);
    const int rows = 64 / a.pieces, mine = lane / a.pieces, piece = lane - mine * a.pieces;
    // the row of the pool that holds position p of the request; -1: none
    auto row_of = [&](int64_t p) -> int64_t {
        if (p < 0 || p >= a.max_keys) return -1;
        const uint32_t page = (uint32_t)a.table[b * a.width + (p >> a.page_log2)];
        if (page >= a.pages) return -1;
        return (((int64_t)page * a.heads + h) << a.page_log2) + (p & ((1 << a.page_log2) - 1));
    };
    for (int64_t i0 = 0; i0 < kept; i0 += rows) {
        const int64_t i = i0 + mine;
        int64_t from = -1, to = -1;
        if (mine < rows && i < kept && ctx >= 0) {
            const int64_t node = a.path[b * a.path_width + i];
            if (node >= 0 && node != i) {
                from = row_of(ctx + node);
                to = row_of(ctx + i);
            }
        }
        const bool live = from >= 0 && to >= 0;
        uint4 x = make_uint4(0, 0, 0, 0);
        uint8_t e = 0;
        if (live) {
            x = reinterpret_cast<const uint4*>(a.data[which])[from * a.pieces + piece];
            if (piece < a.row_exps) e = a.exps[which][from * a.row_exps + piece];
        }
        // every row of the run has been read before any is written (a wave's loads answer for all its lanes)
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_s_waitcnt(0);
        __builtin_amdgcn_sched_barrier(0);
        if (live) {
            reinterpret_cast<uint4*>(a.data[which])[to * a.pieces + piece] = x;
            if (piece < a.row_exps) a.exps[which][to * a.row_exps + piece] = e;
        }
        // and written before the next run is read
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_s_waitcnt(0);
        __builtin_amdgcn_sched_barrier(0);
    }
}

}  // namespace
}  // namespace mx

using namespace mx;

extern "C" mx_status mx_tree_plan(const int32_t* parents, const int32_t* q_start, const int32_t* ctx_len, int64_t requests, int64_t tokens,
                                  int32_t words, uint64_t* masks, int32_t* positions, void* stream) {
    if (requests < 0 || tokens < 0 || words < 1) return MX_ERR_BAD_ARG;
    if (tokens > 0 && masks == nullptr) return MX_ERR_BAD_ARG;
    if (tokens > 0 && requests > 0 && (parents == nullptr || q_start == nullptr || ctx_len == nullptr)) return MX_ERR_BAD_ARG;
    for (const void* p : {(const void*)parents, (const void*)q_start, (const void*)ctx_len, (const void*)positions})
        if (!aligned(p, 4)) return MX_ERR_BAD_ARG;
    if (!aligned(masks, 8)) return MX_ERR_BAD_ARG;
    if (requests > kCacheMaxRequests || tokens > INT32_MAX || words > MX_TREE_MAX_NODES / 64) return MX_ERR_UNSUPPORTED;
    if (tokens == 0) return MX_OK;
    TreeArgs a{parents, q_start, ctx_len, masks, positions, tokens, (int32_t)requests, words};
    const int64_t groups = words == 1 ? ceil_div(requests, kTreeThreads / 64) : requests;
    const unsigned grid = (unsigned)(groups > 0 ? groups : 1);
    if (words == 1) tree_word_kernel<<<grid, kTreeThreads, 0, (hipStream_t)stream>>>(a);
    else tree_words_kernel<<<grid, kTreeThreads, 0, (hipStream_t)stream>>>(a);
    MX_HIP_LAUNCH_CHECK();
    return MX_OK;
}

extern "C" mx_status mx_cache_move(mx_cache c, void* k_data, uint8_t* k_exps, void* v_data, uint8_t* v_exps, const int32_t* table,
                                   int64_t width, const int32_t* ctx_len, const int32_t* path, int64_t path_width, const int32_t* kept,
                                   int64_t requests, void* stream) {
    const mx_status st = cache_status(c);
    if (st == MX_ERR_BAD_ARG || requests < 0 || width < 0 || path_width < 0) return MX_ERR_BAD_ARG;
    if (requests > 0) {
        if (k_data == nullptr || v_data == nullptr || ctx_len == nullptr || kept == nullptr || (width > 0 && table == nullptr) ||
            (path_width > 0 && path == nullptr))
            return MX_ERR_BAD_ARG;
        if (c.f.block != 0 && (k_exps == nullptr || v_exps == nullptr)) return MX_ERR_BAD_ARG;
        if (!aligned(k_data, 16) || !aligned(v_data, 16)) return MX_ERR_BAD_ARG;
        for (const int32_t* p : {table, ctx_len, path, kept})
            if (!aligned(p, 4)) return MX_ERR_BAD_ARG;
    }
    if (st != MX_OK) return st;
    if (requests > kCacheMaxRequests || width > INT32_MAX || path_width > INT32_MAX) return MX_ERR_UNSUPPORTED;
    if (requests == 0 || width == 0 || path_width == 0) return MX_OK;
    MoveArgs a{};
    a.data[0] = (uint8_t*)k_data; a.data[1] = (uint8_t*)v_data;
    a.exps[0] = k_exps; a.exps[1] = v_exps;
    a.table = table; a.ctx = ctx_len; a.path = path; a.kept = kept;
    a.width = width; a.path_width = path_width;
    a.max_keys = width * c.page;
    a.pages = (uint32_t)c.pages;
    a.requests = (int32_t)requests; a.heads = c.heads;
    a.pieces = c.dim * (c.f.block == 0 ? 2 : 1) / 16;
    a.row_exps = c.f.block == 0 ? 0 : c.dim / c.f.block;
    a.page_log2 = log2_of(c.page);
    const int64_t groups = ceil_div(requests * c.heads * 2, 4);
    if (groups >= 1 << 24) return MX_ERR_UNSUPPORTED;       // the threads of a launch are counted in 32 bits
    cache_move_kernel<<<(unsigned)groups, 256, 0, (hipStream_t)stream>>>(a);
    MX_HIP_LAUNCH_CHECK();
    return MX_OK;
}
