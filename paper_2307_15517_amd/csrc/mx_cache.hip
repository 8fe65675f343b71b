// Paged key/value cache: block tables and slot maps from request lengths, and the append of new keys and values.
#include "mx_cache.h"

namespace mx {
namespace {

// ---- mx_cache_plan --------------------------------------------------------------------------------------
// have = ceil(ctx / page), want = ceil((ctx + new) / page), need = want - have; the pages of request b start at the sum of the
// needs before it, its tokens at the sum of the new tokens before it.  Integers only, a few hundred kilobytes at most: bound by
// the latency of one launch and, with prompts, of the searches that a thread makes for its tokens, one after another.  Every
// workgroup scans all requests for itself into LDS (two sums per request), so that nothing is exchanged between workgroups and one
// launch does it; then it takes its share of the requests (a wave each: the new entries of the row) and of the tokens (a thread
// each: its request by binary search in LDS).  4 requests 3.4 us in the kernel, 5.6 a call; 700 requests, 10 percent with prompts of
// up to 1024 tokens, 7.4 a call: of the 1.6 us more than 4 requests take 0.1 are the scan, 0.2 the rows, 1.3 the 32740 tokens.
struct PlanArgs {
    const int32_t* ctx;
    const int32_t* fresh;
    const int32_t* free_pages;
    int64_t n_free;
    int32_t* table;
    int64_t width, tokens;
    int32_t* q_start;
    int32_t* kv_len;
    int32_t* slots;
    int32_t* positions;
    int32_t* counts;
    int32_t requests, page_log2;
};

constexpr int kPlanThreads = 256;

__device__ __forceinline__ int64_t wave_scan(int64_t v) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int64_t o = __shfl_up(v, d, 64);
        v += lane >= d ? o : 0;
    }
    return v;
}

// RUN: neighbouring requests a thread takes of the scan, whose lengths it asks for together
template <int RUN>
__global__ __launch_bounds__(kPlanThreads) void cache_plan_kernel(PlanArgs a) {
    extern __shared__ int32_t plan_lds[];
    int32_t* start = plan_lds;                        // [requests + 1]: first packed token of a request
    int32_t* at = plan_lds + a.requests + 1;          // [requests]: its first page in free_pages; -1: refused
    __shared__ int64_t part[2][kPlanThreads / 64];
    __shared__ int64_t served[2];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int page = 1 << a.page_log2;
    auto length = [](int32_t v) { return (int64_t)(v > 0 ? v : 0); };
    auto pages_of = [&](int64_t tokens) { return (tokens + page - 1) >> a.page_log2; };

    if (tid < 2) served[tid] = 0;
    int64_t page_sum = 0, token_sum = 0, taken = 0, refused = 0;
    for (int base = 0; base < a.requests; base += kPlanThreads * RUN) {
        const int b0 = base + tid * RUN;
        int64_t n[RUN], need[RUN], c[RUN], sum_need = 0, sum_n = 0;
        bool wide[RUN];
#pragma unroll
        for (int i = 0; i < RUN; ++i) {
            const int b = min(b0 + i, a.requests - 1);
            c[i] = length(a.ctx[b]);
            n[i] = length(a.fresh[b]);
        }
#pragma unroll
        for (int i = 0; i < RUN; ++i) {
            if (b0 + i >= a.requests) c[i] = n[i] = 0;
            const int64_t want = pages_of(c[i] + n[i]);
            wide[i] = want > a.width;
            need[i] = wide[i] ? 0 : want - pages_of(c[i]);
            sum_need += need[i];
            sum_n += n[i];
        }
        const int64_t up = wave_scan(sum_need), ut = wave_scan(sum_n);
        __syncthreads();                              // the tile before has read part
        if (lane == 63) { part[0][wave] = up; part[1][wave] = ut; }
        __syncthreads();
        int64_t p = page_sum + up - sum_need, t = token_sum + ut - sum_n;
#pragma unroll
        for (int w = 0; w < kPlanThreads / 64; ++w) {
            if (w < wave) { p += part[0][w]; t += part[1][w]; }
            page_sum += part[0][w];
            token_sum += part[1][w];
        }
#pragma unroll
        for (int i = 0; i < RUN; ++i) {
            p += need[i];
            t += n[i];
            if (b0 + i >= a.requests) break;
            const bool no = wide[i] || (need[i] > 0 && p > a.n_free);
            start[b0 + i + 1] = (int32_t)(t < INT32_MAX ? t : INT32_MAX);
            at[b0 + i] = no ? -1 : need[i] > 0 ? (int32_t)(p - need[i]) : 0;     // served: p <= n_free < 2^31
            taken += no ? 0 : need[i];
            refused += no;
        }
    }
    if (tid == 0) start[0] = 0;
    if (blockIdx.x == 0 && a.counts != nullptr) {
        const int64_t s0 = wave_scan(taken), s1 = wave_scan(refused);
        if (lane == 63) {                             // integer sums: the order does not matter
            atomicAdd((unsigned long long*)&served[0], (unsigned long long)s0);
            atomicAdd((unsigned long long*)&served[1], (unsigned long long)s1);
        }
    }
    __syncthreads();
    if (blockIdx.x == 0 && a.counts != nullptr && tid < 2) a.counts[tid] = (int32_t)served[tid];
    if (blockIdx.x == 0 && tid == 0) a.q_start[0] = 0;

    for (int b = blockIdx.x * (kPlanThreads / 64) + wave; b < a.requests; b += gridDim.x * (kPlanThreads / 64)) {
        const int64_t c = length(a.ctx[b]), total = c + length(a.fresh[b]);
        const int first = at[b];
        if (lane == 0) {
            a.q_start[b + 1] = start[b + 1];
            a.kv_len[b] = first < 0 ? 0 : (int32_t)(total < INT32_MAX ? total : INT32_MAX);
        }
        if (first < 0) continue;
        const int64_t have = pages_of(c), want = pages_of(total);
        for (int64_t j = have + lane; j < want; j += 64) a.table[b * a.width + j] = a.free_pages[first + (j - have)];
    }

    const int64_t step = (int64_t)gridDim.x * kPlanThreads;
    for (int64_t t = (int64_t)blockIdx.x * kPlanThreads + tid; t < a.tokens; t += step) {
        int lo = 0, hi = a.requests;                  // the last b with start[b] <= t; requests when t is past them all
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (start[mid + 1] <= t) lo = mid + 1;
            else hi = mid;
        }
        int32_t slot = -1, position = -1;
        if (lo < a.requests && at[lo] >= 0) {
            const int64_t c = length(a.ctx[lo]), pos = c + (t - start[lo]), have = pages_of(c);
            const int64_t j = pos >> a.page_log2;
            const int32_t entry = j < have ? a.table[lo * a.width + j] : a.free_pages[at[lo] + (j - have)];
            position = (int32_t)(pos < INT32_MAX ? pos : INT32_MAX);
            if (entry >= 0 && entry <= INT32_MAX >> a.page_log2) slot = (int32_t)(((uint32_t)entry << a.page_log2) + (uint32_t)(pos & (page - 1)));
        }
        a.slots[t] = slot;
        if (a.positions != nullptr) a.positions[t] = position;
    }
}

// ---- mx_cache_append ------------------------------------------------------------------------------------
// Every element is read once and written once: bound by memory, by latency at the few tokens of a decode step.  A lane takes
// eight elements of a row (BLOCK/8 neighbouring lanes a block, whose largest magnitude they exchange), both tensors in one
// launch.  The MXInt arithmetic is mx_quantize's, on the bits: E = floor(log2 max|x|) clamped, q = round(x 2^(6 - E)).
// 1999 tokens x 8 heads x 128, fp32 into MXInt: 5.8 us for 20.6 MB, 3.6 TB/s; 8 tokens x 32 heads 2.5 us in the kernel, 5.4 a call.
struct AppendArgs {
    const void* x[2];          // k, v
    void* data[2];
    uint8_t* exps[2];
    const int32_t* slots;
    int64_t ld[2];
    int64_t pages;
    uint32_t octets;           // tokens * heads * dim/8
    int32_t heads, row_octets; // dim/8
    int32_t page_log2, bias, emax, rounding;
};

template <int BLOCK, int TYPE, bool VEC>
__global__ __launch_bounds__(256) void cache_append_kernel(AppendArgs a) {
    constexpr int LPB = BLOCK == 0 ? 1 : BLOCK / 8;
    const int which = blockIdx.y;
    const uint32_t o = blockIdx.x * 256 + threadIdx.x;
    const bool live = o < a.octets;
    const uint32_t row = o / a.row_octets, c8 = o - row * a.row_octets, token = row / a.heads, head = row - token * a.heads;
    int32_t slot = -1;
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (live) {
        slot = a.slots[token];
        load8<TYPE, VEC>(a.x[which], token * a.ld[which] + (int64_t)(row - token * a.heads) * a.row_octets * 8 + c8 * 8, v);
    }
    const bool keep = slot >= 0 && (slot >> a.page_log2) < a.pages;      // the lanes of a block share their token
    const int64_t dst = (((int64_t)(slot >> a.page_log2) * a.heads + head) << a.page_log2) + (slot & ((1 << a.page_log2) - 1));
    const int64_t octet = dst * a.row_octets + c8;
    if constexpr (BLOCK == 0) {
        if (keep)
            static_cast<uint4*>(a.data[which])[octet] =
                make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
    } else {
        uint32_t am = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) am = max(am, __float_as_uint(v[i]) & 0x7fffffffu);
        am = max(am, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)am, 0xB1, 0xF, 0xF, true));               // lane ^ 1
        if constexpr (LPB == 4) am = max(am, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)am, 0x4E, 0xF, 0xF, true));   // ^ 2
        const int ef = (int)(am >> 23);
        const int E = min(max(ef == 0 ? -127 : ef - 127, -a.bias), a.emax);
        uint32_t w[2] = {0, 0};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float s = __builtin_ldexpf(v[i], 6 - E);
            const float r = __builtin_fminf(__builtin_fmaxf(a.rounding == MX_RNE ? __builtin_rintf(s) : __builtin_truncf(s), -127.f), 127.f);
            w[i >> 2] |= ((uint32_t)(int)r & 255u) << (8 * (i & 3));
        }
        if (keep) {
            static_cast<uint2*>(a.data[which])[octet] = make_uint2(w[0], w[1]);
            if ((threadIdx.x & (LPB - 1)) == 0) a.exps[which][octet / LPB] = (uint8_t)(E + a.bias);
        }
    }
}

template <int BLOCK, int TYPE, bool VEC>
mx_status launch_append(const AppendArgs& a, hipStream_t stream) {
    const dim3 grid((unsigned)ceil_div(a.octets, 256), 2);
    cache_append_kernel<BLOCK, TYPE, VEC><<<grid, 256, 0, stream>>>(a);
    MX_HIP_LAUNCH_CHECK();
    return MX_OK;
}

template <int BLOCK>
mx_status append_block(const AppendArgs& a, int32_t type, bool vec, hipStream_t s) {
    if (type == MX_F32) return vec ? launch_append<BLOCK, MX_F32, true>(a, s) : launch_append<BLOCK, MX_F32, false>(a, s);
    return vec ? launch_append<BLOCK, MX_BF16, true>(a, s) : launch_append<BLOCK, MX_BF16, false>(a, s);
}

}  // namespace
}  // namespace mx

using namespace mx;

extern "C" size_t mx_cache_data_bytes(mx_cache c) {
    if (cache_status(c) != MX_OK) return 0;
    return (size_t)c.pages * c.heads * c.page * c.dim * (c.f.block == 0 ? 2 : 1);
}

extern "C" size_t mx_cache_exps_bytes(mx_cache c) {
    if (cache_status(c) != MX_OK || c.f.block == 0) return 0;
    return (size_t)c.pages * c.heads * c.page * (c.dim / c.f.block);
}

extern "C" mx_status mx_cache_plan(const int32_t* ctx_len, const int32_t* new_len, int64_t requests, int32_t page,
                                   const int32_t* free_pages, int64_t n_free, int32_t* table, int64_t width, int64_t tokens,
                                   int32_t* q_start, int32_t* kv_len, int32_t* slots, int32_t* positions, int32_t* counts,
                                   void* stream) {
    if (requests < 0 || n_free < 0 || width < 0 || tokens < 0 || page < 1 || q_start == nullptr) return MX_ERR_BAD_ARG;
    if (requests > 0 && (ctx_len == nullptr || new_len == nullptr || kv_len == nullptr)) return MX_ERR_BAD_ARG;
    if ((requests > 0 && width > 0 && table == nullptr) || (n_free > 0 && free_pages == nullptr) || (tokens > 0 && slots == nullptr))
        return MX_ERR_BAD_ARG;
    for (const void* p : {(const void*)ctx_len, (const void*)new_len, (const void*)free_pages, (const void*)table,
                          (const void*)q_start, (const void*)kv_len, (const void*)slots, (const void*)positions, (const void*)counts})
        if (!aligned(p, 4)) return MX_ERR_BAD_ARG;
    if (!cache_page_ok(page) || requests > kCacheMaxRequests || n_free > INT32_MAX || width > INT32_MAX || tokens > INT32_MAX)
        return MX_ERR_UNSUPPORTED;
    PlanArgs a{ctx_len, new_len, free_pages, n_free, table, width, tokens, q_start, kv_len, slots, positions, counts,
               (int32_t)requests, log2_of(page)};
    const int lds = (int)(2 * requests + 1) * 4;
    static std::atomic<uint64_t> raised{0};
    if (lds > 60 * 1024 && !allow_dynamic_lds((const void*)cache_plan_kernel<4>, (2 * kCacheMaxRequests + 1) * 4, raised))
        return MX_ERR_DEVICE;
    // a workgroup per 1024 tokens or 16 requests: the scan, which all repeat, costs as much as that
    int64_t groups = max(ceil_div(tokens, 1024), ceil_div(requests, 16));
    groups = groups < 1 ? 1 : groups > 512 ? 512 : groups;
    // one round of the scan with a request a thread is enough (60 prompts 6.2 us, four a thread 6.6), or several with four (700
    // requests 7.6 us, one a thread 8.5; 4000 requests of one token 9.8 and 17)
    if (requests <= kPlanThreads) cache_plan_kernel<1><<<(unsigned)groups, kPlanThreads, lds, (hipStream_t)stream>>>(a);
    else cache_plan_kernel<4><<<(unsigned)groups, kPlanThreads, lds, (hipStream_t)stream>>>(a);
    MX_HIP_LAUNCH_CHECK();
    return MX_OK;
}

extern "C" mx_status mx_cache_append(const void* k, const void* v, int32_t type, int64_t tokens, int64_t ldk, int64_t ldv,
                                     mx_cache c, void* k_data, uint8_t* k_exps, void* v_data, uint8_t* v_exps,
                                     const int32_t* slots, void* stream) {
    if (type != MX_F32 && type != MX_BF16) return MX_ERR_BAD_ARG;
    const mx_status st = cache_status(c);
    if (st == MX_ERR_BAD_ARG || tokens < 0) return MX_ERR_BAD_ARG;
    const int64_t row = (int64_t)c.heads * c.dim;
    if (tokens > 0) {
        if (k == nullptr || v == nullptr || k_data == nullptr || v_data == nullptr || slots == nullptr) return MX_ERR_BAD_ARG;
        if (c.f.block != 0 && (k_exps == nullptr || v_exps == nullptr)) return MX_ERR_BAD_ARG;
        if (ldk < row || ldv < row || !aligned(k, type_bytes(type)) || !aligned(v, type_bytes(type)) || !aligned(k_data, 16) ||
            !aligned(v_data, 16) || !aligned(slots, 4))
            return MX_ERR_BAD_ARG;
    }
    if (st != MX_OK) return st;
    const int per = 16 / type_bytes(type);
    const bool vec = aligned(k, 16) && aligned(v, 16) && ldk % per == 0 && ldv % per == 0;
    AppendArgs a{};
    a.data[0] = k_data; a.data[1] = v_data;
    a.exps[0] = k_exps; a.exps[1] = v_exps;
    a.ld[0] = ldk; a.ld[1] = ldv;
    a.pages = c.pages;
    a.heads = c.heads;
    a.row_octets = c.dim / 8;
    a.page_log2 = log2_of(c.page);
    a.bias = exponent_bias(c);
    a.emax = a.bias + 1;
    a.rounding = c.f.rounding;
    const int64_t slice = (((int64_t)1 << 31) - 256) / (row / 8);         // tokens whose octets a launch can number
    for (int64_t t = 0; t < tokens; t += slice) {
        const int64_t n = tokens - t < slice ? tokens - t : slice;
        a.octets = (uint32_t)(n * (row / 8));
        a.x[0] = (const char*)k + t * ldk * type_bytes(type);
        a.x[1] = (const char*)v + t * ldv * type_bytes(type);
        a.slots = slots + t;
        const hipStream_t s = (hipStream_t)stream;
        const mx_status r = c.f.block == 0 ? append_block<0>(a, type, vec, s)
                            : c.f.block == 16 ? append_block<16>(a, type, vec, s) : append_block<32>(a, type, vec, s);
        if (r != MX_OK) return r;
    }
    return MX_OK;
}
