// Attention of new tokens over the paged key/value cache, grouped heads: causal, or (compiled with MX_CACHE_TREE=1, a unit of its own) of
// trees of drafted tokens, where masks say which of the new tokens a token sees.
#include <type_traits>

#include "mx_cache.h"

namespace mx {
namespace {

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));

#ifndef MX_CACHE_TREE
#define MX_CACHE_TREE 0
#endif
constexpr bool kTree = MX_CACHE_TREE;

constexpr int kCounterBytes = 65536;

struct CacheAttnArgs {
    const void* q;
    void* out;
    int64_t ldq, ldo;
    const uint8_t* k;
    const uint8_t* v;
    const uint8_t* k_exps;
    const uint8_t* v_exps;
    const int32_t* table;
    int64_t width;
    const int32_t* q_start;
    const int32_t* kv_len;
    float* part_o;             // [part row][split][dim], unnormalised; part rows: of decode() [unit][part_rows], of chunk() [head][packed row]
    float2* part_ml;           // [part row][split]: row maximum (exp2 domain), row sum
    uint32_t* counters;        // of the workgroups of a unit that have stored their part; zero between calls
    int64_t tokens;
    int64_t max_keys;          // width * page
    uint32_t pages;
    int32_t requests, heads, group, heads_q, dim;
    int32_t page_log2;
    int32_t exp_shift;         // an exponent byte e stands for 2^(e - exp_shift) per mantissa unit
    int32_t splits;            // of this launch, at most
    int32_t run;               // chunk(): tiles of keys that a split is given
    int32_t least, most;       // this launch takes the requests that have least .. most rows (token, head of a group)
    int32_t part_rows;         // decode(): part rows per unit; a request with more rows is not split
    int32_t tiles;             // chunk(): row tiles of all requests, at most
    int32_t sorted;            // the longest requests go first
    int32_t join;              // the workgroup of a unit that comes last joins its parts; else a launch of its own does
    int32_t vec_q, vec_o;      // rows of q / out allow 16-byte (bfloat16 out: 8-byte) accesses
    float c;                   // |scale| * log2(e)
    uint32_t flip;             // sign bit of the scale: carried by q
#if MX_CACHE_TREE                // (the causal kernels take two of these: with more fields scalar registers spill, 3 to 8 % of chunks over MXInt)
    const uint32_t* masks;     // [tokens][mask_words], bit j: new token j of the request is seen
    int32_t mask_words;        // 32-bit words of a token's mask
    int32_t slots;             // cache_tree_kernel: its workgroups; tiles: units, at most
    int32_t small_rows, small_run, least_run;   // rows that a small tile may have; its runs in eighths of a large one's, and of one of 32 rows
#endif
};

// One request as a workgroup sees it, every length bounded by what the arrays hold.
struct Request {
    int t0, n, len;            // first packed token, new tokens, cached tokens
};
__device__ __forceinline__ Request request_of(const CacheAttnArgs& a, int b) {
    Request r;
    const int64_t lo = a.q_start[b], hi = a.q_start[b + 1], len = a.kv_len[b];
    const int64_t t0 = lo < 0 ? 0 : lo > a.tokens ? a.tokens : lo, t1 = hi > a.tokens ? a.tokens : hi;
    r.t0 = (int)t0;
    r.n = (int)(t1 > t0 ? t1 - t0 : 0);
    r.len = (int)(len < 0 ? 0 : len > a.max_keys ? a.max_keys : len);
    return r;
}

#if MX_CACHE_TREE
// Which of 32 keys from new token `at` on (negative: cached ones) packed token `t` sees, a bit each.
__device__ __forceinline__ uint32_t seen_from(const CacheAttnArgs& a, int64_t t, int at) {
    const uint32_t* mask = a.masks + t * a.mask_words;
    const int w = at >> 5;
    const uint32_t lo = mask[min(max(w, 0), a.mask_words - 1)], hi = mask[min(max(w + 1, 0), a.mask_words - 1)];
    return __builtin_amdgcn_alignbit(w + 1 < 0 ? ~0u : w + 1 < a.mask_words ? hi : 0u, w < 0 ? ~0u : w < a.mask_words ? lo : 0u, at & 31);
}
#else
__device__ __forceinline__ uint32_t seen_from(const CacheAttnArgs&, int64_t, int) { return ~0u; }
#endif

// Zeros for the tokens before the first request's and after the last one's.
template <int TYPE>
__device__ __forceinline__ void fill_padding(const CacheAttnArgs& a) {
    const int64_t first = a.q_start[0], end = a.q_start[a.requests];
    const int64_t lead = first < 0 ? 0 : first > a.tokens ? a.tokens : first, tail = end < lead ? lead : end > a.tokens ? a.tokens : end;
    const int64_t n = lead + a.tokens - tail, row = (int64_t)a.heads_q * a.dim;
    for (int64_t t = blockIdx.x; t < n; t += gridDim.x) {
        const int64_t at = (t < lead ? t : tail + t - lead) * a.ldo;
        for (int64_t d = threadIdx.x; d < row; d += blockDim.x) {
            if constexpr (TYPE == MX_F32) static_cast<float*>(a.out)[at + d] = 0.f;
            else static_cast<uint16_t*>(a.out)[at + d] = 0;
        }
    }
}

// N consecutive results (4 or 8) to element `at` of out.
template <int TYPE, int N>
__device__ __forceinline__ void store_out(const CacheAttnArgs& a, int64_t at, const float (&x)[N]) {
    if constexpr (TYPE == MX_F32) {
        float* p = static_cast<float*>(a.out) + at;
        if (a.vec_o) {
#pragma unroll
            for (int i = 0; i < N; i += 4) *reinterpret_cast<float4*>(p + i) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) p[i] = x[i];
        }
    } else {
        uint16_t* p = static_cast<uint16_t*>(a.out) + at;
        if (a.vec_o) {
#pragma unroll
            for (int i = 0; i < N; i += 4) *reinterpret_cast<uint2*>(p + i) = make_uint2(pack_bf16(x[i], x[i + 1]), pack_bf16(x[i + 2], x[i + 3]));
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) p[i] = (uint16_t)pack_bf16(x[i], 0.f);
        }
    }
}

// The pages of one request as a wave walks over its keys: 64 entries of the table row at a time, one per lane, so that a step
// finds its pages without a load (a scalar load among LDS reads makes every wait for one of them a wait for all).
struct PageWindow {
    const int32_t* row_table;
    int base, last, id;        // id: of page `base` + lane, no further than `last`

    // The first window is asked for at once, before the request's length is known (what lies past its pages is not looked at).
    __device__ __forceinline__ PageWindow(const CacheAttnArgs& a, int b) : row_table(a.table + (int64_t)b * a.width), base(0), last(0), id(0) {
        if (a.width > 0) id = row_table[min((int)(threadIdx.x & 63), (int)a.width - 1)];
    }
    __device__ __forceinline__ void set_length(const CacheAttnArgs& a, int len) {
        last = (len - 1) >> a.page_log2;
        asm volatile("" : "+v"(id));               // awaited here, not in the loop
    }
    // The row of the pool that holds key `key` of the request (and those after it in its run of sixteen): `key` is below its
    // length and the same for all lanes.  A page index outside the pool reads as page 0.
    __device__ __forceinline__ int64_t row(const CacheAttnArgs& a, int h, int key) {
        const int page = key >> a.page_log2;
        if ((unsigned)(page - base) >= 64) {
            base = page;
            id = row_table[min(page + (int)(threadIdx.x & 63), last)];
            asm volatile("" : "+v"(id));       // awaited here, once in 64 pages, and not wherever it might just have been loaded
        }
        uint32_t at = (uint32_t)__builtin_amdgcn_readlane(id, page - base);
        at = at < a.pages ? at : 0;
        return (((int64_t)at * a.heads + h) << a.page_log2) + (key & ((1 << a.page_log2) - 1));
    }
};

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// The leading bfloat16 pieces (8 bits, cut) of two floats, which keep the rest
__device__ __forceinline__ uint32_t cut_piece(float& a, float& b) {
    const uint32_t w = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
    a -= __uint_as_float(__float_as_uint(a) & 0xffff0000u);
    b -= __uint_as_float(__float_as_uint(b) & 0xffff0000u);
    return w;
}

// The nearest bfloat16 numbers of two floats, which keep the rest (not for floats that would round to infinity)
__device__ __forceinline__ uint32_t near_piece(float& a, float& b) {
    const uint32_t w = pack_bf16(a, b);
    a -= __uint_as_float(w << 16);
    b -= __uint_as_float(w & 0xffff0000u);
    return w;
}

// A float as one, two or three bfloat16 pieces.  One is the nearest bfloat16 number, which of a bfloat16 activation is all of it.
// Three are all 24 bits: each is cut, and what the last one gets fits it.  Two are rounded each, which leaves 2^-16 of the float at
// most (2^-15 if the first were cut) in as many instructions.
template <int P>
__device__ __forceinline__ void pieces_of(float a, float b, uint32_t (&w)[P]) {
#pragma unroll
    for (int p = 0; p < P; ++p) {
        w[p] = p == P - 1 ? pack_bf16(a, b) : P == 2 ? near_piece(a, b) : cut_piece(a, b);
    }
}

// q of one row as the pieces that a lane holds: N runs of eight elements, run n from element at(n) on (zeros past the head
// dimension).  The loads of all runs go out together: one branch on the alignment around them, none inside.
template <int TYPE, int QP, int N, typename At>
__device__ __forceinline__ void load_q(const CacheAttnArgs& a, int64_t row, At at, v4u (&qf)[QP][N]) {
    float v[N][8];
    if (a.vec_q) {
#pragma unroll
        for (int n = 0; n < N; ++n) load8<TYPE, true>(a.q, row + (at(n) < a.dim ? at(n) : 0), v[n]);
    } else {
#pragma unroll
        for (int n = 0; n < N; ++n) load8<TYPE, false>(a.q, row + (at(n) < a.dim ? at(n) : 0), v[n]);
    }
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const uint32_t keep = at(n) < a.dim ? 0xffffffffu : 0u;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            uint32_t w[QP];
            pieces_of<QP>(__uint_as_float(__float_as_uint(v[n][2 * e]) ^ a.flip), __uint_as_float(__float_as_uint(v[n][2 * e + 1]) ^ a.flip), w);
#pragma unroll
            for (int p = 0; p < QP; ++p) qf[p][n][e] = w[p] & keep;
        }
    }
}

// The largest of three, or two; __builtin_fmaxf spends an instruction on every operand whose origin the compiler cannot see.
__device__ __forceinline__ float max_of(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
__device__ __forceinline__ float max_of(float a, float b) {
    float r;
    asm("v_max_f32 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}
__device__ __forceinline__ float max_across_32(float v) {
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return max_of(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float max_across_16_32(float v) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = max_of(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return max_of(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float sum_across_16_32(float v) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// 2^n as a float, n of any size (below the smallest subnormal: 0)
__device__ __forceinline__ float power2(int n) { return __builtin_ldexpf(1.f, n); }

// ---- few rows: decoding ---------------------------------------------------------------------------------
// A workgroup takes sixteen rows (token, head of the group) of one request and key/value head, and a run of its keys; its four
// waves take blocks of 32 keys in turn and join at the end.  S^T = K Q^T puts a row in a lane's column and four consecutive
// keys of either half block in its registers, which is the right operand of O^T = V^T P^T as it stands; K and V go from memory
// to registers without LDS, each lane a run of one key's row, and V's rows are transposed in registers.
// DT: head dimension padded to 64 or 128 (in registers only).  BLOCK: 0 bfloat16, else MXInt.
// Pieces: K and V are bfloat16 numbers as they are (an MXInt element has 7 bits and a sign).  bfloat16 q is one piece, float q
// three, and the probabilities are three, so that nothing but the result is rounded to fewer than 24 bits.  The matrix instructions
// are idle most of the time here: the third piece takes 1 % (32 ragged sequences, bfloat16: 74.6 us with two, 74.9 to 75.8).
// Bound by the reads of K and V: one sequence of 100003 keys (8 heads x 5, bfloat16) 77 us = 5.3 TB/s of the 5.6 that a bare read
// reaches; 32 of up to 8191 (8 heads x 4, MXInt 32) 75 us = 4.3 TB/s, the vector arithmetic of the MXInt conversion taking as long as
// the reads and the last requests ending alone.  Short calls by the chain of loads (lengths, table, K and V), about 0.9 us a step, and
// the meeting of the splits: 1936 keys of 32 heads 12.5 us, one sequence of 61 keys 6.2.
template <int TYPE>
constexpr int kQueryPieces = TYPE == MX_F32 ? 3 : 1;

// Parts of a row's result pass between workgroups that may sit behind different L2 caches: they are written through to and read
// from the level that all compute units share (device scope), so that no cache has to be written back or invalidated as a whole.
constexpr int kDeviceScope = 0x10;
constexpr int kMaxSplits = 64;
constexpr int kFewRows = 16;           // (token, head of a group) of a request that decode() takes at once

// The parts of `rows` rows (16 or, with 32 lanes a row, eight at a time), `splits` each, of a unit whose workgroups have all
// stored theirs: o = sum_s o_s 2^(m_s - m) / sum_s l_s 2^(m_s - m).  Called by the 256 threads of the workgroup that came last; the
// order of the additions is given by the sizes, not by the order of arrival.  32 lanes take four elements each of a row; the eight
// groups of 32 share a row's splits when there are fewer rows than groups.
template <typename Store>
__device__ __forceinline__ void join_parts(const CacheAttnArgs& a, int64_t part_row, int rows, float4 (*lds)[32], Store store) {
    const int group = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int share = 8;                                                        // groups per row
    while (share > 1 && rows * share > 8) share >>= 1;
    const BufRsrc ro = make_rsrc(a.part_o + part_row * a.splits * a.dim, (uint32_t)(rows * a.splits * a.dim * 4));
    const BufRsrc rm = make_rsrc(a.part_ml + part_row * a.splits, (uint32_t)(rows * a.splits * 8));
    const int d = 4 * lane < a.dim ? 4 * lane : 0;
    for (int r0 = 0; r0 < rows; r0 += 8 / share) {
        const int row = min(r0 + group / share, rows - 1), first = group & (share - 1);
        float m[2], l[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int s = lane + 32 * x;
            const auto t = __builtin_amdgcn_raw_buffer_load_b64(rm, (row * a.splits + min(s, a.splits - 1)) * 8, 0, kDeviceScope);
            m[x] = s < a.splits ? __uint_as_float(t[0]) : -__builtin_inff();
            l[x] = __uint_as_float(t[1]);
        }
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
        float top = __builtin_fmaxf(m[0], m[1]);
#pragma unroll
        for (int e = 1; e < 32; e *= 2) top = __builtin_fmaxf(top, __shfl_xor(top, e, 32));
        const float f0 = m[0] == -__builtin_inff() ? 0.f : exp2_of(m[0] - top), f1 = m[1] == -__builtin_inff() ? 0.f : exp2_of(m[1] - top);
        float sum = (m[0] == -__builtin_inff() ? 0.f : l[0] * f0) + (m[1] == -__builtin_inff() ? 0.f : l[1] * f1);
#pragma unroll
        for (int e = 1; e < 32; e *= 2) sum += __shfl_xor(sum, e, 32);
        for (int s0 = first; s0 < a.splits; s0 += 8 * share) {
            v4u y[8];
#pragma unroll
            for (int u = 0; u < 8; ++u)
                y[u] = __builtin_bit_cast(v4u, __builtin_amdgcn_raw_buffer_load_b128(ro, ((row * a.splits + min(s0 + u * share, a.splits - 1)) * a.dim + d) * 4, 0, kDeviceScope));
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int s = s0 + u * share;
                const float w0 = __shfl(s < 32 ? f0 : f1, s & 31, 32);
                if (s < a.splits) {
                    x.x += __uint_as_float(y[u][0]) * w0; x.y += __uint_as_float(y[u][1]) * w0;
                    x.z += __uint_as_float(y[u][2]) * w0; x.w += __uint_as_float(y[u][3]) * w0;
                }
            }
        }
        if (share > 1) {
            __syncthreads();
            lds[group][lane] = x;
            __syncthreads();
            if (first == 0)
                for (int g = 1; g < share; ++g) {
                    const float4 y = lds[group + g][lane];
                    x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
                }
        }
        if (first == 0 && r0 + group / share < rows && 4 * lane < a.dim) {
            const float inv = sum > 0.f ? 1.f / sum : 0.f;
            const float o[4] = {x.x * inv, x.y * inv, x.z * inv, x.w * inv};
            store(row, 4 * lane, o);
        }
    }
}

// Counts this workgroup in after its parts are stored; true in the one that comes last, which also clears the counter.
__device__ __forceinline__ bool came_last(uint32_t* counter, int splits, uint32_t* flag) {
    // this thread's parts have been written through (the wait), then every thread's (the barrier), then the arrival is counted
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if (threadIdx.x == 0) {
        const uint32_t old = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        *flag = old == (uint32_t)(splits - 1);
        if (*flag) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
    return *flag != 0;
}

template <int DT, int BLOCK>
struct KeyBlock {
    static constexpr int KC = DT / 64;                            // MXInt: 16-byte chunks of a key per lane
    static constexpr int VE = DT / 16;                            // elements of a V row per lane
    v4u k[2][BLOCK == 0 ? DT / 32 : KC];
    int ke[2][KC];
    uint32_t v[8][BLOCK == 0 ? VE / 2 : VE / 4];
    int ve[8];
};

// The request that is number n by length (at most 64 of them; equal lengths in their order).
__device__ __forceinline__ int nth_longest(const CacheAttnArgs& a, int n) {
    const int lane = threadIdx.x & 63;
    const int len = lane < a.requests ? a.kv_len[lane] : INT_MIN;
    int rank = 0;
    for (int j = 0; j < a.requests; ++j) {
        const int other = __builtin_amdgcn_readlane(len, j);
        rank += other > len || (other == len && j < lane);
    }
    return __builtin_ctzll(__ballot(rank == n && lane < a.requests));
}

template <int DT>
struct DecodeLds {
    float o[4][16][DT + 4];
    float2 ml[4][16];
    uint32_t flag;
};

template <int TYPE, int DT, int BLOCK>
__device__ __forceinline__ void decode(const CacheAttnArgs& a, int index, DecodeLds<DT>& lds) {
    constexpr int NS = DT / 32, NJ = DT / 16, VE = DT / 16;
    constexpr int EB = BLOCK == 0 ? 2 : 1;
    constexpr int QP = kQueryPieces<TYPE>, P = 3;
    using Block = KeyBlock<DT, BLOCK>;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int n = lane & 15, g = lane >> 4;

    const int split = index % a.splits;
    const int unit = index / a.splits;
    const int h = unit % a.heads;
    int b = unit / a.heads;
    if (a.sorted) b = nth_longest(a, b);
    PageWindow pages(a, b);
    const Request rq = request_of(a, b);
    const int rows = rq.n * a.group;
    if (rows < a.least || rows > a.most) return;
    const int splits = rows <= a.part_rows ? a.splits : 1;
    if (split >= splits) return;
    const int len = rq.len;
    pages.set_length(a, len);
    // this split's run of keys, in whole blocks of 128
    const int per = (((len + 127) >> 7) + splits - 1) / splits;
    const int begin = min(split * per * 128, len), end = min(begin + per * 128, len);
    const int dim = a.dim;

    for (int r0 = 0; r0 < rows; r0 += 16) {
        // q: column n of the score product, elements d(step, g, i); rows past the last repeat it
        const int r = min(r0 + n, rows - 1);
        const int tok = r / a.group, head = h * a.group + (r - tok * a.group);
        const int last = kTree ? len - 1 : len - rq.n + tok;              // the last key this row sees
        v4u qf[QP][NS];
        // keys past the last one any row of this tile sees are left out
        const int first_last = kTree ? len - rq.n - 1 : len - rq.n + r0 / a.group;   // the last key that all its rows see
        const int stop = kTree ? end : min(end, len - rq.n + min(r0 + 15, rows - 1) / a.group + 1);

        float m = -__builtin_inff(), l = 0.f;
        v4f o[NJ];
#pragma unroll
        for (int j = 0; j < NJ; ++j) o[j] = v4f{0.f, 0.f, 0.f, 0.f};

        // The two runs of sixteen keys of a block lie in one page each; a run past the end reads the last one again (masked).
        const int last_run = (len - 1) & ~15;
        auto load = [&](Block& f, int kb) __attribute__((always_inline)) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int64_t row = pages.row(a, h, min(kb + 16 * t, last_run));
                const uint8_t* kp = a.k + row * dim * EB;
                const uint8_t* vp = a.v + row * dim * EB;
                if constexpr (BLOCK == 0) {
#pragma unroll
                    for (int s = 0; s < NS; ++s) {
                        const int d = 32 * s + 8 * g;
                        f.k[t][s] = *reinterpret_cast<const v4u*>(kp + (n * dim + (d < dim ? d : 0)) * 2);
                    }
                } else {
                    const uint8_t* kx = a.k_exps + row * (dim / BLOCK);
#pragma unroll
                    for (int s = 0; s < Block::KC; ++s) {
                        const int d = 64 * s + 16 * g, e = d < dim ? d : 0;
                        f.k[t][s] = *reinterpret_cast<const v4u*>(kp + n * dim + e);
                        f.ke[t][s] = kx[n * (dim / BLOCK) + e / BLOCK];
                    }
                }
                const int d = VE * n < dim ? VE * n : 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint8_t* src = vp + ((4 * g + i) * dim + d) * EB;
                    if constexpr (VE * EB == 16) {
                        const v4u x = *reinterpret_cast<const v4u*>(src);
#pragma unroll
                        for (int w = 0; w < 4; ++w) f.v[4 * t + i][w] = x[w];
                    } else if constexpr (VE * EB == 8) {
                        const v2u x = *reinterpret_cast<const v2u*>(src);
                        f.v[4 * t + i][0] = x[0];
                        f.v[4 * t + i][1] = x[1];
                    } else {
                        f.v[4 * t + i][0] = *reinterpret_cast<const uint32_t*>(src);
                    }
                    if constexpr (BLOCK != 0) f.ve[4 * t + i] = (a.v_exps + row * (dim / BLOCK))[(4 * g + i) * (dim / BLOCK) + d / BLOCK];
                }
            }
        };
        auto compute = [&](Block& f, int kb) __attribute__((always_inline)) {
            v4f s[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                s[t] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int step = 0; step < NS; ++step) {
                    v4u kf;
                    if constexpr (BLOCK == 0) {
                        kf = f.k[t][step];
                    } else {
                        const float sc = power2(f.ke[t][step >> 1] - a.exp_shift);
#pragma unroll
                        for (int w = 0; w < 4; ++w) {
                            int x = (int)f.k[t][step >> 1][2 * (step & 1) + (w >> 1)];
                            asm("" : "+v"(x));        // the bytes are taken apart here, not when they arrive (four registers for one)
                            const float lo = (float)(int8_t)(x >> (16 * (w & 1))) * sc, hi = (float)(int8_t)(x >> (16 * (w & 1) + 8)) * sc;
                            kf[w] = __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
                        }
                    }
#pragma unroll
                    for (int p = QP - 1; p >= 0; --p)
                        s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, kf), __builtin_bit_cast(v8bf, qf[p][step]),
                                                                       s[t], 0, 0, 0);
                    if constexpr (BLOCK != 0) __builtin_amdgcn_sched_barrier(0);   // few converted elements at a time: registers
                }
            }
            if (kb + 31 > min(first_last, stop - 1)) {
                const int seen = min(last, stop - 1) - kb - 4 * g;
                const uint32_t bits = kTree ? seen_from(a, rq.t0 + tok, kb - (len - rq.n)) >> (4 * g) : ~0u;
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        s[t][e] = 16 * t + e <= seen && (!kTree || (bits >> (16 * t + e) & 1)) ? s[t][e] : -__builtin_inff();
                    }
            }
            float top = -__builtin_inff();
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) top = __builtin_fmaxf(top, s[t][e]);
            const float m_new = __builtin_fmaxf(m, max_across_16_32(top) * a.c);
            const float m_use = m_new == -__builtin_inff() ? 0.f : m_new;
            const float alpha = exp2_of(m - m_use);
            m = m_new;
            float pr[8], sum = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                pr[e] = exp2_of(__builtin_fmaf(s[e >> 2][e & 3], a.c, -m_use));
                sum += pr[e];
            }
            l = l * alpha + sum;
#pragma unroll
            for (int j = 0; j < NJ; ++j) o[j] *= alpha;
            v4u pf[P];
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                uint32_t x[P];
                pieces_of<P>(pr[2 * w], pr[2 * w + 1], x);
#pragma unroll
                for (int p = 0; p < P; ++p) pf[p][w] = x[p];
            }
            // rows past the request's end may hold anything, NaN among it: they count as zeros
            const bool whole = kb + 32 <= len;
            float sc[8];
            if constexpr (BLOCK != 0) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const bool in = whole || kb + 16 * (i >> 2) + 4 * g + (i & 3) < len;
                    sc[i] = in ? power2(f.ve[i] - a.exp_shift) : 0.f;
                }
            } else if (!whole) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const bool in = kb + 16 * (i >> 2) + 4 * g + (i & 3) < len;
#pragma unroll
                    for (int w = 0; w < VE / 2; ++w) f.v[i][w] = in ? f.v[i][w] : 0u;
                }
            }
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                v4u vf;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    if constexpr (BLOCK == 0) {
                        vf[w] = __builtin_amdgcn_perm(f.v[2 * w + 1][j >> 1], f.v[2 * w][j >> 1], (j & 1) ? 0x07060302u : 0x05040100u);
                    } else {
                        int x = (int)f.v[2 * w][j >> 2], y = (int)f.v[2 * w + 1][j >> 2];
                        asm("" : "+v"(x), "+v"(y));
                        const float lo = (float)(int8_t)(x >> (8 * (j & 3))) * sc[2 * w];
                        const float hi = (float)(int8_t)(y >> (8 * (j & 3))) * sc[2 * w + 1];
                        vf[w] = __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
                    }
                }
#pragma unroll
                for (int p = P - 1; p >= 0; --p)
                    o[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, vf), __builtin_bit_cast(v8bf, pf[p]), o[j],
                                                                   0, 0, 0);
                if constexpr (BLOCK != 0) __builtin_amdgcn_sched_barrier(0);
            }
        };
        load_q<TYPE, QP, NS>(a, (int64_t)(rq.t0 + tok) * a.ldq + (int64_t)head * dim,
                             [&](int n) { return BLOCK == 0 ? 32 * n + 8 * g : 64 * (n >> 1) + 16 * g + 8 * (n & 1); }, qf);
        // One block in flight per wave: a second one costs a third wave per SIMD (32 ragged sequences 79 us, 84 with it).
        for (int kb = begin + 32 * wave; kb < stop; kb += 128) {
            Block f;
            load(f, kb);
            compute(f, kb);
        }

        // the four waves join: lane (n, g) holds row n, elements VE*(4g + e) + j
        l = sum_across_16_32(l);
        __syncthreads();                                                  // the tile before has been read
        if (g == 0) lds.ml[wave][n] = make_float2(m, l);
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int j = 0; j < NJ; ++j) lds.o[wave][n][VE * (4 * g + e) + j] = o[j][e];
        __syncthreads();
        const int row = threadIdx.x >> 4, part = threadIdx.x & 15;
        if (r0 + row < rows && VE * part < dim) {
            float mm = -__builtin_inff();
#pragma unroll
            for (int w = 0; w < 4; ++w) mm = __builtin_fmaxf(mm, lds.ml[w][row].x);
            float ll = 0.f, acc[VE];
#pragma unroll
            for (int j = 0; j < VE; ++j) acc[j] = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float2 ml = lds.ml[w][row];
                const float f = ml.x == -__builtin_inff() ? 0.f : exp2_of(ml.x - mm);
                ll += ml.y * f;
#pragma unroll
                for (int j = 0; j < VE; ++j) acc[j] += lds.o[w][row][VE * part + j] * f;
            }
            if (splits == 1) {
                const int tk = (r0 + row) / a.group, hd = h * a.group + (r0 + row - tk * a.group);
                const float inv = ll > 0.f ? 1.f / ll : 0.f;
#pragma unroll
                for (int j = 0; j < VE; ++j) acc[j] *= inv;
                store_out<TYPE, VE>(a, (int64_t)(rq.t0 + tk) * a.ldo + (int64_t)hd * dim + VE * part, acc);
            } else {
                const int at = row * splits + split;
                const int64_t rows0 = (int64_t)unit * a.part_rows * splits;
                const BufRsrc ro = make_rsrc(a.part_o + rows0 * dim, (uint32_t)(rows * splits * dim * 4));
                const BufRsrc rm = make_rsrc(a.part_ml + rows0, (uint32_t)(rows * splits * 8));
                if (part == 0) __builtin_amdgcn_raw_buffer_store_b64(v2u{__float_as_uint(mm), __float_as_uint(ll)}, rm, at * 8, 0, kDeviceScope);
#pragma unroll
                for (int j = 0; j < VE; j += 4)
                    __builtin_amdgcn_raw_buffer_store_b128(v4u{__float_as_uint(acc[j]), __float_as_uint(acc[j + 1]), __float_as_uint(acc[j + 2]), __float_as_uint(acc[j + 3])},
                                                           ro, (at * dim + VE * part + j) * 4, 0, kDeviceScope);
            }
        }
    }
    if (splits == 1 || !a.join) return;
    if (!came_last(a.counters + unit, splits, &lds.flag)) return;
    join_parts(a, (int64_t)unit * a.part_rows, rows, reinterpret_cast<float4(*)[32]>(&lds.o[0][0][0]), [&](int row, int d, const float (&x)[4]) {
        const int tk = row / a.group, hd = h * a.group + (row - tk * a.group);
        store_out<TYPE, 4>(a, (int64_t)(rq.t0 + tk) * a.ldo + (int64_t)hd * dim + d, x);
    });
}

template <int TYPE, int DT, int BLOCK>
__global__ __launch_bounds__(256, 2) void cache_decode_kernel(CacheAttnArgs a) {
    __shared__ __attribute__((aligned(16))) DecodeLds<DT> lds;
    decode<TYPE, DT, BLOCK>(a, blockIdx.x, lds);
    fill_padding<TYPE>(a);     // last: its loads would hold up everything else
}

// ---- many rows: chunks and prompts ----------------------------------------------------------------------
// A workgroup takes 128 rows (token, head of the group) of one request and key/value head, a wave 32 of them, q in registers;
// K and V pass through LDS in tiles of 64 keys.  S^T = K Q^T puts a row in a lane's column, so that its maximum and sum take one
// exchange between the lane halves, and hands the probabilities to O^T = V^T P^T in registers; V is transposed by the LDS reads.
//
// Bound by the matrix instructions and, nearly as much, by the vector arithmetic of the softmax, which run under each other only
// where the program has them side by side.  So the work goes in steps of 32 keys, and step u holds three things that do not
// depend on each other: P V of step u-1, the scores of step u+1, and the softmax of step u, whose instructions stand between
// those matrix instructions.  K's stages are therefore 32 keys ahead of V's.
//
// K and V are bfloat16 numbers as they are, so nothing bounds their sizes.  fp32 activations: three bfloat16 pieces of q and of the
// probabilities, all their bits.  bfloat16 activations: q as it is and two pieces of the probabilities, what is left out being 2^-16
// of one, 2^-8 of what the rounding of the result leaves out.  (Three: 648 us for the five prompts below, 526 with two.  One
// half-precision piece: 485, with 11 bits and V scaled to half precision's range by the largest of sixteen keys, which loses small
// values next to large ones, also to those of tokens that a row must not see.)
//
// Measured: five prompts of 1687 .. 4096 tokens (8 heads x 4 of 128, bfloat16) 530 us = 698 TFLOP/s, 1047 with the second piece
// counted; matrix cores busy 57 % and vector ALUs 56 % of the cycles.  300 tokens on 2000 keys (32 heads, fp32: three times the
// matrix instructions, one wave per SIMD) 69 us, of which 8 join the splits; its 96 row tiles, a third of them with 44 of 128 rows,
// are 192 workgroups on 256 compute units.
//
// DT is the head dimension that LDS is laid out for, 64 or 128, DC the one that is computed with: up to 96 of 128 the matrix
// instructions leave the last quarter out (3 prompts of 1000 tokens, 8 heads x 4 of 96: 57.8 us with 128, 50.7 with 96; MXInt
// 68.5 and 61.5).
constexpr int kTileRows = 128, kTileKeys = 64;
constexpr float kLag = 8.f;            // the maximum that probabilities are taken against follows the rows' own within this power of two

// The request that tile number `tile` belongs to, and which of its tiles of rows it is; b < 0: none.  Every wave looks for itself, 64
// requests at a time.
struct Tile {
    int b, index;
    Request rq;
};
__device__ __forceinline__ Tile find_tile(const CacheAttnArgs& a, int tile) {
    const int lane = threadIdx.x & 63;
    int before = 0;
    for (int base = 0; base < a.requests; base += 64) {
        int count = 0;
        Request r{0, 0, 0};
        if (base + lane < a.requests) {
            r = request_of(a, base + lane);
            const int64_t rows = (int64_t)r.n * a.group;
            if (rows >= a.least && rows <= a.most) count = (int)((rows + kTileRows - 1) / kTileRows);
        }
        int upto = count;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int o = __shfl_up(upto, d, 64);
            upto += lane >= d ? o : 0;
        }
        const uint64_t past = __ballot(before + upto > tile);
        if (past != 0) {
            const int at = __builtin_ctzll(past);
            const int index = tile - before - (__builtin_amdgcn_readlane(upto, at) - __builtin_amdgcn_readlane(count, at));
            return Tile{base + at, index, Request{__builtin_amdgcn_readlane(r.t0, at), __builtin_amdgcn_readlane(r.n, at), __builtin_amdgcn_readlane(r.len, at)}};
        }
        before += __builtin_amdgcn_readlane(upto, 63);
    }
    return Tile{-1, 0, Request{0, 0, 0}};
}

// Part row of row r of a request: the rows of a head lie one after another, as the tokens are packed.
__device__ __forceinline__ int64_t part_row_of(const CacheAttnArgs& a, int h, const Request& rq, int r) {
    return (h * a.tokens + rq.t0) * a.group + r;
}

// The keys of the request that some row of the tile sees, and the splits that they are given: as many as there are runs of them.
__device__ __forceinline__ int keys_seen(const CacheAttnArgs& a, const Tile& t) {
    return max(0, t.rq.len - t.rq.n + min(t.index * kTileRows + kTileRows - 1, t.rq.n * a.group - 1) / a.group + 1);
}
__device__ __forceinline__ int splits_of(const CacheAttnArgs& a, int keys) {
    return max(1, min(((keys + kTileKeys - 1) / kTileKeys + a.run - 1) / a.run, a.splits));
}

// LDS tile of keys by DT elements, rows without padding, 16-byte chunks placed so that neither the reads of K (32 keys, one
// chunk each) nor the transposing reads of V (8 keys, 64 bytes each) meet on a bank more often than they must.
template <int DT>
__device__ __forceinline__ int k_place(int key, int chunk) {
    return DT == 128 ? key * 256 + ((chunk ^ (key & 15)) << 4) : key * 128 + ((chunk ^ ((key >> 1) & 7)) << 4);
}
template <int DT>
__device__ __forceinline__ int v_place(int key, int chunk) {
    return DT == 128 ? key * 256 + ((chunk ^ ((key & 7) << 1)) << 4) : key * 128 + ((chunk ^ ((key & 2) << 1)) << 4);
}

typedef float v16f __attribute__((ext_vector_type(16)));
typedef short v4s __attribute__((ext_vector_type(4)));

// 16 bytes per lane from memory straight into LDS: lane L's bytes land at lds_addr + 16 L.  Awaited with s_waitcnt vmcnt.
__device__ __forceinline__ void copy16_to_lds(const uint8_t* uniform_src, uint32_t lane_offset, uint32_t lds_addr) {
    asm volatile(
        "s_mov_b32 m0, %2\n\t"
        "s_nop 0\n\t"
        "global_load_lds_dwordx4 %0, %1\n\t"
        :
        : "v"(lane_offset), "s"(uniform_src), "s"(lds_addr)
        : "memory", "m0");
}

// Four keys (rows of V in LDS) of one column per lane: lane l of sixteen gives the place of row l/4, columns 4(l%4).. and
// receives column l of the four rows.
__device__ __forceinline__ v2u read_transposed(uint32_t lds) {
    const v4s r = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(uintptr_t)lds);
    return __builtin_bit_cast(v2u, r);
}
__device__ __forceinline__ v4u lds_read(uint32_t lds) { return *(__attribute__((address_space(3))) const v4u*)(uintptr_t)lds; }
__device__ __forceinline__ void lds_write(uint32_t lds, v4u x) { *(__attribute__((address_space(3))) v4u*)(uintptr_t)lds = x; }
// The value is computed before this point: an empty volatile statement is ordered with the scheduling fences, and so, through it,
// is the (otherwise freely movable) arithmetic that gives x.
__device__ __forceinline__ void pin(float x) { asm volatile("" ::"v"(x)); }
__device__ __forceinline__ void pin(uint32_t x) { asm volatile("" ::"v"(x)); }
// A register that the compiler may not look into: what is added to it stays in the instructions' offsets instead of becoming
// a register of its own, one for every place in every stage.
__device__ __forceinline__ void opaque(uint32_t& x) { asm("" : "+v"(x)); }

// The arithmetic of one item: row tile `tile` for head h, run number `split` of its keys.  The causal unit finds that run while the first pages
// are on their way (found before, fp32 chunks take 1 % longer); of trees it is `run`.
struct Run {
    int splits, begin, end;
};
template <int TYPE, int DT, int BLOCK, int DC>
__device__ __forceinline__ void chunk_tile(const CacheAttnArgs& a, const Tile& tile, int h, int split, Run run, uint8_t* smem) {
    constexpr int QP = kQueryPieces<TYPE>, P = TYPE == MX_F32 ? 3 : 2;
    constexpr int NK = DC / 16, ND = DC / 32;
    constexpr int EB = BLOCK == 0 ? 2 : 1;
    constexpr int kTensor = kTileKeys * DT * 2;            // LDS: K stage 0, 1, V stage 0, 1
    constexpr int kVBase = 2 * kTensor;
    constexpr int kLoads = 16 * DT * EB / 1024;            // 16-byte loads per lane that bring a run of sixteen keys
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int i = lane & 31, h2 = lane >> 5;

    const int b = tile.b;
    PageWindow pages(a, b);
    const Request rq = tile.rq;
    const int rows = rq.n * a.group, r0 = tile.index * kTileRows;
    const int len = rq.len, dim = a.dim;
#if MX_CACHE_TREE
    const int splits = run.splits, begin = run.begin, stop = run.end;
#else
    // the keys that some row of the tile sees, and this split's run of them in whole tiles
    const int all = keys_seen(a, tile), splits = splits_of(a, all);
    if (split >= splits) return;
    const int per = (((all + kTileKeys - 1) / kTileKeys) + splits - 1) / splits * kTileKeys;
    const int begin = min(split * per, all), stop = min(begin + per, all);
#endif

    // this wave's rows: q is the right operand of the scores, lane (i, h2) row i, elements 16kk + 8h2 ..
    const int r = min(r0 + 32 * wave + i, rows - 1);
    const int tok = r / a.group, head = h * a.group + (r - tok * a.group);
    const int last = min(kTree ? len - 1 : len - rq.n + tok, stop - 1);   // the last key of this split that the row sees
    // the last one all of the wave's see
    const int all_see = min(kTree ? len - rq.n - 1 : len - rq.n + min(r0 + 32 * wave, rows - 1) / a.group, stop - 1);
    v4u qf[QP][NK];
    load_q<TYPE, QP, NK>(a, (int64_t)(rq.t0 + tok) * a.ldq + (int64_t)head * dim, [&](int n) { return 16 * n + 8 * h2; }, qf);

    // ---- staging: a wave brings one run of sixteen keys of a stage, which lies in one page -------------------
    // bfloat16: copies from memory straight to LDS, 1 KiB each, lane L's bytes at 16 L of it, so the placement of the chunks is done
    // by what each lane reads.  MXInt: through registers.
    constexpr int kLaneRows = 1024 / (DT * EB);                           // rows of a load
    constexpr int kRowLanes = 64 / kLaneRows;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)smem;
    const int last_run = (len - 1) & ~15;
    const int rel = lane / kRowLanes;
    const int lane_d = lane % kRowLanes * (16 / EB);                      // what lies past the head dimension reads its start again
    uint32_t k_from[BLOCK == 0 ? kLoads : 1], v_from[BLOCK == 0 ? kLoads : 1];
    const uint32_t from = (rel * dim + (lane_d < dim ? lane_d : 0)) * EB;
    if constexpr (BLOCK == 0) {
#pragma unroll
        for (int u = 0; u < kLoads; ++u) {
            const int row = u * kLaneRows + rel, chunk = lane % kRowLanes;
            const int kc = 8 * ((k_place<DT>(row, chunk) - row * DT * 2) >> 4), vc = 8 * ((v_place<DT>(row, chunk) - row * DT * 2) >> 4);
            k_from[u] = (row * dim + (kc < dim ? kc : 0)) * 2;
            v_from[u] = (row * dim + (vc < dim ? vc : 0)) * 2;
        }
    }
    const uint32_t e_from = BLOCK == 0 ? 0 : rel * (dim / (BLOCK == 0 ? 1 : BLOCK)) + (lane_d < dim ? lane_d : 0) / (BLOCK == 0 ? 1 : BLOCK);
    uint32_t k_to[kLoads][2], v_to[kLoads][2];                            // places of this lane's chunks in a stage
#pragma unroll
    for (int u = 0; u < kLoads; ++u)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int row = 16 * wave + u * kLaneRows + rel, chunk = lane % kRowLanes * (2 / EB) + x;
            k_to[u][x] = lds0 + k_place<DT>(row, chunk);
            v_to[u][x] = lds0 + kVBase + v_place<DT>(row, chunk);
        }
    v4u sk[BLOCK == 0 ? 1 : kLoads], sv[BLOCK == 0 ? 1 : kLoads];
    int ek[kLoads], ev[kLoads];
    pages.set_length(a, len);
    auto row_of = [&](int key) __attribute__((always_inline)) { return pages.row(a, h, max(min(key + 16 * wave, last_run), 0)); };
    // K stage t: keys begin + 64t + 32 ..; V stage t: keys begin + 64t ..
    auto load_k = [&](int slot, int key0) __attribute__((always_inline)) {
        const int64_t row = row_of(key0);
        const uint8_t* src = a.k + row * dim * EB;
#pragma unroll
        for (int u = 0; u < kLoads; ++u) {
            if constexpr (BLOCK == 0) {
                copy16_to_lds(src, k_from[u], lds0 + slot + wave * (16 * DT * 2) + u * 1024);
            } else {
                sk[u] = *reinterpret_cast<const v4u*>(src + u * kLaneRows * dim + from);
                ek[u] = (a.k_exps + row * (dim / BLOCK) + u * kLaneRows * (dim / BLOCK))[e_from];
            }
        }
    };
    auto load_v = [&](int slot, int key0) __attribute__((always_inline)) {
        const int64_t row = row_of(key0);
        const uint8_t* src = a.v + row * dim * EB;
#pragma unroll
        for (int u = 0; u < kLoads; ++u) {
            if constexpr (BLOCK == 0) {
                copy16_to_lds(src, v_from[u], lds0 + kVBase + slot + wave * (16 * DT * 2) + u * 1024);
            } else {
                sv[u] = *reinterpret_cast<const v4u*>(src + u * kLaneRows * dim + from);
                ev[u] = (a.v_exps + row * (dim / BLOCK) + u * kLaneRows * (dim / BLOCK))[e_from];
            }
        }
    };
    auto widen = [&](const v4u& x, float sc, v4u (&y)[2]) __attribute__((always_inline)) {     // sixteen mantissas to bfloat16 numbers
#pragma unroll
        for (int w = 0; w < 8; ++w) {
            int t = (int)x[w >> 1];
            asm("" : "+v"(t));
            const float lo = (float)(int8_t)(t >> (16 * (w & 1))) * sc, hi = (float)(int8_t)(t >> (16 * (w & 1) + 8)) * sc;
            y[w >> 2][w & 3] = __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
        }
    };
    auto put_k = [&](int slot) __attribute__((always_inline)) {
        if constexpr (BLOCK != 0) {
#pragma unroll
            for (int u = 0; u < kLoads; ++u) {
                v4u y[2];
                widen(sk[u], power2(ek[u] - a.exp_shift), y);
                lds_write(k_to[u][0] + slot, y[0]);
                lds_write(k_to[u][1] + slot, y[1]);
            }
        }
    };
    // What lies past the request's end may be anything, NaN among it, and meets probabilities of zero: it becomes zeros
    // (of bfloat16 V in LDS, before the stage is read).  Past the head dimension lies a repetition, which meets zeros of q or gives
    // results that nobody reads.
    auto put_v = [&](int slot, int key0) __attribute__((always_inline)) {
        if constexpr (BLOCK != 0) {
            const bool whole = key0 + 16 * wave + 16 <= len;
#pragma unroll
            for (int u = 0; u < kLoads; ++u) {
                const bool in = whole || key0 + 16 * wave + u * kLaneRows + rel < len;
                v4u y[2];
                widen(in ? sv[u] : v4u{0, 0, 0, 0}, power2((in ? ev[u] : 0) - a.exp_shift), y);
                lds_write(v_to[u][0] + slot, y[0]);
                lds_write(v_to[u][1] + slot, y[1]);
            }
        }
    };

    // places of this lane's reads in a stage, without the multiples of eight keys that the instructions add
    uint32_t k_at[NK], v_at[ND];
#pragma unroll
    for (int kk = 0; kk < NK; ++kk) k_at[kk] = lds0 + k_place<DT>(i, 2 * kk + h2);
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) {
        const int d = 32 * dt + (lane & 16) + 4 * (lane & 3);
        v_at[dt] = lds0 + kVBase + v_place<DT>(4 * h2 + ((lane & 15) >> 2), d >> 3) + (d & 7) * 2;
    }

    float m = -__builtin_inff(), l = 0.f;
    v16f o[ND];
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[dt][e] = 0.f;
    v16f s[2];                                  // scores of an even and an odd step; register e: key 8(e/4) + 4h2 + e%4
    v4u kf[NK], vf[2][ND], pf[2][P];            // vf, pf: two runs of sixteen keys of the step before
#pragma unroll
    for (int x = 0; x < 2; ++x) {
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) vf[x][dt] = v4u{0, 0, 0, 0};
#pragma unroll
        for (int p = 0; p < P; ++p) pf[x][p] = v4u{0, 0, 0, 0};
    }
    auto read_k = [&](int first, int end_, int at) __attribute__((always_inline)) {
#pragma unroll
        for (int kk = first; kk < end_; ++kk) {
            opaque(k_at[kk]);
            kf[kk] = lds_read(k_at[kk] + at);
        }
    };
    auto read_v = [&](int x, int dt, int at) __attribute__((always_inline)) {
        opaque(v_at[dt]);
#pragma unroll
        for (int jj = 0; jj < 2; ++jj) {
            const v2u y = read_transposed(v_at[dt] + (at + (16 * x + 8 * jj) * DT * 2));
            vf[x][dt][2 * jj] = y[0];
            vf[x][dt][2 * jj + 1] = y[1];
        }
    };
    auto score = [&](int n, auto set_c) __attribute__((always_inline)) {              // matrix instruction n of NK * QP
        constexpr int set = decltype(set_c)::value;
        const int kk = n / QP, p = QP - 1 - n % QP;
        v16f zero;
#pragma unroll
        for (int e = 0; e < 16; ++e) zero[e] = 0.f;
        s[set] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, kf[kk]), __builtin_bit_cast(v8bf, qf[p][kk]),
                                                         n == 0 ? zero : s[set], 0, 0, 0);
    };
    auto out = [&](int n) __attribute__((always_inline)) {                            // matrix instruction n of 2 * P * ND
        const int x = n / (P * ND), p = P - 1 - n / ND % P, dt = n % ND;
        o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, vf[x][dt]), __builtin_bit_cast(v8bf, pf[x][p]), o[dt], 0, 0, 0);
    };

    // One step of 32 keys from kb; k_next: place of the next step's keys in LDS, v_this: of this step's values.
    auto step = [&](auto set_c, int kb, auto k_next_c, auto v_this_c) __attribute__((always_inline)) {
        constexpr int set = decltype(set_c)::value, k_next = decltype(k_next_c)::value, v_this = decltype(v_this_c)::value;
        constexpr int NO = 2 * P * ND, NQ = NK * QP;
        float top = -__builtin_inff();
        // P V of the step before, the maximum of this step's scores under it.  The operands of both products share registers: a
        // half of one is read from LDS when a half of the other has been used.
#pragma unroll
        for (int n = 0; n < NO; ++n) {
            out(n);
            __builtin_amdgcn_sched_barrier(0);
            if (n == NO / 2 - 1) read_k(0, NK / 2, k_next);
            if (n == NO - 1) read_k(NK / 2, NK, k_next);
            if (n == 0 && kb + 31 > all_see) {
                const int most = last - kb - 4 * h2;
                const uint32_t bits = kTree ? seen_from(a, rq.t0 + tok, kb - (len - rq.n)) >> (4 * h2) : ~0u;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int x = 8 * (e >> 2) + (e & 3);
                    s[set][e] = x <= most && (!kTree || (bits >> x & 1)) ? s[set][e] : -__builtin_inff();
                }
            }
            if (n == NO / 2) {
                float t[2];
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    t[x] = max_of(s[set][8 * x], s[set][8 * x + 1], s[set][8 * x + 2]);
                    t[x] = max_of(t[x], s[set][8 * x + 3], s[set][8 * x + 4]);
                    t[x] = max_of(t[x], s[set][8 * x + 5], s[set][8 * x + 6]);
                    t[x] = max_of(t[x], s[set][8 * x + 7]);
                }
                top = max_across_32(max_of(t[0], t[1]) * a.c);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        // The sums are kept against a maximum that follows the rows' own within 2^8: the first step sets it, few later ones move it.
        if (__any(top > m + kLag)) {
            const float m_new = __builtin_fmaxf(m, top);
            const float alpha = m_new == -__builtin_inff() ? 1.f : exp2_of(m - m_new);
            m = m_new;
            l *= alpha;
#pragma unroll
            for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[dt][e] *= alpha;
        }
        const float m_use = m == -__builtin_inff() ? 0.f : m;
        __builtin_amdgcn_sched_barrier(0);
        // the scores of the next step, this step's probabilities under it; its values are read for the step after
        float sum = 0.f;
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            score(n, std::integral_constant<int, set ^ 1>{});
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int x = n * 8 / NQ; x < (n + 1) * 8 / NQ; ++x) {         // probabilities 2x and 2x + 1
                float pr[2];
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    pr[y] = exp2_of(__builtin_fmaf(s[set][2 * x + y], a.c, -m_use));
                    sum += pr[y];
                }
                pin(sum);
                uint32_t w[P];
                pieces_of<P>(pr[0], pr[1], w);
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    pf[x >> 2][p][x & 3] = w[p];
                    pin(w[p]);
                }
                if (x == 7) l += sum;
            }
            if (n == NQ / 2 - 1 || n == NQ - 1) {
#pragma unroll
                for (int dt = 0; dt < ND; ++dt) read_v(n == NQ - 1, dt, v_this);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // A tile of 64 keys in the stages at `slot` (0 or kTensor): its data is awaited and published, the next one's is asked for and,
    // where it passes through registers, put in place after the arithmetic.  One body for both stages: with two, the compiler
    // keeps the accumulators in two places.
    if (begin < stop) {
        // before the loop: the first 32 keys' scores, from what would be K's stage before the first, and the first stages
        load_k(kTensor, begin - 32);
        put_k(kTensor);
        load_v(0, begin);
        load_k(0, begin + 32);
        put_k(0);
        put_v(0, begin);
        if constexpr (BLOCK == 0) __builtin_amdgcn_s_waitcnt(0x0F70);
        __syncthreads();
        read_k(0, NK, kTensor + 32 * DT * 2);
#pragma unroll
        for (int n = 0; n < NK * QP; ++n) score(n, std::integral_constant<int, 0>{});
        int slot = 0;
        for (int kb = begin; kb < stop; kb += kTileKeys) {
            if constexpr (BLOCK == 0) __builtin_amdgcn_s_waitcnt(0x0F70);     // vmcnt(0): the copies
            __syncthreads();
            if (BLOCK == 0 && kb + kTileKeys > len) {
                const v4u zero = {0, 0, 0, 0};                                // rows of the stage lie one after another
                for (int x = (len - kb) * DT * 2 + threadIdx.x * 16; x < kTensor; x += 4096) lds_write(lds0 + kVBase + slot + x, zero);
                __syncthreads();
            }
            const bool more = kb + kTileKeys < stop;
            if (more) {
                load_v(slot ^ kTensor, kb + kTileKeys);
                load_k(slot ^ kTensor, kb + kTileKeys + 32);
            }
            constexpr auto first = std::integral_constant<int, 0>{};
            constexpr auto second = std::integral_constant<int, 32 * DT * 2>{};
            step(std::integral_constant<int, 0>{}, kb, first, first);
            step(std::integral_constant<int, 1>{}, kb + 32, second, second);
            const int to_other = slot ? -kTensor : kTensor;
            slot ^= kTensor;
#pragma unroll
            for (int kk = 0; kk < NK; ++kk) k_at[kk] += to_other;
#pragma unroll
            for (int dt = 0; dt < ND; ++dt) v_at[dt] += to_other;
            if (more) {
                put_k(slot);
                put_v(slot, kb + kTileKeys);
            }
        }
#pragma unroll
        for (int n = 0; n < 2 * P * ND; ++n) out(n);
    }

    // lane (i, h2) holds row i, elements 32dt + 8(e/4) + 4h2 + e%4
    if (r0 + 32 * wave + i < rows) {
        const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
        const float ll = __uint_as_float(both[0]) + __uint_as_float(both[1]);
        const float inv = splits > 1 ? 1.f : ll > 0.f ? 1.f / ll : 0.f;
        const int64_t prow = part_row_of(a, h, rq, r) * a.splits + split;
        const int64_t part0 = part_row_of(a, h, rq, r0) * a.splits;
        const int tile_rows = min(kTileRows, rows - r0), at = (32 * wave + i) * a.splits + split;
        const BufRsrc ro = make_rsrc(a.part_o + part0 * dim, (uint32_t)(tile_rows * a.splits * dim * 4));
        if (splits > 1 && h2 == 0) {
            if (kTree && a.join) __builtin_amdgcn_raw_buffer_store_b64(v2u{__float_as_uint(m), __float_as_uint(ll)}, make_rsrc(a.part_ml + part0, (uint32_t)(tile_rows * a.splits * 8)), at * 8, 0, kDeviceScope);
            else a.part_ml[prow] = make_float2(m, ll);
        }
        const int64_t to = (int64_t)(rq.t0 + tok) * a.ldo + (int64_t)head * dim;
#pragma unroll
        for (int dt = 0; dt < ND; ++dt)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {
                const int d = 32 * dt + 8 * q4 + 4 * h2;
                float x[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = o[dt][4 * q4 + e] * inv;
                if (d < dim) {
                    if (splits == 1) store_out<TYPE, 4>(a, to + d, x);
                    else if (kTree && a.join) __builtin_amdgcn_raw_buffer_store_b128(v4u{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])}, ro, (at * dim + d) * 4, 0, kDeviceScope);
                    else *reinterpret_cast<float4*>(a.part_o + prow * dim + d) = make_float4(x[0], x[1], x[2], x[3]);
                }
            }
    }
}

#if !MX_CACHE_TREE
template <int TYPE, int DT, int BLOCK, int DC>
__device__ __forceinline__ void chunk(const CacheAttnArgs& a, int index, uint8_t* smem) {
    // Workgroup u runs on XCD u % 8: with a multiple of eight heads an XCD takes whole heads, so that its L2 holds few of them.
    // The tiles with the most keys go first.
    const int per_head = a.tiles * a.splits;
    int h, rest;
    if (a.heads % 8 == 0) {
        const int j = index / 8;
        h = index % 8 + 8 * (j / per_head);
        rest = j % per_head;
    } else {
        h = index % a.heads;
        rest = index / a.heads;
    }
    const int split = rest % a.splits, tile_id = a.tiles - 1 - rest / a.splits;
    const Tile tile = find_tile(a, tile_id);
    if (tile.b < 0) return;
    chunk_tile<TYPE, DT, BLOCK, DC>(a, tile, h, split, Run{}, smem);
}
#else
// ---- trees of more than sixteen rows --------------------------------------------------------------------
// o = sum_j p_j v_j over the cached keys and those of the new ones that the row's mask has, in tiles of one request, key/value head and up to
// 128 rows: chunk_tile()'s, without a causal order, or a small tile of up to 32 rows, 64 in bfloat16 calls on an MXInt cache, where a
// large one would convert each key for half as many rows.  A small tile's four waves take blocks of 32 keys in turn, as in decode(), and
// join at the end: K and V go from memory to registers once for all rows, R groups of sixteen, an MXInt block is converted once
// for them, and q, which all waves use, lies in LDS as the matrix instructions read it.  bfloat16 calls have two pieces of P, as
// chunk_tile() has, but three in tiles of up to sixteen rows (R = 1), as decode() has: a request's results are as exact beside larger
// ones as alone (24 requests of 16 rows beside one of 64, 2000 keys of an MXInt cache: 39.5 us, 41.2 as R = 2 with two pieces).  A
// block's K registers are free for the next block's loads when its scores are there, V's after P V, so both are in flight during
// the rest.
// Bound by the issue of vector arithmetic (softmax, pieces of P, MXInt) and of matrix instructions, which two waves a SIMD overlap little:
// 24 requests of 320 to 504 rows, 8 heads, 128 elements, MXInt 32: 368 to 388 us, clock 2.1 GHz, matrix cores 0.30 and vector units 0.49
// of the time (heads over 64 with an MXInt cache: 256 registers and 28 bytes spilled, addresses that the copies of a stage read back).  Eight requests of 36 / 52 / 64 rows on 500 to 4000 keys, 8 heads: MXInt as small tiles 31.6 / 33.0 / 33.7 us, as large ones
// 33.3 / 34.4 / 35.3; a bfloat16 cache as small ones 34.0 / 35.8 / 37.0, as large ones 32.7 / 33.6 / 34.8, but of 20 rows 25.9 and 31.0.
template <int TYPE, int BLOCK>
constexpr int kTreeGroups = TYPE == MX_F32 || BLOCK == 0 ? 2 : 4;

// How a batch is shared out.  A unit is a tile of a request's rows and a key/value head; its keys are cut into runs of as few blocks of 64 as
// leave no more items (a unit's runs) than workgroups.  A block of a large tile takes longer (3.6 us with an MXInt cache, 2.5 with
// bfloat16; of a small one of 64 rows 2.3, of 32 1.6), so small tiles have longer runs.  All know all lengths: there are no items
// without work.  Every wave works it out for itself, a request a lane, 64 at a time (2 to 3 us with the loads of the lengths for up to 64
// requests; of more each pass loads them again: 128, 256, 512 of 20 rows on 20 keys take 18, 38, 82 us in all).
struct TreeItem {
    Tile tile;                 // b < 0: nothing; index: of kTileRows rows
    bool small;                // no more than a.small_rows of them
    int h, split, splits;
    int unit;                  // number of (tile, head)
};

// Lanes' values (none negative) up to and including each as one: from the lane one before in the row of sixteen, two, four, eight; then the
// first and third row's last lane to the row after, the second row's to the second half.
template <int CTRL, int ROWS>
__device__ __forceinline__ int moved(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xF, ROWS == 0xF); }
template <typename Op>
__device__ __forceinline__ int scan_wave(int v, Op op) {
    v = op(v, moved<0x111, 0xF>(v));
    v = op(v, moved<0x112, 0xF>(v));
    v = op(v, moved<0x114, 0xF>(v));
    v = op(v, moved<0x118, 0xF>(v));
    v = op(v, moved<0x142, 0xA>(v));
    return op(v, moved<0x143, 0xC>(v));
}
__device__ __forceinline__ int sums_of(int v) { return scan_wave(v, [](int x, int y) { return x + y; }); }
__device__ __forceinline__ int sum_of(int v) { return __builtin_amdgcn_readlane(sums_of(v), 63); }
__device__ __forceinline__ int largest_of(int v) { return __builtin_amdgcn_readlane(scan_wave(v, [](int x, int y) { return max(x, y); }), 63); }

template <int TYPE>
struct TreePlan {
    static constexpr int kResident = TYPE == MX_F32 ? 256 : 512;       // workgroups that the GPU holds
    const CacheAttnArgs& a;
    int lane, b0, index;       // requests b0 .. b0 + 63 are the lanes', each its `index`
    Request rq;
    int large, small, blocks;
    int eighths;               // of a large tile's run, for the small one's
    int run;

    __device__ __forceinline__ void look_at(int b) {
        if (b == b0) return;
        b0 = b;
        rq = Request{0, 0, 0};
        if (b + lane < a.requests) rq = request_of(a, b + lane);
        const int rows = rq.n * a.group, rest = rows % kTileRows;
        large = rows / kTileRows + (rest > a.small_rows);
        small = rest > 0 && rest <= a.small_rows;
        eighths = rest <= 32 ? a.least_run : a.small_run;
        blocks = max(1, (rq.len + kTileKeys - 1) / kTileKeys);
        index = b + lane;
        if (a.sorted) {                                // the longest first: 64 requests at most
            int rank = 0;
            for (int j = 0; j < a.requests; ++j) {
                const int other = __builtin_amdgcn_readlane(blocks, j);
                rank += other > blocks || (other == blocks && j < lane);
            }
            index = __builtin_amdgcn_ds_permute((lane < a.requests ? rank : lane) * 4, lane);
            rq = Request{__shfl(rq.t0, index), __shfl(rq.n, index), __shfl(rq.len, index)};
            large = __shfl(large, index);
            small = __shfl(small, index);
            eighths = __shfl(eighths, index);
            blocks = __shfl(blocks, index);
        }
    }
    // How many runs of about `of` blocks the request's keys are cut into: any number will do that all agree on, two kernels among them, so
    // what is rounded once is written so
    __device__ __forceinline__ int runs(int of) const {
        return min(max((int)__builtin_fmaf((float)blocks, __builtin_amdgcn_rcpf((float)of), 0.9999f), 1), a.splits);
    }
    // n / d: of small numbers the reciprocal is off by one at most
    static __device__ __forceinline__ int over(int n, int d) {
        if (n >= 1 << 21) return n / d;
        int q = (int)((float)n * __builtin_amdgcn_rcpf((float)d));
        const int r = n - q * d;
        q += r >= d ? 1 : r < 0 ? -1 : 0;
        return q;
    }
    __device__ __forceinline__ int small_run() const { return max(run, run / 8 * eighths + run % 8 * eighths / 8); }

    __device__ __forceinline__ explicit TreePlan(const CacheAttnArgs& args) : a(args), lane(threadIdx.x & 63), b0(-1), run(INT_MAX / 4) {
        look_at(0);
        if (a.splits <= 1) return;                     // one run a unit
        float all = 0.f;
        int most = 1, units = 0;
        for (int base = 0; base < a.requests; base += 64) {
            look_at(base);
            all += (float)sum_of((int)fminf(__builtin_fmaf(8.f * __builtin_amdgcn_rcpf((float)eighths), (float)small, (float)large) * (float)blocks, 1e7f));
            most = max(most, largest_of(blocks));
            units += sum_of(large + small);
        }
        const float work = all * (float)a.heads;       // in blocks of a large tile
        // The smallest run that leaves no more items than there are workgroups.  A unit's last run is half empty on average: a little less than fits
        // is the first guess, then a sixteenth more at a time until the items are few enough, as they are with one run a unit.
        // Items for more than one round even out ragged lengths; where all units fit one round, longer runs may be done sooner.  A run's start and end
        // take as long as kStart blocks, and of the last round half a run stands alone on average.  (30 requests of 52 rows on 200 to 3000 keys of a
        // bfloat16 cache 76 us, 86 in two rounds, of an MXInt one 64 and 75; 32 of 32 rows on 2000 keys 65 and 75.)
        constexpr float kStart = 2.5f;
        int slots = a.slots, several = 0;
        float rounds = 0.f;
#pragma unroll 1
        while (true) {
            const float left = __builtin_fmaf(-0.45f * (float)a.heads, (float)units, (float)slots);
            run = max(a.run, (int)fminf(work * __builtin_amdgcn_rcpf(fmaxf(left, 1.f)), (float)most));
            int64_t items = 0;
#pragma unroll 1
            while (true) {
                items = 0;
                for (int base = 0; base < a.requests; base += 64) {
                    look_at(base);
                    items += sum_of(large * runs(run) + small * runs(small_run()));
                }
                items *= a.heads;
                if (items <= slots || run >= most) break;
                run += max(1, run >> 4);
            }
            if (slots <= kResident) {
                if (several > 0 && (float)run + kStart >= rounds) run = several;
                return;
            }
            if (units * a.heads > kResident) return;
            rounds = __builtin_fmaf(__builtin_fmaf(kStart, (float)items, work), __builtin_amdgcn_rcpf((float)kResident), 0.5f * (float)run);
            several = run;
            slots = kResident;
        }
    }
    __device__ __forceinline__ TreeItem find(int item) {
        int before = 0, units = 0;
        for (int base = 0; base < a.requests; base += 64) {
            look_at(base);
            const int of_large = runs(run), of_small = runs(small_run());
            // (exact below 2^24, which is past all workgroups: only requests whose tokens overlap come there, and they stay in bounds)
            auto items_of = [&](int l, int s) { return (int)fminf((float)(l + s) * (float)a.heads, 0x1p24f); };
            const int count = items_of(large * of_large, small * of_small), many = items_of(large, small);
            const int upto = sums_of(count), units_to = sums_of(many);
            const uint64_t past = __ballot(before + upto > item);
            if (past != 0) {
                const int at = __builtin_ctzll(past);
                auto of = [&](int v) { return __builtin_amdgcn_readlane(v, at); };
                const int n_large = of(large), s_large = of(of_large), s_small = of(of_small);
                const Request r{of(rq.t0), of(rq.n), of(rq.len)};
                // Workgroup u runs on XCD u % 8: with a multiple of eight heads an XCD takes whole heads, so that its L2 holds few of them; the
                // tiles that read the same keys follow one another.
                const int rest = item - before - (of(upto) - of(count)), each = n_large * s_large + (of(small) ? s_small : 0);
                int h, y;
                if (a.heads % 8 == 0) {
                    y = rest >> 3;
                    const int eighth = over(y, each);
                    h = (rest & 7) + 8 * eighth;
                    y -= eighth * each;
                } else {
                    y = over(rest, a.heads);
                    h = rest - y * a.heads;
                }
                const bool is_small = y >= n_large * s_large;
                const int split = is_small ? y - n_large * s_large : over(y, n_large), tile = is_small ? n_large : y - split * n_large;
                const int unit = units + of(units_to) - of(many) + tile * a.heads + h;
                if ((uint32_t)unit >= (uint32_t)a.tiles) break;            // (only where requests' tokens overlap)
                return TreeItem{Tile{of(index), tile, r}, is_small, h, split, is_small ? s_small : s_large, unit};
            }
            before += __builtin_amdgcn_readlane(upto, 63);
            units += __builtin_amdgcn_readlane(units_to, 63);
        }
        return TreeItem{Tile{-1, 0, Request{0, 0, 0}}, false, 0, 0, 0, 0};
    }
    // The runs of the unit that a head's row number `row` of all packed ones belongs to; 0: none
    __device__ __forceinline__ int runs_of_row(int row) {
        for (int base = 0; base < a.requests; base += 64) {
            look_at(base);
            const int r = row - rq.t0 * a.group;
            const uint64_t its = __ballot(r >= 0 && r < rq.n * a.group);
            if (its != 0) return __builtin_amdgcn_readlane(runs(r / kTileRows < large ? run : small_run()), __builtin_ctzll(its));
        }
        return 0;
    }
};

// The parts of 8 U rows as one: eight groups of 32 lanes, a group U of the rows, S splits' parts of all of them in flight.
template <int TYPE, int U, int S, int SCOPE>
__device__ __forceinline__ void join_tile(const CacheAttnArgs& a, const Request& rq, int h, int r0, int rows, int splits) {
    const int64_t part0 = part_row_of(a, h, rq, r0) * a.splits;
    const BufRsrc ro = make_rsrc(a.part_o + part0 * a.dim, (uint32_t)(rows * a.splits * a.dim * 4));
    const BufRsrc rm = make_rsrc(a.part_ml + part0, (uint32_t)(rows * a.splits * 8));
    const int group = threadIdx.x >> 5, lane = threadIdx.x & 31, d = 4 * lane < a.dim ? 4 * lane : 0;
    float x[U][4], m[U], l[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        m[u] = -__builtin_inff();
        l[u] = x[u][0] = x[u][1] = x[u][2] = x[u][3] = 0.f;
    }
    for (int s0 = 0; s0 < splits; s0 += S) {
        v4u y[U][S];
        float2 ml[U][S];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int s = 0; s < S; ++s) {
                const int at = min(group + 8 * u, rows - 1) * a.splits + min(s0 + s, splits - 1);
                const auto t = __builtin_amdgcn_raw_buffer_load_b64(rm, at * 8, 0, SCOPE);
                ml[u][s] = make_float2(__uint_as_float(t[0]), __uint_as_float(t[1]));
                y[u][s] = __builtin_bit_cast(v4u, __builtin_amdgcn_raw_buffer_load_b128(ro, (at * a.dim + d) * 4, 0, SCOPE));
            }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int s = 0; s < S; ++s) {
                if (s0 + s >= splits || ml[u][s].x == -__builtin_inff()) continue;      // a run that the row saw nothing of
                const float top = __builtin_fmaxf(m[u], ml[u][s].x), f = exp2_of(m[u] - top), w = exp2_of(ml[u][s].x - top);
                m[u] = top;
                l[u] = l[u] * f + ml[u][s].y * w;
#pragma unroll
                for (int e = 0; e < 4; ++e) x[u][e] = x[u][e] * f + __uint_as_float(y[u][s][e]) * w;
            }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (group + 8 * u >= rows || 4 * lane >= a.dim) continue;
        const float inv = l[u] > 0.f ? 1.f / l[u] : 0.f;
        const float o[4] = {x[u][0] * inv, x[u][1] * inv, x[u][2] * inv, x[u][3] * inv};
        const int row = r0 + group + 8 * u, tok = row / a.group, head = h * a.group + (row - tok * a.group);
        store_out<TYPE, 4>(a, (int64_t)(rq.t0 + tok) * a.ldo + (int64_t)head * a.dim + d, o);
    }
}

template <int TYPE, int DT, int BLOCK, int R>
__device__ __forceinline__ void tree_tile(const CacheAttnArgs& a, const Tile& tile, int h, int split, int splits, int begin, int end, uint8_t* smem) {
    constexpr int NS = DT / 32, NJ = DT / 16, VE = DT / 16;
    constexpr int EB = BLOCK == 0 ? 2 : 1;
    constexpr int QP = kQueryPieces<TYPE>, P = TYPE == MX_F32 || R == 1 ? 3 : 2;     // (up to sixteen rows: all bits of P, as in decode())
    using Block = KeyBlock<DT, BLOCK>;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int n = lane & 15, g = lane >> 4;
    const Request rq = tile.rq;
    PageWindow pages(a, tile.b);
    const int rows = rq.n * a.group, r0 = tile.index * kTileRows, len = rq.len, dim = a.dim, base = len - rq.n;
    pages.set_length(a, len);
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)smem + lane * 16;

    auto row_at = [&](int r, int i) { return min(r0 + 16 * r + i, rows - 1); };        // rows past the last repeat it
    Block f;
    int64_t at[2];
    const int last_run = (len - 1) & ~15;
    auto load_k = [&](int kb) __attribute__((always_inline)) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            at[t] = pages.row(a, h, min(kb + 16 * t, last_run));
            const uint8_t* kp = a.k + at[t] * dim * EB;
            if constexpr (BLOCK == 0) {
#pragma unroll
                for (int s = 0; s < NS; ++s) {
                    const int d = 32 * s + 8 * g;
                    f.k[t][s] = *reinterpret_cast<const v4u*>(kp + (n * dim + (d < dim ? d : 0)) * 2);
                }
            } else {
                const uint8_t* kx = a.k_exps + at[t] * (dim / BLOCK);
#pragma unroll
                for (int s = 0; s < Block::KC; ++s) {
                    const int d = 64 * s + 16 * g, e = d < dim ? d : 0;
                    f.k[t][s] = *reinterpret_cast<const v4u*>(kp + n * dim + e);
                    f.ke[t][s] = kx[n * (dim / BLOCK) + e / BLOCK];
                }
            }
        }
    };
    auto load_v = [&]() __attribute__((always_inline)) {
        const int d = VE * n < dim ? VE * n : 0;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint8_t* src = a.v + at[t] * dim * EB + ((4 * g + i) * dim + d) * EB;
                if constexpr (VE * EB == 16) {
                    const v4u x = *reinterpret_cast<const v4u*>(src);
#pragma unroll
                    for (int w = 0; w < 4; ++w) f.v[4 * t + i][w] = x[w];
                } else if constexpr (VE * EB == 8) {
                    const v2u x = *reinterpret_cast<const v2u*>(src);
                    f.v[4 * t + i][0] = x[0];
                    f.v[4 * t + i][1] = x[1];
                } else {
                    f.v[4 * t + i][0] = *reinterpret_cast<const uint32_t*>(src);
                }
                if constexpr (BLOCK != 0) f.ve[4 * t + i] = (a.v_exps + at[t] * (dim / BLOCK))[(4 * g + i) * (dim / BLOCK) + d / BLOCK];
            }
    };
    int kb = begin + 32 * wave;
    if (kb < end) {
        load_k(kb);
        load_v();
    }
    for (int r = wave; r < R; r += 4) {
        const int row = row_at(r, n), tok = row / a.group, head = h * a.group + (row - tok * a.group);
        v4u qf[QP][NS];
        load_q<TYPE, QP, NS>(a, (int64_t)(rq.t0 + tok) * a.ldq + (int64_t)head * dim,
                             [&](int x) { return BLOCK == 0 ? 32 * x + 8 * g : 64 * (x >> 1) + 16 * g + 8 * (x & 1); }, qf);
#pragma unroll
        for (int p = 0; p < QP; ++p)
#pragma unroll
            for (int x = 0; x < NS; ++x) lds_write(lds0 + ((r * NS + x) * QP + p) * 1024, qf[p][x]);
    }
    __syncthreads();

    float m[R], l[R];
    v4f o[R][NJ];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        m[r] = -__builtin_inff();
        l[r] = 0.f;
#pragma unroll
        for (int j = 0; j < NJ; ++j) o[r][j] = v4f{0.f, 0.f, 0.f, 0.f};
    }
    for (; kb < end; kb += 128) {
        v4f s[R][2];
#pragma unroll
        for (int r = 0; r < R; ++r) s[r][0] = s[r][1] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int x = 0; x < NS; ++x) {
            v4u kf[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                if constexpr (BLOCK == 0) {
                    kf[t] = f.k[t][x];
                } else {
                    const float sc = power2(f.ke[t][x >> 1] - a.exp_shift);
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        int y = (int)f.k[t][x >> 1][2 * (x & 1) + (w >> 1)];
                        asm("" : "+v"(y));            // the bytes are taken apart here, not when they arrive (four registers for one)
                        const float lo = (float)(int8_t)(y >> (16 * (w & 1))) * sc, hi = (float)(int8_t)(y >> (16 * (w & 1) + 8)) * sc;
                        kf[t][w] = __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
                    }
                }
            }
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int p = QP - 1; p >= 0; --p) {
                    const v4u qf = lds_read(lds0 + ((r * NS + x) * QP + p) * 1024);
#pragma unroll
                    for (int t = 0; t < 2; ++t)
                        s[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, kf[t]), __builtin_bit_cast(v8bf, qf), s[r][t], 0, 0, 0);
                }
            __builtin_amdgcn_sched_barrier(0);
        }
        load_k(kb + 128);                              // (past the end: the last run again, unused)
        // V of this block is at the rows before
        v4u pf[R][P];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (kb + 31 >= base || kb + 31 >= end) {
                const int tok = row_at(r, n) / a.group, seen = end - 1 - kb - 4 * g;
                const uint32_t bits = seen_from(a, rq.t0 + tok, kb - base) >> (4 * g);
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[r][t][e] = 16 * t + e <= seen && (bits >> (16 * t + e) & 1) ? s[r][t][e] : -__builtin_inff();
            }
            float top = max_of(s[r][0][0], s[r][0][1], s[r][0][2]);
            top = max_of(top, s[r][0][3], s[r][1][0]);
            top = max_of(top, s[r][1][1], s[r][1][2]);
            top = max_across_16_32(max_of(top, s[r][1][3])) * a.c;
            // the sums are kept against a maximum that follows the rows' own within 2^8
            if (__any(top > m[r] + kLag)) {
                const float m_new = __builtin_fmaxf(m[r], top);
                const float alpha = m_new == -__builtin_inff() ? 1.f : exp2_of(m[r] - m_new);
                m[r] = m_new;
                l[r] *= alpha;
#pragma unroll
                for (int j = 0; j < NJ; ++j) o[r][j] *= alpha;
            }
            const float m_use = m[r] == -__builtin_inff() ? 0.f : m[r];
            float sum = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float p0 = exp2_of(__builtin_fmaf(s[r][w >> 1][2 * (w & 1)], a.c, -m_use));
                const float p1 = exp2_of(__builtin_fmaf(s[r][w >> 1][2 * (w & 1) + 1], a.c, -m_use));
                sum += p0 + p1;
                uint32_t y[P];
                pieces_of<P>(p0, p1, y);
#pragma unroll
                for (int p = 0; p < P; ++p) pf[r][p][w] = y[p];
            }
            l[r] += sum;
        }
        // what lies past the request's end may be anything, NaN among it: it counts as zeros
        const bool whole = kb + 32 <= len;
        float sc[8];
        if constexpr (BLOCK != 0) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool in = whole || kb + 16 * (i >> 2) + 4 * g + (i & 3) < len;
                sc[i] = in ? power2(f.ve[i] - a.exp_shift) : 0.f;
            }
        } else if (!whole) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool in = kb + 16 * (i >> 2) + 4 * g + (i & 3) < len;
#pragma unroll
                for (int w = 0; w < VE / 2; ++w) f.v[i][w] = in ? f.v[i][w] : 0u;
            }
        }
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            v4u vf;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                if constexpr (BLOCK == 0) {
                    vf[w] = __builtin_amdgcn_perm(f.v[2 * w + 1][j >> 1], f.v[2 * w][j >> 1], (j & 1) ? 0x07060302u : 0x05040100u);
                } else {
                    int x = (int)f.v[2 * w][j >> 2], y = (int)f.v[2 * w + 1][j >> 2];
                    asm("" : "+v"(x), "+v"(y));
                    const float lo = (float)(int8_t)(x >> (8 * (j & 3))) * sc[2 * w];
                    const float hi = (float)(int8_t)(y >> (8 * (j & 3))) * sc[2 * w + 1];
                    vf[w] = __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
                }
            }
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int p = P - 1; p >= 0; --p)
                    o[r][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, vf), __builtin_bit_cast(v8bf, pf[r][p]), o[r][j], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
        load_v();
    }

    // the four waves join, sixteen rows at a time: lane (n, g) holds row n, elements VE*(4g + e) + j
    DecodeLds<DT>& lds = *reinterpret_cast<DecodeLds<DT>*>(smem);
    const int tile_rows = min(16 * R, rows - r0);
    const int64_t part0 = part_row_of(a, h, rq, r0);
    const BufRsrc ro = make_rsrc(a.part_o + part0 * a.splits * dim, (uint32_t)(tile_rows * a.splits * dim * 4));
    const BufRsrc rm = make_rsrc(a.part_ml + part0 * a.splits, (uint32_t)(tile_rows * a.splits * 8));
#pragma unroll
    for (int r = 0; r < R; ++r) {
        l[r] = sum_across_16_32(l[r]);
        __syncthreads();                                                  // q, or the rows before, have been read
        if (g == 0) lds.ml[wave][n] = make_float2(m[r], l[r]);
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int j = 0; j < NJ; ++j) lds.o[wave][n][VE * (4 * g + e) + j] = o[r][j][e];
        __syncthreads();
        const int i = threadIdx.x >> 4, part = threadIdx.x & 15, row = r0 + 16 * r + i;
        if (row < rows && VE * part < dim) {
            float mm = -__builtin_inff();
#pragma unroll
            for (int w = 0; w < 4; ++w) mm = __builtin_fmaxf(mm, lds.ml[w][i].x);
            float ll = 0.f, acc[VE];
#pragma unroll
            for (int j = 0; j < VE; ++j) acc[j] = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float2 ml = lds.ml[w][i];
                const float c = ml.x == -__builtin_inff() ? 0.f : exp2_of(ml.x - mm);
                ll += ml.y * c;
#pragma unroll
                for (int j = 0; j < VE; ++j) acc[j] += lds.o[w][i][VE * part + j] * c;
            }
            if (splits == 1) {
                const int tok = row / a.group, head = h * a.group + (row - tok * a.group);
                const float inv = ll > 0.f ? 1.f / ll : 0.f;
#pragma unroll
                for (int j = 0; j < VE; ++j) acc[j] *= inv;
                store_out<TYPE, VE>(a, (int64_t)(rq.t0 + tok) * a.ldo + (int64_t)head * dim + VE * part, acc);
            } else {
                // written through for the workgroup that joins them in this launch; a launch of its own finds them in any case
                const int to = (16 * r + i) * a.splits + split;
                const v2u ml = {__float_as_uint(mm), __float_as_uint(ll)};
#pragma unroll
                for (int j = 0; j < VE; j += 4) {
                    const v4u x = {__float_as_uint(acc[j]), __float_as_uint(acc[j + 1]), __float_as_uint(acc[j + 2]), __float_as_uint(acc[j + 3])};
                    if (a.join) __builtin_amdgcn_raw_buffer_store_b128(x, ro, (to * dim + VE * part + j) * 4, 0, kDeviceScope);
                    else __builtin_amdgcn_raw_buffer_store_b128(x, ro, (to * dim + VE * part + j) * 4, 0, 0);
                }
                if (part == 0) {
                    if (a.join) __builtin_amdgcn_raw_buffer_store_b64(ml, rm, to * 8, 0, kDeviceScope);
                    else __builtin_amdgcn_raw_buffer_store_b64(ml, rm, to * 8, 0, 0);
                }
            }
        }
    }
}

template <int TYPE, int DT, int BLOCK, int DC>
__global__ __launch_bounds__(256, TYPE == MX_F32 ? 1 : 2) void cache_tree_kernel(CacheAttnArgs a) {
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    constexpr int G = kTreeGroups<TYPE, BLOCK>;
    static_assert(G * (DT / 32) * kQueryPieces<TYPE> * 1024 <= (int)sizeof(DecodeLds<DT>), "q and the waves' results share the workgroup's LDS");
    const TreeItem i = TreePlan<TYPE>(a).find(blockIdx.x);
    if (i.tile.b >= 0) {
        const Request& rq = i.tile.rq;
        const int r0 = i.tile.index * kTileRows, rows = min(rq.n * a.group - r0, kTileRows), len = rq.len;
        const int per = ((len + kTileKeys - 1) / kTileKeys + i.splits - 1) / i.splits * kTileKeys;
        const int begin = min(i.split * per, len), end = min(begin + per, len);
        // (in this order; with tiles of 32 rows, the most frequent ones, last these take 2 % longer)
        if (i.small && rows <= 32 && (TYPE == MX_F32 || rows > kFewRows)) tree_tile<TYPE, DT, BLOCK, 2>(a, i.tile, i.h, i.split, i.splits, begin, end, smem);
        else if (!i.small) chunk_tile<TYPE, DT, BLOCK, DC>(a, i.tile, i.h, i.split, Run{i.splits, begin, end}, smem);
        else if (G == 4 && rows > 32) tree_tile<TYPE, DT, BLOCK, G>(a, i.tile, i.h, i.split, i.splits, begin, end, smem);
        else if constexpr (TYPE == MX_BF16) tree_tile<TYPE, DT, BLOCK, 1>(a, i.tile, i.h, i.split, i.splits, begin, end, smem);
        if (i.splits > 1 && a.join && came_last(a.counters + i.unit, i.splits, reinterpret_cast<uint32_t*>(smem)))
            for (int r = 0; r < rows; r += 64) join_tile<TYPE, 8, 2, kDeviceScope>(a, rq, i.h, r0 + r, min(64, rows - r), i.splits);
    }
    fill_padding<TYPE>(a);
}

// The parts of a row as one: a wave a row, its two halves every other part, kJoinParts of them in flight.  Bound by the latency of the lengths'
// loads and of one or two rounds of parts (972 rows of up to 7 parts 7 us, 2440 of 22 parts 9).
constexpr int kJoinParts = 8, kJoinGrid = 1536;     // (as many workgroups as the GPU holds)
template <int TYPE>
__global__ __launch_bounds__(256) void cache_tree_join_kernel(CacheAttnArgs a) {
    const int rows = (int)a.tokens * a.group, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    TreePlan<TYPE> plan(a);
    for (int64_t item = (int64_t)blockIdx.x * 4 + wave; item < (int64_t)rows * a.heads; item += (int64_t)gridDim.x * 4) {
        const int h = (int)item / rows, row = (int)item - h * rows;
        const int splits = plan.runs_of_row(row);
        if (splits <= 1) continue;
        const int64_t part0 = ((int64_t)h * rows + row) * a.splits;
        const BufRsrc ro = make_rsrc(a.part_o + part0 * a.dim, (uint32_t)(splits * a.dim * 4)), rm = make_rsrc(a.part_ml + part0, (uint32_t)(splits * 8));
        const int half = (threadIdx.x >> 5) & 1, lane = threadIdx.x & 31, d = 4 * lane < a.dim ? 4 * lane : 0;
        float m = -__builtin_inff(), l = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
        // m, l and x take in another part's
        auto take = [&](float pm, float pl, const float (&px)[4]) __attribute__((always_inline)) {
            const float top = __builtin_fmaxf(m, pm), use = top == -__builtin_inff() ? 0.f : top, f = exp2_of(m - use), w = exp2_of(pm - use);
            m = top;
            l = l * f + pl * w;
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = x[e] * f + px[e] * w;
        };
        for (int s0 = half; s0 < splits; s0 += 2 * kJoinParts) {
            v4u y[kJoinParts];
            v2u ml[kJoinParts];
#pragma unroll
            for (int i = 0; i < kJoinParts; ++i) {
                const int at = min(s0 + 2 * i, splits - 1);
                ml[i] = __builtin_amdgcn_raw_buffer_load_b64(rm, at * 8, 0, 0);
                y[i] = __builtin_bit_cast(v4u, __builtin_amdgcn_raw_buffer_load_b128(ro, (at * a.dim + d) * 4, 0, 0));
            }
#pragma unroll
            for (int i = 0; i < kJoinParts; ++i) {
                const float p[4] = {__uint_as_float(y[i][0]), __uint_as_float(y[i][1]), __uint_as_float(y[i][2]), __uint_as_float(y[i][3])};
                if (s0 + 2 * i < splits && __uint_as_float(ml[i][0]) > -__builtin_inff()) take(__uint_as_float(ml[i][0]), __uint_as_float(ml[i][1]), p);
            }
        }
        auto other = [](float v) __attribute__((always_inline)) {
            const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
            return __uint_as_float(r[1]);                  // the upper half's, in both
        };
        const float p[4] = {other(x[0]), other(x[1]), other(x[2]), other(x[3])};
        take(other(m), other(l), p);
        if (half != 0 || 4 * lane >= a.dim) continue;
        const int tok = row / a.group, head = h * a.group + (row - tok * a.group);
        const float inv = l > 0.f ? 1.f / l : 0.f;
        const float o[4] = {x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv};
        store_out<TYPE, 4>(a, (int64_t)tok * a.ldo + (int64_t)head * a.dim + d, o);
    }
}
#endif

#if !MX_CACHE_TREE
// Requests of many rows and, in the workgroups after `chunks`, of few: in a batch that has both they run side by side.
template <int TYPE, int DT, int BLOCK, int DC>
__global__ __launch_bounds__(256, TYPE == MX_F32 ? 1 : 2) void cache_mixed_kernel(CacheAttnArgs many, CacheAttnArgs few, int chunks) {
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    if ((int)blockIdx.x < chunks) chunk<TYPE, DT, BLOCK, DC>(many, blockIdx.x, smem);
    else decode<TYPE, DT, BLOCK>(few, blockIdx.x - chunks, *reinterpret_cast<DecodeLds<DT>*>(smem));
    fill_padding<TYPE>(many);
}
#endif

// ---- joining the splits ---------------------------------------------------------------------------------
// o = sum_s o_s 2^(m_s - m) / sum_s l_s 2^(m_s - m), in an order that the number of splits gives, whatever order they ended in.
// 32 lanes take a row, four elements each.  Many splits: a workgroup a row, its eight groups of 32 sharing the splits.  Few splits of a
// tile: a workgroup 32 rows, a group four of them at a time (eight rows, one a group, took 3 us longer for 44 tiles of 8 heads,
// most of it finding the tile; the last workgroup to arrive joining a tile, 8).
template <int TYPE, bool CHUNK>
__global__ __launch_bounds__(256) void cache_join_kernel(CacheAttnArgs a) {
    __shared__ float4 lds[8][32];
    const int group = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int64_t prow = blockIdx.x;
    const int per_unit = CHUNK ? kTileRows : a.part_rows;
    const int unit = (int)(prow / per_unit), row = (int)(prow - (int64_t)unit * per_unit);
    const int h = unit % a.heads;
    int b = unit / a.heads, r = row, splits = a.splits;
    if constexpr (CHUNK) {
        const Tile t = find_tile(a, b);
        if (t.b < 0) return;
        b = t.b;
        splits = splits_of(a, keys_seen(a, t));
        if (splits == 1) return;
        r += t.index * kTileRows;
    } else {
        if (b >= a.requests) return;
        if (a.sorted) b = nth_longest(a, b);
    }
    const Request rq = request_of(a, b);
    const int64_t rows = (int64_t)rq.n * a.group;
    if (r >= rows || rows < a.least || rows > a.most || (!CHUNK && rows > a.part_rows)) return;
    const int tok = r / a.group, head = h * a.group + (r - tok * a.group);
    if constexpr (CHUNK) prow = part_row_of(a, h, rq, r);

    float2 ml[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) ml[x] = lane + 32 * x < splits ? a.part_ml[prow * a.splits + lane + 32 * x] : make_float2(-__builtin_inff(), 0.f);
    float mm = __builtin_fmaxf(ml[0].x, ml[1].x);
#pragma unroll
    for (int d = 1; d < 32; d *= 2) mm = __builtin_fmaxf(mm, __shfl_xor(mm, d, 32));
    const float f0 = ml[0].x == -__builtin_inff() ? 0.f : exp2_of(ml[0].x - mm);
    const float f1 = ml[1].x == -__builtin_inff() ? 0.f : exp2_of(ml[1].x - mm);
    float ll = ml[0].y * f0 + ml[1].y * f1;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) ll += __shfl_xor(ll, d, 32);

    const int d = 4 * lane;
    const float4* p = reinterpret_cast<const float4*>(a.part_o + prow * a.splits * a.dim + (d < a.dim ? d : 0));
    const int stride = a.dim / 4;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s0 = group; s0 < splits; s0 += 64) {
        float4 y[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) y[u] = p[(int64_t)min(s0 + u * 8, splits - 1) * stride];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int s = s0 + u * 8;
            const float w0 = __shfl(s < 32 ? f0 : f1, s & 31, 32), w = s < splits ? w0 : 0.f;
            x.x += y[u].x * w; x.y += y[u].y * w; x.z += y[u].z * w; x.w += y[u].w * w;
        }
    }
    lds[group][lane] = x;
    __syncthreads();
    if (group != 0) return;
#pragma unroll
    for (int g = 1; g < 8; ++g) {
        const float4 y = lds[g][lane];
        x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
    }
    if (d < a.dim) {
        const float inv = ll > 0.f ? 1.f / ll : 0.f;
        const float o[4] = {x.x * inv, x.y * inv, x.z * inv, x.w * inv};
        store_out<TYPE, 4>(a, (int64_t)(rq.t0 + tok) * a.ldo + (int64_t)head * a.dim + d, o);
    }
}

template <int TYPE>
__global__ __launch_bounds__(256) void cache_join_tiles_kernel(CacheAttnArgs a) {
    const int group = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int unit = blockIdx.x / (kTileRows / 32), base = blockIdx.x % (kTileRows / 32) * 32;
    const int h = unit % a.heads;
    const Tile t = find_tile(a, unit / a.heads);
    if (t.b < 0) return;
    const int first = t.index * kTileRows, rows = min(kTileRows, t.rq.n * a.group - first);
    const int d = 4 * lane < a.dim ? 4 * lane : 0;
    const int64_t part_row = part_row_of(a, h, t.rq, first);
    const int splits = splits_of(a, keys_seen(a, t));
    if (base >= rows || splits == 1) return;                               // (of a single split the rows are there)
    float x[4][4], m[4], l[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        m[u] = -__builtin_inff();
        l[u] = x[u][0] = x[u][1] = x[u][2] = x[u][3] = 0.f;
    }
    for (int s0 = 0; s0 < splits; s0 += 4) {
        float4 y[4][4];
        float2 ml[4][4];
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const int64_t at = (part_row + min(base + group + 8 * u, rows - 1)) * a.splits + min(s0 + s, splits - 1);
                ml[u][s] = a.part_ml[at];
                y[u][s] = *reinterpret_cast<const float4*>(a.part_o + at * a.dim + d);
            }
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                if (s0 + s >= splits || ml[u][s].x == -__builtin_inff()) continue;      // a split that the row saw nothing of
                const float top = __builtin_fmaxf(m[u], ml[u][s].x), f = exp2_of(m[u] - top), w = exp2_of(ml[u][s].x - top);
                m[u] = top;
                l[u] = l[u] * f + ml[u][s].y * w;
                x[u][0] = x[u][0] * f + y[u][s].x * w;
                x[u][1] = x[u][1] * f + y[u][s].y * w;
                x[u][2] = x[u][2] * f + y[u][s].z * w;
                x[u][3] = x[u][3] * f + y[u][s].w * w;
            }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int row = base + group + 8 * u;
        if (row >= rows || 4 * lane >= a.dim) continue;
        const int tok = (first + row) / a.group, head = h * a.group + (first + row - tok * a.group);
        const float inv = l[u] > 0.f ? 1.f / l[u] : 0.f;
        const float o[4] = {x[u][0] * inv, x[u][1] * inv, x[u][2] * inv, x[u][3] * inv};
        store_out<TYPE, 4>(a, (int64_t)(t.rq.t0 + tok) * a.ldo + (int64_t)head * a.dim + d, o);
    }
}

template <int TYPE, bool CHUNK>
mx_status launch_join(const CacheAttnArgs& a, int64_t rows, hipStream_t stream) {
    if constexpr (CHUNK) {
        if (a.splits <= 16) {
            cache_join_tiles_kernel<TYPE><<<(unsigned)(rows / 32), 256, 0, stream>>>(a);
            MX_HIP_LAUNCH_CHECK();
            return MX_OK;
        }
    }
    cache_join_kernel<TYPE, CHUNK><<<(unsigned)rows, 256, 0, stream>>>(a);
    MX_HIP_LAUNCH_CHECK();
    return MX_OK;
}

template <int TYPE>
__global__ __launch_bounds__(256) void cache_zero_kernel(CacheAttnArgs a) {
    const int64_t row = (int64_t)a.heads_q * a.dim;
    for (int64_t t = blockIdx.x; t < a.tokens; t += gridDim.x)
        for (int64_t d = threadIdx.x; d < row; d += 256) {
            if constexpr (TYPE == MX_F32) static_cast<float*>(a.out)[t * a.ldo + d] = 0.f;
            else static_cast<uint16_t*>(a.out)[t * a.ldo + d] = 0;
        }
}

// ---- what a call launches -------------------------------------------------------------------------------
// Requests with at most sixteen rows are the work of decode(), the others of chunk().  The host knows bounds only: when no request can
// have more rows by them, cache_decode_kernel takes all (any number of rows is right there, sixteen at a time), else
// cache_mixed_kernel has workgroups of both, each of which leaves the other's requests alone; a single request needs those of
// the one or the other only.  (24 mixed requests, with one half-precision piece of a probability: 66 us in one launch, 80 in two.)
struct Plan {
    bool decode, chunk;
    int part_rows, splits;         // of cache_decode_kernel
    int tiles, chunk_splits, run;
    int grid;                      // cache_tree_kernel
    bool join;                     // in it
    size_t few_bytes;
};

// Workgroups that split keys, at most: about 40 and 8 times what the GPU holds of either kind, past which finer runs even nothing out.  They
// bound the parts, so that a workspace for a batch serves every smaller one, which may well be split more often.
constexpr int64_t kMostDecode = 32768, kMostChunks = 4096;
constexpr int kDecodeSlots = 768;                  // of bfloat16 calls; 512 of fp32 ones
constexpr int kLongRun = 4096;                     // keys of a run in decode(), at most, while kMostDecode allows it

// Splits of the longest tiles' keys, `tiles` tiles of 64 each, for `groups` workgroups, `slots` of which the GPU holds at once, and
// `other` tiles' time of work beside them.  A workgroup's start and end count as kStart tiles, a part's store and its join as two.
// One request: all have as many keys, so the fewest rounds times tiles.  Several: half as many keys on average (the host knows the
// longest only), so the longest workgroup or the work over the slots, whichever takes longer.  Measured on 168 groups of 47 tiles at
// most beside 21 requests of one token: 1 split 103 us, 2 79, 3 (taken) 70, 4 82; 80 groups of 32 tiles of one request: 1 74 us, 3 42,
// 6 (taken) 43, 8 49; 96 groups of 32 tiles, fp32: 1 109 us, 2 (taken) 70, 3 90, 4 79.
int chunk_splits(int64_t groups, int64_t tiles, int64_t slots, int64_t other, bool one) {
    constexpr int kStart = 5;
    int best = 1;
    double least = 1e300;
    for (int s = 1; s <= kMaxSplits && s <= tiles && (s == 1 || groups * s <= kMostChunks); ++s) {
        const int64_t fixed = kStart + (s > 1 ? 2 : 0), longest = ceil_div(tiles, s) + fixed, rounds = ceil_div(groups * s, slots);
        double cost = (double)(rounds * longest);
        if (!one) {
            const double even = (groups * (0.5 * tiles + fixed * s) + other) / slots + (rounds > 1 ? 0.5 * longest : 0);
            cost = even > longest ? even : longest;
        }
        if (cost < least) { least = cost; best = s; }
    }
    return best;
}

// The last workgroup of a unit to arrive joins its splits, or a launch of its own does when there are many parts of many rows.
bool joined_apart(int rows, int splits) { return rows * splits > 128; }

// Splits of a request's keys in decode(), `blocks` steps of 128 keys in all: a step takes about 0.9 us, the meeting of the splits 2.4 +
// 0.15 each, joining them apart 6.3.  (16 requests of 300 keys, 8 heads x 4: 1 split 9.6 us, 2 11.8, 3 10.9; 2 of 1000: 3 splits 12.2,
// 4 10.8, 8 10.1; 1936 keys of 32 heads: 6 splits 14.2, 8 12.6, 16 13.9; 2 of 4096: 11 splits 14.2, 16 13.6, 32 16.9; 2 of 16000:
// 25 splits 23.4, 48, joined apart, 21.8; one of 9000, one head x 8, joined apart: 18 splits 14.8, 36 11.8.)
int decode_splits(int64_t blocks, int least, int most, int rows) {
    int best = least;
    int64_t lowest = INT64_MAX;
    for (int s = least; s <= most && s <= blocks; ++s) {
        const int64_t cost = 18 * ceil_div(blocks, s) + (s == 1 ? 0 : joined_apart(rows, s) ? 126 : 48 + 3 * s);
        if (cost < lowest) { lowest = cost; best = s; }
    }
    return best;
}

size_t part_bytes(const mx_cache& c, int64_t parts) { return ((size_t)parts * ((size_t)c.dim * 4 + 8) + 255) / 256 * 256; }

Plan plan_of(const mx_cache& c, int32_t type, int64_t tokens, int64_t requests, int32_t heads_q, int64_t max_new, int64_t max_len) {
    Plan p{};
    if (max_len > INT32_MAX) max_len = INT32_MAX;      // no sum or product below leaves 64 bits
    const int64_t group = heads_q / c.heads;
    const int64_t most = (max_new < tokens ? max_new : tokens) * group;
    p.chunk = most > kFewRows;
    p.decode = !p.chunk || requests > 1;
    p.part_rows = (int)(most < kFewRows ? most : kFewRows);
    auto clamp = [](int64_t v, int64_t hi) { return (int)(v > hi ? (hi < 1 ? 1 : hi) : v < 1 ? 1 : v); };
    const int64_t units = requests * c.heads;
    // at most as many workgroups as the GPU holds at once, but no run of keys over kLongRun, which would leave the last ones alone at
    // the end
    const int64_t slots = type == MX_F32 ? 512 : kDecodeSlots, even = units > 0 ? slots / units : 1;
    int64_t fine = ceil_div(max_len, kLongRun);
    if (units > 0 && units * fine > kMostDecode) fine = kMostDecode / units;
    p.splits = units <= kCounterBytes / 4 ? decode_splits(ceil_div(max_len, 128), clamp(fine, kMaxSplits), clamp(even > fine ? even : fine, kMaxSplits),
                                                              p.chunk ? 0 : p.part_rows) : 1;
    const int64_t rows = tokens * group;
    const int64_t big = p.decode ? (rows / (kFewRows + 1) < requests ? rows / (kFewRows + 1) : requests) : 1;   // requests with more rows
    if (kTree && p.chunk) {
        const int64_t big = rows < requests ? rows : requests, units = (rows / kTileRows + big) * c.heads, slots = type == MX_F32 ? 256 : 512;
        p.decode = false;
        p.tiles = clamp(units, INT32_MAX);
        p.run = 2;
        // Few units are cut to fill the GPU once; of many there is room for the longest to be cut, of more than there are counters for none is.
        p.grid = clamp(2 * units > slots ? units + slots : slots, INT32_MAX);
        p.chunk_splits = units > kCounterBytes / 4 ? 1 : clamp(rows * c.heads > 0 ? kMostChunks * kTileRows / (rows * c.heads) : 1, kMaxSplits);
        if (p.chunk_splits > ceil_div(max_len, kTileKeys)) p.chunk_splits = clamp(ceil_div(max_len, kTileKeys), kMaxSplits);
        // More units than the GPU holds workgroups have few parts each, and the last workgroup of a unit to come joins them beside others' work
        // (24 requests of 320 to 504 rows, 8 heads: 375 us, 385 with a launch for the joins); the parts of fewer units are joined by a
        // launch, over the whole GPU (16 requests of 4 to 100 rows: 54 us, 72 without; 30 of 52 rows: 83.9, 87.9).
        p.join = units > slots;
        return p;
    }
    p.tiles = p.chunk ? clamp(p.decode ? rows / kTileRows + big : ceil_div(rows, kTileRows), INT32_MAX) : 0;
    // (128 keys of a request of one token take about as long as a tile)
    p.chunk_splits = p.chunk ? chunk_splits((rows / kTileRows + 1) * c.heads, ceil_div(max_len, kTileKeys), type == MX_F32 ? 256 : 512,
                                            p.decode ? units * (max_len / 128) : 0, requests == 1) : 1;
    p.run = clamp(ceil_div(ceil_div(max_len, kTileKeys), p.chunk_splits), 1 << 24);
    p.few_bytes = p.decode && p.splits > 1 ? part_bytes(c, units * p.part_rows * p.splits) : 0;
    return p;
}

// What any plan for these arguments, or for smaller ones, needs: every term grows with every argument.  Parts of decode(): units * splits is
// at most what the GPU holds, or units times the runs of kLongRun keys; of chunk(): the workgroups that split are at least a
// 128th of the rows.  At most 273 MB a kind with heads of 128.
size_t workspace_bytes(const mx_cache& c, int64_t tokens, int64_t requests, int32_t heads_q, int64_t max_new, int64_t max_len) {
    if (max_len > INT32_MAX) max_len = INT32_MAX;
    auto least = [](int64_t a, int64_t b) { return a < b ? a : b; };
    const int64_t group = heads_q / c.heads, most = least(max_new, tokens) * group;
    const int64_t units = least(requests * c.heads, kCounterBytes / 4), fine = least(ceil_div(max_len, kLongRun), kMaxSplits);
    const int64_t long_runs = fine > 1 ? least(units * fine, kMostDecode) : 0;
    const int64_t few = least(units * least(ceil_div(max_len, 128), kMaxSplits), long_runs > kDecodeSlots ? long_runs : kDecodeSlots);
    const int64_t many = most > kFewRows ? least(tokens * heads_q * least(ceil_div(max_len, kTileKeys), kMaxSplits), kMostChunks * kTileRows) : 0;
    return kCounterBytes + part_bytes(c, few * least(most, kFewRows)) + part_bytes(c, many);
}

template <int TYPE, int DT, int BLOCK, int DC>
mx_status launch_kernels(const CacheAttnArgs& base, const Plan& p, uint8_t* workspace, hipStream_t stream) {
    CacheAttnArgs few = base, many = base;
    uint8_t* parts = workspace + kCounterBytes;
    const int64_t units = (int64_t)base.requests * base.heads;
    int64_t few_rows = 0;
    if (p.decode) {
        few.least = 1;
        few.most = p.chunk ? kFewRows : INT32_MAX;
        few.splits = p.splits;
        few.part_rows = p.part_rows;
        few.counters = (uint32_t*)workspace;
        few_rows = units * p.part_rows;
        few.part_o = (float*)parts;
        few.part_ml = (float2*)(few.part_o + few_rows * p.splits * base.dim);
        few.join = p.chunk || !joined_apart(p.part_rows, p.splits);      // next to chunks the bound of sixteen rows says little
        few.sorted = base.requests > 1 && base.requests <= 64 && units * p.splits > 512;
        parts += p.few_bytes;
    }
    if (p.chunk) {
        many.least = p.decode ? kFewRows + 1 : 1;
        many.most = INT32_MAX;
        many.splits = p.chunk_splits;
        many.run = p.run;
        many.tiles = p.tiles;
        many.part_o = (float*)parts;
        many.part_ml = (float2*)(many.part_o + base.tokens * base.heads_q * p.chunk_splits * base.dim);
#if MX_CACHE_TREE
        many.counters = (uint32_t*)workspace;
        many.slots = p.grid;
        many.small_rows = 16 * kTreeGroups<TYPE, BLOCK>;
        many.small_run = 12;
        many.least_run = BLOCK == 0 ? 14 : 18;
        many.join = p.join;
        many.sorted = 2 * p.tiles > p.grid && base.requests > 1 && base.requests <= 64;
        constexpr int lds = 4 * kTileKeys * DT * 2;
        static_assert(sizeof(DecodeLds<DT>) <= lds, "both kinds of tile share the workgroup's LDS");
        static std::atomic<uint64_t> raised{0};
        if (lds > 60 * 1024 && !allow_dynamic_lds((const void*)cache_tree_kernel<TYPE, DT, BLOCK, DC>, lds, raised)) return MX_ERR_DEVICE;
        cache_tree_kernel<TYPE, DT, BLOCK, DC><<<(unsigned)p.grid, 256, lds, stream>>>(many);
        MX_HIP_LAUNCH_CHECK();
        if (!p.join && p.chunk_splits > 1) {
            many.sorted = 0;
            const int64_t rows = base.tokens * base.heads_q;
            cache_tree_join_kernel<TYPE><<<(unsigned)(rows < 4 * kJoinGrid ? ceil_div(rows, 4) : kJoinGrid), 256, 0, stream>>>(many);
            MX_HIP_LAUNCH_CHECK();
        }
        return MX_OK;
#else
        const int64_t chunks = (int64_t)p.tiles * base.heads * p.chunk_splits;
        constexpr int lds = 4 * kTileKeys * DT * 2;
        static_assert(sizeof(DecodeLds<DT>) <= lds, "both share the workgroup's LDS");
        static std::atomic<uint64_t> raised{0};
        if (lds > 60 * 1024 && !allow_dynamic_lds((const void*)cache_mixed_kernel<TYPE, DT, BLOCK, DC>, lds, raised)) return MX_ERR_DEVICE;
        cache_mixed_kernel<TYPE, DT, BLOCK, DC><<<(unsigned)(chunks + (p.decode ? units * p.splits : 0)), 256, lds, stream>>>(many, few, (int)chunks);
#endif
    } else {
        cache_decode_kernel<TYPE, DT, BLOCK><<<(unsigned)(units * p.splits), 256, 0, stream>>>(few);
    }
    MX_HIP_LAUNCH_CHECK();
    if (p.decode && p.splits > 1 && !few.join) {
        const mx_status st = launch_join<TYPE, false>(few, few_rows, stream);
        if (st != MX_OK) return st;
    }
#if MX_CACHE_TREE
    return MX_OK;
#else
    return p.chunk && p.chunk_splits > 1 ? launch_join<TYPE, true>(many, (int64_t)p.tiles * base.heads * kTileRows, stream) : MX_OK;
#endif
}

template <int TYPE, int DT, int DC>
mx_status launch_block(const CacheAttnArgs& a, const Plan& p, int block, uint8_t* workspace, hipStream_t stream) {
    return block == 0 ? launch_kernels<TYPE, DT, 0, DC>(a, p, workspace, stream)
           : block == 16 ? launch_kernels<TYPE, DT, 16, DC>(a, p, workspace, stream) : launch_kernels<TYPE, DT, 32, DC>(a, p, workspace, stream);
}

template <int TYPE>
mx_status launch(const CacheAttnArgs& a, const Plan& p, int block, uint8_t* workspace, hipStream_t stream) {
    if (a.requests == 0) {
        cache_zero_kernel<TYPE><<<(unsigned)(a.tokens < 65536 ? a.tokens : 65536), 256, 0, stream>>>(a);
        MX_HIP_LAUNCH_CHECK();
        return MX_OK;
    }
    if (a.dim <= 64) return launch_block<TYPE, 64, 64>(a, p, block, workspace, stream);
    return a.dim <= 96 ? launch_block<TYPE, 128, 96>(a, p, block, workspace, stream) : launch_block<TYPE, 128, 128>(a, p, block, workspace, stream);
}

bool attention_args_ok(const mx_cache& c, int64_t tokens, int64_t requests, int32_t heads_q, int64_t max_new, int64_t max_len) {
    return tokens >= 0 && requests >= 0 && heads_q >= 1 && c.heads >= 1 && heads_q % c.heads == 0 && max_new >= 1 && max_len >= 1;
}
// Keys of a request and its rows are counted in 32 bits, and the kernels look past the last one by tiles: of 128 keys for each of 64
// splits, which is the most.
constexpr int32_t kMostCounted = INT32_MAX - 65536;
bool attention_supported(const mx_cache& c, int64_t tokens, int64_t requests, int32_t heads_q) {
    return requests <= kCacheMaxRequests && tokens <= kMostCounted / heads_q && requests * c.heads < ((int64_t)1 << 24);
}


size_t workspace_checked(const mx_cache& c, int64_t tokens, int64_t requests, int32_t heads_q, int64_t max_new, int64_t max_len) {
    if (cache_status(c) != MX_OK || !attention_args_ok(c, tokens, requests, heads_q, max_new, max_len) ||
        !attention_supported(c, tokens, requests, heads_q))
        return 0;
    return workspace_bytes(c, tokens, requests, heads_q, max_new, max_len);
}

mx_status attend(const void* q, int32_t type, int64_t tokens, int64_t ldq, int32_t heads_q, mx_cache c, const void* k_data,
                 const uint8_t* k_exps, const void* v_data, const uint8_t* v_exps, const int32_t* table, int64_t width,
                 const int32_t* q_start, const int32_t* kv_len, const uint64_t* masks, int32_t words, int64_t requests, int64_t max_new,
                 int64_t max_len, float scale, void* workspace, void* out, int64_t ldo, void* stream) {
    if (type != MX_F32 && type != MX_BF16) return MX_ERR_BAD_ARG;
    const mx_status st = cache_status(c);
    if (st == MX_ERR_BAD_ARG || !attention_args_ok(c, tokens, requests, heads_q, max_new, max_len)) return MX_ERR_BAD_ARG;
    if (!__builtin_isfinite(scale) || width < 0 || words < 0 || (kTree && words < 1)) return MX_ERR_BAD_ARG;
    const int64_t row = (int64_t)heads_q * c.dim;
    const int tb = type_bytes(type);
    if (tokens > 0) {
        if (q == nullptr || out == nullptr || !aligned(q, tb) || !aligned(out, tb) || ldq < row || ldo < row) return MX_ERR_BAD_ARG;
        if (workspace == nullptr || !aligned(workspace, 256)) return MX_ERR_BAD_ARG;
        if (requests > 0) {
            if (k_data == nullptr || v_data == nullptr || q_start == nullptr || kv_len == nullptr || (width > 0 && table == nullptr))
                return MX_ERR_BAD_ARG;
            if (c.f.block != 0 && (k_exps == nullptr || v_exps == nullptr)) return MX_ERR_BAD_ARG;
            if (!aligned(k_data, 16) || !aligned(v_data, 16) || !aligned(table, 4) || !aligned(q_start, 4) || !aligned(kv_len, 4))
                return MX_ERR_BAD_ARG;
            if (kTree && (masks == nullptr || !aligned(masks, 8))) return MX_ERR_BAD_ARG;
        }
    }
    if (st != MX_OK) return st;
    if (!attention_supported(c, tokens, requests, heads_q) || width > kMostCounted / c.page || words > MX_TREE_MAX_NODES / 64) return MX_ERR_UNSUPPORTED;
    if (tokens == 0) return MX_OK;
    const Plan p = plan_of(c, type, tokens, requests, heads_q, max_new, max_len);
    // the threads of a launch, 256 a workgroup, are counted in 32 bits (joins, of few workgroups by kMostChunks, stay far below)
    if (kTree ? p.grid >= 1 << 24 : (int64_t)p.tiles * c.heads * p.chunk_splits + (p.decode ? requests * c.heads * p.splits : 0) >= 1 << 24) return MX_ERR_UNSUPPORTED;
    CacheAttnArgs a{};
    a.q = q; a.out = out; a.ldq = ldq; a.ldo = ldo;
    a.k = (const uint8_t*)k_data; a.v = (const uint8_t*)v_data;
    a.k_exps = k_exps; a.v_exps = v_exps;
    a.table = table; a.width = width; a.q_start = q_start; a.kv_len = kv_len;
    a.tokens = tokens;
    a.max_keys = width * c.page;
    a.pages = (uint32_t)c.pages;
    a.requests = (int32_t)requests; a.heads = c.heads; a.group = heads_q / c.heads; a.heads_q = heads_q; a.dim = c.dim;
    a.page_log2 = log2_of(c.page);
    a.exp_shift = exponent_bias(c) + 6;
    a.vec_q = aligned(q, 16) && ldq % (16 / tb) == 0;
    a.vec_o = aligned(out, 4 * tb) && ldo % 4 == 0;
    a.c = __builtin_fmaxf(__builtin_fabsf(scale) * 1.4426950408889634f, 0x1p-126f);   // never 0: minus infinity stays a mask
    a.flip = scale < 0.f ? 0x80000000u : 0u;
#if MX_CACHE_TREE
    a.masks = (const uint32_t*)masks;
    a.mask_words = 2 * words;
#endif
    uint8_t* ws = (uint8_t*)workspace;
    return type == MX_F32 ? launch<MX_F32>(a, p, c.f.block, ws, (hipStream_t)stream) : launch<MX_BF16>(a, p, c.f.block, ws, (hipStream_t)stream);
}

}  // namespace
}  // namespace mx

using namespace mx;

#if MX_CACHE_TREE
extern "C" size_t mx_cache_tree_attention_workspace_bytes(mx_cache c, int64_t tokens, int64_t requests, int32_t heads_q, int64_t max_new,
                                                          int64_t max_len) {
    return workspace_checked(c, tokens, requests, heads_q, max_new, max_len);
}

extern "C" mx_status mx_cache_tree_attention(const void* q, int32_t type, int64_t tokens, int64_t ldq, int32_t heads_q, mx_cache c,
                                             const void* k_data, const uint8_t* k_exps, const void* v_data, const uint8_t* v_exps,
                                             const int32_t* table, int64_t width, const int32_t* q_start, const int32_t* kv_len,
                                             const uint64_t* masks, int32_t words, int64_t requests, int64_t max_new, int64_t max_len,
                                             float scale, void* workspace, void* out, int64_t ldo, void* stream) {
    return attend(q, type, tokens, ldq, heads_q, c, k_data, k_exps, v_data, v_exps, table, width, q_start, kv_len, masks, words, requests,
                  max_new, max_len, scale, workspace, out, ldo, stream);
}
#else
extern "C" size_t mx_cache_attention_workspace_bytes(mx_cache c, int64_t tokens, int64_t requests, int32_t heads_q, int64_t max_new,
                                                     int64_t max_len) {
    return workspace_checked(c, tokens, requests, heads_q, max_new, max_len);
}

extern "C" mx_status mx_cache_attention(const void* q, int32_t type, int64_t tokens, int64_t ldq, int32_t heads_q, mx_cache c,
                                        const void* k_data, const uint8_t* k_exps, const void* v_data, const uint8_t* v_exps,
                                        const int32_t* table, int64_t width, const int32_t* q_start, const int32_t* kv_len,
                                        int64_t requests, int64_t max_new, int64_t max_len, float scale, void* workspace, void* out,
                                        int64_t ldo, void* stream) {
    return attend(q, type, tokens, ldq, heads_q, c, k_data, k_exps, v_data, v_exps, table, width, q_start, kv_len, nullptr, 0, requests,
                  max_new, max_len, scale, workspace, out, ldo, stream);
}
#endif
