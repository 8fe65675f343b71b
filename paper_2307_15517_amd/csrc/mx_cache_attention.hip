// Attention of new tokens over the paged key/value cache, causal, grouped heads.
#include <type_traits>

#include "mx_cache.h"

namespace mx {
namespace {

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));

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
    float* part_o;             // [part row][split][dim], unnormalised
    float2* part_ml;           // [part row][split]: row maximum (exp2 domain), row sum
    int64_t tokens;
    int64_t max_keys;          // width * page
    uint32_t pages;
    int32_t requests, heads, group, heads_q, dim;
    int32_t page_log2;
    int32_t exp_shift;         // an exponent byte e stands for 2^(e - exp_shift) per mantissa unit
    int32_t splits;            // of this launch
    int32_t least, most;       // this launch takes the requests that have least .. most rows (token, head of a group)
    int32_t part_rows;         // part rows per unit; a request with more rows is not split
    int32_t tiles;             // cache_chunk_kernel: row tiles of all requests, at most
    int32_t fill;              // this launch writes the zeros of tokens outside every request
    int32_t vec_q, vec_o;      // rows of q / out allow 16-byte (bfloat16 out: 8-byte) accesses
    float c;                   // |scale| * log2(e)
    uint32_t flip;             // sign bit of the scale: carried by q
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

    __device__ __forceinline__ PageWindow(const CacheAttnArgs& a, int b, int len)
        : row_table(a.table + (int64_t)b * a.width), base(-64), last((len - 1) >> a.page_log2), id(0) {}
    // The row of the pool that holds key `key` of the request (and those after it in its run of sixteen): `key` is below its
    // length and the same for all lanes.  A page index outside the pool reads as page 0.
    __device__ __forceinline__ int64_t row(const CacheAttnArgs& a, int h, int key) {
        const int page = key >> a.page_log2;
        if (page - base >= 64) {
            base = page;
            id = row_table[min(page + (int)(threadIdx.x & 63), last)];
            asm volatile("" : "+v"(id));       // awaited here, once in 64 pages, and not wherever it might just have been loaded
        }
        uint32_t at = (uint32_t)__builtin_amdgcn_readlane(id, page - base);
        at = at < a.pages ? at : 0;
        return (((int64_t)at * a.heads + h) << a.page_log2) + (key & ((1 << a.page_log2) - 1));
    }
};

template <int TYPE>
__device__ __forceinline__ void load_q(const CacheAttnArgs& a, int64_t at, float (&v)[8]) {
    if (a.vec_q) load8<TYPE, true>(a.q, at, v);
    else load8<TYPE, false>(a.q, at, v);
}

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// bfloat16 pieces of a float whose sum is the float's leading 8, 16 or 24 bits; each piece is cut, not rounded, but the last
template <int P>
__device__ __forceinline__ void pieces_of(float a, float b, uint32_t (&w)[P]) {
#pragma unroll
    for (int p = 0; p < P; ++p) {
        if (p == P - 1) {
            w[p] = pack_bf16(a, b);
        } else {
            w[p] = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
            a -= __uint_as_float(__float_as_uint(a) & 0xffff0000u);
            b -= __uint_as_float(__float_as_uint(b) & 0xffff0000u);
        }
    }
}

__device__ __forceinline__ float max_across_32(float v) {
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __builtin_fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float max_across_16_32(float v) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __builtin_fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __builtin_fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
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
// Pieces: K and V are bfloat16 numbers as they are (an MXInt element has 7 bits and a sign).  bfloat16 q is one piece and its
// probabilities are two, 16 bits, so that what is rounded is the result; float q and its probabilities are three, 24 bits.
// The matrix instructions are idle most of the time here, so the pieces cost nothing.
template <int TYPE>
struct Pieces {
    static constexpr int Q = TYPE == MX_F32 ? 3 : 1, P = TYPE == MX_F32 ? 3 : 2;
};

template <int DT, int BLOCK>
struct KeyBlock {
    static constexpr int KC = DT / 64;                            // MXInt: 16-byte chunks of a key per lane
    static constexpr int VE = DT / 16;                            // elements of a V row per lane
    v4u k[2][BLOCK == 0 ? DT / 32 : KC];
    int ke[2][KC];
    uint32_t v[8][BLOCK == 0 ? VE / 2 : VE / 4];
    int ve[8];
};

template <int TYPE, int DT, int BLOCK>
__global__ __launch_bounds__(256, 2) void cache_decode_kernel(CacheAttnArgs a) {
    constexpr int NS = DT / 32, NJ = DT / 16, VE = DT / 16;
    constexpr int EB = BLOCK == 0 ? 2 : 1;
    constexpr int QP = Pieces<TYPE>::Q, P = Pieces<TYPE>::P;
    using Block = KeyBlock<DT, BLOCK>;
    __shared__ float lds_o[4][16][DT + 4];
    __shared__ float2 lds_ml[4][16];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int n = lane & 15, g = lane >> 4;
    if (a.fill) fill_padding<TYPE>(a);

    const int split = blockIdx.x % a.splits;
    const int unit = blockIdx.x / a.splits;
    const int h = unit % a.heads, b = unit / a.heads;
    const Request rq = request_of(a, b);
    const int rows = rq.n * a.group;
    if (rows < a.least || rows > a.most) return;
    const int splits = rows <= a.part_rows ? a.splits : 1;
    if (split >= splits) return;
    const int len = rq.len;
    // this split's run of keys, in whole blocks of 128
    const int per = (((len + 127) >> 7) + splits - 1) / splits;
    const int begin = min(split * per * 128, len), end = min(begin + per * 128, len);
    const int dim = a.dim;

    for (int r0 = 0; r0 < rows; r0 += 16) {
        // q: column n of the score product, elements d(step, g, i); rows past the last repeat it
        const int r = min(r0 + n, rows - 1);
        const int tok = r / a.group, head = h * a.group + (r - tok * a.group);
        const int last = len - rq.n + tok;                                // the last key this row sees
        v4u qf[QP][NS];
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            const int d = BLOCK == 0 ? 32 * s + 8 * g : 64 * (s >> 1) + 16 * g + 8 * (s & 1);
            float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            if (d < dim) load_q<TYPE>(a, (int64_t)(rq.t0 + tok) * a.ldq + (int64_t)head * dim + d, v);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t w[QP];
                pieces_of<QP>(__uint_as_float(__float_as_uint(v[2 * i]) ^ a.flip), __uint_as_float(__float_as_uint(v[2 * i + 1]) ^ a.flip), w);
#pragma unroll
                for (int p = 0; p < QP; ++p) qf[p][s][i] = w[p];
            }
        }
        // keys past the last one any row of this tile sees are left out
        const int first_last = len - rq.n + r0 / a.group;                 // the last key that all its rows see
        const int stop = min(end, len - rq.n + min(r0 + 15, rows - 1) / a.group + 1);

        float m = -__builtin_inff(), l = 0.f;
        v4f o[NJ];
#pragma unroll
        for (int j = 0; j < NJ; ++j) o[j] = v4f{0.f, 0.f, 0.f, 0.f};

        // The two runs of sixteen keys of a block lie in one page each; a run past the end reads the last one again (masked).
        // A block's loads are issued while the one before is computed on; there is one past the end, so that no load is conditional.
        const int last_run = (len - 1) & ~15;
        PageWindow pages(a, b, len);
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
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int key = kb + 16 * t + 4 * g + e;
                        s[t][e] = key <= last && key < stop ? s[t][e] : -__builtin_inff();
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
        int kb = begin + 32 * wave;
        if (kb < stop) {
            Block f0, f1;
            load(f0, kb);
            for (;;) {
                load(f1, kb + 128);
                compute(f0, kb);
                if ((kb += 128) >= stop) break;
                load(f0, kb + 128);
                compute(f1, kb);
                if ((kb += 128) >= stop) break;
            }
        }

        // the four waves join: lane (n, g) holds row n, elements VE*(4g + e) + j
        l = sum_across_16_32(l);
        __syncthreads();                                                  // the tile before has been read
        if (g == 0) lds_ml[wave][n] = make_float2(m, l);
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int j = 0; j < NJ; ++j) lds_o[wave][n][VE * (4 * g + e) + j] = o[j][e];
        __syncthreads();
        const int row = threadIdx.x >> 4, part = threadIdx.x & 15;
        if (r0 + row < rows && VE * part < dim) {
            float mm = -__builtin_inff();
#pragma unroll
            for (int w = 0; w < 4; ++w) mm = __builtin_fmaxf(mm, lds_ml[w][row].x);
            float ll = 0.f, acc[VE];
#pragma unroll
            for (int j = 0; j < VE; ++j) acc[j] = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float2 ml = lds_ml[w][row];
                const float f = ml.x == -__builtin_inff() ? 0.f : exp2_of(ml.x - mm);
                ll += ml.y * f;
#pragma unroll
                for (int j = 0; j < VE; ++j) acc[j] += lds_o[w][row][VE * part + j] * f;
            }
            if (splits == 1) {
                const int tk = (r0 + row) / a.group, hd = h * a.group + (r0 + row - tk * a.group);
                const float inv = ll > 0.f ? 1.f / ll : 0.f;
#pragma unroll
                for (int j = 0; j < VE; ++j) acc[j] *= inv;
                store_out<TYPE, VE>(a, (int64_t)(rq.t0 + tk) * a.ldo + (int64_t)hd * dim + VE * part, acc);
            } else {
                const int64_t at = ((int64_t)unit * a.part_rows + row) * a.splits + split;
                if (part == 0) a.part_ml[at] = make_float2(mm, ll);
#pragma unroll
                for (int j = 0; j < VE; j += 4)
                    *reinterpret_cast<float4*>(a.part_o + at * dim + VE * part + j) = make_float4(acc[j], acc[j + 1], acc[j + 2], acc[j + 3]);
            }
        }
    }
}

// ---- many rows: chunks and prompts ----------------------------------------------------------------------
// A workgroup takes 128 rows (token, head of the group) of one request and key/value head, a wave 32 of them, q in registers;
// K and V pass through LDS in tiles of 64 (fp32: 32) keys as bfloat16 (MXInt elements become that on the way, exactly), two stages, so
// that a tile's loads run under the arithmetic on the one before.  S^T = K Q^T puts a row in a lane's column, so that its
// maximum and sum take one exchange between the lane halves, and hands the probabilities to O^T = V^T P^T in registers;
// V is transposed by the LDS reads.
constexpr int kTileRows = 128;
// keys per tile: 32 with fp32 activations, whose q takes three times the registers
template <int TYPE>
constexpr int kTileKeys = TYPE == MX_F32 ? 32 : 64;

// The request and its tile of rows that tile number `tile` is; b < 0: none.  Every wave looks for itself, 64 requests at a time.
struct Tile {
    int b, index;
};
__device__ __forceinline__ Tile find_tile(const CacheAttnArgs& a, int tile) {
    const int lane = threadIdx.x & 63;
    int before = 0;
    for (int base = 0; base < a.requests; base += 64) {
        int count = 0;
        if (base + lane < a.requests) {
            const Request r = request_of(a, base + lane);
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
            return Tile{base + at, tile - before - (__builtin_amdgcn_readlane(upto, at) - __builtin_amdgcn_readlane(count, at))};
        }
        before += __builtin_amdgcn_readlane(upto, 63);
    }
    return Tile{-1, 0};
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
__device__ __forceinline__ v2u read_transposed(const uint8_t* p) {
    const v4s r = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(uintptr_t)p);
    return __builtin_bit_cast(v2u, r);
}

template <int TYPE, int DT, int BLOCK>
__global__ __launch_bounds__(256, 2) void cache_chunk_kernel(CacheAttnArgs a) {
    constexpr int QP = Pieces<TYPE>::Q, P = Pieces<TYPE>::P;
    constexpr int KT = kTileKeys<TYPE>, NT = KT / 32, NK = DT / 16, ND = DT / 32;
    constexpr int EB = BLOCK == 0 ? 2 : 1;
    constexpr int kTensor = KT * DT * 2, kStage = 2 * kTensor;
    constexpr int kPer = 16, kLanes = DT / kPer;       // MXInt staging: sixteen elements per lane
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int i = lane & 31, h2 = lane >> 5;
    if (a.fill) fill_padding<TYPE>(a);

    // Workgroup u runs on XCD u % 8: with a multiple of eight heads an XCD takes whole heads, so that its L2 holds few of them.
    // The tiles with the most keys go first.
    const int per_head = a.tiles * a.splits;
    int h, rest;
    if (a.heads % 8 == 0) {
        const int j = blockIdx.x / 8;
        h = blockIdx.x % 8 + 8 * (j / per_head);
        rest = j % per_head;
    } else {
        h = blockIdx.x % a.heads;
        rest = blockIdx.x / a.heads;
    }
    const int split = rest % a.splits, tile_id = a.tiles - 1 - rest / a.splits;
    const Tile tile = find_tile(a, tile_id);
    if (tile.b < 0) return;
    const int b = tile.b;
    const Request rq = request_of(a, b);
    const int rows = rq.n * a.group, r0 = tile.index * kTileRows;
    const int len = rq.len, dim = a.dim;

    // the keys that some row of the tile sees, and this split's run of them in whole tiles
    const int all = max(0, len - rq.n + min(r0 + kTileRows - 1, rows - 1) / a.group + 1);
    const int per = (((all + KT - 1) / KT) + a.splits - 1) / a.splits * KT;
    const int begin = min(split * per, all), stop = min(begin + per, all);

    // this wave's rows: q is the right operand of the scores, lane (i, h2) row i, elements 16kk + 8h2 ..
    const int r = min(r0 + 32 * wave + i, rows - 1);
    const int tok = r / a.group, head = h * a.group + (r - tok * a.group);
    const int last = len - rq.n + tok;
    const int first_last = len - rq.n + min(r0 + 32 * wave, rows - 1) / a.group;          // the last key all of its rows see
    const int wave_stop = min(stop, len - rq.n + min(r0 + 32 * wave + 31, rows - 1) / a.group + 1);
    v4u qf[QP][NK];
#pragma unroll
    for (int kk = 0; kk < NK; ++kk) {
        const int d = 16 * kk + 8 * h2;
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (d < dim) load_q<TYPE>(a, (int64_t)(rq.t0 + tok) * a.ldq + (int64_t)head * dim + d, v);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            uint32_t w[QP];
            pieces_of<QP>(__uint_as_float(__float_as_uint(v[2 * e]) ^ a.flip), __uint_as_float(__float_as_uint(v[2 * e + 1]) ^ a.flip), w);
#pragma unroll
            for (int p = 0; p < QP; ++p) qf[p][kk][e] = w[p];
        }
    }

    // Staging.  bfloat16: copies from memory straight to LDS, 1 KiB (whole rows) per wave and instruction, lane L's bytes at
    // 16 L of it, so the placement of the chunks is done by what each lane reads.  MXInt: through registers.
    const int last_run = (len - 1) & ~15;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)smem;
    constexpr int kPieceRows = BLOCK == 0 ? 512 / DT : 64 / kLanes;       // rows of a wave's piece, within a run of sixteen
    constexpr int kPieces = KT / (4 * kPieceRows) > 0 ? KT / (4 * kPieceRows) : 1;
    const int rel = BLOCK == 0 ? lane / (DT / 8) : lane / kLanes;         // this lane's row of the piece
    uint32_t k_from = 0, v_from = 0;                                      // and the place of what it reads in there
    {
        const int row = kPieceRows * wave + rel;                          // the pieces are 4 * kPieceRows rows apart: no matter here
        if constexpr (BLOCK == 0) {
            const int chunk = lane % (DT / 8);
            const int kc = (k_place<DT>(row, chunk) - row * DT * 2) >> 4, vc = (v_place<DT>(row, chunk) - row * DT * 2) >> 4;
            k_from = (rel * dim + (8 * kc < dim ? 8 * kc : 0)) * 2;
            v_from = (rel * dim + (8 * vc < dim ? 8 * vc : 0)) * 2;
        } else {
            const int d = (lane % kLanes) * kPer;
            k_from = v_from = rel * dim + (d < dim ? d : 0);
        }
    }
    const uint32_t e_from = BLOCK == 0 ? 0 : rel * (dim / (BLOCK == 0 ? 1 : BLOCK)) + (k_from - rel * dim) / (BLOCK == 0 ? 1 : BLOCK);
    v4u sk[BLOCK == 0 ? 1 : kPieces], sv[BLOCK == 0 ? 1 : kPieces];
    int ek[BLOCK == 0 ? 1 : kPieces], ev[BLOCK == 0 ? 1 : kPieces];
    PageWindow pages(a, b, len);
    const bool stages = 4 * kPieceRows <= KT || wave < KT / kPieceRows;   // with few keys per tile some waves have none to bring
    auto load = [&](uint32_t stage, int kb) __attribute__((always_inline)) {
        if (!stages) return;
#pragma unroll
        for (int u = 0; u < kPieces; ++u) {
            const int key = kb + (4 * u + wave) * kPieceRows, run = min(key & ~15, last_run);
            const int64_t row = pages.row(a, h, run) + (key & 15);
            const uint8_t* kp = a.k + row * dim * EB;
            const uint8_t* vp = a.v + row * dim * EB;
            if constexpr (BLOCK == 0) {
                const uint32_t to = lds0 + stage + (4 * u + wave) * 1024;
                copy16_to_lds(kp, k_from, to);
                copy16_to_lds(vp, v_from, to + kTensor);
            } else {
                sk[u] = *reinterpret_cast<const v4u*>(kp + k_from);
                sv[u] = *reinterpret_cast<const v4u*>(vp + v_from);
                ek[u] = (a.k_exps + row * (dim / BLOCK))[e_from];
                ev[u] = (a.v_exps + row * (dim / BLOCK))[e_from];
            }
        }
    };
    auto widen = [&](const v4u& x, float sc, v4u (&y)[2]) {               // sixteen mantissas to bfloat16 numbers
#pragma unroll
        for (int w = 0; w < 8; ++w) {
            int t = (int)x[w >> 1];
            asm("" : "+v"(t));
            const float lo = (float)(int8_t)(t >> (16 * (w & 1))) * sc, hi = (float)(int8_t)(t >> (16 * (w & 1) + 8)) * sc;
            y[w >> 2][w & 3] = __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
        }
    };
    // What lies past the request's end may be anything, NaN among it, and meets probabilities of zero: it becomes zeros.  (Past
    // the head dimension lies a repetition; it meets zeros of q, or gives results that nobody reads.)
    auto store = [&](uint8_t* stage, int kb) __attribute__((always_inline)) {
        if constexpr (BLOCK != 0) {
            if (!stages) return;
#pragma unroll
            for (int u = 0; u < kPieces; ++u) {
                const int key = (4 * u + wave) * kPieceRows + rel, chunk = 2 * (lane % kLanes);
                const bool in = kb + key < len;
                v4u y[2];
                widen(sk[u], in ? power2(ek[u] - a.exp_shift) : 0.f, y);
                *reinterpret_cast<v4u*>(stage + k_place<DT>(key, chunk)) = y[0];
                *reinterpret_cast<v4u*>(stage + k_place<DT>(key, chunk + 1)) = y[1];
                widen(sv[u], in ? power2(ev[u] - a.exp_shift) : 0.f, y);
                *reinterpret_cast<v4u*>(stage + kTensor + v_place<DT>(key, chunk)) = y[0];
                *reinterpret_cast<v4u*>(stage + kTensor + v_place<DT>(key, chunk + 1)) = y[1];
            }
        }
    };
    auto clear_past = [&](uint8_t* stage, int kb) __attribute__((always_inline)) {
        if constexpr (BLOCK == 0) {
            const int from = (len - kb) * DT * 2;                         // rows of the V tile lie one after another
            const v4u zero = {0, 0, 0, 0};
            for (int x = from + threadIdx.x * 16; x < kTensor; x += 4096) *reinterpret_cast<v4u*>(stage + kTensor + x) = zero;
        }
    };

    // places of this lane's reads in a stage, without the multiples of eight keys that the instructions add
    const uint8_t* k_at[NK];
    const uint8_t* v_at[ND];
#pragma unroll
    for (int kk = 0; kk < NK; ++kk) k_at[kk] = smem + k_place<DT>(i, 2 * kk + h2);
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) {
        const int d = 32 * dt + (lane & 16) + 4 * (lane & 3);
        v_at[dt] = smem + kTensor + v_place<DT>(4 * h2 + ((lane & 15) >> 2), d >> 3) + (d & 7) * 2;
    }

    float m = -__builtin_inff(), l = 0.f;
    v16f o[ND];
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[dt][e] = 0.f;

    auto compute = [&](auto stage_c, int kb) __attribute__((always_inline)) {
        constexpr int stage = decltype(stage_c)::value * kStage;
        v16f s[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int e = 0; e < 16; ++e) s[t][e] = 0.f;
#pragma unroll
            for (int kk = 0; kk < NK; ++kk) {
                const v4u kf = *reinterpret_cast<const v4u*>(k_at[kk] + (stage + 32 * t * DT * 2));
#pragma unroll
                for (int p = QP - 1; p >= 0; --p)
                    s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, kf), __builtin_bit_cast(v8bf, qf[p][kk]), s[t],
                                                                   0, 0, 0);
            }
        }
        v4u vf[2][ND];
        auto read_v = [&](int step) __attribute__((always_inline)) {                                     // sixteen keys
#pragma unroll
            for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                for (int jj = 0; jj < 2; ++jj) {
                    const v2u x = read_transposed(v_at[dt] + (stage + (16 * step + 8 * jj) * DT * 2));
                    vf[step & 1][dt][2 * jj] = x[0];
                    vf[step & 1][dt][2 * jj + 1] = x[1];
                }
        };
        read_v(0);
        // result register e of half t: key 32t + 8(e/4) + 4h2 + e%4
        if (kb + KT - 1 > min(first_last, wave_stop - 1)) {
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int key = kb + 32 * t + 8 * (e >> 2) + 4 * h2 + (e & 3);
                    s[t][e] = key <= last && key < stop ? s[t][e] : -__builtin_inff();
                }
        }
        float top = -__builtin_inff();
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) top = __builtin_fmaxf(top, s[t][e]);
        top = max_across_32(top) * a.c;
        // The sums are kept against a maximum that follows the rows' own within 2^8: the first tile sets it, few later ones move it.
        if (__any(top > m + 8.f)) {
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
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                s[t][e] = exp2_of(__builtin_fmaf(s[t][e], a.c, -m_use));
                sum += s[t][e];
            }
            l += sum;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int step = 2 * t + half;
                if (step + 1 < 2 * NT) read_v(step + 1);
                v4u pf[P];
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    uint32_t x[P];
                    pieces_of<P>(s[t][8 * half + 2 * w], s[t][8 * half + 2 * w + 1], x);
#pragma unroll
                    for (int p = 0; p < P; ++p) pf[p][w] = x[p];
                }
#pragma unroll
                for (int p = P - 1; p >= 0; --p)
#pragma unroll
                    for (int dt = 0; dt < ND; ++dt)
                        o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, vf[step & 1][dt]),
                                                                        __builtin_bit_cast(v8bf, pf[p]), o[dt], 0, 0, 0);
            }
        }
    };

    // A tile: its data is awaited and published, the next tile's is asked for, and, MXInt, put in place after the arithmetic.
    auto step = [&](auto stage_c, int kb) __attribute__((always_inline)) {
        constexpr int at = decltype(stage_c)::value * kStage, other = kStage - at;
        if constexpr (BLOCK == 0) __builtin_amdgcn_s_waitcnt(0x0F70);     // vmcnt(0): the copies
        __syncthreads();                                                  // the tile is there, and the other stage has been read
        if (BLOCK == 0 && kb + KT > len) {
            clear_past(smem + at, kb);
            __syncthreads();
        }
        const bool more = kb + KT < stop;
        if (more) load(other, kb + KT);
        if (kb < wave_stop) compute(stage_c, kb);
        if (more) store(smem + other, kb + KT);
    };
    if (begin < stop) {
        load(0, begin);
        store(smem, begin);
        for (int kb = begin;;) {
            step(std::integral_constant<int, 0>{}, kb);
            if ((kb += KT) >= stop) break;
            step(std::integral_constant<int, 1>{}, kb);
            if ((kb += KT) >= stop) break;
        }
    }

    // lane (i, h2) holds row i, elements 32dt + 8(e/4) + 4h2 + e%4
    if (r0 + 32 * wave + i < rows) {
        const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
        const float ll = __uint_as_float(both[0]) + __uint_as_float(both[1]);
        const float inv = a.splits > 1 ? 1.f : ll > 0.f ? 1.f / ll : 0.f;
        const int64_t prow = (((int64_t)tile_id * a.heads + h) * kTileRows + 32 * wave + i) * a.splits + split;
        if (a.splits > 1 && h2 == 0) a.part_ml[prow] = make_float2(m, ll);
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
                    if (a.splits == 1) store_out<TYPE, 4>(a, to + d, x);
                    else *reinterpret_cast<float4*>(a.part_o + prow * dim + d) = make_float4(x[0], x[1], x[2], x[3]);
                }
            }
    }
}

// ---- joining the splits ---------------------------------------------------------------------------------
// o = sum_s o_s 2^(m_s - m) / sum_s l_s 2^(m_s - m), in the order of the splits whatever order they ended in.  A workgroup takes
// a row, each wave a quarter of its splits: the loads of a wave do not wait for each other.
constexpr int kMaxSplits = 64;

template <int TYPE, bool CHUNK>
__global__ __launch_bounds__(256) void cache_join_kernel(CacheAttnArgs a) {
    __shared__ float lds[4][128];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t prow = blockIdx.x;
    const int unit = (int)(prow / a.part_rows), row = (int)(prow - (int64_t)unit * a.part_rows);
    const int h = unit % a.heads;
    int b = unit / a.heads, r = row;
    if constexpr (CHUNK) {
        const Tile t = find_tile(a, b);
        if (t.b < 0) return;
        b = t.b;
        r += t.index * kTileRows;
    }
    const Request rq = request_of(a, b);
    const int64_t rows = (int64_t)rq.n * a.group;
    if (r >= rows || rows < a.least || rows > a.most || (!CHUNK && rows > a.part_rows)) return;
    const int tok = r / a.group, head = h * a.group + (r - tok * a.group);

    const float2 ml = lane < a.splits ? a.part_ml[prow * a.splits + lane] : make_float2(-__builtin_inff(), 0.f);
    float mm = ml.x;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) mm = __builtin_fmaxf(mm, __shfl_xor(mm, d, 64));
    const float f = ml.x == -__builtin_inff() ? 0.f : exp2_of(ml.x - mm);
    float ll = ml.y * f;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) ll += __shfl_xor(ll, d, 64);
    const float* p = a.part_o + prow * a.splits * a.dim;
    float x0 = 0.f, x1 = 0.f;
    const bool two = lane + 64 < a.dim, one = lane < a.dim;
    for (int s0 = wave; s0 < a.splits; s0 += 32) {
        float y0[8], y1[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int64_t at = (int64_t)min(s0 + 4 * u, a.splits - 1) * a.dim + lane;
            y0[u] = one ? p[at] : 0.f;
            y1[u] = two ? p[at + 64] : 0.f;
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int s = s0 + 4 * u;
            const float w = s < a.splits ? __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(f), s & 63)) : 0.f;
            x0 += y0[u] * w;
            x1 += y1[u] * w;
        }
    }
    lds[wave][lane] = x0;
    lds[wave][lane + 64] = x1;
    __syncthreads();
    const int d = threadIdx.x * 4;
    if (d < a.dim) {
        const float inv = ll > 0.f ? 1.f / ll : 0.f;
        float x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = (lds[0][d + e] + lds[1][d + e] + lds[2][d + e] + lds[3][d + e]) * inv;
        store_out<TYPE, 4>(a, (int64_t)(rq.t0 + tok) * a.ldo + (int64_t)head * a.dim + d, x);
    }
}

template <int TYPE>
__global__ __launch_bounds__(256) void cache_zero_kernel(CacheAttnArgs a) {
    const int64_t row = (int64_t)a.heads_q * a.dim;
    for (int64_t d = threadIdx.x; d < row; d += 256) {
        if constexpr (TYPE == MX_F32) static_cast<float*>(a.out)[blockIdx.x * a.ldo + d] = 0.f;
        else static_cast<uint16_t*>(a.out)[blockIdx.x * a.ldo + d] = 0;
    }
}

// ---- what a call launches -------------------------------------------------------------------------------
// Requests with at most sixteen rows go to cache_decode_kernel, the others to cache_chunk_kernel.  The host knows bounds only:
// when no request can have more rows by them, the first takes all (any number of rows is right there, sixteen at a time), a
// single request goes to the one or the other, else both are launched and each leaves the other's requests alone.
constexpr int kFewRows = 16;

struct Plan {
    bool decode, chunk;
    int part_rows, splits;         // of cache_decode_kernel
    int tiles, chunk_splits;
    size_t bytes;
};

Plan plan_of(const mx_cache& c, int64_t tokens, int64_t requests, int32_t heads_q, int64_t max_new, int64_t max_len) {
    Plan p{};
    const int64_t group = heads_q / c.heads;
    const int64_t most = (max_new < tokens ? max_new : tokens) * group;
    p.chunk = most > kFewRows;
    p.decode = !p.chunk || requests > 1;
    p.part_rows = (int)(most < kFewRows ? most : kFewRows);
    auto clamp = [](int64_t v, int64_t hi) { return (int)(v > hi ? (hi < 1 ? 1 : hi) : v < 1 ? 1 : v); };
    const int64_t units = requests * c.heads;
    p.splits = units > 0 ? clamp(1024 / units, ceil_div(max_len, 256)) : 1;
    p.splits = p.splits > kMaxSplits ? kMaxSplits : p.splits;
    const int64_t rows = tokens * group;
    const int64_t big = p.decode ? (rows / (kFewRows + 1) < requests ? rows / (kFewRows + 1) : requests) : 1;   // requests with more rows
    p.tiles = p.chunk ? clamp(p.decode ? rows / kTileRows + big : ceil_div(rows, kTileRows), INT32_MAX) : 0;
    p.chunk_splits = p.chunk ? clamp(512 / ((int64_t)p.tiles * c.heads), ceil_div(max_len, 512)) : 1;
    p.chunk_splits = p.chunk_splits > kMaxSplits ? kMaxSplits : p.chunk_splits;
    const size_t part = (size_t)c.dim * 4 + 8;
    const size_t few = p.decode && p.splits > 1 ? (size_t)units * p.part_rows * p.splits * part : 0;
    const size_t many = p.chunk && p.chunk_splits > 1 ? (size_t)p.tiles * c.heads * kTileRows * p.chunk_splits * part : 0;
    p.bytes = ((few > many ? few : many) + 255) / 256 * 256 + kCounterBytes;
    return p;
}

template <int TYPE, int DT, int BLOCK>
mx_status launch_kernels(CacheAttnArgs a, const Plan& p, uint8_t* workspace, hipStream_t stream) {
    const int64_t units = (int64_t)a.requests * a.heads;
    a.fill = 1;
    if (p.decode) {
        a.least = 1;
        a.most = p.chunk ? kFewRows : INT32_MAX;
        a.splits = p.splits;
        a.part_rows = p.part_rows;
        const int64_t rows = units * p.part_rows;
        a.part_o = (float*)(workspace + kCounterBytes);
        a.part_ml = (float2*)(a.part_o + rows * p.splits * a.dim);
        cache_decode_kernel<TYPE, DT, BLOCK><<<(unsigned)(units * p.splits), 256, 0, stream>>>(a);
        MX_HIP_LAUNCH_CHECK();
        a.fill = 0;
        if (p.splits > 1) {
            cache_join_kernel<TYPE, false><<<(unsigned)rows, 256, 0, stream>>>(a);
            MX_HIP_LAUNCH_CHECK();
        }
    }
    if (p.chunk) {
        a.least = p.decode ? kFewRows + 1 : 1;
        a.most = INT32_MAX;
        a.splits = p.chunk_splits;
        a.tiles = p.tiles;
        a.part_rows = kTileRows;
        const int64_t rows = (int64_t)p.tiles * a.heads * kTileRows;
        a.part_o = (float*)(workspace + kCounterBytes);
        a.part_ml = (float2*)(a.part_o + rows * p.chunk_splits * a.dim);
        constexpr int lds = 4 * kTileKeys<TYPE> * DT * 2;
        static std::atomic<uint64_t> raised{0};
        if (lds > 60 * 1024 && !allow_dynamic_lds((const void*)cache_chunk_kernel<TYPE, DT, BLOCK>, lds, raised)) return MX_ERR_DEVICE;
        cache_chunk_kernel<TYPE, DT, BLOCK><<<(unsigned)((int64_t)p.tiles * a.heads * p.chunk_splits), 256, lds, stream>>>(a);
        MX_HIP_LAUNCH_CHECK();
        if (p.chunk_splits > 1) {
            cache_join_kernel<TYPE, true><<<(unsigned)rows, 256, 0, stream>>>(a);
            MX_HIP_LAUNCH_CHECK();
        }
    }
    return MX_OK;
}

template <int TYPE>
mx_status launch(const CacheAttnArgs& a, const Plan& p, int block, uint8_t* workspace, hipStream_t stream) {
    if (a.requests == 0) {
        cache_zero_kernel<TYPE><<<(unsigned)a.tokens, 256, 0, stream>>>(a);
        MX_HIP_LAUNCH_CHECK();
        return MX_OK;
    }
    if (a.dim <= 64)
        return block == 0 ? launch_kernels<TYPE, 64, 0>(a, p, workspace, stream)
               : block == 16 ? launch_kernels<TYPE, 64, 16>(a, p, workspace, stream) : launch_kernels<TYPE, 64, 32>(a, p, workspace, stream);
    return block == 0 ? launch_kernels<TYPE, 128, 0>(a, p, workspace, stream)
           : block == 16 ? launch_kernels<TYPE, 128, 16>(a, p, workspace, stream) : launch_kernels<TYPE, 128, 32>(a, p, workspace, stream);
}

bool attention_args_ok(const mx_cache& c, int64_t tokens, int64_t requests, int32_t heads_q, int64_t max_new, int64_t max_len) {
    return tokens >= 0 && requests >= 0 && heads_q >= 1 && c.heads >= 1 && heads_q % c.heads == 0 && max_new >= 1 && max_len >= 1;
}
bool attention_supported(const mx_cache& c, int64_t tokens, int64_t requests, int32_t heads_q) {
    return requests <= kCacheMaxRequests && tokens < ((int64_t)1 << 31) / heads_q && requests * c.heads < ((int64_t)1 << 24);
}

}  // namespace
}  // namespace mx

using namespace mx;

extern "C" size_t mx_cache_attention_workspace_bytes(mx_cache c, int64_t tokens, int64_t requests, int32_t heads_q, int64_t max_new,
                                                     int64_t max_len) {
    if (cache_status(c) != MX_OK || !attention_args_ok(c, tokens, requests, heads_q, max_new, max_len) ||
        !attention_supported(c, tokens, requests, heads_q))
        return 0;
    return plan_of(c, tokens, requests, heads_q, max_new, max_len).bytes;
}

extern "C" mx_status mx_cache_attention(const void* q, int32_t type, int64_t tokens, int64_t ldq, int32_t heads_q, mx_cache c,
                                        const void* k_data, const uint8_t* k_exps, const void* v_data, const uint8_t* v_exps,
                                        const int32_t* table, int64_t width, const int32_t* q_start, const int32_t* kv_len,
                                        int64_t requests, int64_t max_new, int64_t max_len, float scale, void* workspace, void* out,
                                        int64_t ldo, void* stream) {
    if (type != MX_F32 && type != MX_BF16) return MX_ERR_BAD_ARG;
    const mx_status st = cache_status(c);
    if (st == MX_ERR_BAD_ARG || !attention_args_ok(c, tokens, requests, heads_q, max_new, max_len)) return MX_ERR_BAD_ARG;
    if (!__builtin_isfinite(scale) || width < 0) return MX_ERR_BAD_ARG;
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
        }
    }
    if (st != MX_OK) return st;
    if (!attention_supported(c, tokens, requests, heads_q) || width > INT32_MAX / c.page) return MX_ERR_UNSUPPORTED;
    if (tokens == 0) return MX_OK;
    const Plan p = plan_of(c, tokens, requests, heads_q, max_new, max_len);
    if ((int64_t)p.tiles * c.heads * (p.chunk_splits > 1 ? kTileRows : 1) > INT32_MAX) return MX_ERR_UNSUPPORTED;
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
    a.exp_shift = (1 << (c.f.exp_bits - 1)) - 1 + 6;
    a.vec_q = aligned(q, 16) && ldq % (16 / tb) == 0;
    a.vec_o = aligned(out, 4 * tb) && ldo % 4 == 0;
    a.c = __builtin_fmaxf(__builtin_fabsf(scale) * 1.4426950408889634f, 0x1p-126f);   // never 0: minus infinity stays a mask
    a.flip = scale < 0.f ? 0x80000000u : 0u;
    uint8_t* ws = (uint8_t*)workspace;
    return type == MX_F32 ? launch<MX_F32>(a, p, c.f.block, ws, (hipStream_t)stream) : launch<MX_BF16>(a, p, c.f.block, ws, (hipStream_t)stream);
}
