// Attention of new tokens over the paged key/value cache, causal, grouped heads.
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
    float* part_o;             // [splits][tokens * heads_q][dim], unnormalised
    float2* part_ml;           // [splits][tokens * heads_q]: row maximum (exp2 domain), row sum
    int64_t tokens;
    int64_t max_keys;          // width * page
    uint32_t pages;
    int32_t requests, heads, group, heads_q, dim;
    int32_t page_log2;
    int32_t exp_shift;         // an exponent byte e stands for 2^(e - exp_shift) per mantissa unit
    int32_t splits;
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

    const int split = blockIdx.x % a.splits;
    const int unit = blockIdx.x / a.splits;
    const int h = unit % a.heads, b = unit / a.heads;
    const Request rq = request_of(a, b);
    const int rows = rq.n * a.group;
    const int len = rq.len;
    // this split's run of keys, in whole blocks of 128
    const int blocks128 = (len + 127) >> 7;
    const int per = (blocks128 + a.splits - 1) / a.splits;
    const int begin = min(split * per * 128, len), end = min(begin + per * 128, len);
    const int32_t* row_table = a.table + (int64_t)b * a.width;
    const int page_mask = (1 << a.page_log2) - 1;
    const int dim = a.dim;

    for (int r0 = blockIdx.y * 16; r0 < rows; r0 += gridDim.y * 16) {
        // q: column n of the score product, elements d(step, g, i)
        const int r = min(r0 + n, rows - 1);
        const int tok = r / a.group, head = h * a.group + (r - tok * a.group);
        const int last = r0 + n < rows ? len - rq.n + tok : -1;           // the last key this row sees
        v4u qf[QP][NS];
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            const int d = BLOCK == 0 ? 32 * s + 8 * g : 64 * (s >> 1) + 16 * g + 8 * (s & 1);
            float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            if (d < dim) load8<TYPE, false>(a.q, (int64_t)(rq.t0 + tok) * a.ldq + (int64_t)head * dim + d, v);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t w[QP];
                pieces_of<QP>(__uint_as_float(__float_as_uint(v[2 * i]) ^ a.flip), __uint_as_float(__float_as_uint(v[2 * i + 1]) ^ a.flip), w);
#pragma unroll
                for (int p = 0; p < QP; ++p) qf[p][s][i] = w[p];
            }
        }
        // keys past the last one any row of this tile sees are left out
        const int tile_last = len - rq.n + min(r0 + 15, rows - 1) / a.group;
        const int stop = min(end, tile_last + 1);

        float m = -__builtin_inff(), l = 0.f;
        v4f o[NJ];
#pragma unroll
        for (int j = 0; j < NJ; ++j) o[j] = v4f{0.f, 0.f, 0.f, 0.f};

        for (int kb = begin + 32 * wave; kb < stop; kb += 128) {
            // the two runs of sixteen keys lie in one page each; a run past the end reads the last one again (masked)
            Block f;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int key = kb + 16 * t < len ? kb + 16 * t : (len - 1) & ~15;
                uint32_t id = (uint32_t)row_table[key >> a.page_log2];
                id = id < a.pages ? id : 0;
                const int64_t row = (((int64_t)id * a.heads + h) << a.page_log2) + (key & page_mask);
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
                    if constexpr (BLOCK != 0) f.ve[4 * t + i] = a.v_exps[(row + 4 * g + i) * (dim / BLOCK) + d / BLOCK];
                }
            }

            // scores
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
                            const int x = (int)f.k[t][step >> 1][2 * (step & 1) + (w >> 1)];
                            const float lo = (float)(int8_t)(x >> (16 * (w & 1))) * sc, hi = (float)(int8_t)(x >> (16 * (w & 1) + 8)) * sc;
                            kf[w] = __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
                        }
                    }
#pragma unroll
                    for (int p = QP - 1; p >= 0; --p)
                        s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, kf), __builtin_bit_cast(v8bf, qf[p][step]),
                                                                       s[t], 0, 0, 0);
                }
            }
            float top = -__builtin_inff();
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int key = kb + 16 * t + 4 * g + e;
                    s[t][e] = key <= last && key < stop ? s[t][e] : -__builtin_inff();
                    top = __builtin_fmaxf(top, s[t][e]);
                }
            top = max_across_16_32(top);
            const float m_new = top == -__builtin_inff() ? m : __builtin_fmaxf(m, top * a.c);
            const float m_use = m_new == -__builtin_inff() ? 0.f : m_new;
            const float alpha = exp2_of(m - m_use);
            m = m_new;
            float pr[8];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const bool seen = s[t][e] != -__builtin_inff();       // also where the scale is 0
                    pr[4 * t + e] = seen ? exp2_of(__builtin_fmaf(s[t][e], a.c, -m_use)) : 0.f;
                }
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += pr[e];
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
                        const float lo = (float)(int8_t)((int)f.v[2 * w][j >> 2] >> (8 * (j & 3))) * sc[2 * w];
                        const float hi = (float)(int8_t)((int)f.v[2 * w + 1][j >> 2] >> (8 * (j & 3))) * sc[2 * w + 1];
                        vf[w] = __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
                    }
                }
#pragma unroll
                for (int p = P - 1; p >= 0; --p)
                    o[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, vf), __builtin_bit_cast(v8bf, pf[p]), o[j],
                                                                   0, 0, 0);
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
        if (r0 + row < rows) {
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
            const int tk = (r0 + row) / a.group, hd = h * a.group + (r0 + row - tk * a.group);
            const int64_t token = rq.t0 + tk;
            if (VE * part < dim) {
                if (a.splits == 1) {
                    const float inv = ll > 0.f ? 1.f / ll : 0.f;
                    const int64_t at = token * a.ldo + (int64_t)hd * dim + VE * part;
#pragma unroll
                    for (int j = 0; j < VE; ++j) {
                        if constexpr (TYPE == MX_F32) static_cast<float*>(a.out)[at + j] = acc[j] * inv;
                        else static_cast<uint16_t*>(a.out)[at + j] = (uint16_t)pack_bf16(acc[j] * inv, 0.f);
                    }
                } else {
                    const int64_t at = (int64_t)split * a.tokens * a.heads_q + token * a.heads_q + hd;
                    if (part == 0) a.part_ml[at] = make_float2(mm, ll);
#pragma unroll
                    for (int j = 0; j < VE; ++j) a.part_o[at * dim + VE * part + j] = acc[j];
                }
            }
        }
    }
}

// Joins the splits, in their order; also writes the zeros of tokens outside every request.  A wave takes one row.
template <int TYPE>
__global__ __launch_bounds__(256) void cache_join_kernel(CacheAttnArgs a) {
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    const int64_t rows = a.tokens * a.heads_q;
    if (row >= rows) return;
    const int64_t t = row / a.heads_q;
    const int hd = (int)(row - t * a.heads_q);
    const bool inside = a.requests > 0 && t >= a.q_start[0] && t < a.q_start[a.requests];
    if (inside && a.splits == 1) return;
    float mm = -__builtin_inff();
    if (inside)
        for (int s = 0; s < a.splits; ++s) mm = __builtin_fmaxf(mm, a.part_ml[s * rows + row].x);
    float ll = 0.f, x0 = 0.f, x1 = 0.f;
    if (inside && mm != -__builtin_inff()) {
        for (int s = 0; s < a.splits; ++s) {
            const float2 ml = a.part_ml[s * rows + row];
            const float f = ml.x == -__builtin_inff() ? 0.f : exp2_of(ml.x - mm);
            ll += ml.y * f;
            const float* p = a.part_o + (s * rows + row) * a.dim;
            if (lane < a.dim) x0 += p[lane] * f;
            if (lane + 64 < a.dim) x1 += p[lane + 64] * f;
        }
    }
    const float inv = ll > 0.f ? 1.f / ll : 0.f;
    const int64_t at = t * a.ldo + (int64_t)hd * a.dim + lane;
    if constexpr (TYPE == MX_F32) {
        if (lane < a.dim) static_cast<float*>(a.out)[at] = x0 * inv;
        if (lane + 64 < a.dim) static_cast<float*>(a.out)[at + 64] = x1 * inv;
    } else {
        if (lane < a.dim) static_cast<uint16_t*>(a.out)[at] = (uint16_t)pack_bf16(x0 * inv, 0.f);
        if (lane + 64 < a.dim) static_cast<uint16_t*>(a.out)[at + 64] = (uint16_t)pack_bf16(x1 * inv, 0.f);
    }
}

struct Plan {
    int splits, row_tiles;
    size_t bytes;
};

Plan plan_of(const mx_cache& c, int64_t tokens, int64_t requests, int32_t heads_q, int64_t max_new, int64_t max_len) {
    Plan p;
    const int64_t group = heads_q / c.heads;
    const int64_t most = max_new < tokens ? max_new : tokens;
    int64_t tiles = ceil_div(most * group, 16);
    tiles = tiles < 1 ? 1 : tiles > 65535 ? 65535 : tiles;
    const int64_t units = tiles * requests * c.heads;
    int64_t s = units > 0 ? 1024 / units : 1;
    const int64_t by_len = ceil_div(max_len, 256);
    s = s > by_len ? by_len : s;
    s = s < 1 ? 1 : s > 128 ? 128 : s;
    p.splits = (int)s;
    p.row_tiles = (int)tiles;
    const size_t rows = (size_t)tokens * heads_q;
    p.bytes = kCounterBytes + (s > 1 ? s * rows * ((size_t)c.dim + 2) * 4 : 0);
    p.bytes = (p.bytes + 255) / 256 * 256;
    return p;
}

template <int TYPE, int DT, int BLOCK>
mx_status launch_decode(const CacheAttnArgs& a, const Plan& p, hipStream_t stream) {
    const dim3 grid((unsigned)((int64_t)a.requests * a.heads * p.splits), (unsigned)p.row_tiles);
    cache_decode_kernel<TYPE, DT, BLOCK><<<grid, 256, 0, stream>>>(a);
    MX_HIP_LAUNCH_CHECK();
    return MX_OK;
}

template <int TYPE>
mx_status launch(const CacheAttnArgs& a, const Plan& p, int block, hipStream_t stream) {
    mx_status st = MX_OK;
    if (a.requests > 0) {
        if (a.dim <= 64)
            st = block == 0 ? launch_decode<TYPE, 64, 0>(a, p, stream) : block == 16 ? launch_decode<TYPE, 64, 16>(a, p, stream)
                 : launch_decode<TYPE, 64, 32>(a, p, stream);
        else
            st = block == 0 ? launch_decode<TYPE, 128, 0>(a, p, stream) : block == 16 ? launch_decode<TYPE, 128, 16>(a, p, stream)
                 : launch_decode<TYPE, 128, 32>(a, p, stream);
    }
    if (st != MX_OK) return st;
    cache_join_kernel<TYPE><<<(unsigned)ceil_div(a.tokens * a.heads_q, 4), 256, 0, stream>>>(a);
    MX_HIP_LAUNCH_CHECK();
    return MX_OK;
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
    CacheAttnArgs a{};
    a.q = q; a.out = out; a.ldq = ldq; a.ldo = ldo;
    a.k = (const uint8_t*)k_data; a.v = (const uint8_t*)v_data;
    a.k_exps = k_exps; a.v_exps = v_exps;
    a.table = table; a.width = width; a.q_start = q_start; a.kv_len = kv_len;
    a.part_ml = (float2*)((char*)workspace + kCounterBytes);
    a.part_o = (float*)(a.part_ml + (size_t)p.splits * tokens * heads_q);
    a.tokens = tokens;
    a.max_keys = width * c.page;
    a.pages = (uint32_t)c.pages;
    a.requests = (int32_t)requests; a.heads = c.heads; a.group = heads_q / c.heads; a.heads_q = heads_q; a.dim = c.dim;
    a.page_log2 = log2_of(c.page);
    a.exp_shift = (1 << (c.f.exp_bits - 1)) - 1 + 6;
    a.splits = p.splits;
    a.c = __builtin_fabsf(scale) * 1.4426950408889634f;
    a.flip = scale < 0.f ? 0x80000000u : 0u;
    return type == MX_F32 ? launch<MX_F32>(a, p, c.f.block, (hipStream_t)stream) : launch<MX_BF16>(a, p, c.f.block, (hipStream_t)stream);
}
