// The paged key/value cache as its kernels see it.
#pragma once

#include "mx_common.h"

namespace mx {

constexpr int kCacheMaxRequests = 16384;

inline bool cache_page_ok(int32_t page) { return page >= 16 && page <= 1024 && (page & (page - 1)) == 0; }
inline int log2_of(int32_t power_of_two) { return __builtin_ctz((unsigned)power_of_two); }

// MX_OK when the kernels take this cache.
inline mx_status cache_status(const mx_cache& c) {
    if (c.pages < 1 || c.page < 1 || c.heads < 1 || c.dim < 1) return MX_ERR_BAD_ARG;
    const mx_format& f = c.f;
    if (f.block != 0 && (!format_ok_quant(f) || c.dim % f.block != 0)) return MX_ERR_BAD_ARG;
    if (!cache_page_ok(c.page) || c.dim % 16 != 0 || c.dim > 128 || c.heads > 65535) return MX_ERR_UNSUPPORTED;
    if (c.pages > ((int64_t)1 << 31) / c.page - 1) return MX_ERR_UNSUPPORTED;
    if (f.block != 0 && ((f.block != 16 && f.block != 32) || f.mant_bits != 8 || f.block_rows != 1)) return MX_ERR_UNSUPPORTED;
    return MX_OK;
}

// An exponent byte e stands for 2^(e - bias) of a block's elements.  With bfloat16 elements the format's other fields may be anything.
inline int exponent_bias(const mx_cache& c) { return c.f.block == 0 ? 0 : (1 << (c.f.exp_bits - 1)) - 1; }

inline bool aligned(const void* p, uintptr_t n) { return (uintptr_t)p % n == 0; }

// Floats of type MX_F32 or MX_BF16: bytes, and eight of them from memory that is (VEC) or need not be 16-byte aligned.
inline int type_bytes(int32_t type) { return type == MX_F32 ? 4 : 2; }

template <int TYPE, bool VEC>
__device__ __forceinline__ void load8(const void* base, int64_t element, float (&v)[8]) {
    if constexpr (TYPE == MX_F32) {
        const float* p = static_cast<const float*>(base) + element;
        if constexpr (VEC) {
            const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
            v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = p[i];
        }
    } else {
        const uint16_t* p = static_cast<const uint16_t*>(base) + element;
        if constexpr (VEC) {
            const uint4 a = *reinterpret_cast<const uint4*>(p);
            const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[2 * i] = __uint_as_float(w[i] << 16);
                v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = __uint_as_float((uint32_t)p[i] << 16);
        }
    }
}

// Two floats to the nearest bfloat16 numbers, ties to even, NaN stays NaN: one instruction on gfx950.
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
    v2bf r;
    r[0] = (__bf16)lo;
    r[1] = (__bf16)hi;
    return __builtin_bit_cast(uint32_t, r);
}

}  // namespace mx
