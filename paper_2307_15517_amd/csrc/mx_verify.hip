// Verification of drafted tokens against the model's logits, from given random numbers.
#include <type_traits>

#include "mx_cache.h"

namespace mx {
namespace {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef f4 f4u __attribute__((aligned(4)));          // rows of odd lengths start anywhere: 16 bytes from any element on
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef u4 u4u __attribute__((aligned(2)));

struct VerifyArgs {
    const void* logits;
    const void* draft;         // null: drafted tokens count as certain
    const int32_t* ids;
    const int32_t* parents;
    const int32_t* q_start;
    const float* temperature;
    const float* uniform;
    const float* noise;
    int32_t* path;
    int32_t* kept;
    int32_t* next;
    int64_t tokens, ldl, ldd, ldn, width;
    int32_t vocab, requests;
};

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr size_t kCounterBytes = 65536;
constexpr int kNodes = MX_TREE_MAX_NODES;

// 2^((x) log2(e) / T), x <= 0: the factor as two floats, and what the product is rounded by as a factor of the result, so that the
// result is off by little more than the instruction's last bit however large x is.
struct Heat {
    float hi, lo;
    double inv;
    __device__ __forceinline__ explicit Heat(float t) {
        inv = 1.0 / fmin(fmax((double)t, 1e-30), 1e30);     // so that 0 and minus infinity times it are what they are
        const double c = inv * 1.4426950408889634;
        hi = (float)c;
        lo = (float)(c - (double)hi);
    }
    __device__ __forceinline__ float exp_of(float x) const {
        const float y = x * hi, rest = __builtin_fmaf(x, hi, -y) + x * lo;
        const float e = __builtin_amdgcn_exp2f(y);
        return y < -126.f ? 0.f : __builtin_fmaf(e, rest * 0.6931471805599453f, e);
    }
};

template <int TYPE>
__device__ __forceinline__ float value_at(const void* row, int64_t i) {
    if constexpr (TYPE == MX_F32) return static_cast<const float*>(row)[i];
    else return __uint_as_float((uint32_t)static_cast<const uint16_t*>(row)[i] << 16);
}
template <int TYPE>
__device__ __forceinline__ void values8(const void* row, int64_t i, float (&v)[8]) {
    if constexpr (TYPE == MX_F32) {
        const float* p = static_cast<const float*>(row) + i;
        const f4 a = *reinterpret_cast<const f4u*>(p), b = *reinterpret_cast<const f4u*>(p + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) { v[e] = a[e]; v[4 + e] = b[e]; }
    } else {
        const u4 a = *reinterpret_cast<const u4u*>(static_cast<const uint16_t*>(row) + i);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[2 * e] = __uint_as_float(a[e] << 16);
            v[2 * e + 1] = __uint_as_float(a[e] & 0xffff0000u);
        }
    }
}

template <int TYPE>
__device__ __forceinline__ const void* row_at(const void* base, int64_t element) {
    return static_cast<const char*>(base) + element * (TYPE == MX_F32 ? 4 : 2);
}

// What a pass over a row of logits finds: the largest and the first place that has it, the sum of exp((x - top) / T), and of the
// race exp((x - top) / T) / noise the winner, the first of equal ones, among the tokens that are not tried as children.
struct Found {
    float top;
    int top_at;
    double sum;
    float best;
    int best_at;               // -1: none with a probability above 0
};

struct Child {
    int node, token;
    float uniform;
    bool tried_before;         // an earlier sibling has the same token
    double p, q;
};

struct Shared {
    float top[kWaves];
    int top_at[kWaves];
    double sum[kWaves];
    float best[kWaves];
    int best_at[kWaves];
    Child child[kNodes];
};

__device__ __forceinline__ bool is_child(const Shared& s, int children, int token) {
    for (int k = 0; k < children; ++k)
        if (s.child[k].token == token) return true;
    return false;
}

// The parts of all threads as one, the same in every thread.
__device__ __forceinline__ Found join(Found f, const Heat& heat, Shared& s) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    auto add = [&](float top, int top_at, double sum, float best, int best_at) __attribute__((always_inline)) {
        const float m = __builtin_fmaxf(f.top, top);
        const float mine = f.top == m ? 1.f : heat.exp_of(f.top - m), its = top == m ? 1.f : heat.exp_of(top - m);
        f.top_at = f.top > top ? f.top_at : top > f.top ? top_at : min(f.top_at, top_at);
        f.top = m;
        f.sum = f.sum * mine + sum * its;
        const float x = f.best * mine, y = best * its;
        f.best_at = x > y ? f.best_at : y > x ? best_at : (int)min((uint32_t)f.best_at, (uint32_t)best_at);
        f.best = __builtin_fmaxf(x, y);
    };
#pragma unroll
    for (int d = 1; d < 64; d *= 2)
        add(__shfl_xor(f.top, d), __shfl_xor(f.top_at, d), __shfl_xor(f.sum, d), __shfl_xor(f.best, d), __shfl_xor(f.best_at, d));
    __syncthreads();
    if (lane == 0) {
        s.top[wave] = f.top;
        s.top_at[wave] = f.top_at;
        s.sum[wave] = f.sum;
        s.best[wave] = f.best;
        s.best_at[wave] = f.best_at;
    }
    __syncthreads();
    f = Found{s.top[0], s.top_at[0], s.sum[0], s.best[0], s.best_at[0]};
    for (int w = 1; w < kWaves; ++w) add(s.top[w], s.top_at[w], s.sum[w], s.best[w], s.best_at[w]);
    return f;
}

// RACE: with the race against the random numbers; `children` of s.child do not take part in it.
template <int TYPE, bool RACE>
__device__ __forceinline__ Found pass(const VerifyArgs& a, const void* row, const float* noise, const Heat& heat, int children, Shared& s) {
    Found f{-__builtin_inff(), INT_MAX, 0.0, 0.f, -1};
    auto take = [&](int at, const float* x, const float* z, auto count_c) __attribute__((always_inline)) {
        constexpr int N = decltype(count_c)::value;
        float top = x[0];
#pragma unroll
        for (int e = 1; e < N; ++e) top = __builtin_fmaxf(top, x[e]);
        if (top > f.top) {
#pragma unroll
            for (int e = N - 1; e >= 0; --e)
                if (x[e] == top) f.top_at = at + e;
            const float less = f.top == -__builtin_inff() ? 0.f : heat.exp_of(f.top - top);
            f.sum *= less;
            f.best *= less;
            f.top = top;
        }
        if (f.top == -__builtin_inff()) return;
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float p = heat.exp_of(x[e] - f.top);
            sum += p;
            if constexpr (RACE) {
                const float score = p / z[e];
                if (score > f.best && !is_child(s, children, at + e)) {
                    f.best = score;
                    f.best_at = at + e;
                }
            }
        }
        f.sum += sum;
    };
    const int octets = a.vocab / 8;
    for (int o = threadIdx.x; o < octets; o += kThreads) {
        float x[8], z[8];
        values8<TYPE>(row, 8 * (int64_t)o, x);
        if constexpr (RACE) values8<MX_F32>(noise, 8 * (int64_t)o, z);
        take(8 * o, x, z, std::integral_constant<int, 8>{});
    }
    if (const int at = 8 * octets + threadIdx.x; at < a.vocab) {
        float x[1] = {value_at<TYPE>(row, at)}, z[1] = {RACE ? noise[at] : 1.f};
        take(at, x, z, std::integral_constant<int, 1>{});
    }
    return join(f, heat, s);
}

// r = max(p - c q, 0): its sum, or with RACE the winner of r / noise.
template <int TYPE, bool RACE>
__device__ __forceinline__ Found residual(const VerifyArgs& a, const void* row, const Found& p, const void* drafted, const Found& q, double c,
                                          const float* noise, const Heat& heat, Shared& s) {
    const float fp = (float)(1.0 / p.sum), fq = (float)(c / q.sum);
    Found f{0.f, 0, 0.0, 0.f, -1};
    auto take = [&](int at, float x, float y, float z) __attribute__((always_inline)) {
        const float r = __builtin_fmaxf(__builtin_fmaf(heat.exp_of(x - p.top), fp, -(heat.exp_of(y - q.top) * fq)), 0.f);
        if constexpr (RACE) {
            const float score = r / z;
            if (score > f.best) {
                f.best = score;
                f.best_at = at;
            }
        }
        return r;
    };
    const int octets = a.vocab / 8;
    for (int o = threadIdx.x; o < octets; o += kThreads) {
        float x[8], y[8], z[8], sum = 0.f;
        values8<TYPE>(row, 8 * (int64_t)o, x);
        values8<TYPE>(drafted, 8 * (int64_t)o, y);
        if constexpr (RACE) values8<MX_F32>(noise, 8 * (int64_t)o, z);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += take(8 * o + e, x[e], y[e], z[e]);
        f.sum += sum;
    }
    if (const int at = 8 * octets + threadIdx.x; at < a.vocab)
        f.sum += take(at, value_at<TYPE>(row, at), value_at<TYPE>(drafted, at), RACE ? noise[at] : 1.f);
    return join(f, heat, s);
}

// A workgroup a request: it reads the rows of the nodes that the walk comes to, one after another.
template <int TYPE>
__global__ __launch_bounds__(kThreads) void verify_kernel(VerifyArgs a) {
    __shared__ Shared s;
    const int b = blockIdx.x, lane = threadIdx.x & 63;
    const int64_t lo = a.q_start[b], hi = a.q_start[b + 1];
    const int64_t t0 = lo < 0 ? 0 : lo > a.tokens ? a.tokens : lo, t1 = hi > a.tokens ? a.tokens : hi;
    const int n = (int)min(max(t1 - t0, (int64_t)0), (int64_t)kNodes);
    const float t = a.temperature[b];
    const bool cold = !(t > 0.f);
    const Heat heat(cold ? 1.f : t);
    const float* noise = a.noise + b * a.ldn;
    int64_t kept = n > 0;
    int node = 0, next = -1;
    if (threadIdx.x == 0 && n > 0) a.path[b * a.width] = 0;
    while (n > 0) {
        // the children, in the order of their numbers
        int children = 0;
        if (kept < a.width) {
            __syncthreads();
            for (int base = node + 1; base < n; base += 64) {
                const int i = base + lane;
                const bool is = i < n && a.parents[t0 + i] == node;
                const uint64_t all = __ballot(is);
                if (is && threadIdx.x < 64) {
                    Child& c = s.child[children + __popcll(all & ((1ull << lane) - 1))];
                    c.node = i;
                    c.token = a.ids[t0 + i];
                    c.uniform = a.uniform[t0 + i];
                }
                children += __popcll(all);
            }
            __syncthreads();
        }
        const void* row = row_at<TYPE>(a.logits, (t0 + node) * a.ldl);
        const void* drafted = a.draft ? row_at<TYPE>(a.draft, (t0 + node) * a.ldd) : nullptr;
        const bool with_q = drafted != nullptr && children > 0 && !cold;
        const Found p = cold || with_q ? pass<TYPE, false>(a, row, noise, heat, 0, s) : pass<TYPE, true>(a, row, noise, heat, children, s);
        Found q{};
        if (with_q) q = pass<TYPE, false>(a, drafted, noise, heat, 0, s);
        if (cold) {
            int to = -1;
            for (int k = 0; k < children && to < 0; ++k)
                if (s.child[k].token == p.top_at && p.top > -__builtin_inff()) to = s.child[k].node;
            if (to < 0) {
                next = p.top == -__builtin_inff() ? -1 : p.top_at;
                break;
            }
            node = to;
        } else {
            for (int k = threadIdx.x; k < children; k += kThreads) {
                Child& c = s.child[k];
                const bool in = c.token >= 0 && c.token < a.vocab;
                bool before = !in;
                for (int j = 0; j < k && !with_q; ++j) before |= s.child[j].token == c.token;
                c.tried_before = before;
                c.p = in && p.sum > 0 ? exp(((double)value_at<TYPE>(row, in ? c.token : 0) - (double)p.top) * heat.inv) / p.sum : 0.0;
                c.q = !with_q ? 1.0 : in && q.sum > 0 ? exp(((double)value_at<TYPE>(drafted, in ? c.token : 0) - (double)q.top) * heat.inv) / q.sum : 0.0;
            }
            __syncthreads();
            int to = -1;
            double mass = 1.0, c = 0.0;
            for (int k = 0; k < children; ++k) {
                const Child& d = s.child[k];
                const double r = with_q ? fmax(d.p - c * d.q, 0.0) : d.tried_before ? 0.0 : d.p;
                if ((double)d.uniform * mass * d.q < r) {
                    to = d.node;
                    break;
                }
                if (!with_q) {
                    mass = fmax(mass - r, 0.0);
                } else {
                    c += mass;
                    if (k + 1 < children) mass = residual<TYPE, false>(a, row, p, drafted, q, c, noise, heat, s).sum;
                }
            }
            if (to < 0) {
                int best = p.best_at;
                if (with_q) best = residual<TYPE, true>(a, row, p, drafted, q, c, noise, heat, s).best_at;
                if (best < 0 && p.top > -__builtin_inff()) best = pass<TYPE, true>(a, row, noise, heat, 0, s).best_at;   // nothing is left: from p itself
                next = best;
                break;
            }
            node = to;
        }
        if (threadIdx.x == 0) a.path[b * a.width + kept] = node;
        ++kept;
    }
    for (int64_t i = kept + threadIdx.x; i < a.width; i += kThreads) a.path[b * a.width + i] = -1;
    if (threadIdx.x == 0) {
        a.kept[b] = (int32_t)kept;
        a.next[b] = next;
    }
}

}  // namespace
}  // namespace mx

using namespace mx;

extern "C" size_t mx_verify_workspace_bytes(int64_t tokens, int64_t requests, int64_t vocab) {
    if (tokens < 0 || requests < 0 || vocab < 1 || requests > kCacheMaxRequests || tokens > INT32_MAX || vocab > MX_VERIFY_MAX_VOCAB) return 0;
    return kCounterBytes;
}

extern "C" mx_status mx_verify(const void* logits, const void* draft, int32_t type, int64_t tokens, int64_t vocab, int64_t ldl, int64_t ldd,
                               const int32_t* ids, const int32_t* parents, const int32_t* q_start, int64_t requests,
                               const float* temperature, const float* uniform, const float* noise, int64_t ldn, void* workspace,
                               int32_t* path, int64_t path_width, int32_t* kept, int32_t* next, void* stream) {
    if (type != MX_F32 && type != MX_BF16) return MX_ERR_BAD_ARG;
    if (tokens < 0 || requests < 0 || vocab < 1 || path_width < 1) return MX_ERR_BAD_ARG;
    if (requests > 0) {
        if (q_start == nullptr || temperature == nullptr || path == nullptr || kept == nullptr || next == nullptr) return MX_ERR_BAD_ARG;
        if (tokens > 0 && (logits == nullptr || ids == nullptr || parents == nullptr || uniform == nullptr || noise == nullptr || workspace == nullptr))
            return MX_ERR_BAD_ARG;
        if (ldl < vocab || (draft != nullptr && ldd < vocab) || ldn < vocab) return MX_ERR_BAD_ARG;
        if (!aligned(logits, type_bytes(type)) || !aligned(draft, type_bytes(type)) || !aligned(workspace, 256)) return MX_ERR_BAD_ARG;
        for (const void* p : {(const void*)ids, (const void*)parents, (const void*)q_start, (const void*)temperature, (const void*)uniform,
                              (const void*)noise, (const void*)path, (const void*)kept, (const void*)next})
            if (!aligned(p, 4)) return MX_ERR_BAD_ARG;
    }
    if (requests > kCacheMaxRequests || tokens > INT32_MAX || vocab > MX_VERIFY_MAX_VOCAB || path_width > INT32_MAX) return MX_ERR_UNSUPPORTED;
    if (requests == 0) return MX_OK;
    VerifyArgs a{logits, draft, ids, parents, q_start, temperature, uniform, noise, path, kept, next, tokens, ldl, ldd, ldn, path_width,
                 (int32_t)vocab, (int32_t)requests};
    if (type == MX_F32) verify_kernel<MX_F32><<<(unsigned)requests, kThreads, 0, (hipStream_t)stream>>>(a);
    else verify_kernel<MX_BF16><<<(unsigned)requests, kThreads, 0, (hipStream_t)stream>>>(a);
    MX_HIP_LAUNCH_CHECK();
    return MX_OK;
}
