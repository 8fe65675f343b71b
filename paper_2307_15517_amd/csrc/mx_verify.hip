// Verification of drafted tokens against the model's logits, from given random numbers.  (Compiled with MX_VERIFY_EARLY=1 for a test: the
// workspace says who does not wait for whom.)
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
    struct Control* control;
    uint64_t* parts;           // [request][2][kSlots][3]
    int32_t team;              // workgroups a request
    int32_t finest;            // segments of a row, at most
    int32_t wide;              // a request with so many nodes or fewer has the rows of all of them read at once
    int32_t ahead;             // else so many children's rows with a node's
};

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kNodes = MX_TREE_MAX_NODES;
constexpr int kMostRows = 16;              // nodes whose rows are read at once
constexpr int kMostSegments = 64;          // of a row, a lane each where they are joined
constexpr int kMostMembers = 1024, kMostTeams = 512;
constexpr int kSlots = 64 * kWaves + 2 * kMostRows;   // parts of a job: rows times segments, no more than the waves of a team or the rows
constexpr int kExcluded = 16;
constexpr int kMostPolls = 512;
constexpr size_t kControlBytes = 65536;

// exp(x / T).  The subtraction that gives x, the factor and the product are rounded once each, which moves the exponent y (of e) by 3 |y| 2^-24 at
// most; the instruction is off by one unit in the last place, 2 2^-24.  A row's exponentials are rescaled on the way to its top, through steps
// of T or more and three others (the end of the lane's part, the wave, the row), each with an error of that kind; a value may lie T above
// what it is first taken against.  In all 3 (y + 2) + 2 (y + 1) + 2 (1 + 3) = 5 y + 16 of 2^-24.
struct Heat {
    float t;                   // T
    float scale;               // log2(e) / T
    double inv;                // 1 / T
    __device__ __forceinline__ explicit Heat(float temperature) {
        t = (float)fmin(fmax((double)temperature, 1e-30), 1e30);    // so that 0 and minus infinity times 1 / T are what they are
        inv = 1.0 / (double)t;
        scale = (float)(inv * 1.4426950408889634);
    }
    __device__ __forceinline__ float exp_of(float x) const { return __builtin_amdgcn_exp2f(x * scale); }
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

// 1 / noise, no more than 2^126, so that no score is infinite: exponentials are no larger than e where they meet it
__device__ __forceinline__ float inverse_of(float noise) { return __builtin_amdgcn_rcpf(__builtin_amdgcn_fmed3f(noise, 0x1p-126f, 0x1p127f)); }

// All lanes' values as one, in every lane, without LDS: neighbours, quads, rows of sixteen mirrored, then the rows.
template <int STEP>
__device__ __forceinline__ void pair_of(uint32_t v, uint32_t& x, uint32_t& y) {
    if constexpr (STEP < 4) {
        constexpr int ctrl = STEP == 0 ? 0xB1 : STEP == 1 ? 0x4E : STEP == 2 ? 0x141 : 0x140;
        x = v;
        y = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, ctrl, 0xF, 0xF, true);
    } else {
        const auto r = STEP == 4 ? __builtin_amdgcn_permlane16_swap(v, v, false, false) : __builtin_amdgcn_permlane32_swap(v, v, false, false);
        x = r[0];
        y = r[1];
    }
}
template <int STEP = 0, typename Op>
__device__ __forceinline__ uint32_t over_wave(uint32_t v, Op op) {
    if constexpr (STEP == 6) {
        return v;
    } else {
        uint32_t x, y;
        pair_of<STEP>(v, x, y);
        return over_wave<STEP + 1>(op(x, y), op);
    }
}
template <int STEP = 0, typename Op>
__device__ __forceinline__ uint64_t over_wave64(uint64_t v, Op op) {
    if constexpr (STEP == 6) {
        return v;
    } else {
        uint32_t x0, y0, x1, y1;
        pair_of<STEP>((uint32_t)v, x0, y0);
        pair_of<STEP>((uint32_t)(v >> 32), x1, y1);
        return over_wave64<STEP + 1>(op((uint64_t)x1 << 32 | x0, (uint64_t)y1 << 32 | y0), op);
    }
}

// What a pass over a part of a row finds: the largest and the first place that has it, the sum of exp((x - top) / T), and of the race
// exp((x - top) / T) / noise the winner, the first of equal ones, among the tokens that are not excluded.
struct Found {
    float top;
    int top_at;
    double sum;
    float best;
    int best_at;               // -1: none with a probability above 0

    // The parts of a wave's lanes as one
    __device__ __forceinline__ void join(const Heat& heat) {
        const float m = __uint_as_float(over_wave(__float_as_uint(top), [](uint32_t x, uint32_t y) {
            return __float_as_uint(__builtin_fmaxf(__uint_as_float(x), __uint_as_float(y)));
        }));
        const float f = top == m ? 1.f : heat.exp_of(top - m);
        top_at = (int)over_wave(top == m ? (uint32_t)top_at : INT_MAX, [](uint32_t x, uint32_t y) { return min(x, y); });
        top = m;
        sum = __builtin_bit_cast(double, over_wave64(__builtin_bit_cast(uint64_t, sum * f), [](uint64_t x, uint64_t y) {
            return __builtin_bit_cast(uint64_t, __builtin_bit_cast(double, x) + __builtin_bit_cast(double, y));
        }));
        // scores are not negative: their bits are in their order, and of equal ones the smaller place is to win
        best *= f;
        const uint64_t key = over_wave64(best > 0.f ? (uint64_t)__float_as_uint(best) << 32 | (uint32_t)~best_at : 0ull,
                                         [](uint64_t x, uint64_t y) { return x > y ? x : y; });
        best = __uint_as_float((uint32_t)(key >> 32));
        best_at = key == 0 ? -1 : (int)~(uint32_t)key;
    }
};
constexpr Found kNothing{-__builtin_inff(), INT_MAX, 0.0, 0.f, -1};

// What a team works on: rows of logits (kRows), or of one node what is left of p when c q is taken off, its sum (kSum) or the winner of its
// race (kRace; c < 0 stands for p itself, whatever was tried).
enum { kRows = 0, kSum = 1, kRace = 2 };
struct Job {
    int kind, node, kept;
    int next_child;            // kSum: where the next child is looked for
    float p_top, q_top;
    double c, mass, p_sum, q_sum;
};

// Of the workspace, zero before its first use and the calls' own from then on.  A call's number is `number`; the last of its workgroups that
// has read it puts the next one there.
struct Control {
    uint64_t number;
    uint32_t teams;                     // of this call, whose members have all read the number
    uint32_t early;                     // with MX_VERIFY_EARLY: from job number early & 0xffff on members do not look out for others, those
                                        // of odd numbers only with 1 << 16; 0: they do
    uint32_t members[kMostTeams];       // of a team
    uint64_t posted[kMostMembers];      // number << 16 | jobs done, of every member
};
static_assert(sizeof(Control) <= kControlBytes, "the workspace's first part");

struct Shared {
    Found found[2 * kMostRows];
    Job job;                            // (not in registers: the walk's state is read between the passes only)
    uint64_t part[kMostSegments][3];    // of a row that a workgroup reads alone
    int excluded[kWaves][kExcluded];
    uint32_t all_here;
    int parent[kNodes], id[kNodes];
    float uniform[kNodes], lp[kNodes], lq[kNodes];   // lp, lq: the logits of node i's token in the rows of its parent
};

__device__ __forceinline__ void put(uint64_t* p, uint64_t v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ uint64_t get(const uint64_t* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ uint64_t both(uint32_t lo, uint32_t hi) { return (uint64_t)hi << 32 | lo; }
// What this wave has stored is where every compute unit sees it
__device__ __forceinline__ void stored() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
    __builtin_amdgcn_s_waitcnt(0);
}

// Once for every workgroup, after it has read the call's number
__device__ __forceinline__ void team_counts_in(const VerifyArgs& a, int b, uint64_t number) {
    Control* c = a.control;
    if (__hip_atomic_fetch_add(&c->members[b], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != (uint32_t)a.team - 1) return;
    __hip_atomic_store(&c->members[b], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (__hip_atomic_fetch_add(&c->teams, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != (uint32_t)a.requests - 1) return;
    __hip_atomic_store(&c->teams, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    put(&c->number, number + 1);
}

// Sums of the lanes' values up to and including each
template <int CTRL, int ROWS>
__device__ __forceinline__ double moved(double v) {
    const uint64_t x = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)x, CTRL, ROWS, 0xF, ROWS == 0xF);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(x >> 32), CTRL, ROWS, 0xF, ROWS == 0xF);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double scan_wave(double v) {
    v += moved<0x111, 0xF>(v);                          // from the lane one before in the row of sixteen, two, four, eight
    v += moved<0x112, 0xF>(v);
    v += moved<0x114, 0xF>(v);
    v += moved<0x118, 0xF>(v);
    v += moved<0x142, 0xA>(v);                          // the first and third row's last lane to the row after
    v += moved<0x143, 0xC>(v);                          // the second row's last lane to the second half
    return v;
}

__device__ __forceinline__ double lane_of(double v, int lane) {
    const uint64_t x = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)x, lane), hi = __builtin_amdgcn_readlane((uint32_t)(x >> 32), lane);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

template <int TYPE>
struct Team {
    const VerifyArgs& a;
    Shared& s;
    int b, member, n;
    int64_t t0;
    bool cold, drafted;
    Heat heat;
    const float* noise;
    int lane, wave;
    int base, up, id;          // of node base + lane: parent, token, random number, its logits in its parent's rows
    float uniform, lp, lq;
    int nodes, row0, row1, row2;   // on the list of rows
    bool every;
    int segments;              // of a row, in this job: as many as give every wave of the team one

    __device__ __forceinline__ Team(const VerifyArgs& args, Shared& shared)
        : a(args), s(shared), b(blockIdx.x / args.team), member(blockIdx.x % args.team), heat(1.f), lane(threadIdx.x & 63),
          wave(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)), base(-1) {
        const int64_t lo = a.q_start[b], hi = a.q_start[b + 1];
        const float t = a.temperature[b];
        t0 = lo < 0 ? 0 : lo > a.tokens ? a.tokens : lo;
        const int64_t t1 = hi > a.tokens ? a.tokens : hi;
        n = (int)min(max(t1 - t0, (int64_t)0), (int64_t)kNodes);
        cold = !(t > 0.f);
        drafted = a.draft != nullptr && !cold;
        heat = Heat(cold ? 1.f : t);
        noise = a.noise + b * a.ldn;
    }
    __device__ __forceinline__ const void* logits_of(int node) const { return row_at<TYPE>(a.logits, (t0 + node) * a.ldl); }
    __device__ __forceinline__ const void* draft_of(int node) const { return row_at<TYPE>(a.draft, (t0 + node) * a.ldd); }

    // Lane i holds node base + i
    __device__ __forceinline__ void look_at(int to) {
        if (to == base) return;
        base = to;
        const int k = min(base + lane, kNodes - 1);
        up = base + lane < n ? s.parent[k] : -2;
        id = s.id[k];
        uniform = s.uniform[k];
        lp = s.lp[k];
        lq = s.lq[k];
    }
    // The logits of the nodes' tokens in their parents' rows, thread i of `step`: nothing needs them before the first decision
    __device__ __forceinline__ void look_up(int i, int step) const {
        for (; i < n; i += step) {
            const int p = s.parent[i], x = s.id[i];
            const bool in = p >= 0 && x >= 0 && x < a.vocab;
            s.lp[i] = in ? value_at<TYPE>(logits_of(p), x) : 0.f;
            s.lq[i] = in && a.draft != nullptr ? value_at<TYPE>(draft_of(p), x) : 0.f;
        }
    }
    // The first child of `node` from number `from` on, n when there is none
    __device__ __forceinline__ int child_from(int node, int from) {
        while (from < n) {
            look_at(from & ~63);
            const uint64_t is = __ballot(up == node) & ~0ull << (from & 63);
            if (is != 0) return __builtin_amdgcn_readfirstlane(base + __builtin_ctzll(is));
            from = base + 64;
        }
        return n;
    }
    // Without a draft: the first child that is accepted, -1 for none.  Both sides of the test are left as they are summed; a lane a child,
    // 64 nodes at a time: what its earlier siblings leave is the sum less theirs.
    __device__ __forceinline__ int first_accepted(int node, const Found& p) {
        double mass = p.sum;
        for (int at = (node + 1) & ~63; at < n; at += 64) {
            look_at(at);
            const uint64_t kids = __ballot(up == node);
            if (kids == 0) continue;
            bool again = false;                          // an earlier sibling has the same token
            for (uint64_t k = kids; k != 0; k &= k - 1) {
                const int i = __builtin_ctzll(k);
                again |= lane > i && id == __builtin_amdgcn_readlane(id, i);
                if (at > ((node + 1) & ~63) && tried_before(node, base + i)) again |= lane == i;
            }
            const bool counts = up == node && !again && id >= 0 && id < a.vocab && p.sum > 0.0;
            const double e = counts ? exp(((double)lp - (double)p.top) * heat.inv) : 0.0;
            const double upto = scan_wave(e);
            const uint64_t yes = __ballot(counts && (double)uniform * fmax(mass - (upto - e), 0.0) < e);
            if (yes != 0) return base + __builtin_ctzll(yes);
            mass = fmax(mass - lane_of(upto, 63), 0.0);
        }
        return -1;
    }
    // Whether a child of `node` before number `i` (which is looked at) has the same token
    __device__ __forceinline__ bool tried_before(int node, int i) {
        const int token = __builtin_amdgcn_readlane(id, i - base);
        if ((__ballot(up == node && id == token) & ((1ull << (i - base)) - 1)) != 0) return true;
        for (int at = (node + 1) & ~63; at < base; at += 64)
            if (__ballot(s.parent[at + lane] == node && s.id[at + lane] == token) != 0) return true;
        return false;
    }

    // The nodes whose rows the walk may come to next: all of a small tree, or the node and its first children, a.ahead (two) of them at most.  Each
    // counts for two rows, its logits and its draft's, when the draft plays a part.
    __device__ __forceinline__ void list_rows(int node, bool all) {
        every = all;
        nodes = all ? n : 1;
        if (all) return;
        row0 = node;
        row1 = a.ahead > 0 ? child_from(node, node + 1) : n;
        row2 = a.ahead > 1 && row1 < n ? child_from(node, row1 + 1) : n;
        nodes += (row1 < n) + (row2 < n);
    }
    __device__ __forceinline__ int rows() const { return drafted ? 2 * nodes : nodes; }
    __device__ __forceinline__ int node_of(int row) const {
        const int k = drafted ? row >> 1 : row;
        return __builtin_amdgcn_readfirstlane(every ? k : k == 0 ? row0 : k == 1 ? row1 : row2);
    }
    __device__ __forceinline__ int row_of(int node) const {              // -1: not on the list
        const int k = every ? node : node == row1 ? 1 : node == row2 ? 2 : -1;
        return k < 0 ? -1 : drafted ? 2 * k : k;
    }

    // Elements 8 o0 .. 8 o1 of a row (`tail`: and those behind them), by one wave; with `race` the race too, without the `excludes` tokens of
    // node's children that lie there.
    __device__ __forceinline__ Found scan(const void* row, int o0, int o1, bool tail, bool race, int node, int excludes) {
        Found f = kNothing;
        constexpr int U = 2;                       // octets of a lane at a time; the next ones are in flight
        float ref = -__builtin_inff();
        // N elements from place `at` on, none larger than ref + T
        auto take = [&](int at, const float* x, float* z, auto count_c) __attribute__((always_inline)) {
            constexpr int N = decltype(count_c)::value;
            float p[N];
            double sum[2] = {0.0, 0.0};
#pragma unroll
            for (int e = 0; e < N; ++e) {
                p[e] = heat.exp_of(x[e] - ref);
                sum[e & 1] += (double)p[e];
            }
            f.sum += sum[0] + sum[1];
            if (!race) return;
            auto exclude = [&](int token) __attribute__((always_inline)) {
#pragma unroll
                for (int e = 0; e < N; ++e) p[e] = token == at + e ? 0.f : p[e];
            };
            if (excludes <= kExcluded) {
                for (int k = 0; k < excludes; ++k) exclude(s.excluded[wave][k]);
            } else {                               // more than there is room for: all nodes are looked through
                for (int i = node + 1; i < n; ++i) exclude(s.parent[i] == node ? s.id[i] : -1);
            }
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float score = p[e] * inverse_of(z[e]);
                if (score > f.best) {
                    f.best = score;
                    f.best_at = at + e;
                }
            }
        };
        // exp((x - ref) / T) is what is added up: ref follows the top when it is left behind by T, and at the end, so that a row that rises all
        // along is rescaled no more often than its exponent grows.  The best score is rescaled in 64 bits, its roundings do not add up.
        double best = 0.0;
        auto raise = [&](float top) __attribute__((always_inline)) {
            const double less = ref == -__builtin_inff() ? 0.f : heat.exp_of(ref - top);
            if ((float)best != f.best) best = (double)f.best;         // another winner since
            best *= less;
            f.sum *= less;
            f.best = (float)best;
            ref = top;
        };
        float x[U][8], z[U][8], next_x[U][8], next_z[U][8];
        auto load = [&](int o) __attribute__((always_inline)) {
#pragma unroll
            for (int u = 0; u < U; ++u) values8<TYPE>(row, 8 * (int64_t)min(o + u * 64, o1 - 1), next_x[u]);
            if (race) {
#pragma unroll
                for (int u = 0; u < U; ++u) values8<MX_F32>(noise, 8 * (int64_t)min(o + u * 64, o1 - 1), next_z[u]);
            }
        };
        if (o0 < o1) load(o0 + lane);
#pragma unroll 1
        for (int o = o0; o < o1; o += 64 * U) {
            const int mine = o + lane;
            float top = -__builtin_inff();
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    x[u][e] = mine + u * 64 < o1 ? next_x[u][e] : -__builtin_inff();
                    if (race) z[u][e] = next_z[u][e];
                    top = __builtin_fmaxf(top, x[u][e]);
                }
            if (o + 64 * U < o1) load(mine + 64 * U);
            if (top > f.top) {
                f.top = top;
                if (cold) {
#pragma unroll
                    for (int e = 8 * U - 1; e >= 0; --e)
                        if (x[e / 8][e % 8] == top) f.top_at = 8 * (mine + e / 8 * 64) + e % 8;
                }
            }
            if (!cold && top - ref > heat.t) raise(top);
            if (!cold && ref > -__builtin_inff()) {
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (u == 0 || mine + u * 64 < o1) take(8 * (mine + u * 64), x[u], z[u], std::integral_constant<int, 8>{});
            }
        }
        if (const int at = 8 * o1 + lane; tail && at < a.vocab) {
            float x[1] = {value_at<TYPE>(row, at)}, z[1] = {race ? noise[at] : 1.f};
            if (x[0] > f.top) {
                f.top = x[0];
                f.top_at = at;
            }
            if (!cold && x[0] - ref > heat.t) raise(x[0]);
            if (!cold && ref > -__builtin_inff()) take(at, x, z, std::integral_constant<int, 1>{});
        }
        if (!cold && f.top > ref) raise(f.top);
        return f;
    }

    // r = max(p - c q, 0) of a part of the rows: its sum, and with `race` the winner of r / noise
    __device__ __forceinline__ Found residual(int o0, int o1, bool tail, bool race) {
        const Job& j = s.job;
        const int node = __builtin_amdgcn_readfirstlane(j.node);
        const bool whole = j.c < 0.0;
        const void* row = logits_of(node);
        const void* other = whole ? row : draft_of(node);
        const float fp = (float)(1.0 / j.p_sum), fq = whole ? 0.f : (float)(j.c / j.q_sum);
        const float p_top = j.p_top, q_top = whole ? j.p_top : j.q_top;
        Found f{0.f, 0, 0.0, 0.f, -1};
        constexpr int U = 2;
        auto take = [&](int at, const float* x, const float* y, const float* z, auto count_c) __attribute__((always_inline)) {
            constexpr int N = decltype(count_c)::value;
            double sum[2] = {0.0, 0.0};
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float r = __builtin_fmaxf(__builtin_fmaf(heat.exp_of(x[e] - p_top), fp, -(heat.exp_of(y[e] - q_top) * fq)), 0.f);
                sum[e & 1] += (double)r;
                const float score = r * inverse_of(z[e]);
                if (score > f.best) {
                    f.best = score;
                    f.best_at = at + e;
                }
            }
            f.sum += sum[0] + sum[1];
        };
#pragma unroll 1
        for (int o = o0 + lane; o < o1; o += 64 * U) {
            float x[U][8], y[U][8], z[U][8];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t at = 8 * (int64_t)min(o + u * 64, o1 - 1);
                values8<TYPE>(row, at, x[u]);
                values8<TYPE>(other, at, y[u]);
            }
            if (race) {
#pragma unroll
                for (int u = 0; u < U; ++u) values8<MX_F32>(noise, 8 * (int64_t)min(o + u * 64, o1 - 1), z[u]);
            } else {
#pragma unroll
                for (int e = 0; e < 8 * U; ++e) z[e / 8][e % 8] = 1.f;
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (o + u * 64 < o1) take(8 * (o + u * 64), x[u], y[u], z[u], std::integral_constant<int, 8>{});
        }
        if (const int at = 8 * o1 + lane; tail && at < a.vocab) {
            float x[1] = {value_at<TYPE>(row, at)}, y[1] = {value_at<TYPE>(other, at)}, z[1] = {race ? noise[at] : 1.f};
            take(at, x, y, z, std::integral_constant<int, 1>{});
        }
        return f;
    }

    // Segment number `segment` of row number `r` of a job, by one wave; three words
    __device__ __forceinline__ void work(int kind, int r, int segment, uint64_t (&words)[3]) {
        const int octets = a.vocab / 8, each = (octets + segments - 1) / segments;
        const int o0 = min(segment * each, octets), o1 = min(o0 + each, octets);
        const bool tail = segment == segments - 1;
        Found f;
        if (kind == kRows) {
            const int node = node_of(r);
            const bool second = drafted && (r & 1);
            const int first = child_from(node, node + 1);
            if (second && first >= n) return;          // nobody looks at it
            const bool race = !(cold || second || (drafted && first < n));
            int excludes = 0;
            if (race) {                                // the children do not take part: it counts when all were rejected
                const int lo = 8 * o0, hi = tail ? a.vocab : 8 * o1;
                for (int i = first; i < n; i = child_from(node, i + 1)) {
                    const int x = __builtin_amdgcn_readlane(id, i - base);
                    if (x < lo || x >= hi) continue;
                    if (lane == 0 && excludes < kExcluded) s.excluded[wave][excludes] = x;
                    ++excludes;
                }
            }
            base = -1;                                 // (what it stands for is not kept in registers over the pass)
            f = scan(second ? draft_of(node) : logits_of(node), o0, o1, tail, race, node, excludes);
        } else {
            base = -1;
            f = residual(o0, o1, tail, kind == kRace);
        }
        f.join(heat);
        words[0] = both(__float_as_uint(f.top), (uint32_t)f.top_at);
        words[1] = __builtin_bit_cast(uint64_t, f.sum);
        words[2] = both(__float_as_uint(f.best), (uint32_t)f.best_at);
    }

    // What the segments of a row found together, lane i holding segment i's words; by a whole wave
    __device__ __forceinline__ void keep(int r, uint64_t x, uint64_t y, uint64_t z) {
        Found f = kNothing;
        if (lane < segments)
            f = Found{__uint_as_float((uint32_t)x), (int)(x >> 32), __builtin_bit_cast(double, y), __uint_as_float((uint32_t)z), (int)(z >> 32)};
        f.join(heat);
        if (lane == 0) s.found[r] = f;
    }

    __device__ __forceinline__ void finish(int kept, int next) {
        if (member != 0) return;
        for (int64_t i = kept + threadIdx.x; i < a.width; i += kThreads) a.path[b * a.width + i] = -1;
        if (threadIdx.x == 0) {
            a.kept[b] = kept;
            a.next[b] = next;
        }
    }

    // After a job: walks on as far as what is known goes, and says what is wanted next; false: nothing, the walk has ended.  All threads of all
    // members take the same way.
    __device__ __forceinline__ bool decide(Job& j) {
        int node = j.node, child = j.next_child;
        bool leaf = false;
        if (j.kind == kRace) {
            const int best = s.found[0].best_at;
            if (best < 0 && j.c >= 0.0) {                // nothing is left: from p itself
                j.c = -1.0;
                return true;
            }
            finish(j.kept, best);
            return false;
        }
        if (j.kind == kSum) j.mass = s.found[0].sum;
        int at = 0;
        while (true) {
            Found p{};
            if (j.kind == kRows) {
                p = s.found[at];
                j.p_top = p.top;
                j.p_sum = p.sum;
                if (drafted) {
                    j.q_top = s.found[at + 1].top;
                    j.q_sum = s.found[at + 1].sum;
                }
                child = child_from(node, node + 1);
                leaf = child >= n;
                j.c = 0.0;
                j.mass = 1.0;
            }
            const bool full = j.kept >= a.width;
            int to = -1;
            if (cold) {
                for (int i = full ? n : child; i < n && to < 0; i = child_from(node, i + 1))
                    if (__builtin_amdgcn_readlane(id, i - base) == p.top_at && p.top > -__builtin_inff()) to = i;
                if (to < 0) {
                    finish(j.kept, p.top > -__builtin_inff() ? p.top_at : -1);
                    return false;
                }
            } else {
                if (!drafted) {
                    if (!full) to = first_accepted(node, p);
                } else if (!full && child < n) {
                    // one child a job: what is left of p when it is rejected takes a pass
                    look_at(child & ~63);
                    const bool in = id >= 0 && id < a.vocab;
                    const double pc = in && j.p_sum > 0.0 ? exp(((double)lp - (double)j.p_top) * heat.inv) / j.p_sum : 0.0;
                    const double qc = in && j.q_sum > 0.0 ? exp(((double)lq - (double)j.q_top) * heat.inv) / j.q_sum : 0.0;
                    const bool yes = (double)uniform * j.mass * qc < fmax(pc - j.c * qc, 0.0);
                    if (__ballot(yes) >> (child - base) & 1) {
                        to = child;
                    } else {
                        j.c += j.mass;
                        j.node = node;
                        j.next_child = child_from(node, child + 1);
                        j.kind = j.next_child < n ? kSum : kRace;
                        return true;
                    }
                }
                if (to < 0) {
                    if (j.kind == kRows && (leaf || (!drafted && !full && p.best_at >= 0))) {
                        finish(j.kept, p.best_at);
                        return false;
                    }
                    if (!(j.p_top > -__builtin_inff())) {
                        finish(j.kept, -1);
                        return false;
                    }
                    j.kind = kRace;                      // the path is full, or nothing but its children was left: from p itself
                    j.node = node;
                    j.c = -1.0;
                    return true;
                }
            }
            if (member == 0 && threadIdx.x == 0) a.path[b * a.width + j.kept] = to;
            ++j.kept;
            node = to;
            at = j.kind == kRows ? row_of(node) : -1;
            j.kind = kRows;
            j.node = node;
            if (at < 0) return true;
        }
    }
};

// p and q are never written: what a walk needs of a row is its largest value, the sum of exp((x - top) / T), the logits of the children's tokens
// and the winner of the race, all from one pass.  After j rejected children r = max(p - c q, 0) with c the sum of the Z so far, so r too is one
// pass over both rows.  Without a draft r is p without the tokens tried, its sum p's less theirs, and needs no pass.
// A walk reads few rows (16 trees over a vocabulary of 128000: 44 MB, half of it rows that no walk came to; 8 us of a copy's rate) but one after another, so it is bound by
// the latency of a job: 2.5 to 5 us of reading, 2 to 4 until all members' parts are seen, 1 to fetch them, 2 to decide.  With the call, a
// chain of five over 32000 tokens / 24 chains with their drafts over 50272 / those trees / six trees drawn from bfloat16 drafts, 100003: a
// workgroup a request 27 / 156 / 250 / 184 us; teams 13 / 33 / 45 / 52; segments over all waves of a team 13 / 28 / 36 / 47; a lane a child
// 11 / 26 / 33 / 45; sums in 64 bits 11 / 27 / 34 / 46.  The rows of the first two children are read with a node's (36 us for the trees; 44 with four or with none), those
// of all nodes where a tree has eight on average or fewer.
// A team of workgroups a request.  A job's rows are read in segments, each by a wave of its own; members hand in what their segments gave,
// look out for the others' a bounded number of times, join all parts in the order of the segments and decide, every one for itself
// and all alike, what the next job is.  A member that has looked in vain goes on alone and reads all segments itself, with the same
// result: nobody has to wait for a workgroup that may not be running.  Member 0 writes the results.
template <int TYPE>
__global__ __launch_bounds__(kThreads, 3) void verify_kernel(VerifyArgs a) {
    __shared__ Shared s;
    Team<TYPE> team(a, s);
    const int n = team.n, b = team.b, tid = threadIdx.x, lane = team.lane, wave = team.wave;
    const bool shared = a.team > 1;
    const uint64_t number = shared ? get(&a.control->number) : 0;
    for (int i = tid; i < n; i += kThreads) {
        const int p = a.parents[team.t0 + i];
        s.parent[i] = p >= 0 && p < i ? p : -1;           // so children come after their parent, here and wherever nodes are compared with it
        s.id[i] = a.ids[team.t0 + i];
        s.uniform[i] = a.uniform[team.t0 + i];
    }
    __syncthreads();
    if (!shared) team.look_up(tid, kThreads);
    if (team.member == 0 && tid == 0 && n > 0) a.path[b * a.width] = 0;
    if (tid == 0) {
        s.job = Job{};
        s.job.kept = 1;
    }
    __syncthreads();
    bool alone = !shared, more = n > 0;
    uint64_t* posted = shared ? a.control->posted + b * a.team : nullptr;
    uint64_t* parts = a.parts + (int64_t)b * 2 * kSlots * 3;
    if (!more) team.finish(0, -1);
    for (uint32_t jobs = 1; more; ++jobs) {
        const int kind = __builtin_amdgcn_readfirstlane(s.job.kind);
        if (kind == kRows) team.list_rows(__builtin_amdgcn_readfirstlane(s.job.node), jobs == 1 && n <= a.wide);
        const int rows = kind == kRows ? team.rows() : 1;
        team.segments = min(max((shared ? a.team : 4) * kWaves / rows, 1), a.finest);
        // together with the others first; alone, a row at a time, when they are not seen
        for (int r = alone ? 0 : -1; r < rows; ++r) {
            const bool mine = r >= 0;
            uint64_t* to = parts + (jobs & 1 ? 0 : (int64_t)kSlots * 3);
            __syncthreads();
            for (int i = mine ? wave : team.member * kWaves + wave; i < (mine ? 1 : rows) * team.segments; i += mine ? kWaves : a.team * kWaves) {
                uint64_t words[3] = {0, 0, 0};
                team.work(kind, mine ? r : i / team.segments, i % team.segments, words);
                if (lane < 3) {
                    const uint64_t word = lane == 0 ? words[0] : lane == 1 ? words[1] : words[2];
                    if (mine) s.part[i][lane] = word;
                    else put(to + (int64_t)i * 3 + lane, word);
                }
            }
            if (mine) {
                __syncthreads();
                if (wave == 0) {
                    const int at = min(lane, team.segments - 1);
                    team.keep(r, s.part[at][0], s.part[at][1], s.part[at][2]);
                }
                continue;
            }
            stored();
            __syncthreads();
            const uint64_t want = number << 16 | jobs;
            if (tid == 0) put(posted + team.member, want);
            if (wave == 0) {
                bool here = false;
                int polls = 0;
#if MX_VERIFY_EARLY
                const uint32_t early = __hip_atomic_load(&a.control->early, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                if (early != 0 && jobs >= (early & 0xffff) && (team.member & 1) >= (int)(early >> 16)) polls = kMostPolls;
#endif
                for (; !here && polls < kMostPolls; ++polls)
                    here = __ballot(lane < a.team && get(posted + min(lane, a.team - 1)) < want) == 0;
                if (lane == 0) s.all_here = here;
            } else if (wave == 3 && jobs == 1) {
                if (lane == 0) team_counts_in(a, b, number);
            } else if (jobs == 1) {
                team.look_up(tid - 64, 128);
            }
            __syncthreads();
            if (jobs == 1) team.base = -1;
            alone = s.all_here == 0;
            if (alone) continue;
            for (int x = wave; x < rows; x += kWaves) {
                const uint64_t* from = to + ((int64_t)x * team.segments + min(lane, team.segments - 1)) * 3;
                team.keep(x, get(from), get(from + 1), get(from + 2));
            }
            break;
        }
        __syncthreads();
        Job job = s.job;
        more = team.decide(job);
        __syncthreads();
        if (tid == 0) s.job = job;
        __syncthreads();
    }
    if (shared && n == 0 && tid == 0) team_counts_in(a, b, number);
}

struct Plan {
    int team, finest, wide, ahead;
};

Plan plan_of(int64_t tokens, int64_t requests, int64_t vocab, int rows_each) {
    Plan p{};
    if (requests < 1) requests = 1;
    const int64_t nodes = ceil_div(tokens, requests);
    auto clamp = [](int64_t v, int64_t lo, int64_t hi) { return (int)(v < lo ? lo : v > hi ? hi : v); };
    p.wide = nodes <= 8 ? kMostRows : 1;
    p.ahead = rows_each == 1 ? 2 : 1;
    const int64_t rows = (p.wide > 1 ? nodes : 1 + (nodes - 1 < p.ahead ? nodes - 1 : p.ahead)) * rows_each;
    p.finest = clamp(ceil_div(vocab, 512), 1, kMostSegments);
    p.team = requests > kMostTeams ? 1 : clamp(ceil_div(p.finest * rows, kWaves), 1, clamp(kMostMembers * 3 / 4 / requests, 1, 64));
    return p;
}

// Parts of a team's rows, twice (a member may be a job ahead of another); a team of one keeps them in LDS.
size_t workspace_bytes(int64_t requests) {
    const int64_t teams = requests < kMostTeams ? requests : kMostTeams;
    return kControlBytes + (size_t)teams * 2 * kSlots * 24;
}

}  // namespace
}  // namespace mx

using namespace mx;

extern "C" size_t mx_verify_workspace_bytes(int64_t tokens, int64_t requests, int64_t vocab) {
    if (tokens < 0 || requests < 0 || vocab < 1 || requests > kCacheMaxRequests || tokens > INT32_MAX || vocab > MX_VERIFY_MAX_VOCAB) return 0;
    return workspace_bytes(requests);
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
    VerifyArgs a{};
    a.logits = logits; a.draft = draft; a.ids = ids; a.parents = parents; a.q_start = q_start;
    a.temperature = temperature; a.uniform = uniform; a.noise = noise;
    a.path = path; a.kept = kept; a.next = next;
    a.tokens = tokens; a.ldl = ldl; a.ldd = ldd; a.ldn = ldn; a.width = path_width;
    a.vocab = (int32_t)vocab; a.requests = (int32_t)requests;
    const Plan p = plan_of(tokens, requests, vocab, draft != nullptr ? 2 : 1);
    a.team = p.team; a.finest = p.finest; a.wide = p.wide; a.ahead = p.ahead;
    a.control = (Control*)workspace;
    a.parts = (uint64_t*)((uint8_t*)workspace + kControlBytes);
    const unsigned grid = (unsigned)(requests * p.team);
    if (type == MX_F32) verify_kernel<MX_F32><<<grid, kThreads, 0, (hipStream_t)stream>>>(a);
    else verify_kernel<MX_BF16><<<grid, kThreads, 0, (hipStream_t)stream>>>(a);
    MX_HIP_LAUNCH_CHECK();
    return MX_OK;
}
