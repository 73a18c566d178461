// Log probabilities of given tokens with the row's entropy, log-sum-exp and likeliest
// columns, in one pass over the logits, and their gradient.
//
// Row z, token x:  lse = m + log l,  l = sum_v exp(z_v - m),  logprob = z_x - lse,
//   entropy = -sum_v p_v log p_v = log l - sum_v exp(z_v - m) (z_v - m) / l,  p = exp(z - lse);
// gradient of a g_lp logprob + g_h entropy:
//   dz_v = g_lp ([v = x] - p_v) - g_h p_v (log p_v + entropy).
// A thread keeps (m, l, s = sum exp(z - m) (z - m)) in fp32 over the columns it walks and
// moves l and s to a new maximum when it finds one; threads, then blocks, join in a fixed order.
//
// Bound: HBM, a read of the logits (and a write of as much for the gradient); the
// exponential unit and the arithmetic take about half of that time.  So: 16-byte loads, four a
// thread in flight and two rounds more on their way into L2, a row a block, or a warp where rows
// are short, and where there are fewer rows than places for blocks a row in several parts, whose
// last block to end joins them.  8192 bf16 rows of 151936: 330 to 348 us, 7.2 to 7.5 TB/s (without
// the rounds ahead 371), their gradient 739 us.
//
// The likeliest columns come along in the same pass: a column is a candidate while its key
// (order of the value, then of the index) is above a bar that k columns reach.  The bar is the
// k-th largest of the threads' maxima so far, taken in rounds 0, 2, 8, 26, ...: about 2 k columns
// pass it from one of these to the next.  (A bar takes a warp 150 instructions, a candidate 100:
// rounds 0, 1, 3, 7, ... are slower for few columns, 435 against 417 us at 8192 rows of 151936 and
// one column, and faster for many, 542 against 557 with 20.)  Each warp keeps its candidates in
// shared memory (a block's warps need not wait for one another: a maximum that has moved on since
// it was read only makes the bar too low), its lanes look together at the columns of a lane whose
// maximum passes, and cuts them down to the best k where they are many.  What bounds it then is
// the instructions: 640 rows of 151936 take 38.5 us alone, 49 with one column and 64 with 20.  A
// bar from the first columns alone, and each lane at its own columns, took 122 us.
#include <cmath>

#include <math_constants.h>

#include "serve.h"
#include "serve_ptx.cuh"

namespace sas {
namespace {

constexpr int kThreads = 256;
constexpr int kBlocks = 4;            // a multiprocessor, as many as their registers allow
constexpr int kMaxParts = 32;         // of a row: a lane each at the join
constexpr int kAhead = 3;             // rounds of a block's from its loads to its farthest prefetch (2 or 4: within 2%, 6 slower)
constexpr int kBarStep = 3;           // from a bar's round to the next one's
constexpr int kMinPart = 4096;        // columns: a round of fp32
// Columns of rows that a warp takes, for the gradient: 16384 bf16 rows of 4096 take 46 us by warps and 60 by blocks,
// of 16384 182 and 171, 152 rows of 16384 19 and 9.
constexpr int kSmallRow = 4096;
constexpr int kStatusBadInput = 1;    // == SAS_ERR_INVALID_ARG
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.69314718055994531f;
// Below this exponent 2^y is 0 in fp32; y itself is kept finite, as 0 times it is added.
constexpr float kLowest = -1000.f;
constexpr float kNone = -HUGE_VALF;   // maximum of no column

__device__ __forceinline__ float max_nan(float a, float b) {   // NaN if either is
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}

// 16 bytes of logits as fp32.
template <class E>
struct Vec;
template <>
struct Vec<bf16> {
    static constexpr int N = 8, UNROLL = 4;
    __device__ __forceinline__ static void unpack(const uint4& u, float* f) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    __device__ __forceinline__ static uint4 pack(const float* f) {
        return make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
    }
    __device__ __forceinline__ static uint4 nothing() { return make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u); }
    // The largest number, NaN passed over (-infinity if there is no other).
    __device__ __forceinline__ static uint32_t max2(uint32_t a, uint32_t b) {
        uint32_t d;
        asm("max.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
        return d;
    }
    template <int U>
    __device__ __forceinline__ static float top(const uint4 (&u)[U]) {
        uint32_t m = 0xff80ff80u;
#pragma unroll
        for (int i = 0; i < U; ++i) m = max2(max2(m, u[i].x), max2(max2(u[i].y, u[i].z), u[i].w));
        return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
    }
    __device__ __forceinline__ static float one(const bf16* p) { return __bfloat162float(load(p)); }
    __device__ __forceinline__ static void put(bf16* p, float v) { *p = __float2bfloat16_rn(v); }
};
template <>
struct Vec<float> {
    static constexpr int N = 4, UNROLL = 4;
    __device__ __forceinline__ static void unpack(const uint4& u, float* f) {
        f[0] = __uint_as_float(u.x);
        f[1] = __uint_as_float(u.y);
        f[2] = __uint_as_float(u.z);
        f[3] = __uint_as_float(u.w);
    }
    __device__ __forceinline__ static uint4 pack(const float* f) {
        return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
    __device__ __forceinline__ static uint4 nothing() { return make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u); }
    template <int U>
    __device__ __forceinline__ static float top(const uint4 (&u)[U]) {
        float m = -CUDART_INF_F;
#pragma unroll
        for (int i = 0; i < U; ++i) {
            m = max3f(m, __uint_as_float(u[i].x), __uint_as_float(u[i].y));
            m = max3f(m, __uint_as_float(u[i].z), __uint_as_float(u[i].w));
        }
        return m;
    }
    __device__ __forceinline__ static float one(const float* p) { return load(p); }
    __device__ __forceinline__ static void put(float* p, float v) { *p = v; }
};

// Columns [v0, v1) of a row as 16-byte vectors: vector j holds columns first + j N .., the
// first and the last one maybe in part.
template <class E>
struct Span {
    const E* row;
    int v0, v1, first, count;
    __device__ __forceinline__ Span(const E* row_, int v0_, int v1_) : row(row_), v0(v0_), v1(v1_) {
        const int off = static_cast<int>((reinterpret_cast<uintptr_t>(row + v0) & 15u) / sizeof(E));
        first = v0 - off;
        count = (v1 - first + Vec<E>::N - 1) / Vec<E>::N;
    }
    __device__ __forceinline__ int column(int j) const { return first + j * Vec<E>::N; }
    __device__ __forceinline__ int head() const { return count > 0 && !whole(0); }   // its first vector is partial
    __device__ __forceinline__ bool whole(int j) const { return column(j) >= v0 && column(j) + Vec<E>::N <= v1; }
};

// Sums over columns relative to the maximum m, in the log2 domain: y = (z - m) log2(e).  (One FMA, z
// log2(e) - m log2(e), would not be 0 at the maximum.)
struct Sums {
    float m, l, s;   // sums of 2^y and of 2^y y
    __device__ __forceinline__ Sums() : m(kNone), l(0.f), s(0.f) {}
    __device__ __forceinline__ Sums(float m_, float l_, float s_) : m(m_), l(l_), s(s_) {}
    // To another maximum.  No column so far (or none but NaN): nothing to move.
    __device__ __forceinline__ void move(float to) {
        if (m == -CUDART_INF_F) {
            m = to;
            return;
        }
        const float d = (m - to) * kLog2e;
        if (d == 0.f || to == -CUDART_INF_F) return;
        const float f = exp2f(d);
        s = f * fmaf(max_nan(d, kLowest), l, s);
        l *= f;
        m = to;
    }
    __device__ __forceinline__ void join(Sums o) {
        const float to = fmaxf(m, o.m);
        move(to);
        o.move(to);
        l += o.l;
        s += o.s;
    }
};

__device__ __forceinline__ Sums shfl_xor(const Sums& x, int o) {
    return Sums(__shfl_xor_sync(0xffffffffu, x.m, o), __shfl_xor_sync(0xffffffffu, x.l, o), __shfl_xor_sync(0xffffffffu, x.s, o));
}

// The same in every lane: which of two joined sums is the left one must not matter, so both
// lanes of a pair add them in lane order.
template <int LANES = 32>
__device__ __forceinline__ Sums warp_join(Sums x) {   // of every LANES neighbours
#pragma unroll
    for (int o = 1; o < LANES; o <<= 1) {
        const Sums y = shfl_xor(x, o);
        Sums a = (lane_id() & o) ? y : x;
        a.join((lane_id() & o) ? x : y);
        x = a;
    }
    return x;
}

// The order of a value, as a whole number; zeros of both signs are equal.
__device__ __forceinline__ uint32_t order_of(float z) {
    const uint32_t b = __float_as_uint(z + 0.f);
    return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
// Keys order columns by value, equal ones by index; 0 is below every column.
__device__ __forceinline__ unsigned long long key_of(float z, int v) {
    return (static_cast<unsigned long long>(order_of(z)) << 32) | (0xffffffffu - static_cast<uint32_t>(v));
}
__device__ __forceinline__ float value_of(uint32_t o) { return __uint_as_float((o & 0x80000000u) ? (o & 0x7fffffffu) : ~o); }
__device__ __forceinline__ float key_value(unsigned long long k) {
    return value_of(static_cast<uint32_t>(k >> 32));
}
__device__ __forceinline__ int key_index(unsigned long long k) { return static_cast<int>(0xffffffffu - static_cast<uint32_t>(k)); }

constexpr int kMaxTop = 32;    // a warp's lanes put them out
constexpr int kCand = 128;     // candidates of a warp
constexpr int kCut = 64;       // cut down at the end of a round that leaves this many
constexpr int kJoin = 512;     // candidates that the block joins at a time
constexpr int kGroups = kThreads / 4;
static_assert(kMaxTop <= kGroups, "the k-th of the groups' maxima");
static_assert(kThreads / 32 * kMaxTop + kMaxTop <= kJoin, "the warps' best at a time");

// A team: a block, or one of its warps.
template <int TEAM>
struct Team {
    __device__ __forceinline__ static int rank() { return TEAM == 32 ? lane_id() : threadIdx.x; }
    __device__ __forceinline__ static void sync() {
        if constexpr (TEAM == 32) __syncwarp();
        else __syncthreads();
    }
};
struct Cand {   // of a warp
    unsigned long long key[kCand];
    unsigned long long top[kMaxTop];
};

// The best k of n keys, best first, into their place (keys of 0, of no column, fill one place at most: the
// others are 0 as well).  Returns how many there are.
template <int TEAM>
__device__ __forceinline__ int cut(unsigned long long* key, unsigned long long* top, int n, int k) {
    for (int i = Team<TEAM>::rank(); i < k; i += TEAM) top[i] = 0;
    Team<TEAM>::sync();
    for (int i = Team<TEAM>::rank(); i < n; i += TEAM) {
        const unsigned long long mine = key[i];
        int above = 0;
        for (int j = 0; j < n; ++j) above += key[j] > mine;
        if (above < k) top[above] = mine;
    }
    Team<TEAM>::sync();
    n = min(n, k);
    for (int i = Team<TEAM>::rank(); i < n; i += TEAM) key[i] = top[i];
    Team<TEAM>::sync();
    return n;
}

__device__ __forceinline__ void prefetch_l2(const void* p, uint32_t bytes) {
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(p), "r"(bytes) : "memory");
}

// What a row gives, by one thread.
__device__ __forceinline__ void put_row(const LogpArgs& a, int row, const Sums& x, float zx) {
    const float ll = logf(x.l);
    // a row without a finite column: its sum is 0 and everything but lse is undefined
    a.lse[row] = x.l == 0.f ? -CUDART_INF_F : x.m + ll;
    a.logprob[row] = x.l == 0.f ? CUDART_NAN_F : (zx - x.m) - ll;
    a.entropy[row] = x.l == 0.f ? CUDART_NAN_F : ll - kLn2 * (x.s / x.l);
}

template <class E, int TEAM, bool TOP>
__global__ void __launch_bounds__(kThreads, kBlocks) logp_kernel(LogpArgs a) {
    using V = Vec<E>;
    constexpr int N = V::N, U = V::UNROLL, ROUND = TEAM * U, TEAMS = kThreads / TEAM;
    static_assert(N * U <= 32, "a thread's columns of a round, a lane each");
    static_assert(kMaxTop < kCut && kCut + 32 <= kCand, "room for a lane's columns");
    __shared__ Cand cands[TOP ? kThreads / 32 : 1];
    __shared__ unsigned long long all[TOP && TEAM == kThreads ? kJoin : 1], all_top[kMaxTop];
    __shared__ uint4 seen[TOP ? U * kThreads : 1];
    __shared__ float tops[TOP && TEAM == kThreads ? kGroups : 1];   // maxima so far, of four threads each
    __shared__ int sh_held[kThreads / 32];
    __shared__ float3 joined[kThreads / 32];
    __shared__ int sh_last;
    const int rank = Team<TEAM>::rank(), part = TEAM == kThreads ? blockIdx.x % a.parts : 0;
    const int row = TEAM == kThreads ? blockIdx.x / a.parts : blockIdx.x * TEAMS + static_cast<int>(warp_id());
    Cand& c = cands[TOP ? warp_id() : 0];
    grid_dep_wait();
    if (TEAM == 32 && row >= a.rows) return;
    const int x = load(a.tokens + row);
    if (x < 0 || x >= a.V) {   // a row that does not count: its logits are not read
        if (part == 0) {
            if (rank == 0) {
                if (x != -1) atomicExch(a.status, kStatusBadInput);
                a.logprob[row] = 0.f;
                a.entropy[row] = 0.f;
                a.lse[row] = 0.f;
            }
            if (TOP) {
                for (int i = rank; i < a.k; i += TEAM) {
                    a.top_index[static_cast<size_t>(row) * a.k + i] = -1;
                    a.top_logprob[static_cast<size_t>(row) * a.k + i] = 0.f;
                }
            }
        }
        return;
    }
    const E* const z = static_cast<const E*>(a.logits) + static_cast<size_t>(row) * a.ld;
    const float zx = rank == 0 ? V::one(z + x) : 0.f;   // of use at the end
    const int v0 = part * a.chunk;
    const Span<E> sp(z, v0, min(a.V, v0 + a.chunk));
    Sums t;
    unsigned long long bar = 0;
    float bar_value = -CUDART_INF_F;   // below it no column is a candidate
    int held = 0;                      // the warp's candidates
    // Whole vectors in whole rounds, then the others, of which the row's first may be one.
    const int head = sp.head(), rounds = (sp.count - head - (sp.count > head && !sp.whole(sp.count - 1))) / ROUND;
    const int late = rounds * ROUND + head, others = sp.count - late + head;   // where they begin, how many
    const int all_rounds = rounds + (others + ROUND - 1) / ROUND;
    const E* from = z + sp.column(head + rank);
    // whole rounds, on their way into L2
    auto prefetch = [&](int r) {
        if (TEAM == kThreads && rank == 0 && r < rounds) prefetch_l2(z + sp.column(head) + static_cast<size_t>(r) * (ROUND * N), ROUND * 16);
    };
    for (int r = 1; r < kAhead; ++r) prefetch(r);
    // The bar: the k-th largest of the maxima of four threads each (k columns are no smaller), down to the upper 16 bits of its order: the
    // largest such number that k of them reach.
    auto put_max = [&] {   // of a block
        float v = fmaxf(t.m, __shfl_xor_sync(0xffffffffu, t.m, 1));
        v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 2));
        if (rank % 4 == 0) tops[rank / 4] = v;
    };
    auto raise_bar = [&] {
        constexpr int M = TEAM == 32 ? 1 : kGroups / 32;
        uint32_t o[M], low = 0xffffffffu, high = 0;
#pragma unroll
        for (int i = 0; i < M; ++i) {
            o[i] = order_of(TEAM == 32 ? t.m : *static_cast<volatile float*>(&tops[i * 32 + lane_id()]));
            low = min(low, o[i]);
            high = max(high, o[i]);
        }
        low = __reduce_min_sync(0xffffffffu, low);
        high = __reduce_max_sync(0xffffffffu, high);
        uint32_t bit = 0x80000000u >> __clz((low ^ high) | 1u);   // the first that is not the same in all
        uint32_t at = high & ~(2 * bit - 1) & 0xffff0000u;
#pragma unroll 1
        for (; bit >= 0x10000u; bit >>= 1) {
            int n = 0;
#pragma unroll
            for (int i = 0; i < M; ++i) n += o[i] >= (at | bit);
            if (__reduce_add_sync(0xffffffffu, n) >= a.k) at |= bit;
        }
        if (at > order_of(-CUDART_INF_F)) bar_value = fmaxf(bar_value, value_of(at));
    };
    int next_bar = 0;
    for (int round = 0; round < all_rounds; ++round) {
        prefetch(round + kAhead);
        // this thread's u-th vector
        auto vector = [&](int u, int rank) {
            const int q = (round < rounds ? round : round - rounds) * ROUND + u * TEAM + rank;
            return round < rounds ? head + q : q < head ? 0 : late + q - head;
        };
        uint4 raw[U];
        if (round < rounds) {
#pragma unroll
            for (int u = 0; u < U; ++u) raw[u] = __ldcs(reinterpret_cast<const uint4*>(from + u * (TEAM * N)));
            from += ROUND * N;
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int j = vector(u, rank), v = sp.column(j);
                raw[u] = V::nothing();
                if (j >= sp.count) continue;
                if (sp.whole(j)) {
                    raw[u] = __ldcs(reinterpret_cast<const uint4*>(z + v));
                } else {   // columns of the row alone, -infinity for the others
                    float f[N];
#pragma unroll
                    for (int e = 0; e < N; ++e) f[e] = v + e >= sp.v0 && v + e < sp.v1 ? V::one(z + v + e) : -CUDART_INF_F;
                    raw[u] = V::pack(f);
                }
            }
        }
        const float top = V::top(raw);
        if (top > t.m) t.move(top);
        const float m = t.m == -CUDART_INF_F ? 0.f : t.m;
        float l = 0.f, s = CUDART_NAN_F;
        if (round < rounds) {
            const uint64_t scale2 = f32x2(kLog2e, kLog2e), off2 = f32x2(-m, -m);
            uint64_t l2[2] = {0, 0}, s2[2] = {0, 0};
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float f[N];
                V::unpack(raw[u], f);
#pragma unroll
                for (int e = 0; e < N; e += 2) {
                    const uint64_t y = mul_f32x2(add_f32x2(f32x2(f[e], f[e + 1]), off2), scale2);
                    float y0, y1;
                    f32x2_split(y, y0, y1);
                    const uint64_t p = f32x2(fast_exp2(y0), fast_exp2(y1));
                    l2[e >> 1 & 1] = add_f32x2(l2[e >> 1 & 1], p);
                    s2[e >> 1 & 1] = fma_f32x2(p, y, s2[e >> 1 & 1]);
                }
            }
            float a0, a1;
            f32x2_split(add_f32x2(l2[0], l2[1]), a0, a1);
            l = a0 + a1;
            f32x2_split(add_f32x2(s2[0], s2[1]), a0, a1);
            s = a0 + a1;
        }
        if (s != s) {   // columns of -infinity (0 times y) or none at all, unless it is NaN's
            l = s = 0.f;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (vector(u, rank - static_cast<int>(lane_id())) >= sp.count) continue;   // none of the warp's
                float f[N];
                V::unpack(raw[u], f);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const float y = max_nan((f[e] - m) * kLog2e, kLowest);
                    const float p = fast_exp2(y);
                    l += p;
                    s = fmaf(p, y, s);
                }
            }
        }
        t.l += l;
        t.s += s;
        if constexpr (TOP) {
            if (round == next_bar) {
                next_bar = kBarStep * next_bar + kBarStep - 1;
                if constexpr (TEAM == kThreads) {
                    put_max();
                    if (round == 0) __syncthreads();
                    else __syncwarp();
                }
                raise_bar();
            }
            unsigned pass = __ballot_sync(0xffffffffu, top >= bar_value);   // lanes with a candidate, maybe
            if (pass != 0) {
                if (top >= bar_value) {
#pragma unroll
                    for (int u = 0; u < U; ++u) seen[u * kThreads + threadIdx.x] = raw[u];
                }
                __syncwarp();
                const int i = lane_id(), u = i / N, e = i % N;   // a lane's N U columns, one of them each
                const E* const column = reinterpret_cast<const E*>(seen + (u < U ? u : 0) * kThreads + threadIdx.x - i) + e;
#pragma unroll 1
                for (; pass != 0; pass &= pass - 1) {
                    const int at = __ffs(pass) - 1;
                    const float f = u < U ? V::one(column + at * N) : CUDART_NAN_F;
                    unsigned who = __ballot_sync(0xffffffffu, f >= bar_value);
                    if (who == 0) continue;   // it has moved
                    const int j = vector(u, rank - i + at), v = sp.column(j) + e;
                    if (bar != 0 || bar_value == -CUDART_INF_F)   // (what is no column has come as -infinity)
                        who = __ballot_sync(0xffffffffu, f >= bar_value && key_of(f, v) > bar && j < sp.count && v >= sp.v0 && v < sp.v1);
                    if (who >> i & 1u) c.key[held + __popc(who & ((1u << i) - 1))] = key_of(f, v);
                    held += __popc(who);
                    if (held >= kCut) {
                        __syncwarp();
                        held = cut<32>(c.key, c.top, held, a.k);
                        if (held == a.k) {
                            bar = c.key[a.k - 1];
                            bar_value = fmaxf(bar_value, key_value(bar));
                        }
                    }
                }
                __syncwarp();   // before other columns are put there
            }
        }
    }
    t = warp_join(t);
    if constexpr (TEAM == kThreads) {
        if (lane_id() == 0) joined[warp_id()] = make_float3(t.m, t.l, t.s);
        __syncthreads();
        if (warp_id() == 0) {   // whose alone are a row's and a part's results
            const float3 q = joined[lane_id() % (kThreads / 32)];   // in every lane: each may put out a column
            t = warp_join<kThreads / 32>(Sums(q.x, q.y, q.z));
        }
    }
    unsigned long long* best = c.key;   // the best k, and how many of them are columns
    if constexpr (TOP) {
        __syncwarp();
        if constexpr (TEAM == kThreads) {   // what is still above the bar, most often a few
            int kept = 0;
            for (int i0 = 0; i0 < held; i0 += 32) {
                const int i = i0 + static_cast<int>(lane_id());
                const unsigned long long key = i < held ? c.key[i] : 0ull;
                const bool stays = i < held && key_value(key) >= bar_value;
                const unsigned who = __ballot_sync(0xffffffffu, stays);
                if (stays) c.key[kept + __popc(who & ((1u << lane_id()) - 1))] = key;
                kept += __popc(who);
                __syncwarp();
            }
            held = kept;
        }
        if (TEAM == 32 || held > a.k) held = cut<32>(c.key, c.top, held, a.k);
        if constexpr (TEAM == kThreads) {
            best = all;
            if (lane_id() == 0) sh_held[warp_id()] = held;
            __syncthreads();
            int before = 0, sum = 0;
#pragma unroll
            for (int w = 0; w < kThreads / 32; ++w) {
                if (w == static_cast<int>(warp_id())) before = sum;
                sum += sh_held[w];
            }
            for (int i = lane_id(); i < held; i += 32) all[before + i] = c.key[i];
            __syncthreads();
            held = cut<TEAM>(all, all_top, sum, a.k);
        }
    }
    if (TEAM == kThreads && a.parts > 1) {
        // the part's results; the row's last block joins them in their order
        const size_t at = static_cast<size_t>(row) * a.parts + part;
        if (rank < 32) {
            if (rank == 0) a.part[at] = make_float4(t.m, t.l, t.s, 0.f);
            if (TOP && rank < a.k) a.part_top[at * kMaxTop + rank] = rank < held ? best[rank] : 0ull;
            __threadfence();
            __syncwarp();
            if (rank == 0) sh_last = atomicAdd(a.count + row, 1) == a.parts - 1;
        }
        __syncthreads();
        if (!sh_last) return;
        __threadfence();
        if (rank == 0) a.count[row] = 0;
        const size_t row0 = static_cast<size_t>(row) * a.parts;
        if (warp_id() == 0) {
            t = Sums();
            if (static_cast<int>(lane_id()) < a.parts) {
                const float4 q = __ldcg(a.part + row0 + lane_id());
                t = Sums(q.x, q.y, q.z);
            }
            t = warp_join(t);
        }
        if constexpr (TOP) {
            held = 0;
            const int step = (kJoin - kMaxTop) / kMaxTop;   // parts whose candidates fit beside the best so far
            for (int p0 = 0; p0 < a.parts; p0 += step) {
                const int np = min(step, a.parts - p0);
                for (int i = rank; i < np * a.k; i += TEAM)
                    all[held + i] = __ldcg(a.part_top + (row0 + p0 + i / a.k) * kMaxTop + i % a.k);
                __syncthreads();
                held = cut<TEAM>(all, all_top, held + np * a.k, a.k);
            }
        }
    }
    if (rank == 0) put_row(a, row, t, zx);
    if constexpr (TOP) {
        for (int i = rank; i < a.k; i += TEAM) {
            const unsigned long long key = i < held ? best[i] : 0ull;
            const size_t at = static_cast<size_t>(row) * a.k + i;
            a.top_index[at] = key == 0 ? -1 : key_index(key);
            a.top_logprob[at] = key == 0 || t.l == 0.f ? CUDART_NAN_F : (key_value(key) - t.m) - logf(t.l);
        }
    }
}

// ------------------------------------------------------------------ gradient

template <class E, int TEAM>
__global__ void __launch_bounds__(kThreads) logp_bwd_kernel(LogpBwdArgs a) {
    using V = Vec<E>;
    constexpr int N = V::N, U = V::UNROLL, TEAMS = kThreads / TEAM;
    const int rank = Team<TEAM>::rank(), part = TEAM == kThreads ? blockIdx.x % a.parts : 0;
    const int row = TEAM == kThreads ? blockIdx.x / a.parts : blockIdx.x * TEAMS + static_cast<int>(warp_id());
    grid_dep_wait();
    if (TEAM == 32 && row >= a.rows) return;
    const int x = load(a.tokens + row);
    const bool counts = x >= 0 && x < a.V;
    if (!counts && x != -1 && part == 0 && rank == 0) atomicExch(a.status, kStatusBadInput);
    const E* const z = static_cast<const E*>(a.logits) + static_cast<size_t>(row) * a.ld;
    E* const dz = static_cast<E*>(a.dlogits) + static_cast<size_t>(row) * a.ld_d;
    float lse = 0.f, h = 0.f, gl = 0.f, gh = 0.f;
    if (counts) {
        lse = load(a.lse + row);
        h = load(a.entropy + row);
        gl = load(a.dlogprob + row);
        if (a.dentropy != nullptr) gh = load(a.dentropy + row);
    }
    // with y = log p:  dz = -p (gl + gh (y + h)), and gl more at the token
    const float base = fmaf(gh, h, gl);
    auto grad = [&](float zv, int v) {
        const float y = max_nan(zv - lse, kLowest);
        return fmaf(-exp2f(y * kLog2e), fmaf(gh, y, base), v == x ? gl : 0.f);
    };
    const int v0 = part * a.chunk;
    const Span<E> sp(z, v0, min(a.V, v0 + a.chunk));
    // output vectors of the same columns; where the results' rows lie otherwise within 16 bytes than the logits', stores
    // of one element (4096 bf16 rows of 32003 out of rows of 32064: 324 us into rows of 32003, 86 into rows of 32064;
    // fp32 169 and 161)
    const bool same = ((reinterpret_cast<uintptr_t>(dz) ^ reinterpret_cast<uintptr_t>(z)) & 15u) == 0;
    for (int j0 = rank; j0 < sp.count; j0 += U * TEAM) {
        uint4 raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = j0 + u * TEAM;
            if (counts && j < sp.count && sp.whole(j)) raw[u] = __ldcs(reinterpret_cast<const uint4*>(z + sp.column(j)));
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = j0 + u * TEAM, v = sp.column(j);
            if (j >= sp.count) continue;
            float f[N];
            if (sp.whole(j)) {
                if (counts) {
                    V::unpack(raw[u], f);
#pragma unroll
                    for (int e = 0; e < N; ++e) f[e] = grad(f[e], v + e);
                } else {
#pragma unroll
                    for (int e = 0; e < N; ++e) f[e] = 0.f;
                }
                if (same) {
                    __stcs(reinterpret_cast<uint4*>(dz + v), V::pack(f));
                } else {
#pragma unroll
                    for (int e = 0; e < N; ++e) V::put(dz + v + e, f[e]);
                }
            } else {
                for (int e = 0; e < N; ++e)
                    if (v + e >= sp.v0 && v + e < sp.v1) V::put(dz + v + e, counts ? grad(V::one(z + v + e), v + e) : 0.f);
            }
        }
    }
}

// Parts of a row, so that all places for blocks are taken, and a part's columns.
void split_rows(int rows, int V, int places, int& parts, int& chunk) {
    const int most = (V + kMinPart - 1) / kMinPart;
    parts = places / rows;
    if (parts > kMaxParts) parts = kMaxParts;
    if (parts > most) parts = most;
    if (parts < 1) parts = 1;
    chunk = ((V + parts - 1) / parts + 63) / 64 * 64;   // whole vectors, if the row begins with one
    parts = (V + chunk - 1) / chunk;
}

// Whether a warp takes a row.  A block's row costs 3 us whatever its length, a warp's waits for one load after the
// other, and for its k columns more than all.  By a warp and by a block, us (k columns of bf16 rows):
//                          columns 1024       4096         8192         16384        32000
//   608 rows    k = 0        8.0, 8.2    7.8, 7.6    7.6, 12.8   11.3, 12.5   27.8, 16.8
//               k = 5       10.8, 9.6   11.9, 9.0   17.2, 21.3   24.3, 20.3   42.8, 26.0
//               k = 20      9.3, 10.9  23.4, 10.4   32.9, 23.4   46.6, 22.8   72.2, 30.8
//   2432 rows   k = 0       7.4, 13.4   9.9, 15.9   10.6, 15.7   17.4, 21.5   33.3, 34.2
//               k = 5       8.6, 26.6  13.5, 26.8   20.9, 26.5   31.6, 35.1   50.6, 53.7
//               k = 20     10.4, 33.8  27.7, 31.7   40.7, 31.3   57.7, 43.8   82.7, 65.1
//   4864 rows   k = 0       7.9, 24.4   8.7, 29.9   14.2, 30.7   25.5, 39.6   48.0, 63.2
//               k = 5       9.3, 50.2  18.9, 51.2   29.8, 51.1   42.3, 64.9   70.5, 100
//               k = 20     15.7, 64.1  42.9, 60.4   62.1, 60.4   87.9, 81.5    125, 123
//   16384 rows  k = 0      12.1, 77.3  27.6, 97.3   47.2, 93.8  89.9, 123.7   165, 203
//               k = 5      25.3, 162   55.2, 167    84.9, 161    130, 206     221, 321
//               k = 20     46.0, 205    128, 196     189, 190    267, 259     382, 393
// and for 2432 rows of 65536 without any 62, 56.  (Not by k: a row's numbers are the same with and without
// alternatives.)
bool row_by_warp(const LogpArgs& a) {
    const int per_sm = a.rows / device_sm_count();
    return a.V <= (per_sm >= 32 ? 32768 : per_sm >= 16 ? 4096 : 1024);
}

template <class E>
cudaError_t launch_fwd(LogpArgs a, const KernelEnv& env) {
    const bool small = row_by_warp(a);
    a.parts = 1;
    a.chunk = a.V;
    if (!small) split_rows(a.rows, a.V, logp_max_splits(), a.parts, a.chunk);
    const dim3 grid(small ? (a.rows + kThreads / 32 - 1) / (kThreads / 32) : a.rows * a.parts);
    if (a.k > 0) return launch_early(small ? logp_kernel<E, 32, true> : logp_kernel<E, kThreads, true>, grid, kThreads, 0, env.stream, a);
    return launch_early(small ? logp_kernel<E, 32, false> : logp_kernel<E, kThreads, false>, grid, kThreads, 0, env.stream, a);
}

template <class E>
cudaError_t launch_bwd(LogpBwdArgs a, const KernelEnv& env) {
    const bool small = a.V <= kSmallRow;
    a.parts = 1;
    a.chunk = a.V;
    // several waves of blocks, which have nothing to join at their end, in parts of as many bytes for either type (us, of
    // 777 rows of 32003: fp32 with 32 places a multiprocessor 32.9, with 6 37.7; bf16 with 16 21.3, with 32 22.6)
    const int places = 8 * static_cast<int>(sizeof(E)) * device_sm_count();
    if (!small) split_rows(a.rows, a.V, places, a.parts, a.chunk);
    const dim3 grid(small ? (a.rows + kThreads / 32 - 1) / (kThreads / 32) : a.rows * a.parts);
    return launch_early(small ? logp_bwd_kernel<E, 32> : logp_bwd_kernel<E, kThreads>, grid, kThreads, 0, env.stream, a);
}

}  // namespace

const char* logp_check(int V, int dtype, const void* logits, long long ld) {
    if (V < 1 || V > (1 << 30)) return "V must be 1 .. 2^30";
    if (dtype != 0 && dtype != 1) return "dtype must be SAS_DTYPE_BF16 or SAS_DTYPE_FP32";
    if (ld < V) return "a row stride is below V";
    if ((reinterpret_cast<uintptr_t>(logits) & (dtype == 0 ? 1u : 3u)) != 0) return "misaligned pointer";
    return nullptr;
}

// As many parts as blocks have places, no second wave: 152 rows of 32000 take 8.2 us (14.6 with 20 columns), in two
// waves 12.9 (24.7), 608 rows of 151936 29.5 us and 35.7.
int logp_max_splits() { return kBlocks * device_sm_count(); }
int logp_max_top() { return kMaxTop; }

cudaError_t launch_logp(const LogpArgs& a, const KernelEnv& env) {
    return a.is_bf16 ? launch_fwd<bf16>(a, env) : launch_fwd<float>(a, env);
}

cudaError_t launch_logp_bwd(const LogpBwdArgs& a, const KernelEnv& env) {
    return a.is_bf16 ? launch_bwd<bf16>(a, env) : launch_bwd<float>(a, env);
}

}  // namespace sas
