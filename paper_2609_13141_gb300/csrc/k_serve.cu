// Bookkeeping of a serving step: the page plan and the verification of drafts.
#include "serve.h"
#include "serve_ptx.cuh"

namespace sas {
namespace {

constexpr int kStatusBadInput = 1;   // == SAS_ERR_INVALID_ARG
constexpr int kStatusNoPages = 5;    // == SAS_ERR_OOM

// ------------------------------------------------------------------ page plan
//
// Request b has s tokens and gets n more: its pages grow from ceil(max(s, held) / 64) to
// ceil((s + n) / 64), the new ones taken from the free list in request order, and
// new token i sits at position s + i, slot page * 64 + (s + i) % 64.
//
// Latency-bound: tens of bytes a request.  So it is one launch without
// communication between blocks: every block scans all requests itself (8 bytes
// each, from L2 after the first block) into shared memory, then blocks share the
// tokens, the new pages and the requests.  In a captured row of calls 5.1 us for 256
// requests of one token and 7.1 for 1500 requests and 371104 tokens (4.5 MB out); called
// from the host 8.2 and 8.6.

constexpr int kPlanThreads = 512;
constexpr int kTokens = 4;   // of a thread

// Exclusive sums over the block's threads of (x, y), and the totals.
__device__ __forceinline__ void block_scan2(long long& x, int& y, long long& tx, int& ty) {
    __shared__ long long wx[kPlanThreads / 32];
    __shared__ int wy[kPlanThreads / 32];
    const int lane = lane_id(), warp = warp_id();
    long long ix = x;
    int iy = y;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long ax = __shfl_up_sync(0xffffffffu, ix, o);
        const int ay = __shfl_up_sync(0xffffffffu, iy, o);
        if (lane >= o) {
            ix += ax;
            iy += ay;
        }
    }
    if (lane == 31) {
        wx[warp] = ix;
        wy[warp] = iy;
    }
    __syncthreads();
    long long bx = 0;
    int by = 0;
    tx = 0;
    ty = 0;
#pragma unroll
    for (int w = 0; w < kPlanThreads / 32; ++w) {
        if (w == warp) {
            bx = tx;
            by = ty;
        }
        tx += wx[w];
        ty += wy[w];
    }
    x = bx + ix - x;
    y = by + iy - y;
}

// The last index i with sums[i] <= v (sums ascending, sums[0] <= v).
__device__ __forceinline__ int owner(const int* sums, int n, int v) {
    int lo = 0, hi = n;   // sums[lo] <= v, sums[hi] > v or hi == n
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (sums[mid] <= v) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Pages request b holds.
__device__ __forceinline__ int pages_held(const PlanArgs& a, int b, int s) {
    return ((a.held_lens != nullptr ? max(s, load(a.held_lens + b)) : s) + 63) / 64;
}

__global__ void __launch_bounds__(kPlanThreads) plan_kernel(PlanArgs a) {
    extern __shared__ int sm[];
    int* cu = sm;              // [B] first new token of each request
    int* off = sm + a.B;       // [B] first new page (counted over all requests)
    const int t = threadIdx.x;
    const long long cap = 64LL * a.max_blocks;
    int bad = 0;
    grid_dep_wait();
    for (int b = t; b < a.B; b += kPlanThreads) {
        const int s = load(a.seq_lens + b), n = load(a.new_lens + b);
        const int held = a.held_lens != nullptr ? load(a.held_lens + b) : 0;
        const bool wrong = s < 0 || n < 0 || static_cast<long long>(s) + n > cap || held < 0 || held > cap;
        bad |= wrong;
        cu[b] = wrong ? 0 : n;
        off[b] = wrong ? 0 : max(0, (s + n + 63) / 64 - (max(s, held) + 63) / 64);
    }
    bad = __syncthreads_or(bad);
    const int per = (a.B + kPlanThreads - 1) / kPlanThreads;
    const int b0 = min(a.B, t * per), b1 = min(a.B, b0 + per);
    long long n_off = 0, n_all;
    int p_off = 0, p_all;
    for (int b = b0; b < b1; ++b) {
        n_off += cu[b];
        p_off += off[b];
    }
    block_scan2(n_off, p_off, n_all, p_all);
    const int begin = load(a.free_begin);
    const bool invalid = bad || n_all > a.T || begin < 0 || begin > a.num_free;
    const bool short_ = !invalid && p_all > a.num_free - begin;
    const bool fits = !invalid && !short_;
    if (!fits && blockIdx.x == 0 && t == 0) atomicExch(a.status, short_ ? kStatusNoPages : kStatusBadInput);
    for (int b = b0; b < b1; ++b) {   // counts to exclusive sums
        const int n = cu[b], p = off[b];
        cu[b] = fits ? static_cast<int>(n_off) : 0;
        off[b] = fits ? p_off : 0;
        n_off += n;
        p_off += p;
    }
    __syncthreads();
    const int total = fits ? static_cast<int>(n_all) : 0, pages = fits ? p_all : 0;
    const int at = blockIdx.x * kPlanThreads + t, step = gridDim.x * kPlanThreads;
    for (int b = at; b < a.B; b += step) {
        a.kv_lens[b] = load(a.seq_lens + b) + (fits ? load(a.new_lens + b) : 0);
        a.cu_new[b] = cu[b];
    }
    if (at == 0) {
        a.cu_new[a.B] = total;
        *a.free_end = begin + pages;
    }
    for (int p = at; p < pages; p += step) {
        const int b = owner(off, a.B, p);
        const int blk = pages_held(a, b, load(a.seq_lens + b)) + p - off[b];
        int page = load(a.free_pages + begin + p);
        if (page < 0 || page >= a.num_pages) {
            atomicExch(a.status, kStatusBadInput);
            page = -1;
        }
        a.block_table[static_cast<size_t>(b) * a.max_blocks + blk] = page;
    }
    // kTokens neighbouring tokens a thread: one search, and a page looked up once, for most
    const bool wide = ((reinterpret_cast<uintptr_t>(a.positions) | reinterpret_cast<uintptr_t>(a.slots)) & 15u) == 0;
    for (long long i0 = static_cast<long long>(at) * kTokens; i0 < a.T; i0 += static_cast<long long>(step) * kTokens) {
        int pos[kTokens];
        long long slot[kTokens];
        int b = i0 < total ? owner(cu, a.B, static_cast<int>(i0)) : 0, s = 0, have = 0, last = -1, page = -1;
        bool fresh = true;
#pragma unroll
        for (int j = 0; j < kTokens; ++j) {
            const int i = static_cast<int>(i0) + j;
            pos[j] = -1;
            slot[j] = -1;
            if (i0 + j >= total) continue;
            while (b + 1 < a.B && cu[b + 1] <= i) {
                ++b;
                fresh = true;
            }
            if (fresh) {
                s = load(a.seq_lens + b);
                have = pages_held(a, b, s);
                last = -1;
                fresh = false;
            }
            const int p = s + i - cu[b], blk = p >> 6;
            if (blk != last) {
                // a page of this call comes from the free list: its table entry may not be written yet
                page = blk < have ? a.block_table[static_cast<size_t>(b) * a.max_blocks + blk]
                                  : load(a.free_pages + begin + off[b] + blk - have);
                last = blk;
                if (page < 0 || page >= a.num_pages) {
                    atomicExch(a.status, kStatusBadInput);
                    page = -1;
                }
            }
            if (page >= 0) {
                pos[j] = p;
                slot[j] = static_cast<long long>(page) * 64 + (p & 63);
            }
        }
        if (wide && i0 + kTokens <= a.T) {
            *reinterpret_cast<int4*>(a.positions + i0) = make_int4(pos[0], pos[1], pos[2], pos[3]);
            *reinterpret_cast<longlong2*>(a.slots + i0) = make_longlong2(slot[0], slot[1]);
            *reinterpret_cast<longlong2*>(a.slots + i0 + 2) = make_longlong2(slot[2], slot[3]);
        } else {
#pragma unroll
            for (int j = 0; j < kTokens; ++j) {
                if (i0 + j < a.T) {
                    a.positions[i0 + j] = pos[j];
                    a.slots[i0 + j] = slot[j];
                }
            }
        }
    }
}

// ------------------------------------------------------------------ drafts
//
// Request b drafted x_0 .. x_{n-1}, x_j from q_j; the target gives p_0 .. p_n.  x_j
// is accepted while u_j q_j(x_j) < p_j(x_j) (probability min(1, p / q)).  At the
// first rejection the next token is drawn from max(p - q, 0) (from p past the last
// draft), as argmax_v w_v / e_v with e_v ~ Exp(1) given: exponential clocks of rates
// w_v ring first at v with probability w_v / sum w, so no sum is needed and the
// choice does not depend on the order of any addition.
//
// HBM-bound: one row of p, q and e a request, read once by several blocks (6.5 TB/s at
// 128 rows of 151936 columns, 36 us).  The division is made only where w could beat the thread's best: w >= best e, a
// product smaller by more than both roundings (with the underflow range let
// through).  Blocks join by a maximum over (quotient bits, ~index): quotients are
// not negative, so their bits order like the values, and ties go to the lower index.  Below
// all of these is the key of a row that has weight only where e cannot be divided by: its
// residual is not empty, so the target does not stand in for it.

constexpr int kVerifyThreads = 256;
constexpr int kVerifyBlocks = 5;   // a multiprocessor

__device__ __forceinline__ void prefetch_l2(const void* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }

constexpr unsigned long long kWeightOnly = 1;   // < any candidate's key: indices stay below 2^30

struct Best {
    float v = -1.f;   // below a quotient that underflows to zero
    int i = -1;
    bool weight = false;   // some column has w > 0
    __device__ __forceinline__ void take(float w, float e, int idx) {
        weight |= w > 0.f;
        const float bar = v * e * 0.999999f;
        if (w > 0.f && e > 0.f && (w >= bar || bar < 1e-30f)) {
            const float s = __fdiv_rn(w, e);
            if (s > v) {   // a thread walks its indices upwards: the first of equals stays
                v = s;
                i = idx;
            }
        }
    }
};

// The block's best (value bits, ~index), kWeightOnly if no column with a weight has a positive e, 0 if no column
// has a weight; in every thread of warp 0.
__device__ __forceinline__ unsigned long long block_best(const Best& m) {
    __shared__ unsigned long long wk[kVerifyThreads / 32];
    unsigned long long k =
        m.i < 0 ? (m.weight ? kWeightOnly : 0ull)
                : (static_cast<unsigned long long>(__float_as_uint(m.v)) << 32) | (0xffffffffu - m.i);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const unsigned long long x = __shfl_xor_sync(0xffffffffu, k, o);
        k = x > k ? x : k;
    }
    __syncthreads();
    if (lane_id() == 0) wk[warp_id()] = k;
    __syncthreads();
    k = lane_id() < kVerifyThreads / 32 ? wk[lane_id()] : 0ull;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const unsigned long long x = __shfl_xor_sync(0xffffffffu, k, o);
        k = x > k ? x : k;
    }
    return k;
}

// Best of columns [v0, v1): w = max(p - q, 0), or p where q is null.
template <bool VEC>
__device__ __forceinline__ void scan_row(Best& m, const float* p, const float* q, const float* e, int drop, int v0,
                                         int v1) {
    if constexpr (VEC) {
        constexpr int U = 2;
        for (int c = v0 + 4 * threadIdx.x; c < v1; c += U * 4 * kVerifyThreads) {
            float4 pv[U], qv[U], ev[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int x = c + u * 4 * kVerifyThreads;
                pv[u] = qv[u] = ev[u] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (x + 3 < v1) {
                    pv[u] = __ldcs(reinterpret_cast<const float4*>(p + x));
                    ev[u] = __ldcs(reinterpret_cast<const float4*>(e + x));
                    if (q != nullptr) qv[u] = __ldcs(reinterpret_cast<const float4*>(q + x));
                } else if (x < v1) {   // the row's last columns
                    pv[u].x = p[x];
                    ev[u].x = e[x];
                    if (q != nullptr) qv[u].x = q[x];
                    if (x + 1 < v1) {
                        pv[u].y = p[x + 1];
                        ev[u].y = e[x + 1];
                        if (q != nullptr) qv[u].y = q[x + 1];
                    }
                    if (x + 2 < v1) {
                        pv[u].z = p[x + 2];
                        ev[u].z = e[x + 2];
                        if (q != nullptr) qv[u].z = q[x + 2];
                    }
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int x = c + u * 4 * kVerifyThreads;
                m.take(x == drop ? 0.f : pv[u].x - qv[u].x, ev[u].x, x);
                m.take(x + 1 == drop ? 0.f : pv[u].y - qv[u].y, ev[u].y, x + 1);
                m.take(x + 2 == drop ? 0.f : pv[u].z - qv[u].z, ev[u].z, x + 2);
                m.take(x + 3 == drop ? 0.f : pv[u].w - qv[u].w, ev[u].w, x + 3);
            }
        }
    } else {
        constexpr int U = 8;
        for (int c = v0 + threadIdx.x; c < v1; c += U * kVerifyThreads) {
            float pv[U], qv[U], ev[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int x = c + u * kVerifyThreads;
                pv[u] = x < v1 ? __ldcs(p + x) : 0.f;
                ev[u] = x < v1 ? __ldcs(e + x) : 0.f;
                qv[u] = x < v1 && q != nullptr ? __ldcs(q + x) : 0.f;
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int x = c + u * kVerifyThreads;
                m.take(x == drop ? 0.f : pv[u] - qv[u], ev[u], x);
            }
        }
    }
}

template <bool VEC>
__global__ void __launch_bounds__(kVerifyThreads, kVerifyBlocks) verify_kernel(VerifyArgs a) {
    __shared__ int sh_a, sh_last;
    const int b = blockIdx.y, t = threadIdx.x;
    grid_dep_wait();
    const int c0 = load(a.cu + b), c1 = load(a.cu + b + 1);
    if (c0 < 0 || c1 < c0 || c1 > a.Td || c1 - c0 > a.W) {
        if (blockIdx.x == 0) {
            if (t == 0) {
                atomicExch(a.status, kStatusBadInput);
                a.accepted[b] = 0;
            }
            for (int j = t; j <= a.W; j += kVerifyThreads) a.out[static_cast<size_t>(b) * (a.W + 1) + j] = -1;
        }
        return;
    }
    const float* e = a.noise + static_cast<size_t>(b) * a.lde;
    const int v0 = blockIdx.x * a.chunk, v1 = min(a.V, v0 + a.chunk);
    // the noise is read whatever is accepted: it travels while that is found out
    for (int v = v0 + 32 * t; v < v1; v += 32 * kVerifyThreads) prefetch_l2(e + v);
    const int n = c1 - c0;
    const float* P = a.target + static_cast<size_t>(c0 + b) * a.ldp;   // the request's n + 1 rows
    const float* Qd = a.draft == nullptr ? nullptr : a.draft + static_cast<size_t>(c0) * a.ldq;
    if (t < 32) {
        int acc = n;
        for (int j0 = 0; j0 < n; j0 += 32) {
            const int j = j0 + t;
            bool ok = true;
            if (j < n) {
                const int x = load(a.tokens + c0 + j);
                if (x < 0 || x >= a.V) {
                    if (blockIdx.x == 0) atomicExch(a.status, kStatusBadInput);
                    ok = false;
                } else {
                    const float q = Qd == nullptr ? 1.f : load(Qd + static_cast<size_t>(j) * a.ldq + x);
                    ok = __fmul_rn(load(a.u + c0 + j), q) < load(P + static_cast<size_t>(j) * a.ldp + x);
                }
            }
            const unsigned no = __ballot_sync(0xffffffffu, !ok);
            if (no != 0) {
                acc = j0 + __ffs(no) - 1;
                break;
            }
        }
        if (t == 0) sh_a = acc;
    }
    __syncthreads();
    const int acc = sh_a;
    const float* p = P + static_cast<size_t>(acc) * a.ldp;
    const float* q = acc < n && Qd != nullptr ? Qd + static_cast<size_t>(acc) * a.ldq : nullptr;
    // without draft probabilities the draft is certain: its token leaves the residual
    const int drop = acc < n && Qd == nullptr ? load(a.tokens + c0 + acc) : -1;
    Best m;
    scan_row<VEC>(m, p, q, e, drop, v0, v1);
    const unsigned long long mine = block_best(m);
    if (t == 0) {
        if (mine != 0) atomicMax(a.key + b, mine);
        __threadfence();
        sh_last = atomicAdd(a.count + b, 1) == static_cast<int>(gridDim.x) - 1;
    }
    __syncthreads();
    if (!sh_last) return;
    // the request's last block: zero the workspace for the next launch and write
    __threadfence();
    unsigned long long best = 0;
    if (t < 32) best = t == 0 ? atomicExch(a.key + b, 0ull) : 0ull;
    if (t == 0) {
        a.count[b] = 0;
        sh_a = best != 0;
    }
    __syncthreads();
    if (!sh_a && acc < n) {   // the residual is empty (p <= q everywhere): p itself
        Best r;
        scan_row<VEC>(r, p, nullptr, e, -1, 0, a.V);
        best = block_best(r);
    }
    int32_t* out = a.out + static_cast<size_t>(b) * (a.W + 1);
    for (int j = t; j <= a.W; j += kVerifyThreads)
        if (j != acc) out[j] = j < acc ? load(a.tokens + c0 + j) : -1;
    if (t == 0) {
        a.accepted[b] = acc;
        out[acc] = best > kWeightOnly ? static_cast<int>(0xffffffffu - static_cast<unsigned>(best)) : -1;
        if (best <= kWeightOnly) atomicExch(a.status, kStatusBadInput);   // no column can be chosen
    }
}

}  // namespace

size_t plan_smem(int B) { return static_cast<size_t>(B) * 2 * sizeof(int); }

cudaError_t plan_prepare(int max_seqs) {
    return ensure_smem_attr(reinterpret_cast<const void*>(plan_kernel), plan_smem(max_seqs));
}

cudaError_t launch_plan(const PlanArgs& a, const KernelEnv& env) {
    const int most = 2 * device_sm_count();
    const int need = (max((a.T + kTokens - 1) / kTokens, a.B) + kPlanThreads - 1) / kPlanThreads;
    return launch_early(plan_kernel, dim3(need < most ? need : most), kPlanThreads, plan_smem(a.B), env.stream, a);
}

cudaError_t launch_verify(VerifyArgs a, const KernelEnv& env) {
    // All blocks at once (a second wave would find out again what is accepted, with its
    // memory idle: 44 us against 39.5 at 128 rows of 151936 columns), of at least 2048
    // columns.
    const int splits = a.B < kVerifyBlocks * device_sm_count() ? kVerifyBlocks * device_sm_count() / a.B : 1;
    const int chunk = (a.V + splits - 1) / splits;
    a.chunk = ((chunk < 2048 ? 2048 : chunk) + 1023) / 1024 * 1024;
    if (a.chunk > a.V) a.chunk = a.V;
    const dim3 grid((a.V + a.chunk - 1) / a.chunk, a.B);
    auto al = [](const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; };
    const bool vec = al(a.target) && al(a.draft) && al(a.noise) && a.ldp % 4 == 0 && a.ldq % 4 == 0 && a.lde % 4 == 0 &&
                     a.chunk % 4 == 0;
    return launch_early(vec ? verify_kernel<true> : verify_kernel<false>, grid, kVerifyThreads, 0, env.stream, a);
}

}  // namespace sas
