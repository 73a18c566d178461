// Dense causal attention of new tokens over an 8-bit paged cache: e4m3 keys and values, a
// scale for each page and KV head.
//
//   O_i = sum_j softmax_j(scale s_K(j) q_i.k_j) s_V(j) v_j,  LSE_i = log sum_j exp(scale s_K(j) q_i.k_j),
// j over the tokens of the request up to i, s_K(j) and s_V(j) the scales of j's page.
//
// Work is cut as chunk_work.cuh says.  A tile has few rows here (8 or 16: R tokens times the G
// heads of a KV group), and each of four teams of two warps takes whole pages of the item, each
// warp half of the keys, with a running maximum, sum and output of its own, which the block joins
// at the item's end.  (Teams of four have half the registers a warp, and take 156 us where two
// take 108.)  Another warp loads the pages by TMA into rings of shared memory.  A ring has a
// multiple of four places, so that a place is always the same team's: one that waited for a place
// of another's could find it two loads behind, which a barrier's parity does not tell from loaded
// (loads end out of order by microseconds when HBM is busy).
//
// Bound: HBM, 2 d bytes a token and KV head.  What stands between a byte in shared memory and
// the tensor core is its conversion, exact, to f16 (two numbers an instruction; HBM brings a
// multiprocessor 23 a cycle).  It is done once, in registers: the keys are the
// left operand of S^T = K Q^T, the values of O^T = V^T P^T (mma.sync m16n8k16: 16 keys or 16
// dims by 8 rows), so that their numbers go from shared memory to the registers where the
// instruction wants them, and nothing converted is written back: the tensor memory's way
// would store two bytes for each one that HBM brings and read them again, more than shared
// memory moves in that time.  Both products accumulate in fp32.  96 single tokens over 250000
// keys in all, 8 KV heads of 128: 107 us, of which HBM needs 76 (4.8 TB/s) and start, end and join
// of the two launches 12 to 15; one token over 32000 keys 24 us, 9.7 of them HBM's.
//
// Which dim or key stands in which place of an operand is free, as long as both operands agree:
//   * S^T: a lane's four dims of a step are four neighbouring bytes of a key's row;
//   * keys stand in the order PI, for which the lanes' 16-byte reads of eight keys (and of the
//     values of eight keys) fall into different banks under TMA's swizzle;
//   * O^T: lane group g has D / 8 neighbouring dims, two a step.
// P^T passes from one product's accumulators to the other's operand by an 8 x 8 transpose.
//
// Q is f16 too, each row under a power of two of its own that brings its largest number to
// 2^14: bf16 numbers down to 2^-31 of the row's largest are exact, less is below the sum's own
// rounding.  P is f16, at most 2^8 (the maximum is moved when a row's sum would pass that) times
// the page's value scale over that of the accumulator, within 2^-6 .. 2^6 (the accumulator is
// moved where a page's is further off; where it cannot follow, chunk8.cuh, P is smaller).
#include <cuda_fp16.h>

#include "chunk8.cuh"
#include "chunk_work.cuh"

namespace sas {
namespace {

constexpr int kTeams = 4;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kRescaleThreshold = 8.0f;       // log2 units
constexpr float kScaleRange = 64.f;
constexpr int kItemSlots = 4;
constexpr int kStatusLayout = 3;

// NT: 8-row steps of a tile.
template <int D, int NT>
struct Cfg {
    static constexpr int TEAM = 2;                          // warps of a team
    static constexpr int WARPS = kTeams * TEAM;            // that compute
    static constexpr int THREADS = (WARPS + 4) * 32;       // a warpgroup beside them, of which one warp is at work: registers move by warpgroups
    static_assert(THREADS >= kRangeThreads, "find_range");
    static constexpr int ROWS = 8 * NT;
    static constexpr int PAGE = kBN * D;
    static constexpr int ST = D == 128 ? 12 : 24;          // pages of the rings
    static_assert(ST % kTeams == 0, "a place of the rings is one team's");
    static constexpr int OFF_V = ST * PAGE;
    static constexpr int OFF_SUM = 2 * ST * PAGE;          // the warps' outputs of RR rows, joined
    static constexpr int RR = 8 / TEAM;
    static constexpr int SUM_LD = D + 4;
    static constexpr int SUM_BYTES = WARPS * RR * SUM_LD * 4;
    static constexpr int OFF_Q = OFF_SUM + SUM_BYTES;
    static constexpr int Q_LD = 2 * D + 8;                 // bytes: the lanes' 8-byte reads fall into different banks
    static constexpr int OFF_ML = OFF_Q + ROWS * Q_LD;     // [warp][row] (max, sum)
    static constexpr int OFF_CTL = OFF_ML + WARPS * ROWS * 8;
    static constexpr int SMEM = OFF_CTL + 2048;
    static_assert(SMEM <= 232448 && OFF_SUM % 16 == 0 && OFF_Q % 16 == 0 && OFF_CTL % 16 == 0, "shared memory");
    // Registers of the loading and of the computing warpgroups; the sum is what the block is launched with:
    // 128 x 88 + 256 x 208 = 384 x 168.
    static constexpr int FEWER = 88, MORE = 208;
};

struct Ctl {
    uint64_t k_full[24], k_empty[24], v_full[24], v_empty[24];
    uint64_t item_full[kItemSlots], item_empty[kItemSlots];
    float ks[24], vs[24];       // the pages' scales
    float row_scale[16];        // of the item's rows: log2(e) scale over the row's power of two
    Item item[kItemSlots];
    int abort_flag;
};
static_assert(sizeof(Ctl) + sizeof(Shares) <= 2048, "control block");

__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Two e4m3 numbers (the low or high half of w) as f16.
__device__ __forceinline__ uint32_t f16_lo(uint32_t w) {
    uint32_t r;
    asm("{\n\t.reg .b16 x, y;\n\tmov.b32 {x, y}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, x;\n\t}" : "=r"(r) : "r"(w));
    return r;
}
__device__ __forceinline__ uint32_t f16_hi(uint32_t w) {
    uint32_t r;
    asm("{\n\t.reg .b16 x, y;\n\tmov.b32 {x, y}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, y;\n\t}" : "=r"(r) : "r"(w));
    return r;
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
// 8 x 8 of 16 bits: lane (g, t) has row g, columns 2t and 2t + 1, and gets them of the transpose.
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
// Waits for the computing threads; true if any of them says so.
template <int THREADS>
__device__ __forceinline__ bool compute_sync_or(bool x) {
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, 1, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(r)
        : "r"(static_cast<uint32_t>(x)), "n"(THREADS)
        : "memory");
    return r != 0;
}

// The key, of eight, in place i of an operand.  Even and odd places differ in the bit that moves
// a 64-byte half (D = 128) or a row's half of 128 bytes (D = 64) in a read of two keys by four lanes
// each, and the even (odd) ones of the four lane pairs differ in the bits that move 32 bytes.
template <int D>
__device__ __forceinline__ int place(int i) {
    const int p = i >> 1;
    if constexpr (D == 128) return (i & 1) ? ((2 * p) ^ 4) + 1 : 2 * p;
    else return (p & 1) + 4 * (p >> 1) + ((i & 1) ? ((p & 1) ? 1 : 3) : 0);
}

template <int D, int NT>
__global__ void __launch_bounds__(Cfg<D, NT>::THREADS, 1)
chunk8_kernel(const __grid_constant__ CUtensorMap mapK, const __grid_constant__ CUtensorMap mapV, ChunkArgs a, float scale_log2,
              int rl, long long limit) {
    using C = Cfg<D, NT>;
    constexpr int MT = D / 16;             // 16-dim steps of O^T
    constexpr int kWarps = C::WARPS;
    auto compute_sync = [] { named_bar_sync(1, kWarps * 32); };
    extern __shared__ __align__(1024) uint8_t smem[];
    if ((smem_u32(smem) & 1023u) != 0) {
        grid_dep_wait();
        if (threadIdx.x == 0) {
            atomicExch(a.status, kStatusLayout);
            a.joins[2 * blockIdx.x] = make_int4(0, 0, 0, 0);
        }
        return;
    }
    Ctl& ctl = *reinterpret_cast<Ctl*>(smem + C::OFF_CTL);
    Shares& sh = *reinterpret_cast<Shares*>(smem + C::OFF_CTL + (sizeof(Ctl) + 15) / 16 * 16);
    const uint32_t warp = warp_id(), lane = lane_id();
    if (threadIdx.x == 0) {
        for (int s = 0; s < C::ST; ++s) {
            mbar_init(&ctl.k_full[s], 1);
            mbar_init(&ctl.k_empty[s], C::TEAM);
            mbar_init(&ctl.v_full[s], 1);
            mbar_init(&ctl.v_empty[s], C::TEAM);
        }
        for (int s = 0; s < kItemSlots; ++s) {
            mbar_init(&ctl.item_full[s], 1);
            mbar_init(&ctl.item_empty[s], kWarps);
        }
        ctl.abort_flag = 0;
        fence_barrier_init();
    }
    __syncthreads();
    const WaitCtl wc{&ctl.abort_flag, a.status, limit};
    grid_dep_wait();   // whatever the stream ran before: lengths, table, cache
    const bool any = find_range(a, rl, sh);
    grid_dep_launch();   // the join's blocks may take the places that open up (they wait for this grid's end)

    // Every warp walks the same items and counts pages over all of them (g): ring slots and
    // barrier phases follow g across item boundaries, and page g is team g % kTeams's.
    if (warp >= kWarps) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::FEWER));
        if (warp != kWarps) return;
        if (lane == 0) {
            tma_prefetch_desc(&mapK);
            tma_prefetch_desc(&mapV);
        }
        Walk walk(a, rl, sh, any);
        int g = 0, gv = 0;
        bool ok = true;
        for (int r = 0; ok; ++r) {
            const Item x = walk.next(a, rl);
            const int slot = r % kItemSlots;
            if (!mbar_wait_warp(&ctl.item_empty[slot], ((r / kItemSlots) & 1) ^ 1u, wc)) { ok = false; break; }
            if (lane == 0) {
                ctl.item[slot] = x;
                mbar_arrive(&ctl.item_full[slot]);
            }
            __syncwarp();
            if (x.head < 0) break;
            int rows = 0;
            float ks = 1.f, vs = 1.f;
            for (int m = x.blk0; m < x.blk1; ++m, ++g) {
                const int j = (m - x.blk0) & 31;
                if (j == 0) {
                    rows = page_row(a, x, m, lane);
                    const bool real = m + static_cast<int>(lane) < x.blk1 && rows < a.num_pages * a.Hkv;
                    ks = real ? load(a.k_scale + rows) : 1.f;
                    vs = real ? load(a.v_scale + rows) : 1.f;
                }
                const int row = __shfl_sync(0xffffffffu, rows, j);
                const float ksj = __shfl_sync(0xffffffffu, ks, j), vsj = __shfl_sync(0xffffffffu, vs, j);
                const int s = g % C::ST;
                const uint32_t phase = ((g / C::ST) & 1) ^ 1u;
                if (!mbar_wait_warp(&ctl.k_empty[s], phase, wc)) { ok = false; break; }
                if (lane == 0) {
                    ctl.ks[s] = ksj;
                    ctl.vs[s] = vsj;
                    mbar_arrive_expect_tx(&ctl.k_full[s], C::PAGE);
                    tma_load_3d(smem + s * C::PAGE, &mapK, &ctl.k_full[s], 0, 0, row);
                }
                __syncwarp();
                if (!mbar_wait_warp(&ctl.v_empty[s], phase, wc)) { ++g; ok = false; break; }
                if (lane == 0) {
                    mbar_arrive_expect_tx(&ctl.v_full[s], C::PAGE);
                    tma_load_3d(smem + C::OFF_V + s * C::PAGE, &mapV, &ctl.v_full[s], 0, 0, row);
                }
                ++gv;
                __syncwarp();
            }
        }
        walk.record(a, rl, sh);
        if (!ok && lane == 0) {   // the last loads may be in flight
            for (int q = g - 1; q >= 0 && q >= g - C::ST; --q)
                mbar_wait_drain(&ctl.k_full[q % C::ST], (q / C::ST) & 1, limit, a.status);
            for (int q = gv - 1; q >= 0 && q >= gv - C::ST; --q)
                mbar_wait_drain(&ctl.v_full[q % C::ST], (q / C::ST) & 1, limit, a.status);
        }
        return;
    }

    // ---------------- the computing warps
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::MORE));
    const int gq = lane >> 2, t = lane & 3;   // the lane's group of four and its place there
    const int gl = 31 - __clz(a.G);
    const int key_a = place<D>(gq);                                  // S^T: the lane's key, of eight
    const int key_0 = place<D>(2 * t), key_1 = place<D>(2 * t + 1);  // O^T: its two keys, of eight
    float2* const ml = reinterpret_cast<float2*>(smem + C::OFF_ML);
    float* const sums = reinterpret_cast<float*>(smem + C::OFF_SUM);
    bool ok = true;
    int g0 = 0;   // pages of the items before
    for (int r = 0;; ++r) {
        Item x;
        x.head = -1;
        x.blk0 = x.blk1 = 0;
        {
            const int slot = r % kItemSlots;
            ok = ok && mbar_poll_warp(&ctl.item_full[slot], (r / kItemSlots) & 1, wc);
            if (ok) {
                x = ctl.item[slot];
                __syncwarp();
                if (lane == 0) mbar_arrive(&ctl.item_empty[slot]);
            }
        }
        // the warps leave together: none waits at a barrier that another does not reach
        if (compute_sync_or<kWarps * 32>(!ok) || x.head < 0) break;
        const int nrow = x.ntok << gl, nt = (nrow + 7) >> 3;

        // ---- Q as f16 in shared memory, a row by D / 8 lanes
        {
            constexpr int LPR = D / 8;
            for (int i = threadIdx.x; i < nt * 8 * LPR; i += kWarps * 32) {
                const int row = i / LPR, c = i % LPR;
                uint4 raw = make_uint4(0, 0, 0, 0);
                if (row < nrow) {
                    const size_t at = (static_cast<size_t>(x.tok0) + (row >> gl)) * a.Hq + static_cast<size_t>(x.head) * a.G + (row & (a.G - 1));
                    raw = load(reinterpret_cast<const uint4*>(a.Q + at * D) + c);
                }
                float f[8];
                const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
                float top = 0.f;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    f[2 * k] = __uint_as_float(w[k] << 16);
                    f[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
                    top = max3f(top, fabsf(f[2 * k]), fabsf(f[2 * k + 1]));
                }
#pragma unroll
                for (int o = LPR / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                // 2^e <= top < 2^(e + 1): times 2^(14 - e)
                const int e = max(-100, min(127, static_cast<int>(__float_as_uint(top) >> 23) - 127));
                const float up = __uint_as_float(static_cast<uint32_t>(127 + 14 - e) << 23);
                if (c == 0) ctl.row_scale[row] = scale_log2 * __uint_as_float(static_cast<uint32_t>(127 - 14 + e) << 23);
                uint2* const dst = reinterpret_cast<uint2*>(smem + C::OFF_Q + row * C::Q_LD + c * 16);
                dst[0] = make_uint2(pack_f16x2(f[0] * up, f[1] * up), pack_f16x2(f[2] * up, f[3] * up));
                dst[1] = make_uint2(pack_f16x2(f[4] * up, f[5] * up), pack_f16x2(f[6] * up, f[7] * up));
            }
        }
        compute_sync();

        float o[MT][NT][4];
        float m_use[NT][2], l[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            m_use[n][0] = m_use[n][1] = -CUDART_INF_F;
            l[n][0] = l[n][1] = 0.f;
#pragma unroll
            for (int i = 0; i < MT; ++i) o[i][n][0] = o[i][n][1] = o[i][n][2] = o[i][n][3] = 0.f;
        }
        float v_ref = 0.f;   // what one of o stands for; 0: nothing yet
        bool large = false;  // a scale was above kLargeScale
        const int np = x.blk1 - x.blk0;
        for (int i = (static_cast<int>(warp / C::TEAM) - g0) & (kTeams - 1); ok && i < np; i += kTeams) {
            const int g = g0 + i, s = g % C::ST, m = x.blk0 + i;
            const uint32_t phase = (g / C::ST) & 1;
            const uint8_t* const K = smem + s * C::PAGE;
            const uint8_t* const V = smem + C::OFF_V + s * C::PAGE;
            if (!mbar_wait_warp(&ctl.k_full[s], phase, wc)) { ok = false; break; }
            const float ks = ctl.ks[s], vs = ctl.vs[s];
            const int first = m * kBN;
            const bool late = first + kBN - 1 > x.pos0;   // some row does not see all of the page
            constexpr int KT = 4 / C::TEAM;   // 16-key steps of a warp's share
            const int share = warp % C::TEAM;
            if (v_ref == 0.f) v_ref = vs;
            large |= vs > kLargeScale;
            if (!(vs <= kScaleRange * v_ref && vs * kScaleRange >= v_ref)) {
                float f = v_ref / vs;
                if (f <= 1.f) {
                    if (f < kFarRise) {
                        f = v_ref * kRiseRest / vs;
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int y = 0; y < MT; ++y)
#pragma unroll
                                for (int e = 0; e < 4; ++e) o[y][n][e] *= kRiseStep;
                    }
                    v_ref = vs;
                } else {
                    float top = 0.f;
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int y = 0; y < MT; ++y)
#pragma unroll
                            for (int e = 0; e < 4; ++e) top = fmaxf(top, finite_size(o[y][n][e]));
#pragma unroll
                    for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                    f = move_unit(v_ref, vs, top);
                }
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int y = 0; y < MT; ++y)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[y][n][e] *= f;
            }
            const float ratio = vs / v_ref;
            // ---- S^T = K Q^T
            float c[KT][NT][4];
#pragma unroll
            for (int k = 0; k < KT; ++k)
#pragma unroll
                for (int n = 0; n < NT; ++n) c[k][n][0] = c[k][n][1] = c[k][n][2] = c[k][n][3] = 0.f;
#pragma unroll
            for (int j = 0; j < D / 64; ++j) {
                uint4 w[KT][2];
#pragma unroll
                for (int k = 0; k < KT; ++k) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int key = (share * KT + k) * 16 + h * 8 + key_a;
                        const int chunk = D == 128 ? (4 * j + t) ^ (key_a & 7) : t ^ ((key_a >> 1) & 3);
                        w[k][h] = *reinterpret_cast<const uint4*>(K + key * D + chunk * 16);
                    }
                }
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    uint2 b[NT];
#pragma unroll
                    for (int n = 0; n < NT; ++n)
                        if (n < nt) b[n] = *reinterpret_cast<const uint2*>(smem + C::OFF_Q + (n * 8 + gq) * C::Q_LD + (64 * j + 16 * t + 4 * q) * 2);
#pragma unroll
                    for (int k = 0; k < KT; ++k) {
                        const uint32_t w0 = q == 0 ? w[k][0].x : q == 1 ? w[k][0].y : q == 2 ? w[k][0].z : w[k][0].w;
                        const uint32_t w1 = q == 0 ? w[k][1].x : q == 1 ? w[k][1].y : q == 2 ? w[k][1].z : w[k][1].w;
                        const uint32_t a0 = f16_lo(w0), a1 = f16_lo(w1), a2 = f16_hi(w0), a3 = f16_hi(w1);
#pragma unroll
                        for (int n = 0; n < NT; ++n)
                            if (n < nt) mma_f16(c[k][n], a0, a1, a2, a3, b[n].x, b[n].y);
                    }
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&ctl.k_empty[s]);
            // ---- softmax
            uint32_t p[KT][NT][2];
            float mx[NT][2], cr[NT][2];
            bool need = false;
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                if (n >= nt) continue;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int row = n * 8 + 2 * t + e;
                    cr[n][e] = score_factor(ctl.row_scale[row], ks);
                    if (late) {
                        const int lim = x.pos0 + (row >> gl) - first;   // its last key of the page
#pragma unroll
                        for (int k = 0; k < KT; ++k) {
                            const int key = (share * KT + k) * 16 + key_a;
                            if (key > lim) c[k][n][e] = -CUDART_INF_F;
                            if (key + 8 > lim) c[k][n][2 + e] = -CUDART_INF_F;
                        }
                    }
                    float top = -CUDART_INF_F;
#pragma unroll
                    for (int k = 0; k < KT; ++k) top = max3f(top, c[k][n][e], c[k][n][2 + e]);
                    mx[n][e] = top * cr[n][e];
                    need |= mx[n][e] > m_use[n][e] + kRescaleThreshold;
                }
            }
            if (__any_sync(0xffffffffu, need)) {
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    if (n >= nt) continue;
                    float f[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float top = mx[n][e];
#pragma unroll
                        for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                        const float m_new = top > m_use[n][e] + kRescaleThreshold ? top : m_use[n][e];
                        f[e] = m_new == m_use[n][e] ? 1.f : fast_exp2(m_use[n][e] - m_new);
                        m_use[n][e] = m_new;
                        l[n][e] *= f[e];
                    }
#pragma unroll
                    for (int y = 0; y < MT; ++y) {
                        o[y][n][0] *= f[0];
                        o[y][n][1] *= f[1];
                        o[y][n][2] *= f[0];
                        o[y][n][3] *= f[1];
                    }
                }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                if (n >= nt) continue;
                float off[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) off[e] = m_use[n][e] == -CUDART_INF_F ? 0.f : -m_use[n][e];
#pragma unroll
                for (int k = 0; k < KT; ++k) {
                    float v[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        v[e] = fast_exp2(fmaf(c[k][n][e], cr[n][e & 1], off[e & 1]));
                        l[n][e & 1] += v[e];
                    }
                    p[k][n][0] = pack_f16x2(v[0] * ratio, v[1] * ratio);
                    p[k][n][1] = pack_f16x2(v[2] * ratio, v[3] * ratio);
                }
            }
            // ---- O^T += V^T P^T
            if (!mbar_wait_warp(&ctl.v_full[s], phase, wc)) { ok = false; break; }
            const int end = x.pos0 + x.ntok - first;   // keys from here on belong to no row: their P is 0, but 0 times NaN is not
#pragma unroll
            for (int k = 0; k < KT; ++k) {
                const int key = (share * KT + k) * 16;
                constexpr int W = D / 32;   // words of a lane's dims
                uint32_t v[4][W];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int in8 = e & 1 ? key_1 : key_0, at = key + (e >> 1) * 8 + in8;
                    if constexpr (D == 128) {
                        const uint4 y = *reinterpret_cast<const uint4*>(V + at * D + ((gq ^ (in8 & 7)) << 4));
                        v[e][0] = y.x;
                        v[e][1] = y.y;
                        v[e][2] = y.z;
                        v[e][3] = y.w;
                    } else {
                        const uint2 y = *reinterpret_cast<const uint2*>(V + at * D + ((((gq >> 1) ^ (in8 >> 1)) & 3) << 4) + (gq & 1) * 8);
                        v[e][0] = y.x;
                        v[e][1] = y.y;
                    }
                    if (late && at >= end) {
#pragma unroll
                        for (int y = 0; y < W; ++y) v[e][y] = 0;
                    }
                }
                uint32_t b[NT][2];
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    if (n >= nt) continue;
                    b[n][0] = transpose8(p[k][n][0]);
                    b[n][1] = transpose8(p[k][n][1]);
                }
#pragma unroll
                for (int y = 0; y < W; ++y) {
                    // bytes (dim, dim + 1) of two keys: pairs of keys by dim
                    const uint32_t a01 = __byte_perm(v[0][y], v[1][y], 0x5140), a23 = __byte_perm(v[2][y], v[3][y], 0x5140);
                    const uint32_t b01 = __byte_perm(v[0][y], v[1][y], 0x7362), b23 = __byte_perm(v[2][y], v[3][y], 0x7362);
                    const uint32_t q0 = f16_lo(a01), q1 = f16_hi(a01), q2 = f16_lo(a23), q3 = f16_hi(a23);
                    const uint32_t r0 = f16_lo(b01), r1 = f16_hi(b01), r2 = f16_lo(b23), r3 = f16_hi(b23);
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        if (n >= nt) continue;
                        mma_f16(o[2 * y][n], q0, q1, q2, q3, b[n][0], b[n][1]);
                        mma_f16(o[2 * y + 1][n], r0, r1, r2, r3, b[n][0], b[n][1]);
                    }
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&ctl.v_empty[s]);
        }
        g0 += np;
        if (large) {
            v_ref *= kShrinkFactor;
#pragma unroll
            for (int n = 0; n < NT; ++n) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    m_use[n][e] += kShrink;
                    l[n][e] *= kShrinkFactor;
                }
            }
        }

        // ---- the warps' results, joined in the warps' order
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            if (n >= nt) continue;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], d);
                if (gq == 0) ml[warp * C::ROWS + n * 8 + 2 * t + e] = make_float2(m_use[n][e], l[n][e]);
            }
        }
        compute_sync();
        constexpr int QUADS = D / 4;
        const int jr = threadIdx.x / QUADS, jq = threadIdx.x % QUADS;   // the row, of RR, and the columns this thread joins
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float f[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                if (n >= nt) continue;
                const int row = n * 8 + 2 * t + e;
                float top = -CUDART_INF_F;
#pragma unroll
                for (int w = 0; w < kWarps; ++w) top = fmaxf(top, ml[w * C::ROWS + row].x);
                // a warp whose rows saw no key has 0 (or NaN, which has to come through)
                f[e] = (top == -CUDART_INF_F ? 1.f : m_use[n][e] == -CUDART_INF_F ? l[n][e] : fast_exp2(m_use[n][e] - top)) * v_ref;
            }
#pragma unroll
            for (int h = 0; h < 8 / C::RR; ++h) {
                if (n * 8 + h * C::RR >= nrow) continue;
                if (n + h > 0) compute_sync();   // the rows before have been read
                if (t / (C::RR / 2) == h) {
                    float* const dst = sums + (warp * C::RR + 2 * (t % (C::RR / 2))) * C::SUM_LD + gq * (D / 8);
#pragma unroll
                    for (int y = 0; y < MT; y += 2) {
                        *reinterpret_cast<float4*>(dst + 2 * y) =
                            make_float4(o[y][n][0] * f[0], o[y][n][2] * f[0], o[y + 1][n][0] * f[0], o[y + 1][n][2] * f[0]);
                        *reinterpret_cast<float4*>(dst + C::SUM_LD + 2 * y) =
                            make_float4(o[y][n][1] * f[1], o[y][n][3] * f[1], o[y + 1][n][1] * f[1], o[y + 1][n][3] * f[1]);
                    }
                }
                compute_sync();
                const int row = n * 8 + h * C::RR + jr;
                if (jr >= C::RR || row >= nrow || !ok) continue;
                float top = -CUDART_INF_F, sum = 0.f;
#pragma unroll
                for (int w = 0; w < kWarps; ++w) top = fmaxf(top, ml[w * C::ROWS + row].x);
                float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int w = 0; w < kWarps; ++w) {
                    const float2 z = ml[w * C::ROWS + row];
                    if (z.x == -CUDART_INF_F && z.y == 0.f) continue;   // no key: whatever its output holds
                    sum += z.x == -CUDART_INF_F ? z.y : z.y * fast_exp2(z.x - top);
                    const float4 q = *reinterpret_cast<const float4*>(sums + (w * C::RR + jr) * C::SUM_LD + jq * 4);
                    y.x += q.x;
                    y.y += q.y;
                    y.z += q.z;
                    y.w += q.w;
                }
                if (x.part < 0) {
                    const size_t at = (static_cast<size_t>(x.tok0) + (row >> gl)) * a.Hq + static_cast<size_t>(x.head) * a.G + (row & (a.G - 1));
                    const float inv = 1.f / sum;
                    *reinterpret_cast<uint2*>(a.O + at * D + jq * 4) = make_uint2(pack_bf16x2(y.x * inv, y.y * inv), pack_bf16x2(y.z * inv, y.w * inv));
                    if (jq == 0 && a.LSE != nullptr) a.LSE[at] = top * kLn2 + logf(sum);
                } else {
                    reinterpret_cast<float4*>(a.part_o)[(static_cast<size_t>(x.part) * QUADS + jq) * kBM + row] = y;
                    if (jq == 0) a.part_ml[static_cast<size_t>(x.part) * kBM + row] = make_float2(top, sum);
                }
            }
        }
    }
}

template <int D, int NT>
cudaError_t launch_d(const ChunkArgs& a, const KernelEnv& env, const char** err) {
    using C = Cfg<D, NT>;
    cudaError_t e = ensure_smem_attr(reinterpret_cast<const void*>(chunk8_kernel<D, NT>), C::SMEM);
    if (e != cudaSuccess) { *err = "cudaFuncSetAttribute(8-bit attention)"; return e; }
    CUtensorMap mk, mv;
    const uint64_t rows = static_cast<uint64_t>(a.num_pages) * a.Hkv;
    if (make_tmap_u8_3d(&mk, a.K8, D, kBN, rows) != 0 || make_tmap_u8_3d(&mv, a.V8, D, kBN, rows) != 0) {
        *err = "tensor map";
        return cudaErrorInvalidValue;
    }
    const int rl = 31 - __builtin_clz(C::ROWS / a.G);
    e = launch_early(chunk8_kernel<D, NT>, dim3(a.blocks), C::THREADS, C::SMEM, env.stream, mk, mv, a, a.sm_scale * kLog2e, rl, env.limit);
    if (e != cudaSuccess) { *err = "8-bit attention launch"; return e; }
    e = launch_early(chunk_join_kernel<D>, dim3(a.blocks), kJoinThreads, 0, env.stream, a);
    if (e != cudaSuccess) *err = "8-bit attention join launch";
    return e;
}

template <int D>
cudaError_t launch_rows(const ChunkArgs& a, const KernelEnv& env, const char** err) {
    // tiles as high as the requests' rows are on average (12 requests of 8 rows over 8000 to 20000: 60.5 us with tiles of
    // 8 rows, 62.1 of 16)
    const long long rows = static_cast<long long>(a.T) * a.G;
    if (rows <= 8LL * a.B) return launch_d<D, 1>(a, env, err);
    return launch_d<D, 2>(a, env, err);
}

template <int D>
cudaError_t prepare() {
    cudaError_t e = ensure_smem_attr(reinterpret_cast<const void*>(chunk8_kernel<D, 1>), Cfg<D, 1>::SMEM);
    if (e == cudaSuccess) e = ensure_smem_attr(reinterpret_cast<const void*>(chunk8_kernel<D, 2>), Cfg<D, 2>::SMEM);
    return e;
}

}  // namespace

cudaError_t chunk8_prepare(int d) {
    const cudaError_t e = d == 128 ? prepare<128>() : prepare<64>();
    return e == cudaSuccess ? chunk8_tile_prepare(d) : e;
}

cudaError_t launch_chunk8(ChunkArgs a, const KernelEnv& env, const char** err) {
    // Requests of more than 16 rows on average: tiles of 128 rows, whose products cost the same however many of
    // the rows there are (12 requests over 8000 to 20000, 8 heads of 128: 90 us at 20 rows, 91 at 16, 81 at 8; here 76 at
    // 16 and 61 at 8, and 172 at 20 with tiles of 32 rows, whose outputs take all registers; heads of 64: 67 us at 20
    // rows, 58 at 16, 73 at 8; here 60 at 16 and 70 at 8).  The average is the batch's: 255 single tokens take 189 us and a
    // prompt chunk of 2048 tokens 40 (8 heads), but one call of both 488, the chunk in tiles of 16 rows here.
    if (static_cast<long long>(a.T) * a.G > 16LL * a.B) return launch_chunk8_tile(a, env, err);
    a.blocks = device_sm_count();   // one a multiprocessor
    if (a.d == 128) return launch_rows<128>(a, env, err);
    if (a.d == 64) return launch_rows<64>(a, env, err);
    *err = "8-bit attention: unsupported head dim";
    return cudaErrorInvalidValue;
}

}  // namespace sas
