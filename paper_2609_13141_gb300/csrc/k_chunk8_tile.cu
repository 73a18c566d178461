// Dense causal attention of new tokens over an 8-bit paged cache, for requests of many rows:
// 128-row tiles on the tensor cores (tcgen05).  The formulas and the cache are k_chunk8.cu's,
// the work is cut as chunk_work.cuh says.
//
// The tensor core takes 8-bit numbers only beside 8-bit numbers, and rounding queries and
// weights to 8 bits would show.  So the pages' numbers become f16, exactly, in shared memory:
//   * warp 0 takes work items, publishes them and loads 8-bit pages by bulk copies (one ring,
//     K and V pages in turn);
//   * warps 2 and 3 convert, half of a page's rows each, into rings of f16 tiles in the tensor
//     core's layout, value rows of no key as zero;
//   * warp 1 issues S = Q K^T and O += P V (P read from tensor memory);
//   * warps 4-7, a thread per row: Q as f16 under a power of two of the row's own (k_chunk8.cu),
//     mask, online softmax in the log2 domain, P as f16 pairs into tensor memory, O rescaled
//     only when the maximum grows by 2^8, or where a page's value scale leaves 2^-6 .. 2^6 times
//     the one that O stands under.
#include <cuda_fp16.h>

#include "chunk_work.cuh"

namespace sas {
namespace {

constexpr int kThreads = 256;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kRescaleThreshold = 8.0f;   // log2 units
constexpr float kScaleRange = 64.f;
constexpr int kItemSlots = 4;     // work items in flight between warp 0 and the other roles
constexpr int kItemReaders = 7;   // the MMA issuer, two that convert, four softmax warps
constexpr int kStatusLayout = 3;
static_assert(kThreads == kRangeThreads, "find_range");

// As in k_chunk.cu: a step is KPS pages, whose scores, softmax and product go through the
// pipeline together; half of Q in tensor memory at d = 128.
template <int D>
struct Cfg {
    static constexpr int KPS = D == 64 ? 2 : 1;
    static constexpr bool QT = D == 128;
    static constexpr int Q_BYTES = kBM * 128;        // 64 dims of the rows in shared memory
    static constexpr int QST = D == 64 ? 2 : 1;      // Q tiles (of the item at work, and the next one's)
    static constexpr int KV_BYTES = kBN * D * 2;
    static constexpr int PAGE = kBN * D;
    static constexpr int KST = D == 64 ? 4 : 2;      // f16 pages of a ring
    static constexpr int SST = D == 64 ? 4 : 4;      // 8-bit pages
    static constexpr int OFF_K = QST * Q_BYTES;
    static constexpr int OFF_V = OFF_K + KST * KV_BYTES;
    static constexpr int OFF_S = OFF_V + KST * KV_BYTES;
    static constexpr int OFF_CTL = OFF_S + SST * PAGE;
    static constexpr int SMEM = OFF_CTL + 1024;      // barriers and items, then Shares
    static_assert(2 * (SMEM + 1024) <= 233472, "two blocks a multiprocessor");
    static constexpr int TMEM_COLS = 256;
    static constexpr int TMEM_O = 0;
    static constexpr int TMEM_S = D;
    static constexpr int TMEM_P = TMEM_S + KPS * kBN;   // keys packed in pairs
    static constexpr int TMEM_Q = TMEM_P + 32 * KPS;    // the row's first 64 dims packed in pairs
    static_assert(TMEM_Q + (QT ? 32 : 0) <= TMEM_COLS, "tensor memory");
    static constexpr uint32_t IDESC_S = idesc_f16(kBM, kBN, 0, 0);
    static constexpr uint32_t IDESC_O = idesc_f16(kBM, D, 0, 1);
};

// Moves registers between the block's two warpgroups (the sum stays within what it was
// launched with: 128 threads x (64 + 184) <= 256 x 128).
template <int D>
__device__ __forceinline__ void give_registers() {
    if constexpr (Cfg<D>::KPS == 2) asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
}
template <int D>
__device__ __forceinline__ void take_registers() {
    if constexpr (Cfg<D>::KPS == 2) asm volatile("setmaxnreg.inc.sync.aligned.u32 184;");
}

struct Ctl {
    uint64_t s_full[4], s_empty[4], k_full[4], k_empty[4], v_full[4], v_empty[4];
    uint64_t sc_full, sc_free, p_full, pv_done, q_ready, drain_bar;
    uint64_t item_full[kItemSlots], item_empty[kItemSlots];
    float ks[16], vs[16];      // scales of page g at g % 16 (the loads are 8 pages ahead of the softmax at most)
    Item item[kItemSlots];
    uint32_t tmem_base;
    int abort_flag;
    int again;                 // the step's product comes in two parts
};
static_assert(sizeof(Ctl) <= 720 && sizeof(Shares) <= 304, "control block");
constexpr int kSharesAt = 720;

__device__ __forceinline__ bool read_item(Ctl& ctl, int r, const WaitCtl& wc, Item& x) {
    const int slot = r % kItemSlots;
    if (!mbar_poll_warp(&ctl.item_full[slot], (r / kItemSlots) & 1, wc)) return false;
    x = ctl.item[slot];
    __syncwarp();
    if (lane_id() == 0) mbar_arrive(&ctl.item_empty[slot]);
    return true;
}

__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
// Four e4m3 numbers as f16.
__device__ __forceinline__ void to_f16(uint32_t w, uint32_t& lo, uint32_t& hi) {
    asm("{\n\t.reg .b16 x, y;\n\tmov.b32 {x, y}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, x;\n\tcvt.rn.f16x2.e4m3x2 %1, y;\n\t}"
        : "=r"(lo), "=r"(hi)
        : "r"(w));
}

// Half of a page's rows (32 half ..) from bytes to a 128-byte-swizzled f16 tile [D / 64][64][64];
// rows from `live` on become zero.  Reads are 16 bytes a lane in order; a lane writes two
// neighbouring 16-byte pieces, at D = 128 in an order that keeps eight lanes' pieces in
// different banks.
template <int D>
__device__ __forceinline__ void convert(uint8_t* dst, const uint8_t* src, int half, int lane, int live) {
    constexpr int CH = D / 16, N = 32 * CH / 32;   // 16-byte chunks of a row, of a lane
#pragma unroll
    for (int i0 = 0; i0 < N; i0 += 4) {
        uint4 w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = *reinterpret_cast<const uint4*>(src + half * (32 * D) + ((i0 + i) * 32 + lane) * 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int at = (i0 + i) * 32 + lane, row = half * 32 + at / CH, c = at % CH;
            uint4 a, b;
            to_f16(w[i].x, a.x, a.y);
            to_f16(w[i].y, a.z, a.w);
            to_f16(w[i].z, b.x, b.y);
            to_f16(w[i].w, b.z, b.w);
            if (row >= live) a = b = make_uint4(0, 0, 0, 0);
            const int h = c >> 2, p = (2 * c) & 7, x = row & 7;
            uint8_t* const to = dst + h * (kBN * 128) + row * 128;
            const bool swap = h != 0;
            *reinterpret_cast<uint4*>(to + (((p + swap) ^ x) << 4)) = swap ? b : a;
            *reinterpret_cast<uint4*>(to + (((p + !swap) ^ x) << 4)) = swap ? a : b;
        }
    }
}

template <int D>
__global__ void __launch_bounds__(kThreads, 2) chunk8_tile_kernel(ChunkArgs a, float scale_log2, long long limit) {
    using C = Cfg<D>;
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
    const uint32_t warp = warp_id(), lane = lane_id();
    if (threadIdx.x == 0) {
        for (int s = 0; s < C::SST; ++s) { mbar_init(&ctl.s_full[s], 1); mbar_init(&ctl.s_empty[s], 2); }
        for (int s = 0; s < C::KST; ++s) { mbar_init(&ctl.k_full[s], 2); mbar_init(&ctl.k_empty[s], 1); }
        for (int s = 0; s < C::KST; ++s) { mbar_init(&ctl.v_full[s], 2); mbar_init(&ctl.v_empty[s], 1); }
        mbar_init(&ctl.sc_full, 1);
        mbar_init(&ctl.sc_free, 4);
        mbar_init(&ctl.pv_done, 1);
        mbar_init(&ctl.p_full, 4);
        mbar_init(&ctl.q_ready, 4);
        mbar_init(&ctl.drain_bar, 1);
        for (int s = 0; s < kItemSlots; ++s) {
            mbar_init(&ctl.item_full[s], 1);
            mbar_init(&ctl.item_empty[s], kItemReaders);
        }
        ctl.abort_flag = 0;
        ctl.again = 0;
        fence_barrier_init();
    }
    if (warp == 1) {
        tmem_alloc(&ctl.tmem_base, C::TMEM_COLS);
        tmem_relinquish();
    }
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = ctl.tmem_base;
    const WaitCtl wc{&ctl.abort_flag, a.status, limit};
    Shares& sh = *reinterpret_cast<Shares*>(smem + C::OFF_CTL + kSharesAt);
    grid_dep_wait();   // whatever the stream ran before: lengths, table, cache
    const int rl = 31 - __clz(kBM / a.G);   // 2^rl tokens of a tile (G is 1, 2, 4 or 8)
    const bool any = find_range(a, rl, sh);
    grid_dep_launch();   // the join's blocks may take the places that open up (they wait for this grid's end)

    // Every role walks the same items and counts pages over all of them (g): ring slots, score
    // buffers and barrier phases follow g across item boundaries.  K page g is the 8-bit ring's
    // 2 g, V page g its 2 g + 1.
    if (warp < 4) {
        give_registers<D>();
        if (warp == 0) {
            // ---------------- items and 8-bit pages
            Walk walk(a, rl, sh, any);
            int n = 0;   // pages loaded
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
                for (int m = x.blk0; ok && m < x.blk1; ++m) {
                    const int j = (m - x.blk0) & 31;
                    if (j == 0) {
                        rows = page_row(a, x, m, lane);
                        const bool real = m + static_cast<int>(lane) < x.blk1 && rows < a.num_pages * a.Hkv;
                        ks = real ? load(a.k_scale + rows) : 1.f;
                        vs = real ? load(a.v_scale + rows) : 1.f;
                    }
                    const int row = __shfl_sync(0xffffffffu, rows, j);
                    const float ksj = __shfl_sync(0xffffffffu, ks, j), vsj = __shfl_sync(0xffffffffu, vs, j);
                    const bool bad = row >= a.num_pages * a.Hkv;   // reads as zero
                    for (int v = 0; v < 2; ++v, ++n) {
                        const int s = n % C::SST;
                        if (!mbar_wait_warp(&ctl.s_empty[s], ((n / C::SST) & 1) ^ 1u, wc)) { ok = false; break; }
                        uint8_t* const dst = smem + C::OFF_S + s * C::PAGE;
                        if (bad) {
                            for (int i = lane; i < C::PAGE / 16; i += 32) reinterpret_cast<uint4*>(dst)[i] = make_uint4(0, 0, 0, 0);
                            __syncwarp();
                        }
                        if (lane == 0) {
                            if (v == 0) {
                                ctl.ks[(n >> 1) % 16] = ksj;
                                ctl.vs[(n >> 1) % 16] = vsj;
                            }
                            if (bad) {
                                mbar_arrive(&ctl.s_full[s]);
                            } else {
                                mbar_arrive_expect_tx(&ctl.s_full[s], C::PAGE);
                                bulk_load(dst, (v == 0 ? a.K8 : a.V8) + static_cast<size_t>(row) * C::PAGE, C::PAGE, &ctl.s_full[s]);
                            }
                        }
                        __syncwarp();
                    }
                }
            }
            walk.record(a, rl, sh);
            if (!ok && lane == 0) {   // the last SST loads may be in flight
                for (int q = n - 1; q >= 0 && q >= n - C::SST; --q)
                    mbar_wait_drain(&ctl.s_full[q % C::SST], (q / C::SST) & 1, limit, a.status);
            }
        } else if (warp >= 2) {
            // ---------------- 8-bit pages to f16 tiles
            const int half = warp - 2;
            int g = 0;
            bool ok = true;
            for (int r = 0; ok; ++r) {
                Item x;
                if (!read_item(ctl, r, wc, x)) { ok = false; break; }
                if (x.head < 0) break;
                const int end = x.pos0 + x.ntok;   // keys from here on belong to no row of the tile
                for (int m = x.blk0; ok && m < x.blk1; ++m, ++g) {
#pragma unroll
                    for (int v = 0; v < 2; ++v) {
                        const int n = 2 * g + v, ss = n % C::SST, s = g % C::KST;
                        if (!mbar_wait_warp(v == 0 ? &ctl.k_empty[s] : &ctl.v_empty[s], ((g / C::KST) & 1) ^ 1u, wc) ||
                            !mbar_wait_warp(&ctl.s_full[ss], (n / C::SST) & 1, wc)) {
                            ok = false;
                            break;
                        }
                        // P is 0 past the end, and 0 times a stale NaN is NaN: such value rows become zero.  Keys
                        // there may be anything.
                        convert<D>(smem + (v == 0 ? C::OFF_K : C::OFF_V) + s * C::KV_BYTES, smem + C::OFF_S + ss * C::PAGE, half, lane,
                                   v == 0 ? kBN : end - m * kBN);
                        fence_proxy_async_smem();
                        __syncwarp();
                        if (lane == 0) {
                            mbar_arrive(v == 0 ? &ctl.k_full[s] : &ctl.v_full[s]);
                            mbar_arrive(&ctl.s_empty[ss]);
                        }
                        __syncwarp();
                    }
                }
            }
        } else {
            // ---------------- products: S of a step ahead of the P V of the one before
            const uint64_t dq0 = smem_desc_sw128(smem_u32(smem), 16, 1024);
            const uint64_t dk0 = smem_desc_sw128(smem_u32(smem + C::OFF_K), 16, 1024);
            const uint64_t dv0 = smem_desc_sw128(smem_u32(smem + C::OFF_V), kBN * 128, 1024);
            int g = 0, gp = 0, tc = 0;   // steps, pages, items
            int vp = 0, np = 0;          // pages of finished products, arrivals of P
            int left = 0;                // pages of the step whose product is due
            bool start = false, ok = true;
            auto product = [&]() {       // P V of the step before; its first page starts a new accumulator
                if (left == 0) return true;
                bool fresh = start;
                for (bool more = true; more;) {
                    for (int i = 0; i < left; ++i)
                        if (!mbar_wait_warp(&ctl.v_full[(vp + i) % C::KST], ((vp + i) / C::KST) & 1, wc)) return false;
                    if (!mbar_wait_warp(&ctl.p_full, np & 1, wc)) return false;
                    ++np;
                    more = C::KPS > 1 && *static_cast<volatile int*>(&ctl.again) != 0;
                    tc_fence_after();
                    for (int i = 0; i < left; ++i) {
                        const int vs = (vp + i) % C::KST;
                        const uint64_t dv = dv0 + static_cast<uint64_t>((vs * C::KV_BYTES) >> 4);
                        if (elect_one()) {
#pragma unroll
                            for (int k = 0; k < kBN / 16; ++k)
                                umma_bf16_ta(tmem_base + C::TMEM_O, tmem_base + C::TMEM_P + i * 32 + k * 8, dv + ((k * 2048) >> 4),
                                             C::IDESC_O, (!fresh || i > 0 || k > 0) ? 1u : 0u);
                            if (!more) umma_commit(&ctl.v_empty[vs]);
                        }
                        __syncwarp();
                    }
                    if (elect_one()) umma_commit(&ctl.pv_done);
                    __syncwarp();
                    fresh = false;
                }
                vp += left;
                left = 0;
                return true;
            };
            for (int r = 0; ok; ++r, ++tc) {
                Item x;
                if (!read_item(ctl, r, wc, x)) { ok = false; break; }
                if (!product()) { ok = false; break; }
                if (x.head < 0) break;
                const int qs = tc % C::QST;
                const uint64_t dq = dq0 + static_cast<uint64_t>((qs * C::Q_BYTES) >> 4);
                if (!mbar_wait_warp(&ctl.q_ready, tc & 1, wc)) { ok = false; break; }
                for (int m = x.blk0; ok && m < x.blk1; m += C::KPS, ++g) {
                    if (g >= 1 && !mbar_wait_warp(&ctl.sc_free, (g - 1) & 1, wc)) { ok = false; break; }
                    int pages = 0;
                    for (int i = 0; i < C::KPS && m + i < x.blk1; ++i, ++gp, ++pages) {
                        const int s = gp % C::KST;
                        if (!mbar_wait_warp(&ctl.k_full[s], (gp / C::KST) & 1, wc)) { ok = false; break; }
                        tc_fence_after();
                        const uint64_t dk = dk0 + static_cast<uint64_t>((s * C::KV_BYTES) >> 4);
                        if (elect_one()) {
#pragma unroll
                            for (int k = 0; k < D / 16; ++k) {
                                const uint32_t off_q = (k & 3) * 32;
                                const uint32_t off_k = (k >> 2) * (kBN * 128) + (k & 3) * 32;
                                if (C::QT && k < 4)
                                    umma_bf16_ta(tmem_base + C::TMEM_S, tmem_base + C::TMEM_Q + k * 8, dk + (off_k >> 4), C::IDESC_S, k > 0);
                                else
                                    umma_bf16(tmem_base + C::TMEM_S + i * kBN, dq + (off_q >> 4), dk + (off_k >> 4), C::IDESC_S, k > 0);
                            }
                            umma_commit(&ctl.k_empty[s]);
                        }
                        __syncwarp();
                    }
                    if (!ok) break;
                    if (elect_one()) umma_commit(&ctl.sc_full);
                    __syncwarp();
                    if (!product()) { ok = false; break; }
                    left = pages;
                    start = m == x.blk0;
                }
            }
            if (elect_one()) {
                umma_commit(&ctl.drain_bar);
                mbar_wait_drain(&ctl.drain_bar, 0, limit, a.status);
            }
            __syncwarp();
        }
    } else {
        // ---------------- softmax, one thread per row
        take_registers<D>();
        constexpr int NK = C::KPS * kBN;   // keys of a step
        const int q = warp - 4;
        const int row = q * 32 + lane;
        const int tok = row / a.G, hq = row - tok * a.G;
        const uint32_t lane_addr = tmem_base + (static_cast<uint32_t>(q * 32) << 16);
        float row_scale = 0.f, next_scale = 0.f;
        // the r-th item, and its rows as f16: the first 64 dims of 128 into tensor memory, the others into
        // shared memory (the products of the item before, which read the ones there, are done: this warp has
        // seen their scores)
        auto take_item = [&](int r, Item& x) {
            if (!read_item(ctl, r, wc, x)) return false;
            if (x.head < 0) return true;
            if (q * 32 < x.ntok * a.G) {
                // twice 64 dims at a time, rather than 128 held: the second time they come out of L2
                const size_t at = (static_cast<size_t>(x.tok0) + tok) * a.Hq + static_cast<size_t>(x.head) * a.G + hq;
                const uint4* const src = reinterpret_cast<const uint4*>(a.Q + at * D);
                uint4 raw[8];
                auto fetch = [&](int h) {
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        raw[c] = make_uint4(0, 0, 0, 0);
                        if (tok < x.ntok) raw[c] = load(src + h * 8 + c);
                    }
                };
                float top = 0.f;
                auto big = [&](uint32_t w) { top = max3f(top, fabsf(__uint_as_float(w << 16)), fabsf(__uint_as_float(w & 0xffff0000u))); };
#pragma unroll 1
                for (int h = 0; h < D / 64; ++h) {
                    fetch(h);
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        big(raw[c].x);
                        big(raw[c].y);
                        big(raw[c].z);
                        big(raw[c].w);
                    }
                }
                // 2^e <= top < 2^(e + 1): times 2^(14 - e)
                const int e = max(-100, min(127, static_cast<int>(__float_as_uint(top) >> 23) - 127));
                const float up = __uint_as_float(static_cast<uint32_t>(127 + 14 - e) << 23);
                next_scale = scale_log2 * __uint_as_float(static_cast<uint32_t>(127 - 14 + e) << 23);
                auto half2 = [&](uint32_t w) { return pack_f16x2(__uint_as_float(w << 16) * up, __uint_as_float(w & 0xffff0000u) * up); };
                // the second half is at hand
                uint8_t* const dst = smem + (r % C::QST) * C::Q_BYTES + row * 128;
#pragma unroll
                for (int c = 0; c < 8; ++c)   // 16-byte chunks, swizzled within the 128-byte row
                    *reinterpret_cast<uint4*>(dst + ((c ^ (row & 7)) << 4)) =
                        make_uint4(half2(raw[c].x), half2(raw[c].y), half2(raw[c].z), half2(raw[c].w));
                if constexpr (C::QT) {
                    fetch(0);
                    uint32_t w[32];
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        w[4 * c] = half2(raw[c].x);
                        w[4 * c + 1] = half2(raw[c].y);
                        w[4 * c + 2] = half2(raw[c].z);
                        w[4 * c + 3] = half2(raw[c].w);
                    }
                    tmem_st32(lane_addr + C::TMEM_Q, w);
                    tmem_wait_st();
                }
                fence_proxy_async_smem();
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&ctl.q_ready);
            return true;
        };
        int g = 0, gp = 0, np = 0;   // steps, pages, arrivals of P
        Item x, nx;
        bool ok = take_item(0, x);
        for (int r = 1; ok && x.head >= 0; x = nx, ++r) {
            row_scale = next_scale;
            const bool valid = tok < x.ntok;
            const bool warp_rows = q * 32 < x.ntok * a.G;   // else nothing of this warp is ever read
            const int pos = x.pos0 + tok;
            float m_use = -CUDART_INF_F, l = 0.f;
            float v_ref = 0.f;   // what one of O stands for
            for (int m = x.blk0; ok && m < x.blk1; m += C::KPS, ++g) {
                const int pages = min(C::KPS, x.blk1 - m);
                // last key column of the step that this row sees (< 0: none; none of a page that is not
                // there).  Rows of no token are never read: they go unmasked.
                const int lim = valid ? min(min(NK - 1, pos - m * kBN), (x.blk1 - m) * kBN - 1) : NK - 1;
                if (!mbar_wait_warp(&ctl.sc_full, g & 1, wc)) { ok = false; break; }
                float ks[C::KPS], vs[C::KPS];
#pragma unroll
                for (int i = 0; i < C::KPS; ++i) {
                    ks[i] = i < pages ? ctl.ks[(gp + i) % 16] : 1.f;
                    vs[i] = i < pages ? ctl.vs[(gp + i) % 16] : vs[0];
                }
                gp += pages;
                if (v_ref == 0.f) v_ref = vs[0];
                auto near = [](float v, float ref) { return v <= kScaleRange * ref && v * kScaleRange >= ref; };
                // a step whose pages cannot stand under one scale has its product in two parts
                const bool parts = C::KPS == 2 && !(near(vs[0], v_ref) && near(vs[C::KPS - 1], v_ref)) && !near(vs[C::KPS - 1], vs[0]);
                // P is free once the product before has read it
                auto p_free = [&] {
                    if (np >= 1 && !mbar_wait_warp(&ctl.pv_done, (np - 1) & 1, wc)) return false;
                    tc_fence_after();
                    return true;
                };
                auto p_ready = [&] {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&ctl.p_full);
                    ++np;
                };
                auto move_to = [&](float v) {   // the factor that O takes
                    const float by = v_ref / v;
                    v_ref = v;
                    return by;
                };
                if (!warp_rows) {
                    if (lane == 0) mbar_arrive(&ctl.sc_free);
                    if (!near(vs[0], v_ref) || (!parts && !near(vs[C::KPS - 1], v_ref))) v_ref = vs[0];
                    if (parts && !near(vs[C::KPS - 1], v_ref)) v_ref = vs[C::KPS - 1];
                    for (int i = 0; ok && i <= static_cast<int>(parts); ++i) {
                        ok = p_free();
                        if (ok) p_ready();
                    }
                    continue;
                }
                tc_fence_after();
                float xs[NK];
                {
                    uint32_t u[NK / 32][32];
#pragma unroll
                    for (int c = 0; c < NK / 32; ++c) tmem_ld32(lane_addr + C::TMEM_S + c * 32, u[c]);
                    tmem_wait_ld();
#pragma unroll
                    for (int k = 0; k < NK; ++k) xs[k] = __uint_as_float(u[k / 32][k % 32]);
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&ctl.sc_free);
                float cr[C::KPS];
                if (__any_sync(0xffffffffu, lim < NK - 1)) {
#pragma unroll
                    for (int k = 0; k < NK; ++k) xs[k] = k <= lim ? xs[k] : -CUDART_INF_F;
                }
                float mb = -CUDART_INF_F;
#pragma unroll
                for (int i = 0; i < C::KPS; ++i) {
                    float mx[4] = {-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F};
#pragma unroll
                    for (int k = i * kBN; k < (i + 1) * kBN; k += 8) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) mx[j] = max3f(mx[j], xs[k + 2 * j], xs[k + 2 * j + 1]);
                    }
                    cr[i] = row_scale * ks[i];
                    mb = fmaxf(mb, fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * cr[i]);
                }
                bool need = valid && mb > m_use + kRescaleThreshold;
                const float m_new = need ? mb : m_use;
                const float off = m_new == -CUDART_INF_F ? 0.f : -m_new;
                float factor = need ? (m_use == -CUDART_INF_F ? 0.f : fast_exp2(m_use - m_new)) : 1.f;
                m_use = m_new;
                l *= factor;
                // O to another maximum, or under another value scale: once the product before is done
                auto rescale = [&](bool change, float by) {
                    if (!__any_sync(0xffffffffu, change)) return true;
                    if (!mbar_wait_warp(&ctl.pv_done, (np - 1) & 1, wc)) return false;
                    tc_fence_after();
#pragma unroll 1
                    for (int cc = 0; cc < D / 32; ++cc) {
                        uint32_t o[32];
                        tmem_ld32(lane_addr + C::TMEM_O + cc * 32, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * by);
                        tmem_st32(lane_addr + C::TMEM_O + cc * 32, o);
                    }
                    tmem_wait_st();
                    return true;
                };
                // P = 2^(z - m) of page i, times its value scale over O's; the row's sum
                auto weights = [&](int i, uint32_t (&pk)[32]) {
                    const float ratio = vs[i] / v_ref;
                    float lr;
                    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(lr) : "f"(ratio));
                    const uint64_t scale2 = f32x2(cr[i], cr[i]), off2 = f32x2(off + lr, off + lr);
                    uint64_t acc[4] = {0, 0, 0, 0};
#pragma unroll
                    for (int k = 0; k < kBN; k += 2) {
                        float a0, a1;
                        f32x2_split(fma_f32x2(f32x2(xs[i * kBN + k], xs[i * kBN + k + 1]), scale2, off2), a0, a1);
                        const float e0 = fast_exp2(a0), e1 = fast_exp2(a1);
                        acc[(k >> 1) & 3] = add_f32x2(acc[(k >> 1) & 3], f32x2(e0, e1));
                        pk[k >> 1] = pack_f16x2(e0, e1);
                    }
                    float s0, s1;
                    f32x2_split(add_f32x2(add_f32x2(acc[0], acc[1]), add_f32x2(acc[2], acc[3])), s0, s1);
                    l = fmaf(s0 + s1, 1.f / ratio, l);
                };
                if (parts) {
                    // rare: a page at a time, the other one's weights zero
#pragma unroll
                    for (int i = 0; i < C::KPS; ++i) {
                        const bool move = !near(vs[i], v_ref);
                        if (move) factor *= move_to(vs[i]);
                        uint32_t pk[32];
                        if ((m > x.blk0 || i > 0) && !rescale(need || move, factor)) { ok = false; break; }
                        weights(i, pk);
                        if (!p_free()) { ok = false; break; }
                        tmem_st32(lane_addr + C::TMEM_P + i * 32, pk);
#pragma unroll
                        for (int k = 0; k < 32; ++k) pk[k] = 0;
                        tmem_st32(lane_addr + C::TMEM_P + (1 - i) * 32, pk);
                        tmem_wait_st();
                        if (threadIdx.x == 128) ctl.again = i == 0;   // warp 4 has rows whenever there are any
                        p_ready();
                        factor = 1.f;
                        need = false;
                    }
                    if (!ok) break;
                    continue;
                }
                bool move = false;
#pragma unroll
                for (int i = 0; i < C::KPS; ++i) move |= !near(vs[i], v_ref);
                if (move) factor *= move_to(vs[0]);
                if (m > x.blk0 && !rescale(need || move, factor)) { ok = false; break; }
                uint32_t pk[C::KPS][32];
#pragma unroll
                for (int i = 0; i < C::KPS; ++i) weights(i, pk[i]);
                if (!p_free()) { ok = false; break; }
#pragma unroll
                for (int i = 0; i < C::KPS; ++i) tmem_st32(lane_addr + C::TMEM_P + i * 32, pk[i]);
                tmem_wait_st();
                p_ready();
            }
            // the next item's Q goes ahead of this one's epilogue: its first product runs during it
            if (!ok || !take_item(r, nx)) { ok = false; break; }
            // The next item's first PV overwrites O only after this warp's next arrival on
            // p_full, which follows the reads below.
            if (!mbar_wait_warp(&ctl.pv_done, (np - 1) & 1, wc)) { ok = false; break; }
            tc_fence_after();
            const size_t orow = (static_cast<size_t>(x.tok0) + tok) * a.Hq + static_cast<size_t>(x.head) * a.G + hq;
            if (x.part < 0) {
                if (warp_rows) {
                    const float inv = v_ref / l;
#pragma unroll 1
                    for (int cc = 0; cc < D / 32; ++cc) {
                        uint32_t o[32];
                        tmem_ld32(lane_addr + C::TMEM_O + cc * 32, o);
                        tmem_wait_ld();
                        if (valid) {
                            uint4* dst = reinterpret_cast<uint4*>(a.O + orow * D + cc * 32);
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                uint4 v;
                                v.x = pack_bf16x2(__uint_as_float(o[8 * e + 0]) * inv, __uint_as_float(o[8 * e + 1]) * inv);
                                v.y = pack_bf16x2(__uint_as_float(o[8 * e + 2]) * inv, __uint_as_float(o[8 * e + 3]) * inv);
                                v.z = pack_bf16x2(__uint_as_float(o[8 * e + 4]) * inv, __uint_as_float(o[8 * e + 5]) * inv);
                                v.w = pack_bf16x2(__uint_as_float(o[8 * e + 6]) * inv, __uint_as_float(o[8 * e + 7]) * inv);
                                dst[e] = v;
                            }
                        }
                    }
                    if (valid && a.LSE != nullptr) a.LSE[orow] = m_use * kLn2 + logf(l);
                }
                tc_fence_before();
                continue;
            }
            // ---- a split: (max, sum) and the unnormalised O of every row in fp32, laid out
            // [quad of columns][row], so that a warp's 32 rows write 512 bytes at a time
            if (warp_rows) {
                float4* po = reinterpret_cast<float4*>(a.part_o) + static_cast<size_t>(x.part) * (D / 4) * kBM + row;
#pragma unroll 1
                for (int cc = 0; cc < D / 32; ++cc) {
                    uint32_t o[32];
                    tmem_ld32(lane_addr + C::TMEM_O + cc * 32, o);
                    tmem_wait_ld();
                    if (valid) {
                        auto at = [&](int e) { return __uint_as_float(o[e]) * v_ref; };
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            po[(cc * 8 + e) * kBM] = make_float4(at(4 * e), at(4 * e + 1), at(4 * e + 2), at(4 * e + 3));
                    }
                }
                if (valid) a.part_ml[static_cast<size_t>(x.part) * kBM + row] = make_float2(m_use, l);
            }
            tc_fence_before();
        }
    }
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem_base, C::TMEM_COLS);
    }
}

template <int D>
cudaError_t launch_d(const ChunkArgs& a, const KernelEnv& env, const char** err) {
    using C = Cfg<D>;
    cudaError_t e = ensure_smem_attr(reinterpret_cast<const void*>(chunk8_tile_kernel<D>), C::SMEM);
    if (e != cudaSuccess) { *err = "cudaFuncSetAttribute(8-bit tile attention)"; return e; }
    // Two blocks a multiprocessor: their shared memory and tensor memory both fit twice.
    e = launch_early(chunk8_tile_kernel<D>, dim3(a.blocks), kThreads, C::SMEM, env.stream, a, a.sm_scale * kLog2e, env.limit);
    if (e != cudaSuccess) { *err = "8-bit tile attention launch"; return e; }
    e = launch_early(chunk_join_kernel<D>, dim3(a.blocks), kJoinThreads, 0, env.stream, a);
    if (e != cudaSuccess) *err = "8-bit attention join launch";
    return e;
}

}  // namespace

cudaError_t chunk8_tile_prepare(int d) {
    return d == 128 ? ensure_smem_attr(reinterpret_cast<const void*>(chunk8_tile_kernel<128>), Cfg<128>::SMEM)
                    : ensure_smem_attr(reinterpret_cast<const void*>(chunk8_tile_kernel<64>), Cfg<64>::SMEM);
}

cudaError_t launch_chunk8_tile(const ChunkArgs& a, const KernelEnv& env, const char** err) {
    return a.d == 128 ? launch_d<128>(a, env, err) : launch_d<64>(a, env, err);
}

}  // namespace sas
