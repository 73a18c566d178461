// Dense causal attention of a chunk of new tokens per sequence over a paged cache.
//
// Token i of a sequence (position p_i in it) attends keys j <= p_i of its pages:
//   O_i = sum_j softmax_j(scale q_i.k_j) v_j,  LSE_i = log sum_j exp(scale q_i.k_j).
//
// A tile is 128 rows: R = 128 / G consecutive tokens of one sequence times the G
// query heads of one KV group (row = token * G + head), so the group's keys are
// read once for its G heads, and a single token fills G rows.  The tile walks the
// 64-key pages 0 .. floor(p_last / 64) with a running maximum and sum:
//   * warp 0 takes work items, publishes them to the other roles and loads K pages
//     by TMA (ring), warp 1 loads V pages (own ring) and the Q tile;
//   * warp 2 issues S = Q K^T, warp 3 O += P V (tcgen05.mma, P read from TMEM);
//   * warps 4-7, a thread per row: mask, online softmax in the log2 domain, P as
//     bf16 pairs into TMEM, O rescaled only when the maximum grows by 2^8.
// P is rounded to bf16 for the tensor core (its row sum is taken before, in fp32).
//
// Work is cut as chunk_work.cuh says, a tile being 128 rows.  A block takes its whole units
// first: units of one sequence then walk the same pages at about the same time on many blocks,
// out of L2.
//
// Measured: 6.3 TB/s of keys and values for 96 single tokens over 100 to 12000 (124 us),
// 6.3 TB/s for 6 x 5 tokens over 20000 to 32000 (106 us), 1653 TFLOP/s for 4096 tokens
// over 32096 (1220 us; 1450 and 1390 us once the card is at its power limit, at 1.64
// GHz), all d = 128 with 32 and 8 heads.  d = 64: 920 TFLOP/s for 2048 tokens over 10048
// (165 us), bound by the softmax warps' chain of waits and arithmetic (Cfg).
//
// Keys past a sequence's end in its last page may hold anything: scores there are
// replaced, not weighted by zero, and values past the tile's last position are
// zeroed in shared memory before the product.  (A value of the tile's own later tokens that
// is not finite does reach the rows that do not see it, as 0 times it.)  A table entry out of range is never
// used as an address: it becomes the row past the cache, which TMA reads as zero.
#include "chunk_work.cuh"

namespace sas {
namespace {

constexpr int kThreads = 256;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kRescaleThreshold = 8.0f;   // log2 units
constexpr int kItemSlots = 4;     // work items in flight between warp 0 and the other roles
constexpr int kItemReaders = 7;   // V producer, two MMA issuers, four softmax warps
constexpr int kStatusLayout = 3;

// ------------------------------------------------------------------ attention

// A step is KPS pages: their scores, softmax and product go through the pipeline together.
// Beside its arithmetic a step costs the softmax warps 760 cycles of barriers, votes and
// tensor-memory loads and stores.  At d = 128 the products of the multiprocessor's two
// blocks cover that.  They are bound by the operands' way out of shared memory: with 64
// keys a product step reads 4 KB of Q and 2 KB of K in 48 cycles, for 32 of arithmetic.
// With the first half of Q in tensor memory (O 128 + S 64 + P 32 + Q 32 columns: no room
// for more) a page takes 571 cycles of the tensor pipe instead of 618.  At d = 64 the
// products are half as long and nothing covers the waits: two pages a step, O 64 + S
// 128 + P 64 columns, with the score rows in registers (184 a softmax thread, 64 for the
// others, of the 128 the block is launched with).  Such a step takes 1650 cycles with one
// block on the multiprocessor (700 of them exponentials and P, 185 the maximum) and 2370
// with two, of 1024 that both need the exponential unit.
template <int D>
struct Cfg {
    static constexpr int KPS = D == 64 ? 2 : 1;
    static constexpr bool QT = D == 128;            // half of Q in tensor memory
    static constexpr int QST = D == 64 ? 2 : 1;     // Q tiles (of the item at work, and the next one's)
    static constexpr int Q_BYTES = kBM * D * 2;
    static constexpr int KV_BYTES = kBN * D * 2;
    static constexpr int KST = D == 64 ? 4 : 2;     // pages of the rings
    static constexpr int VST = KST;
    static constexpr int OFF_K = QST * Q_BYTES;
    static constexpr int OFF_V = OFF_K + KST * KV_BYTES;
    static constexpr int OFF_CTL = OFF_V + VST * KV_BYTES;
    static constexpr int SMEM = OFF_CTL + 768;   // barriers and items, then Shares
    static constexpr int TMEM_COLS = 256;
    static constexpr int TMEM_O = 0;
    static constexpr int TMEM_S = D;
    static constexpr int TMEM_P = TMEM_S + KPS * kBN;   // keys packed in pairs
    static constexpr int TMEM_Q = TMEM_P + 32 * KPS;    // the row's first 64 dims packed in pairs
    static_assert(TMEM_Q + (QT ? 32 : 0) <= TMEM_COLS, "tensor memory");
    static constexpr uint32_t IDESC_S = idesc_bf16(kBM, kBN, 0, 0);
    static constexpr uint32_t IDESC_O = idesc_bf16(kBM, D, 0, 1);
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
    uint64_t q_full[2], q_empty[2], k_full[4], k_empty[4], v_full[4], v_empty[4];
    uint64_t s_full, s_free, p_full, pv_done, q_ready, drain_bar;
    uint64_t item_full[kItemSlots], item_empty[kItemSlots];
    Item item[kItemSlots];
    uint32_t tmem_base;
    int abort_flag;
};
static_assert(sizeof(Ctl) <= 512 && sizeof(Shares) <= 256, "control block");

__device__ __forceinline__ bool read_item(Ctl& ctl, int r, const WaitCtl& wc, Item& x) {
    const int slot = r % kItemSlots;
    if (!mbar_poll_warp(&ctl.item_full[slot], (r / kItemSlots) & 1, wc)) return false;
    x = ctl.item[slot];
    __syncwarp();
    if (lane_id() == 0) mbar_arrive(&ctl.item_empty[slot]);
    return true;
}

template <int D>
__global__ void __launch_bounds__(kThreads, 2)
chunk_attn_kernel(const __grid_constant__ CUtensorMap mapQ, const __grid_constant__ CUtensorMap mapK,
                  const __grid_constant__ CUtensorMap mapV, ChunkArgs a, float scale_log2, long long limit) {
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
        for (int s = 0; s < C::QST; ++s) { mbar_init(&ctl.q_full[s], 1); mbar_init(&ctl.q_empty[s], 1); }
        for (int s = 0; s < C::KST; ++s) { mbar_init(&ctl.k_full[s], 1); mbar_init(&ctl.k_empty[s], 1); }
        for (int s = 0; s < C::VST; ++s) { mbar_init(&ctl.v_full[s], 1); mbar_init(&ctl.v_empty[s], 1); }
        mbar_init(&ctl.s_full, 1);
        mbar_init(&ctl.s_free, 4);
        mbar_init(&ctl.pv_done, 1);
        mbar_init(&ctl.p_full, 4);
        mbar_init(&ctl.q_ready, 4);
        mbar_init(&ctl.drain_bar, 2);
        for (int s = 0; s < kItemSlots; ++s) {
            mbar_init(&ctl.item_full[s], 1);
            mbar_init(&ctl.item_empty[s], kItemReaders);
        }
        ctl.abort_flag = 0;
        fence_barrier_init();
    }
    if (warp == 3) {
        tmem_alloc(&ctl.tmem_base, C::TMEM_COLS);
        tmem_relinquish();
    }
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = ctl.tmem_base;
    const WaitCtl wc{&ctl.abort_flag, a.status, limit};
    Shares& sh = *reinterpret_cast<Shares*>(smem + C::OFF_CTL + 512);
    grid_dep_wait();   // whatever the stream ran before: lengths, table, cache
    const int rl = 31 - __clz(kBM / a.G);   // 2^rl tokens of a tile (G is 1, 2, 4 or 8)
    const bool any = find_range(a, rl, sh);
    grid_dep_launch();   // the join's blocks may take the places that open up (they wait for this grid's end)

    // Every role walks the same items and counts pages over all of them (g): ring
    // slots, score buffers and barrier phases follow g across item boundaries.
    if (warp < 4) {
        give_registers<D>();
        if (warp == 0) {
            // ---------------- items and K pages
            if (lane == 0) tma_prefetch_desc(&mapK);
            Walk walk(a, rl, sh, any);
            int g = 0;
            bool ok = true;
            for (int r = 0; ok; ++r) {
                const Item x = walk.next(a, rl);
                const int slot = r % kItemSlots;
                if (!mbar_wait_warp(&ctl.item_empty[slot], ((r / kItemSlots) & 1) ^ 1u, wc)) { ok = false; break; }
                if (lane == 0) {
                    ctl.item[slot] = x;
                    mbar_arrive(&ctl.item_full[slot]);
                    if (x.head >= 0) {   // its Q tile is loaded when the item before is done with its own: into L2 now
#pragma unroll
                        for (int h = 0; h < D / 64; ++h) tma_prefetch_3d(&mapQ, h * 64, x.head * a.G, x.tok0);
                    }
                }
                __syncwarp();
                if (x.head < 0) break;
                int rows = 0;
                for (int m = x.blk0; m < x.blk1; ++m, ++g) {
                    const int j = (m - x.blk0) & 31;
                    if (j == 0) rows = page_row(a, x, m, lane);
                    const int row = __shfl_sync(0xffffffffu, rows, j);
                    const int s = g % C::KST;
                    if (!mbar_wait_warp(&ctl.k_empty[s], ((g / C::KST) & 1) ^ 1u, wc)) { ok = false; break; }
                    if (lane == 0) {
                        uint8_t* dst = smem + C::OFF_K + s * C::KV_BYTES;
                        mbar_arrive_expect_tx(&ctl.k_full[s], C::KV_BYTES);
#pragma unroll
                        for (int h = 0; h < D / 64; ++h) tma_load_3d(dst + h * (kBN * 128), &mapK, &ctl.k_full[s], h * 64, 0, row);
                    }
                    __syncwarp();
                }
            }
            walk.record(a, rl, sh);
            if (!ok && lane == 0) {   // the last KST loads may be in flight
                for (int q = g - 1; q >= 0 && q >= g - C::KST; --q)
                    mbar_wait_drain(&ctl.k_full[q % C::KST], (q / C::KST) & 1, limit, a.status);
            }
        } else if (warp == 1) {
            // ---------------- V pages and the Q tile
            if (lane == 0) {
                tma_prefetch_desc(&mapQ);
                tma_prefetch_desc(&mapV);
            }
            int g = 0, nq = 0;
            bool ok = true;
            for (int r = 0; ok; ++r) {
                Item x;
                if (!read_item(ctl, r, wc, x)) { ok = false; break; }
                if (x.head < 0) break;
                const int qs = nq % C::QST;
                if (!mbar_wait_warp(&ctl.q_empty[qs], ((nq / C::QST) & 1) ^ 1u, wc)) { ok = false; break; }
                if (lane == 0) {
                    mbar_arrive_expect_tx(&ctl.q_full[qs], C::Q_BYTES);
#pragma unroll
                    for (int h = 0; h < D / 64; ++h)
                        tma_load_3d(smem + qs * C::Q_BYTES + h * (kBM * 128), &mapQ, &ctl.q_full[qs], h * 64, x.head * a.G, x.tok0);
                }
                ++nq;
                int rows = 0;
                for (int m = x.blk0; m < x.blk1; ++m, ++g) {
                    const int j = (m - x.blk0) & 31;
                    if (j == 0) rows = page_row(a, x, m, lane);
                    const int row = __shfl_sync(0xffffffffu, rows, j);
                    const int s = g % C::VST;
                    if (!mbar_wait_warp(&ctl.v_empty[s], ((g / C::VST) & 1) ^ 1u, wc)) { ok = false; break; }
                    if (lane == 0) {
                        uint8_t* dst = smem + C::OFF_V + s * C::KV_BYTES;
                        mbar_arrive_expect_tx(&ctl.v_full[s], C::KV_BYTES);
#pragma unroll
                        for (int h = 0; h < D / 64; ++h) tma_load_3d(dst + h * (kBN * 128), &mapV, &ctl.v_full[s], h * 64, 0, row);
                    }
                    __syncwarp();
                }
            }
            if (!ok && lane == 0) {
                for (int q = nq - 1; q >= 0 && q >= nq - C::QST; --q)
                    mbar_wait_drain(&ctl.q_full[q % C::QST], (q / C::QST) & 1, limit, a.status);
                for (int q = g - 1; q >= 0 && q >= g - C::VST; --q)
                    mbar_wait_drain(&ctl.v_full[q % C::VST], (q / C::VST) & 1, limit, a.status);
            }
        } else if (warp == 2) {
            // ---------------- S = Q K^T of step g, once the softmax warps have loaded S of step g - 1
            const uint64_t dq0 = smem_desc_sw128(smem_u32(smem), 16, 1024);
            const uint64_t dk0 = smem_desc_sw128(smem_u32(smem + C::OFF_K), 16, 1024);
            int g = 0, gp = 0, tc = 0;   // steps, pages, items
            bool ok = true;
            for (int r = 0; ok; ++r, ++tc) {
                Item x;
                if (!read_item(ctl, r, wc, x)) { ok = false; break; }
                if (x.head < 0) break;
                const int qs = tc % C::QST;
                const uint64_t dq = dq0 + static_cast<uint64_t>((qs * C::Q_BYTES) >> 4);
                if (!mbar_wait_warp(&ctl.q_full[qs], (tc / C::QST) & 1, wc)) { ok = false; break; }
                if (C::QT && !mbar_wait_warp(&ctl.q_ready, tc & 1, wc)) { ok = false; break; }
                for (int m = x.blk0; ok && m < x.blk1; m += C::KPS, ++g) {
                    if (g >= 1 && !mbar_wait_warp(&ctl.s_free, (g - 1) & 1, wc)) { ok = false; break; }
                    for (int i = 0; i < C::KPS && m + i < x.blk1; ++i, ++gp) {
                        const int s = gp % C::KST;
                        if (!mbar_wait_warp(&ctl.k_full[s], (gp / C::KST) & 1, wc)) { ok = false; break; }
                        tc_fence_after();
                        const uint64_t dk = dk0 + static_cast<uint64_t>((s * C::KV_BYTES) >> 4);
                        if (elect_one()) {
#pragma unroll
                            for (int k = 0; k < D / 16; ++k) {
                                const uint32_t off_q = (k >> 2) * (kBM * 128) + (k & 3) * 32;
                                const uint32_t off_k = (k >> 2) * (kBN * 128) + (k & 3) * 32;
                                if (C::QT && k < 4)
                                    umma_bf16_ta(tmem_base + C::TMEM_S, tmem_base + C::TMEM_Q + k * 8, dk + (off_k >> 4),
                                                 C::IDESC_S, k > 0);
                                else
                                    umma_bf16(tmem_base + C::TMEM_S + i * kBN, dq + (off_q >> 4), dk + (off_k >> 4),
                                              C::IDESC_S, k > 0);
                            }
                            umma_commit(&ctl.k_empty[s]);
                        }
                        __syncwarp();
                    }
                    if (!ok) break;
                    if (elect_one()) {
                        umma_commit(&ctl.s_full);
                        if (m + C::KPS >= x.blk1) umma_commit(&ctl.q_empty[qs]);
                    }
                    __syncwarp();
                }
            }
            if (elect_one()) {
                umma_commit(&ctl.drain_bar);
                mbar_wait_drain(&ctl.drain_bar, 0, limit, a.status);
            }
            __syncwarp();
        } else if (warp == 3) {
            // ---------------- O += P V of step g; an item's first page starts a new accumulator
            const uint64_t dv0 = smem_desc_sw128(smem_u32(smem + C::OFF_V), kBN * 128, 1024);
            int g = 0, gp = 0;
            bool ok = true;
            for (int r = 0; ok; ++r) {
                Item x;
                if (!read_item(ctl, r, wc, x)) { ok = false; break; }
                if (x.head < 0) break;
                const int end = x.pos0 + x.ntok;   // keys from here on belong to no row of the tile
                for (int m0 = x.blk0; ok && m0 < x.blk1; m0 += C::KPS, ++g) {
                    for (int i = 0; i < C::KPS && m0 + i < x.blk1; ++i, ++gp) {
                        const int m = m0 + i;
                        const int vs = gp % C::VST;
                        if (!mbar_wait_warp(&ctl.v_full[vs], (gp / C::VST) & 1, wc)) { ok = false; break; }
                        if (end < (m + 1) * kBN) {
                            // zero value rows: P is 0 there, and 0 times a stale infinity or NaN is NaN
                            const int r0 = max(0, end - m * kBN);
                            uint8_t* v = smem + C::OFF_V + vs * C::KV_BYTES;
                            for (int j = r0 * 8 + lane; j < kBN * 8; j += 32) {
#pragma unroll
                                for (int h = 0; h < D / 64; ++h)
                                    *reinterpret_cast<uint4*>(v + h * (kBN * 128) + j * 16) = make_uint4(0, 0, 0, 0);
                            }
                            fence_proxy_async_smem();
                            __syncwarp();
                        }
                        if (i == 0 && !mbar_wait_warp(&ctl.p_full, g & 1, wc)) { ok = false; break; }
                        tc_fence_after();
                        const uint64_t dv = dv0 + static_cast<uint64_t>((vs * C::KV_BYTES) >> 4);
                        if (elect_one()) {
#pragma unroll
                            for (int k = 0; k < kBN / 16; ++k)
                                umma_bf16_ta(tmem_base + C::TMEM_O,
                                             tmem_base + C::TMEM_P + i * 32 + k * 8,
                                             dv + ((k * 2048) >> 4), C::IDESC_O, (m > x.blk0 || k > 0) ? 1u : 0u);
                            umma_commit(&ctl.v_empty[vs]);
                        }
                        __syncwarp();
                    }
                    if (!ok) break;
                    if (elect_one()) umma_commit(&ctl.pv_done);
                    __syncwarp();
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
        const uint64_t scale2 = f32x2(scale_log2, scale_log2);
        // the r-th item, and its rows' first 64 dims from shared into tensor memory (the products of
        // the item before, which read the ones there, are done: this warp has seen their scores)
        auto take_item = [&](int r, Item& x) {
            if (!read_item(ctl, r, wc, x)) return false;
            if (!C::QT || x.head < 0) return true;
            if (!mbar_wait_warp(&ctl.q_full[0], r & 1, wc)) return false;
            if (q * 32 < x.ntok * a.G) {
                uint32_t w[32];
#pragma unroll
                for (int c = 0; c < 8; ++c) {   // 16-byte chunks, swizzled within the 128-byte row
                    const uint4 v = *reinterpret_cast<const uint4*>(smem + row * 128 + ((c ^ (row & 7)) << 4));
                    w[4 * c] = v.x;
                    w[4 * c + 1] = v.y;
                    w[4 * c + 2] = v.z;
                    w[4 * c + 3] = v.w;
                }
                tmem_st32(lane_addr + C::TMEM_Q, w);
                tmem_wait_st();
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&ctl.q_ready);
            return true;
        };
        int g = 0;
        Item x, nx;
        bool ok = take_item(0, x);
        for (int r = 1; ok && x.head >= 0; x = nx, ++r) {
            const bool valid = tok < x.ntok;
            const bool warp_rows = q * 32 < x.ntok * a.G;   // else nothing of this warp is ever read
            const int pos = x.pos0 + tok;
            float m_use = -CUDART_INF_F, l = 0.f;
            for (int m = x.blk0; m < x.blk1; m += C::KPS, ++g) {
                // last key column of the step that this row sees (< 0: none; none of a page that is not
                // there).  Rows of no token are never read: they go unmasked.
                const int lim = valid ? min(min(NK - 1, pos - m * kBN), (x.blk1 - m) * kBN - 1) : NK - 1;
                if (!mbar_wait_warp(&ctl.s_full, g & 1, wc)) { ok = false; break; }
                if (!warp_rows) {
                    if (lane == 0) mbar_arrive(&ctl.s_free);
                    if (g >= 1 && !mbar_wait_warp(&ctl.pv_done, (g - 1) & 1, wc)) { ok = false; break; }
                    if (lane == 0) mbar_arrive(&ctl.p_full);
                    __syncwarp();
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
                if (lane == 0) mbar_arrive(&ctl.s_free);
                if (__any_sync(0xffffffffu, lim < NK - 1)) {
#pragma unroll
                    for (int k = 0; k < NK; ++k) xs[k] = k <= lim ? xs[k] : -CUDART_INF_F;
                }
                float mx[4] = {-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F};
#pragma unroll
                for (int k = 0; k < NK; k += 8) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) mx[j] = max3f(mx[j], xs[k + 2 * j], xs[k + 2 * j + 1]);
                }
                const float mb = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * scale_log2;
                const bool need = valid && mb > m_use + kRescaleThreshold;
                const float m_new = need ? mb : m_use;
                const float off = m_new == -CUDART_INF_F ? 0.f : -m_new;
                const uint64_t off2 = f32x2(off, off);
                uint64_t acc[4] = {0, 0, 0, 0};
                uint32_t pk[C::KPS][32];
#pragma unroll
                for (int k = 0; k < NK; k += 2) {
                    float a0, a1;
                    f32x2_split(fma_f32x2(f32x2(xs[k], xs[k + 1]), scale2, off2), a0, a1);
                    const float e0 = fast_exp2(a0), e1 = fast_exp2(a1);
                    acc[(k >> 1) & 3] = add_f32x2(acc[(k >> 1) & 3], f32x2(e0, e1));
                    pk[k / 64][(k % 64) >> 1] = pack_bf16x2(e0, e1);
                }
                float s0, s1, s2, s3, s4, s5, s6, s7;
                f32x2_split(acc[0], s0, s1);
                f32x2_split(acc[1], s2, s3);
                f32x2_split(acc[2], s4, s5);
                f32x2_split(acc[3], s6, s7);
                const float rs = ((s0 + s1) + (s2 + s3)) + ((s4 + s5) + (s6 + s7));
                float factor = 1.f;
                if (need) factor = m_use == -CUDART_INF_F ? 0.f : fast_exp2(m_use - m_new);
                if (m > x.blk0 && __any_sync(0xffffffffu, need)) {
                    // rescaling O needs the previous step's PV done
                    if (!mbar_wait_warp(&ctl.pv_done, (g - 1) & 1, wc)) { ok = false; break; }
                    tc_fence_after();
#pragma unroll 1
                    for (int cc = 0; cc < D / 32; ++cc) {
                        uint32_t o[32];
                        tmem_ld32(lane_addr + C::TMEM_O + cc * 32, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * factor);
                        tmem_st32(lane_addr + C::TMEM_O + cc * 32, o);
                    }
                    tmem_wait_st();
                }
                l = l * factor + rs;
                m_use = m_new;
                // P is free once the PV of step g - 1 has read it
                if (g >= 1 && !mbar_wait_warp(&ctl.pv_done, (g - 1) & 1, wc)) { ok = false; break; }
                tc_fence_after();
#pragma unroll
                for (int i = 0; i < C::KPS; ++i) tmem_st32(lane_addr + C::TMEM_P + i * 32, pk[i]);
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&ctl.p_full);
            }
            // the next item's Q goes ahead of this one's epilogue: its first product runs during it
            if (!ok || !take_item(r, nx)) { ok = false; break; }
            // The next item's first PV overwrites O only after this warp's next arrival on
            // p_full, which follows the reads below.
            if (!mbar_wait_warp(&ctl.pv_done, (g - 1) & 1, wc)) { ok = false; break; }
            tc_fence_after();
            const size_t orow = (static_cast<size_t>(x.tok0) + tok) * a.Hq + static_cast<size_t>(x.head) * a.G + hq;
            if (x.part < 0) {
                if (warp_rows) {
                    const float inv = 1.f / l;
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
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            po[(cc * 8 + e) * kBM] = make_float4(__uint_as_float(o[4 * e]), __uint_as_float(o[4 * e + 1]),
                                                                 __uint_as_float(o[4 * e + 2]), __uint_as_float(o[4 * e + 3]));
                    }
                }
                if (valid) a.part_ml[static_cast<size_t>(x.part) * kBM + row] = make_float2(m_use, l);
            }
            tc_fence_before();
        }
    }
    __syncthreads();
    if (warp == 3) {
        tc_fence_after();
        tmem_dealloc(tmem_base, C::TMEM_COLS);
    }
}

template <int D>
cudaError_t launch_d(const ChunkArgs& a, const KernelEnv& env, const char** err) {
    using C = Cfg<D>;
    cudaError_t e = ensure_smem_attr(reinterpret_cast<const void*>(chunk_attn_kernel<D>), C::SMEM);
    if (e != cudaSuccess) { *err = "cudaFuncSetAttribute(chunk attention)"; return e; }
    CUtensorMap mq, mk, mv;
    const uint64_t rows = static_cast<uint64_t>(a.num_pages) * a.Hkv;
    if (make_tmap_bf16_box(&mq, a.Q, D, a.Hq, a.T, 64, a.G, kBM / a.G) != 0 ||
        make_tmap_bf16_3d(&mk, a.K_cache, D, kBN, rows, 64, kBN) != 0 ||
        make_tmap_bf16_3d(&mv, a.V_cache, D, kBN, rows, 64, kBN) != 0) {
        *err = "tensor map";
        return cudaErrorInvalidValue;
    }
    // Two blocks a multiprocessor: their shared memory and tensor memory both fit twice.
    e = launch_early(chunk_attn_kernel<D>, dim3(a.blocks), kThreads, C::SMEM, env.stream, mq, mk, mv, a, a.sm_scale * kLog2e,
                     env.limit);
    if (e != cudaSuccess) { *err = "chunk attention launch"; return e; }
    e = launch_early(chunk_join_kernel<D>, dim3(a.blocks), kJoinThreads, 0, env.stream, a);
    if (e != cudaSuccess) *err = "chunk join launch";
    return e;
}

}  // namespace

int chunk_blocks() { return 2 * device_sm_count(); }

cudaError_t chunk_attn_prepare(int d) {
    return d == 128 ? ensure_smem_attr(reinterpret_cast<const void*>(chunk_attn_kernel<128>), Cfg<128>::SMEM)
                    : ensure_smem_attr(reinterpret_cast<const void*>(chunk_attn_kernel<64>), Cfg<64>::SMEM);
}

cudaError_t launch_chunk_attn(const ChunkArgs& a, const KernelEnv& env, const char** err) {
    if (a.d == 128) return launch_d<128>(a, env, err);
    if (a.d == 64) return launch_d<64>(a, env, err);
    *err = "chunk attention: unsupported head dim";
    return cudaErrorInvalidValue;
}

}  // namespace sas
