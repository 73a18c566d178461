// Dense causal attention of new tokens over an 8-bit paged cache, for requests of many rows:
// 128-row tiles on the tensor cores (tcgen05).  The formulas and the cache are k_chunk8.cu's,
// the work is cut as chunk_work.cuh says.
//
// The tensor core takes 8-bit numbers only beside 8-bit numbers, and rounding queries and
// weights to 8 bits would show.  So the pages' numbers become f16, exactly, in shared memory:
//   * warp 0 takes work items, publishes them and loads their Q by TMA;
//   * four warps load pages into registers, two of them keys and two values, each every other
//     page or half of every page, one ahead, and convert them into rings of f16 tiles in the tensor
//     core's layout, value rows of no key as zero;
//   * two warps issue the products, S = Q K^T and O += P V (P read from tensor memory): one each of a
//     block's one tile, or one tile each of two;
//   * four warps a tile, a thread per row: Q as f16 under a power of two of the row's own
//     (k_chunk8.cu), mask, online softmax in the log2 domain, P as f16 pairs into tensor memory,
//     O rescaled only when the maximum grows by 2^8, or where a page's value scale leaves 2^-6 ..
//     2^6 times the one that O stands under.
//
// TILES: 128-row tiles of a block, which share its converted pages.  The conversion costs shared
// memory 128 d bytes a page and matrix, beside the products' operands (which take it for two
// thirds of the time that the tensor core needs), so at d = 128 long requests have two tiles a
// block and one block a multiprocessor; requests of fewer rows, and those of d = 64, one tile a
// block and two blocks, each with its own pages.
//
// Bound: the tensor core for prompts, HBM for drafts.  4096 tokens after 28000, 32 query and 8 KV
// heads of 128, take 1452 to 1482 us (73% of the tensor core's rate): the softmax and the wait for it set
// the pace, 1900 cycles a page of two tiles, of which the exponentials take 650, the maxima 320.
// At d = 64 they do all the more, against half the products: a ragged batch of 2626 tokens and 24
// heads 130 us (22%), 2100 cycles a page with two blocks at a time.  Drafts of 20 rows over 152000
// keys in all, 8 heads of 128, 86 us, HBM's 46 (54%): the blocks' rows are mostly of no token.
// The forms of one tile keep 48 to 56 bytes a thread in local memory: 80 registers at launch do not hold every role.
// Units that value scales of any distance need (chunk8.cuh) are 1.1 to 1.6% of these times.
#include <cuda_fp16.h>

#include "chunk8.cuh"
#include "chunk_work.cuh"

namespace sas {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kRescaleThreshold = 8.0f;   // log2 units
constexpr float kScaleRange = 6.f;              // log2 units
constexpr float kLeast = 1099511627776.f, kLeastLog = 40.f;   // a unit over a page's scale, in P: 2^40
constexpr int kItemSlots = 4;     // work items in flight between warp 0 and the other roles
constexpr int kStatusLayout = 3;
// Rows of a request on average above which blocks have two tiles, at d = 128: 12 requests over 8000 to 20000, 8 KV heads,
// in us with one tile and with two: 64 rows 96, 119; 128 rows 108, 132; 160 rows 178, 140; 256 rows 177, 147; 1024 rows
// 712, 562.
constexpr long long kTwoTiles = 128;

// As in k_chunk.cu, half of Q is in tensor memory at d = 128.  A step is one page, with the next
// one's scores made ahead at d = 64.  Two pages a step, which helps bf16 pages at d = 64, would
// need registers that the converting warps hold here; with the second page's scores read twice
// instead, and no scores ahead, a ragged batch of 2626 tokens and 24 heads of 64 takes 144 us
// instead of 128.
template <int D, int TILES>
struct Cfg {
    static constexpr bool QT = D == 128;
    static constexpr int THREADS = 256 + 128 * TILES;
    static constexpr int CONV0 = 4, CONV = 4;                   // the warps that convert
    static constexpr int SHARES = D == 128 && TILES == 1 ? 2 : 1;   // of a page's keys or values: as registers allow
    static constexpr int SOFT0 = 8;                             // the softmax warps, four a tile
    static constexpr bool SPLIT = TILES == 1;                   // a warp for scores and one for P V
    static constexpr int READERS = 2 + CONV + 4 * TILES;       // of an item
    static constexpr int Q_BYTES = kBM * D * 2;      // of a tile
    static constexpr int QST = D == 64 ? 2 : 1;      // Q of the item at work, and the next one's
    static constexpr int KV_BYTES = kBN * D * 2;
    static constexpr int PAGE = kBN * D;
    static constexpr int KST = D == 64 ? 4 : (TILES == 2 ? 4 : 2);   // f16 pages of a ring
    static_assert(SHARES == 2 || KST % 2 == 0, "a place of the rings is one warp's: see k_chunk8.cu");
    static constexpr int SCALES = 16;                // pages' scales: the loads are KST + 4 pages ahead of the softmax at most
    static_assert(KST + 4 <= SCALES, "scales");
    static constexpr int OFF_K = QST * TILES * Q_BYTES;
    static constexpr int OFF_V = OFF_K + KST * KV_BYTES;
    static constexpr int OFF_CTL = OFF_V + KST * KV_BYTES;
    static constexpr int SMEM = OFF_CTL + 1024;      // barriers and items, then Shares
    static_assert(2 / TILES * (SMEM + 1024) <= 233472, "blocks a multiprocessor");
    static constexpr int TMEM_COLS = 256;               // of a tile
    static constexpr int TMEM_O = 0;
    static constexpr int TMEM_S = D;
    static constexpr int NS = D == 64 ? 2 : 1;          // scores of a page at work, and the next one's
    static constexpr int TMEM_P = TMEM_S + NS * kBN;    // keys packed in pairs
    static constexpr int TMEM_Q = TMEM_P + 32;          // the row's first 64 dims packed in pairs
    static_assert(TMEM_Q + (QT ? 32 : 0) <= TMEM_COLS, "tensor memory");
    static constexpr uint32_t IDESC_S = idesc_f16(kBM, kBN, 0, 0);
    static constexpr uint32_t IDESC_O = idesc_f16(kBM, D, 0, 1);
};

// Moves registers between the block's warpgroups (the sum stays within what it was launched
// with: 128 x (40 + 72 + 128) = 384 x 80, 128 x (56 + 120 + 2 x 168) = 512 x 128).
template <int N>
__device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int TILES>
__device__ __forceinline__ void give_registers() {
    if (warp_id() < 4) fewer_registers<TILES == 1 ? 40 : 56>();
    else fewer_registers<TILES == 1 ? 72 : 120>();
}
template <int TILES>
__device__ __forceinline__ void take_registers() {
    more_registers<TILES == 1 ? 128 : 168>();
}

template <class C, int TILES>
struct Ctl {
    uint64_t q_full[C::QST], q_empty[C::QST], k_full[C::KST], k_empty[C::KST], v_full[C::KST], v_empty[C::KST];
    uint64_t sc_full[TILES][C::NS], sc_free[TILES][C::NS], p_full[TILES], pv_done[TILES], q_ready[TILES], drain_bar;
    uint64_t item_full[kItemSlots], item_empty[kItemSlots];
    float4 scale[C::SCALES];   // of page g at g % SCALES: the keys', the values' log2, inverse and itself
    Item item[kItemSlots];
    uint32_t tmem_base;
    int abort_flag;
};
constexpr int kSharesAt = 872;

template <class K>
__device__ __forceinline__ bool read_item(K& ctl, int r, const WaitCtl& wc, Item& x) {
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

// The share-th of NC shares of a page's rows: from memory, and as a 128-byte-swizzled f16 tile [D /
// 64][64][64], rows from `live` on as zero.  Eight lanes take 64 bytes of a row and 64 of the next
// one, at D = 128 the other half of it, which puts the two 16-byte pieces that each of them writes
// into different banks, at offsets that are a lane's own all the way.
template <int D, int NC>
struct Piece {
    static constexpr int ROWS = kBN / NC, PASS = D / 64, N = ROWS / 8 * PASS;
    uint4 w[N];
    __device__ __forceinline__ static int row(int share, int lane) { return share * ROWS + (lane >> 2); }
    __device__ __forceinline__ static int half(int lane, int i) { return PASS == 2 ? (lane >> 2 & 1) ^ (i & 1) : 0; }
    __device__ __forceinline__ void fetch(const uint8_t* page, bool there, int share, int lane) {   // nothing there: zeros
        page += row(share, lane) * D + (lane & 3) * 16;
#pragma unroll
        for (int i = 0; i < N; ++i) {   // 8 rows further every PASS pieces
            w[i] = make_uint4(0, 0, 0, 0);
            if (there) w[i] = __ldcg(reinterpret_cast<const uint4*>(page + i / PASS * 8 * D + half(lane, i) * 64));
        }
    }
    __device__ __forceinline__ void convert(uint8_t* dst, int share, int lane, int live) {
        const int r = row(share, lane), at = ((2 * (lane & 3)) ^ (r & 7)) << 4;
        dst += r * 128;
        if (live < kBN) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (r + i / PASS * 8 >= live) w[i] = make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            uint4 a, b;
            to_f16(w[i].x, a.x, a.y);
            to_f16(w[i].y, a.z, a.w);
            to_f16(w[i].z, b.x, b.y);
            to_f16(w[i].w, b.z, b.w);
            uint8_t* const to = dst + i / PASS * 8 * 128 + half(lane, i) * (kBN * 128);
            *reinterpret_cast<uint4*>(to + at) = a;
            *reinterpret_cast<uint4*>(to + (at ^ 16)) = b;
        }
    }
};
constexpr int kAhead = 6;   // pages that are on their way into L2

__device__ __forceinline__ void prefetch_page(const void* p, uint32_t bytes) {
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(p), "r"(bytes) : "memory");
}

template <int D, int TILES>
__global__ void __launch_bounds__(Cfg<D, TILES>::THREADS, 2 / TILES) chunk8_tile_kernel(const __grid_constant__ CUtensorMap mapQ, ChunkArgs a, float scale_log2, long long limit) {
    using C = Cfg<D, TILES>;
    using K = Ctl<C, TILES>;
    static_assert(sizeof(K) <= kSharesAt && kSharesAt + sizeof(Shares) <= 1024, "control block");
    extern __shared__ __align__(1024) uint8_t smem[];
    if ((smem_u32(smem) & 1023u) != 0) {
        grid_dep_wait();
        if (threadIdx.x == 0) {
            atomicExch(a.status, kStatusLayout);
            a.joins[2 * blockIdx.x] = make_int4(0, 0, 0, 0);
        }
        return;
    }
    K& ctl = *reinterpret_cast<K*>(smem + C::OFF_CTL);
    const uint32_t warp = warp_id(), lane = lane_id();
    if (threadIdx.x == 0) {
        for (int s = 0; s < C::QST; ++s) { mbar_init(&ctl.q_full[s], 1); mbar_init(&ctl.q_empty[s], TILES); }
        for (int s = 0; s < C::KST; ++s) { mbar_init(&ctl.k_full[s], C::SHARES); mbar_init(&ctl.k_empty[s], TILES); }
        for (int s = 0; s < C::KST; ++s) { mbar_init(&ctl.v_full[s], C::SHARES); mbar_init(&ctl.v_empty[s], TILES); }
        for (int t = 0; t < TILES; ++t) {
            for (int s = 0; s < C::NS; ++s) { mbar_init(&ctl.sc_full[t][s], 1); mbar_init(&ctl.sc_free[t][s], 4); }
            mbar_init(&ctl.pv_done[t], 1);
            mbar_init(&ctl.p_full[t], 4);
            mbar_init(&ctl.q_ready[t], 4);
        }
        mbar_init(&ctl.drain_bar, 2);
        for (int s = 0; s < kItemSlots; ++s) {
            mbar_init(&ctl.item_full[s], 1);
            mbar_init(&ctl.item_empty[s], C::READERS);
        }
        ctl.abort_flag = 0;
        fence_barrier_init();
    }
    if (warp == 1) {
        tmem_alloc(&ctl.tmem_base, TILES * C::TMEM_COLS);
        tmem_relinquish();
    }
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = ctl.tmem_base;
    const WaitCtl wc{&ctl.abort_flag, a.status, limit};
    Shares& sh = *reinterpret_cast<Shares*>(smem + C::OFF_CTL + kSharesAt);
    grid_dep_wait();   // whatever the stream ran before: lengths, table, cache
    const int R = kBM / a.G;                           // tokens of a tile (G is 1, 2, 4 or 8)
    const int rl = 31 - __clz(TILES * R);   // 2^rl tokens of an item
    const bool any = find_range(a, rl, sh);
    grid_dep_launch();   // the join's blocks may take the places that open up (they wait for this grid's end)

    // Every role walks the same items and counts pages over all of them (g): ring slots, score
    // buffers and barrier phases follow g across item boundaries.
    if (warp < C::SOFT0) {
        give_registers<TILES>();
        if (warp == 0) {
            // ---------------- items and their Q
            if (lane == 0) tma_prefetch_desc(&mapQ);
            Walk walk(a, rl, sh, any);
            int n = 0;   // items with Q on its way
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
                const int qs = r % C::QST, tiles = TILES == 2 && x.ntok > R ? 2 : 1;
                if (!mbar_wait_warp(&ctl.q_empty[qs], ((r / C::QST) & 1) ^ 1u, wc)) { ok = false; break; }
                if (lane == 0) {
                    mbar_arrive_expect_tx(&ctl.q_full[qs], tiles * C::Q_BYTES);
                    for (int t = 0; t < tiles; ++t)
#pragma unroll
                        for (int h = 0; h < D / 64; ++h)
                            tma_load_3d(smem + (qs * TILES + t) * C::Q_BYTES + h * (kBM * 128), &mapQ, &ctl.q_full[qs], h * 64,
                                        x.head * a.G, x.tok0 + t * R);
                }
                ++n;
                __syncwarp();
            }
            walk.record(a, rl, sh);
            if (!ok && lane == 0) {   // the last loads may be in flight
                for (int q = n - 1; q >= 0 && q >= n - C::QST; --q)
                    mbar_wait_drain(&ctl.q_full[q % C::QST], (q / C::QST) & 1, limit, a.status);
            }
        } else if (warp >= C::CONV0) {
            // ---------------- pages to f16 tiles
            const bool keys = warp < C::CONV0 + 2;
            const int mine = warp & 1, share = C::SHARES == 2 ? mine : 0;
            constexpr int STEP = 3 - C::SHARES;   // pages from one of this warp's to the next
            const uint8_t* const cache = keys ? a.K8 : a.V8;
            uint8_t* const ring = smem + (keys ? C::OFF_K : C::OFF_V);
            uint64_t* const full = keys ? ctl.k_full : ctl.v_full;
            uint64_t* const empty = keys ? ctl.k_empty : ctl.v_empty;
            int g = 0;
            bool ok = true;
            for (int r = 0; ok; ++r) {
                Item x;
                if (!read_item(ctl, r, wc, x)) { ok = false; break; }
                if (x.head < 0) break;
                const int np = x.blk1 - x.blk0, none = a.num_pages * a.Hkv;
                const int end = keys ? kBN * 32768 : x.pos0 + x.ntok - x.blk0 * kBN;   // values from here on are no row's
                int rows = 0, batch = -1;  // of 32 pages, a lane each
                float4 sc = make_float4(1.f, 0.f, 1.f, 1.f);
                Piece<D, C::SHARES> piece;
                // Page i of the item into registers, the scales to the softmax, the pages behind it into L2.
                auto fetch = [&](int i) {
                    const int j = i & 31;
                    if (i >> 5 != batch) {
                        batch = i >> 5;
                        const int m = x.blk0 + batch * 32;
                        rows = page_row(a, x, m, lane);
                        sc = make_float4(1.f, 0.f, 1.f, 1.f);
                        if (m + static_cast<int>(lane) < x.blk1 && rows < none) {
                            if (keys) {
                                const float vs = load(a.v_scale + rows);
                                sc = make_float4(load(a.k_scale + rows), log2f(vs), 1.f / vs, vs);
                            }
                            if (lane < kAhead && (lane & (STEP - 1)) == (j & (STEP - 1)))
                                prefetch_page(cache + static_cast<size_t>(rows) * C::PAGE, C::PAGE);
                        }
                    }
                    const int row = __shfl_sync(0xffffffffu, rows, j), far = __shfl_sync(0xffffffffu, rows, (j + kAhead) & 31);
                    if (lane == 0 && share == 0 && j + kAhead < 32 && i + kAhead < np && far < none)
                        prefetch_page(cache + static_cast<size_t>(far) * C::PAGE, C::PAGE);
                    if (keys && share == 0 && static_cast<int>(lane) == j) ctl.scale[(g + i) % C::SCALES] = sc;
                    piece.fetch(cache + static_cast<size_t>(row) * C::PAGE, row < none, share, lane);
                };
                int i = STEP == 2 ? (g ^ mine) & 1 : 0;
                if (i < np) fetch(i);
                for (; i < np; i += STEP) {
                    const int s = (g + i) % C::KST;
                    if (!mbar_wait_warp(&empty[s], (((g + i) / C::KST) & 1) ^ 1u, wc)) { ok = false; break; }
                    // P is 0 past the end, and 0 times a stale NaN is NaN: such value rows become zero
                    piece.convert(ring + s * C::KV_BYTES, share, lane, end - i * kBN);
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&full[s]);
                    __syncwarp();
                    if (i + STEP < np) fetch(i + STEP);
                }
                g += np;
            }
        } else if (warp <= 2) {
            // ---------------- products: a warp for the scores and one for P V, or, of two tiles, a warp a tile for both, S
            // of a step, then P V of the one before
            const int t = C::SPLIT ? 0 : warp - 1;
            const bool scores = !C::SPLIT || warp == 1, products = !C::SPLIT || warp == 2;
            const uint32_t tile = tmem_base + t * C::TMEM_COLS;
            const uint64_t dq0 = smem_desc_sw128(smem_u32(smem + t * C::Q_BYTES), 16, 1024);
            const uint64_t dk0 = smem_desc_sw128(smem_u32(smem + C::OFF_K), 16, 1024);
            const uint64_t dv0 = smem_desc_sw128(smem_u32(smem + C::OFF_V), kBN * 128, 1024);
            bool ok = true;
            int ns = 0, np = 0;   // scores, arrivals of P
            auto product = [&](int g, bool fresh) {   // fresh: a new accumulator
                const int vs = g % C::KST;
                if (!mbar_wait_warp(&ctl.v_full[vs], (g / C::KST) & 1, wc) || !mbar_wait_warp(&ctl.p_full[t], np & 1, wc)) return false;
                ++np;
                tc_fence_after();
                if (elect_one()) {
                    const uint64_t dv = dv0 + static_cast<uint64_t>((vs * C::KV_BYTES) >> 4);
#pragma unroll
                    for (int k = 0; k < kBN / 16; ++k)
                        umma_bf16_ta(tile + C::TMEM_O, tile + C::TMEM_P + k * 8, dv + ((k * 2048) >> 4), C::IDESC_O, (!fresh || k > 0) ? 1u : 0u);
                    umma_commit(&ctl.v_empty[vs]);
                    umma_commit(&ctl.pv_done[t]);
                }
                __syncwarp();
                return true;
            };
            // (the dims in tensor memory come first)
            auto score = [&](uint64_t dq, int g, uint64_t* q_free) {   // q_free: Q's place is free after it
                const int s = g % C::KST;
                if (!mbar_wait_warp(&ctl.k_full[s], (g / C::KST) & 1, wc)) return false;
                const int buf = ns % C::NS;
                if (ns >= C::NS && !mbar_wait_warp(&ctl.sc_free[t][buf], (ns / C::NS - 1) & 1, wc)) return false;
                ++ns;
                const uint32_t to = tile + C::TMEM_S + buf * kBN;
                tc_fence_after();
                if (elect_one()) {
                    const uint64_t dk = dk0 + static_cast<uint64_t>((s * C::KV_BYTES) >> 4);
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) {
                        const uint32_t off_q = (k >> 2) * (kBM * 128) + (k & 3) * 32;
                        const uint32_t off_k = (k >> 2) * (kBN * 128) + (k & 3) * 32;
                        if (C::QT && k < 4)
                            umma_bf16_ta(to, tile + C::TMEM_Q + k * 8, dk + (off_k >> 4), C::IDESC_S, k > 0);
                        else
                            umma_bf16(to, dq + (off_q >> 4), dk + (off_k >> 4), C::IDESC_S, k > 0);
                    }
                    umma_commit(&ctl.k_empty[s]);
                    umma_commit(&ctl.sc_full[t][buf]);
                    if (q_free != nullptr) umma_commit(q_free);
                }
                __syncwarp();
                return true;
            };
            int g = 0, nq = 0;   // pages; items of the tile
            for (int r = 0; ok; ++r) {
                Item x;
                if (!read_item(ctl, r, wc, x)) { ok = false; break; }
                if (x.head < 0) break;
                const int qs = r % C::QST;
                const uint64_t dq = dq0 + static_cast<uint64_t>((qs * TILES * C::Q_BYTES) >> 4);
                uint64_t* const q_free = &ctl.q_empty[qs];
                if (!C::SPLIT && t * R >= x.ntok) {   // nothing to do but to let all go, once it is there: arrivals of these phases
                    ok = mbar_wait_warp(&ctl.q_ready[t], nq++ & 1, wc);
                    if (ok && lane == 0) mbar_arrive(q_free);
                    for (int m = x.blk0; ok && m < x.blk1; ++m, ++g) {
                        const int s = g % C::KST, phase = (g / C::KST) & 1;
                        ok = mbar_wait_warp(&ctl.k_full[s], phase, wc) && mbar_wait_warp(&ctl.v_full[s], phase, wc);
                        if (ok && lane == 0) {
                            mbar_arrive(&ctl.k_empty[s]);
                            mbar_arrive(&ctl.v_empty[s]);
                        }
                    }
                    continue;
                }
                const int np_item = x.blk1 - x.blk0;
                if (scores) ok = mbar_wait_warp(&ctl.q_ready[t], nq++ & 1, wc) && score(dq, g, np_item == 1 ? q_free : nullptr);
                for (int i = 0; ok && i < np_item; ++i, ++g) {
                    if (scores && i + 1 < np_item) ok = score(dq, g + 1, i + 2 == np_item ? q_free : nullptr);
                    if (products) ok = ok && product(g, i == 0);
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
        take_registers<TILES>();
        constexpr int NK = kBN;
        const int tile = (warp - C::SOFT0) >> 2, q = warp & 3;
        const int row = q * 32 + lane;                          // of the tile
        const int tok = tile * R + row / a.G, hq = row % a.G;   // of the item
        const uint32_t lane_addr = tmem_base + tile * C::TMEM_COLS + (static_cast<uint32_t>(q * 32) << 16);
        // whether anything of this warp is ever read, of this tile
        auto warp_has_rows = [&](const Item& x) { return tile * R * a.G + q * 32 < x.ntok * a.G; };
        auto tile_has_rows = [&](const Item& x) { return tile * R < x.ntok; };
        float row_scale = 0.f, next_scale = 0.f;
        // the r-th item, and its rows as f16, in place (a tile without rows waits and arrives all the same: a barrier
        // that is passed over one phase does not tell the next one); the first 64 dims of 128 into tensor memory (the products
        // of the item before, which read the ones there, are done: this warp has seen their scores)
        auto take_item = [&](int r, Item& x) {
            if (!read_item(ctl, r, wc, x)) return false;
            if (x.head < 0) return true;
            const int qs = r % C::QST;
            if (!mbar_wait_warp(&ctl.q_full[qs], (r / C::QST) & 1, wc)) return false;
            if (warp_has_rows(x)) {
                // 64 dims at a time, 16-byte chunks swizzled within the 128-byte row
                uint8_t* const mine = smem + (qs * TILES + tile) * C::Q_BYTES + row * 128;
                auto chunk = [&](int h, int c) { return reinterpret_cast<uint4*>(mine + h * (kBM * 128) + ((c ^ (row & 7)) << 4)); };
                uint4 raw[8];
                auto fetch = [&](int h) {
#pragma unroll
                    for (int c = 0; c < 8; ++c) raw[c] = *chunk(h, c);
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
#pragma unroll
                for (int c = 0; c < 8; ++c)
                    *chunk(D / 64 - 1, c) = make_uint4(half2(raw[c].x), half2(raw[c].y), half2(raw[c].z), half2(raw[c].w));
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
            if (lane == 0) mbar_arrive(&ctl.q_ready[tile]);
            return true;
        };
        int g = 0, gt = 0;   // pages; the tile's
        Item x, nx;
        bool ok = take_item(0, x);
        for (int r = 1; ok && x.head >= 0; x = nx, ++r) {
            row_scale = next_scale;
            const bool valid = tok < x.ntok;
            const bool warp_rows = warp_has_rows(x);
            if (!tile_has_rows(x)) {
                g += x.blk1 - x.blk0;
                if (!take_item(r, nx)) { ok = false; break; }
                continue;
            }
            const int pos = x.pos0 + tok;
            float m_use = -CUDART_INF_F, l = 0.f;
            float v_ref = 0.f, v_log = 0.f;   // what one of O stands for
            bool large = false;               // a scale was above kLargeScale
            for (int m = x.blk0; m < x.blk1; ++m, ++g, ++gt) {
                // last key column of the page that this row sees (< 0: none).  Rows of no token are never read: they
                // go unmasked.
                const int lim = valid ? min(NK - 1, pos - m * kBN) : NK - 1;
                const int buf = gt % C::NS;
                if (!mbar_wait_warp(&ctl.sc_full[tile][buf], (gt / C::NS) & 1, wc)) { ok = false; break; }
                float4 sc = ctl.scale[g % C::SCALES];
                if (m == x.blk0) {
                    v_log = sc.y;
                    v_ref = sc.w;
                    large = v_ref > kLargeScale;
                }
                // P is free, and O another product's no more, once the product before has read and written them
                auto product_done = [&] { return gt == 0 || mbar_wait_warp(&ctl.pv_done[tile], (gt - 1) & 1, wc); };
                if (!warp_rows) {
                    if (lane == 0) mbar_arrive(&ctl.sc_free[tile][buf]);
                    if (!product_done()) { ok = false; break; }
                    if (lane == 0) mbar_arrive(&ctl.p_full[tile]);
                    __syncwarp();
                    continue;
                }
                tc_fence_after();
                float xs[NK];
                {
                    uint32_t u[NK / 32][32];
#pragma unroll
                    for (int c = 0; c < NK / 32; ++c) tmem_ld32(lane_addr + C::TMEM_S + buf * kBN + c * 32, u[c]);
                    tmem_wait_ld();
#pragma unroll
                    for (int k = 0; k < NK; ++k) xs[k] = __uint_as_float(u[k / 32][k % 32]);
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&ctl.sc_free[tile][buf]);
                if (m * kBN + NK - 1 > x.pos0 + tile * R) {   // some row does not see all of it
#pragma unroll
                    for (int k = 0; k < NK; ++k) xs[k] = k <= lim ? xs[k] : -CUDART_INF_F;
                }
                float mx[4] = {-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F};
#pragma unroll
                for (int k = 0; k < NK; k += 8) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) mx[j] = max3f(mx[j], xs[k + 2 * j], xs[k + 2 * j + 1]);
                }
                const float cr = score_factor(row_scale, sc.x);
                const float mb = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * cr;
                const bool need = valid && mb > m_use + kRescaleThreshold;
                const float m_new = need ? mb : m_use;
                const float off = m_new == -CUDART_INF_F ? 0.f : -m_new;
                float factor = need ? (m_use == -CUDART_INF_F ? 0.f : fast_exp2(m_use - m_new)) : 1.f;
                m_use = m_new;
                l *= factor;
                // O stands under another value scale from here on
                const bool move = !(fabsf(sc.y - v_log) <= kScaleRange);
                if (m > x.blk0 && __any_sync(0xffffffffu, need || move)) {
                    if (!product_done()) { ok = false; break; }
                    tc_fence_after();
                    if (__any_sync(0xffffffffu, move)) {
                        float fall = v_ref * sc.z;
                        const bool falls = !(fall <= 1.f), far = move && fall < kFarRise;
                        if (far) fall = v_ref * kRiseRest * sc.z;
                        const float step = far ? kRiseStep : 1.f;
                        float top = 0.f;
#pragma unroll 1
                        for (int cc = 0; cc < D / 32; ++cc) {
                            uint32_t o[32];
                            tmem_ld32(lane_addr + C::TMEM_O + cc * 32, o);
                            tmem_wait_ld();
#pragma unroll
                            for (int e = 0; e < 32; ++e) {
                                top = fmaxf(top, fabsf(__uint_as_float(o[e])));
                                o[e] = __float_as_uint(__uint_as_float(o[e]) * step);
                            }
                            tmem_st32(lane_addr + C::TMEM_O + cc * 32, o);
                        }
                        tmem_wait_st();
                        if (move) {
                            v_log = sc.y;
                            if (falls) fall = move_unit(v_ref, sc.w, top * factor);
                            else v_ref = sc.w;
                            factor *= fall;
                            large |= sc.w > kLargeScale;
                            if (v_ref != sc.w) {
                                // under a unit that could not follow, P goes no lower than where nothing is left of it in f16: the row's
                                // sum needs its exponentials
                                v_log = log2f(v_ref);
                                sc.y = fmaxf(sc.y, v_log - kLeastLog);
                                sc.z = fminf(sc.z, kLeast / v_ref);
                            }
                        }
                    }
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
                // P = 2^(z - m) times the page's value scale over O's; the row's sum without it
                uint32_t pk[32];
                {
                    const float by = off + (sc.y - v_log);
                    const uint64_t scale2 = f32x2(cr, cr), off2 = f32x2(by, by);
                    uint64_t acc[4] = {0, 0, 0, 0};
#pragma unroll
                    for (int k = 0; k < NK; k += 2) {
                        float a0, a1;
                        f32x2_split(fma_f32x2(f32x2(xs[k], xs[k + 1]), scale2, off2), a0, a1);
                        const float e0 = fast_exp2(a0), e1 = fast_exp2(a1);
                        acc[(k >> 1) & 3] = add_f32x2(acc[(k >> 1) & 3], f32x2(e0, e1));
                        pk[k >> 1] = pack_f16x2(e0, e1);
                    }
                    float s0, s1;
                    f32x2_split(add_f32x2(add_f32x2(acc[0], acc[1]), add_f32x2(acc[2], acc[3])), s0, s1);
                    l = fmaf(s0 + s1, sc.z * v_ref, l);
                }
                if (!product_done()) { ok = false; break; }
                tc_fence_after();
                tmem_st32(lane_addr + C::TMEM_P, pk);
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&ctl.p_full[tile]);
            }
            // the next item's Q goes ahead of this one's epilogue: its first product runs during it
            if (!ok || !take_item(r, nx)) { ok = false; break; }
            // The next item's first PV overwrites O only after this warp's next arrival on
            // p_full, which follows the reads below.
            if (!mbar_wait_warp(&ctl.pv_done[tile], (gt - 1) & 1, wc)) { ok = false; break; }
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
                if (large) {
                    v_ref *= kShrinkFactor;
                    m_use += kShrink;
                    l *= kShrinkFactor;
                }
                float4* po = reinterpret_cast<float4*>(a.part_o) + (static_cast<size_t>(x.part) * TILES + tile) * (D / 4) * kBM + row;
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
                if (valid) a.part_ml[(static_cast<size_t>(x.part) * TILES + tile) * kBM + row] = make_float2(m_use, l);
            }
            tc_fence_before();
        }
    }
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem_base, TILES * C::TMEM_COLS);
    }
}

template <int D, int TILES>
cudaError_t launch_d(ChunkArgs a, const KernelEnv& env, const char** err) {
    using C = Cfg<D, TILES>;
    cudaError_t e = ensure_smem_attr(reinterpret_cast<const void*>(chunk8_tile_kernel<D, TILES>), C::SMEM);
    if (e != cudaSuccess) { *err = "cudaFuncSetAttribute(8-bit tile attention)"; return e; }
    a.blocks = 2 / TILES * device_sm_count();   // their shared memory and tensor memory fit at once
    CUtensorMap mq;
    if (make_tmap_bf16_box(&mq, a.Q, D, a.Hq, a.T, 64, a.G, kBM / a.G) != 0) {
        *err = "tensor map";
        return cudaErrorInvalidValue;
    }
    e = launch_early(chunk8_tile_kernel<D, TILES>, dim3(a.blocks), C::THREADS, C::SMEM, env.stream, mq, a, a.sm_scale * kLog2e, env.limit);
    if (e != cudaSuccess) { *err = "8-bit tile attention launch"; return e; }
    e = launch_early(chunk_join_kernel<D, TILES>, dim3(a.blocks), kJoinThreads, 0, env.stream, a);
    if (e != cudaSuccess) *err = "8-bit attention join launch";
    return e;
}

}  // namespace

cudaError_t chunk8_tile_prepare(int d) {
    if (d == 64) return ensure_smem_attr(reinterpret_cast<const void*>(chunk8_tile_kernel<64, 1>), Cfg<64, 1>::SMEM);
    const cudaError_t e = ensure_smem_attr(reinterpret_cast<const void*>(chunk8_tile_kernel<128, 1>), Cfg<128, 1>::SMEM);
    return e == cudaSuccess ? ensure_smem_attr(reinterpret_cast<const void*>(chunk8_tile_kernel<128, 2>), Cfg<128, 2>::SMEM) : e;
}

cudaError_t launch_chunk8_tile(const ChunkArgs& a, const KernelEnv& env, const char** err) {
    if (a.d == 64) return launch_d<64, 1>(a, env, err);
    return static_cast<long long>(a.T) * a.G > kTwoTiles * a.B ? launch_d<128, 2>(a, env, err) : launch_d<128, 1>(a, env, err);
}

}  // namespace sas
