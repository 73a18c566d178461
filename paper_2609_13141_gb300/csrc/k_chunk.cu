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
// Few new tokens over a long cache leave few tiles: a tile's pages are then split
// over several items (chunk_tiles_kernel), each writing its (max, sum, O) in fp32,
// and the last item of a tile to finish joins them in the order of the splits, so
// equal inputs give equal outputs.
//
// Keys past a sequence's end in its last page may hold anything: scores there are
// replaced, not weighted by zero, and values past the tile's last position are
// zeroed in shared memory before the product.  A table entry out of range is never
// used as an address: it becomes the row past the cache, which TMA reads as zero.
#include <math_constants.h>

#include "internal.h"
#include "ptx.cuh"

namespace sas {
namespace {

constexpr int kBM = 128;          // rows of a tile
constexpr int kBN = 64;           // keys of a page
constexpr int kThreads = 256;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.69314718055994531f;
constexpr float kRescaleThreshold = 8.0f;   // log2 units
constexpr int kItemSlots = 4;     // work items in flight between warp 0 and the other roles
constexpr int kItemReaders = 7;   // V producer, two MMA issuers, four softmax warps
constexpr int kStatusBadInput = 1;
constexpr int kStatusLayout = 3;
constexpr int kJoin = 8;          // rows of a warp in flight when splits are joined
constexpr int kPlanThreads = 1024;
constexpr int kBuckets = 64;

__device__ __forceinline__ void grid_dep_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void grid_dep_launch() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// ------------------------------------------------------------------ work list
//
// One block: tiles of every sequence (prefix sum over sequences), the total number
// of pages they walk, from it the split length that gives about `target` items, and
// the items, longest first (64 classes of length; the order within a class does not
// change any result).

__global__ void __launch_bounds__(kPlanThreads) chunk_tiles_kernel(ChunkArgs a, int R) {
    __shared__ int wsum[32];
    __shared__ int hist[kBuckets], carry, npart, maxlen;
    __shared__ unsigned long long work;
    grid_dep_launch();
    const int t = threadIdx.x, lane = lane_id(), warp = warp_id();
    if (t == 0) {
        carry = 0;
        npart = 0;
        maxlen = 1;
        work = 0;
        a.sched[0] = 0;
    }
    if (t < kBuckets) hist[t] = 0;
    int bad = 0;
    for (int b = t; b < a.B; b += kPlanThreads) {
        const int c0 = __ldg(a.cu + b), c1 = __ldg(a.cu + b + 1);
        bad |= c0 < 0 || c1 < c0 || c1 > a.T;
    }
    bad = __syncthreads_or(bad);
    if (bad) {   // offsets that overlap could ask for more tiles than there is room for
        if (t == 0) {
            atomicExch(a.status, kStatusBadInput);
            *a.nitems = 0;
        }
        return;
    }
    for (int base = 0; base < a.B; base += kPlanThreads) {
        const int b = base + t;
        int nt = 0;
        if (b < a.B) {
            const int n = __ldg(a.cu + b + 1) - __ldg(a.cu + b), L = __ldg(a.kv_lens + b);
            if (L < n || L > 64LL * a.max_blocks) atomicExch(a.status, kStatusBadInput);
            else nt = (n + R - 1) / R;
        }
        int inc = nt;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, inc, o);
            if (lane >= o) inc += x;
        }
        if (lane == 31) wsum[warp] = inc;
        __syncthreads();
        if (warp == 0) {
            int v = wsum[lane];
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int x = __shfl_up_sync(0xffffffffu, v, o);
                if (lane >= o) v += x;
            }
            wsum[lane] = v;
        }
        __syncthreads();
        if (b < a.B) a.tile_off[b] = carry + (warp > 0 ? wsum[warp - 1] : 0) + inc - nt;
        __syncthreads();
        if (t == 0) carry += wsum[31];
        __syncthreads();
    }
    const int ntiles = carry;
    unsigned long long mine = 0;
    int longest = 1;
    for (int i = t; i < ntiles; i += kPlanThreads) {
        int lo = 0, hi = a.B;   // the last sequence whose first tile is <= i (empty ones share theirs with the next)
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (a.tile_off[mid] <= i) lo = mid;
            else hi = mid;
        }
        const int c0 = __ldg(a.cu + lo), n = __ldg(a.cu + lo + 1) - c0, L = __ldg(a.kv_lens + lo);
        const int k = (i - a.tile_off[lo]) * R;
        const int nt = min(R, n - k), pos0 = L - n + k;
        a.tiles[i] = make_int4(lo, c0 + k, nt, pos0);
        const int nb = ((pos0 + nt - 1) >> 6) + 1;
        mine += nb;
        longest = max(longest, nb);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        mine += __shfl_xor_sync(0xffffffffu, mine, o);
        longest = max(longest, __shfl_xor_sync(0xffffffffu, longest, o));
    }
    if (lane == 0) {
        atomicAdd(&work, mine);
        atomicMax(&maxlen, longest);
    }
    __syncthreads();
    const unsigned long long per_item = (work * a.Hkv + a.target - 1) / a.target;
    const int len = per_item < kChunkMinSplit ? kChunkMinSplit
                                              : (per_item < (1u << 20) ? static_cast<int>(per_item) : (1 << 20));
    const int top = min(maxlen, len);
    // longest first: class of a split length
    auto cls = [&](int per) { return kBuckets - 1 - static_cast<int>(static_cast<long long>(per) * (kBuckets - 1) / top); };
    for (int pass = 0; pass < 2; ++pass) {
        for (int i = t; i < ntiles; i += kPlanThreads) {
            const int4 x = a.tiles[i];
            const int nb = ((x.w + x.z - 1) >> 6) + 1;
            const int want = (nb + len - 1) / len;
            const int per = (nb + want - 1) / want, ns = (nb + per - 1) / per;
            const int c = max(0, min(kBuckets - 1, cls(per)));
            const int at = atomicAdd(&hist[c], ns);
            if (pass == 0) continue;
            int part = -1;
            if (ns > 1) {
                part = atomicAdd(&npart, ns);
                for (int h = 0; h < a.Hkv; ++h) a.counts[static_cast<size_t>(part) * a.Hkv + h] = 0;
            }
            for (int s = 0; s < ns; ++s) {
                a.items[2 * (at + s)] = x;
                a.items[2 * (at + s) + 1] = make_int4(s * per, min(nb, (s + 1) * per), part, (s << 16) | ns);
            }
        }
        __syncthreads();
        if (pass == 0) {
            if (t == 0) {
                int sum = 0;
                for (int c = 0; c < kBuckets; ++c) {
                    const int x = hist[c];
                    hist[c] = sum;
                    sum += x;
                }
                *a.nitems = sum;
            }
            __syncthreads();
        }
    }
}

// ------------------------------------------------------------------ attention

template <int D>
struct Cfg {
    static constexpr int Q_BYTES = kBM * D * 2;
    static constexpr int KV_BYTES = kBN * D * 2;
    static constexpr int KST = 2;
    static constexpr int VST = 2;
    static constexpr int OFF_K = Q_BYTES;
    static constexpr int OFF_V = OFF_K + KST * KV_BYTES;
    static constexpr int OFF_CTL = OFF_V + VST * KV_BYTES;
    static constexpr int SMEM = OFF_CTL + 512;
    static constexpr int TMEM_COLS = 256;    // O [0,D)  S [128,192)  P0 [192,224)  P1 [224,256)
    static constexpr int TMEM_O = 0;
    static constexpr int TMEM_S = 128;
    static constexpr int TMEM_P = 192;
    static constexpr uint32_t IDESC_S = idesc_bf16(kBM, kBN, 0, 0);
    static constexpr uint32_t IDESC_O = idesc_bf16(kBM, D, 0, 1);
};

// A work item as the roles read it: one split of one tile of one KV group.
struct Item {
    int head;                 // KV group, or -1: no more work
    int seq, tok0, ntok, pos0;
    int blk0, blk1;           // its pages
    int part, split, ns;      // partial results (part < 0: the whole tile)
};

struct Ctl {
    uint64_t q_full, q_empty, k_full[4], k_empty[4], v_full[4], v_empty[4];
    uint64_t s_full, s_free, p_full[2], pv_done[2], drain_bar;
    uint64_t part_done, last_known;   // a split's results written by the four softmax warps; ctl.last set
    uint64_t item_full[kItemSlots], item_empty[kItemSlots];
    Item item[kItemSlots];
    uint32_t tmem_base;
    int abort_flag, last;
};
static_assert(sizeof(Ctl) <= 512, "control block");

__device__ __forceinline__ bool read_item(Ctl& ctl, int r, const WaitCtl& wc, Item& x) {
    const int slot = r % kItemSlots;
    if (!mbar_poll_warp(&ctl.item_full[slot], (r / kItemSlots) & 1, wc)) return false;
    x = ctl.item[slot];
    __syncwarp();
    if (lane_id() == 0) mbar_arrive(&ctl.item_empty[slot]);
    return true;
}

// Row of the cache's [page][KV group] axis that holds logical page m + lane of the
// item's sequence (lanes past blk1: unused).
__device__ __forceinline__ int page_row(const ChunkArgs& a, const Item& x, int m, int lane) {
    if (m + lane >= x.blk1) return 0;
    int page = __ldg(a.block_table + static_cast<size_t>(x.seq) * a.max_blocks + m + lane);
    if (page < 0 || page >= a.num_pages) {
        atomicExch(a.status, kStatusBadInput);
        return a.num_pages * a.Hkv;   // past the end: TMA fills with zero
    }
    return page * a.Hkv + x.head;
}

template <int D>
__global__ void __launch_bounds__(kThreads, 2)
chunk_attn_kernel(const __grid_constant__ CUtensorMap mapQ, const __grid_constant__ CUtensorMap mapK,
                  const __grid_constant__ CUtensorMap mapV, ChunkArgs a, float scale_log2, long long limit) {
    using C = Cfg<D>;
    extern __shared__ __align__(1024) uint8_t smem[];
    if ((smem_u32(smem) & 1023u) != 0) {
        if (threadIdx.x == 0) atomicExch(a.status, kStatusLayout);
        return;
    }
    Ctl& ctl = *reinterpret_cast<Ctl*>(smem + C::OFF_CTL);
    const uint32_t warp = warp_id(), lane = lane_id();
    if (threadIdx.x == 0) {
        mbar_init(&ctl.q_full, 1);
        mbar_init(&ctl.q_empty, 1);
        for (int s = 0; s < C::KST; ++s) { mbar_init(&ctl.k_full[s], 1); mbar_init(&ctl.k_empty[s], 1); }
        for (int s = 0; s < C::VST; ++s) { mbar_init(&ctl.v_full[s], 1); mbar_init(&ctl.v_empty[s], 1); }
        mbar_init(&ctl.s_full, 1);
        mbar_init(&ctl.s_free, 4);
        for (int s = 0; s < 2; ++s) {
            mbar_init(&ctl.pv_done[s], 1);
            mbar_init(&ctl.p_full[s], 4);
        }
        mbar_init(&ctl.drain_bar, 2);
        mbar_init(&ctl.part_done, 4);
        mbar_init(&ctl.last_known, 1);
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
    grid_dep_wait();   // the work list, and through its kernel everything before it

    // Every role walks the same items and counts pages over all of them (g): ring
    // slots, score buffers and barrier phases follow g across item boundaries.
    if (warp == 0) {
        // ---------------- items and K pages
        if (lane == 0) tma_prefetch_desc(&mapK);
        const long long W = static_cast<long long>(*a.nitems) * a.Hkv;
        long long w = blockIdx.x;
        int g = 0;
        bool ok = true;
        for (int r = 0; ok; ++r) {
            const int slot = r % kItemSlots;
            if (!mbar_wait_warp(&ctl.item_empty[slot], ((r / kItemSlots) & 1) ^ 1u, wc)) { ok = false; break; }
            Item x;
            x.head = -1;
            x.blk0 = x.blk1 = 0;
            int next = 0;
            if (w < W) {
                if (lane == 0) next = atomicAdd(a.sched, 1);   // used when this item's pages are issued
                const long long e = w / a.Hkv;
                const int4 v0 = a.items[2 * e], v1 = a.items[2 * e + 1];
                x = Item{static_cast<int>(w - e * a.Hkv), v0.x, v0.y, v0.z, v0.w, v1.x, v1.y, v1.z, v1.w >> 16, v1.w & 0xffff};
            }
            if (lane == 0) {
                ctl.item[slot] = x;
                mbar_arrive(&ctl.item_full[slot]);
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
            w = gridDim.x + static_cast<long long>(__shfl_sync(0xffffffffu, next, 0));
        }
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
            if (!mbar_wait_warp(&ctl.q_empty, (nq & 1) ^ 1u, wc)) { ok = false; break; }
            if (lane == 0) {
                mbar_arrive_expect_tx(&ctl.q_full, C::Q_BYTES);
#pragma unroll
                for (int h = 0; h < D / 64; ++h)
                    tma_load_3d(smem + h * (kBM * 128), &mapQ, &ctl.q_full, h * 64, x.head * a.G, x.tok0);
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
            if (nq > 0) mbar_wait_drain(&ctl.q_full, (nq - 1) & 1, limit, a.status);
            for (int q = g - 1; q >= 0 && q >= g - C::VST; --q)
                mbar_wait_drain(&ctl.v_full[q % C::VST], (q / C::VST) & 1, limit, a.status);
        }
    } else if (warp == 2) {
        // ---------------- S = Q K_g^T, once the softmax warps have loaded S_{g-1}
        const uint64_t dq0 = smem_desc_sw128(smem_u32(smem), 16, 1024);
        const uint64_t dk0 = smem_desc_sw128(smem_u32(smem + C::OFF_K), 16, 1024);
        int g = 0, tc = 0;
        bool ok = true;
        for (int r = 0; ok; ++r, ++tc) {
            Item x;
            if (!read_item(ctl, r, wc, x)) { ok = false; break; }
            if (x.head < 0) break;
            if (!mbar_wait_warp(&ctl.q_full, tc & 1, wc)) { ok = false; break; }
            for (int m = x.blk0; m < x.blk1; ++m, ++g) {
                const int s = g % C::KST;
                if (!mbar_wait_warp(&ctl.k_full[s], (g / C::KST) & 1, wc)) { ok = false; break; }
                if (g >= 1 && !mbar_wait_warp(&ctl.s_free, (g - 1) & 1, wc)) { ok = false; break; }
                tc_fence_after();
                const uint64_t dk = dk0 + static_cast<uint64_t>((s * C::KV_BYTES) >> 4);
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) {
                        const uint32_t off_q = (k >> 2) * (kBM * 128) + (k & 3) * 32;
                        const uint32_t off_k = (k >> 2) * (kBN * 128) + (k & 3) * 32;
                        umma_bf16(tmem_base + C::TMEM_S, dq0 + (off_q >> 4), dk + (off_k >> 4), C::IDESC_S, k > 0);
                    }
                    umma_commit(&ctl.s_full);
                    umma_commit(&ctl.k_empty[s]);
                    if (m == x.blk1 - 1) umma_commit(&ctl.q_empty);
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
        // ---------------- O += P_g V_g; an item's first page starts a new accumulator
        const uint64_t dv0 = smem_desc_sw128(smem_u32(smem + C::OFF_V), kBN * 128, 1024);
        int g = 0;
        bool ok = true;
        for (int r = 0; ok; ++r) {
            Item x;
            if (!read_item(ctl, r, wc, x)) { ok = false; break; }
            if (x.head < 0) break;
            const int end = x.pos0 + x.ntok;   // keys from here on belong to no row of the tile
            for (int m = x.blk0; m < x.blk1; ++m, ++g) {
                const int vs = g % C::VST;
                if (!mbar_wait_warp(&ctl.v_full[vs], (g / C::VST) & 1, wc)) { ok = false; break; }
                if (end < (m + 1) * kBN) {
                    // zero value rows: P is 0 there, and 0 times a stale infinity or NaN is NaN
                    const int r0 = max(0, end - m * kBN);
                    uint8_t* v = smem + C::OFF_V + vs * C::KV_BYTES;
                    for (int i = r0 * 8 + lane; i < kBN * 8; i += 32) {
#pragma unroll
                        for (int h = 0; h < D / 64; ++h)
                            *reinterpret_cast<uint4*>(v + h * (kBN * 128) + i * 16) = make_uint4(0, 0, 0, 0);
                    }
                    fence_proxy_async_smem();
                    __syncwarp();
                }
                if (!mbar_wait_warp(&ctl.p_full[g & 1], (g >> 1) & 1, wc)) { ok = false; break; }
                tc_fence_after();
                const uint64_t dv = dv0 + static_cast<uint64_t>((vs * C::KV_BYTES) >> 4);
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < kBN / 16; ++k)
                        umma_bf16_ta(tmem_base + C::TMEM_O, tmem_base + C::TMEM_P + (g & 1) * 32 + k * 8,
                                     dv + ((k * 2048) >> 4), C::IDESC_O, (m > x.blk0 || k > 0) ? 1u : 0u);
                    umma_commit(&ctl.pv_done[g & 1]);
                    umma_commit(&ctl.v_empty[vs]);
                }
                __syncwarp();
            }
        }
        if (elect_one()) {
            umma_commit(&ctl.drain_bar);
            mbar_wait_drain(&ctl.drain_bar, 0, limit, a.status);
        }
        __syncwarp();
    } else {
        // ---------------- softmax, one thread per row
        const int q = warp - 4;
        const int row = q * 32 + lane;
        const int tok = row / a.G, hq = row - tok * a.G;
        const uint32_t lane_addr = tmem_base + (static_cast<uint32_t>(q * 32) << 16);
        const uint64_t scale2 = f32x2(scale_log2, scale_log2);
        int g = 0, np = 0;   // pages and splits over all items
        bool ok = true;
        for (int r = 0; ok; ++r) {
            Item x;
            if (!read_item(ctl, r, wc, x)) { ok = false; break; }
            if (x.head < 0) break;
            const bool valid = tok < x.ntok;
            const bool warp_rows = q * 32 < x.ntok * a.G;   // else nothing of this warp is ever read
            const int pos = x.pos0 + tok;
            float m_use = -CUDART_INF_F, l = 0.f;
            for (int m = x.blk0; m < x.blk1; ++m, ++g) {
                const int pb = g & 1;
                // last key column of page m that this row sees (< 0: none)
                const int lim = valid ? min(kBN - 1, pos - m * kBN) : -1;
                if (!mbar_wait_warp(&ctl.s_full, g & 1, wc)) { ok = false; break; }
                if (g >= 2 && !mbar_wait_warp(&ctl.pv_done[pb], ((g - 2) >> 1) & 1, wc)) { ok = false; break; }
                if (!warp_rows) {
                    if (lane == 0) {
                        mbar_arrive(&ctl.s_free);
                        mbar_arrive(&ctl.p_full[pb]);
                    }
                    __syncwarp();
                    continue;
                }
                tc_fence_after();
                float xs[64];
                {
                    uint32_t u0[32], u1[32];
                    tmem_ld32(lane_addr + C::TMEM_S, u0);
                    tmem_ld32(lane_addr + C::TMEM_S + 32, u1);
                    tmem_wait_ld();
#pragma unroll
                    for (int k = 0; k < 32; ++k) {
                        xs[k] = __uint_as_float(u0[k]);
                        xs[k + 32] = __uint_as_float(u1[k]);
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&ctl.s_free);
                if (__any_sync(0xffffffffu, lim < kBN - 1)) {
#pragma unroll
                    for (int k = 0; k < 64; ++k) xs[k] = k <= lim ? xs[k] : -CUDART_INF_F;
                }
                float mx0 = -CUDART_INF_F, mx1 = -CUDART_INF_F;
#pragma unroll
                for (int k = 0; k < 64; k += 4) {
                    mx0 = max3f(mx0, xs[k], xs[k + 1]);
                    mx1 = max3f(mx1, xs[k + 2], xs[k + 3]);
                }
                const float mb = fmaxf(mx0, mx1) * scale_log2;
                const bool need = mb > m_use + kRescaleThreshold;
                const float m_new = need ? mb : m_use;
                const float off = m_new == -CUDART_INF_F ? 0.f : -m_new;
                const uint64_t off2 = f32x2(off, off);
                uint64_t acc[4] = {0, 0, 0, 0};
                uint32_t pk[32];
#pragma unroll
                for (int k = 0; k < 64; k += 2) {
                    float a0, a1;
                    f32x2_split(fma_f32x2(f32x2(xs[k], xs[k + 1]), scale2, off2), a0, a1);
                    const float e0 = fast_exp2(a0), e1 = fast_exp2(a1);
                    acc[(k >> 1) & 3] = add_f32x2(acc[(k >> 1) & 3], f32x2(e0, e1));
                    pk[k >> 1] = pack_bf16x2(e0, e1);
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
                    // rescaling O needs the previous page's PV done
                    if (!mbar_wait_warp(&ctl.pv_done[(g - 1) & 1], ((g - 1) >> 1) & 1, wc)) { ok = false; break; }
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
                tmem_st32(lane_addr + C::TMEM_P + pb * 32, pk);
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&ctl.p_full[pb]);
            }
            if (!ok) break;
            // The next item's first PV overwrites O only after this warp's next arrival on
            // p_full, which follows the reads below.
            const int gl = g - 1;
            if (!mbar_wait_warp(&ctl.pv_done[gl & 1], (gl >> 1) & 1, wc)) { ok = false; break; }
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
            // ---- a split: (max, sum) and the unnormalised O of every row in fp32
            const size_t pslot = (static_cast<size_t>(x.part) + x.split) * a.Hkv + x.head;
            if (warp_rows) {
                float* po = a.part_o + (pslot * kBM + row) * D;
#pragma unroll 1
                for (int cc = 0; cc < D / 32; ++cc) {
                    uint32_t o[32];
                    tmem_ld32(lane_addr + C::TMEM_O + cc * 32, o);
                    tmem_wait_ld();
                    if (valid) {
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            reinterpret_cast<uint4*>(po + cc * 32)[e] =
                                make_uint4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
                    }
                }
                if (valid) a.part_ml[pslot * kBM + row] = make_float2(m_use, l);
            }
            tc_fence_before();
            // (barriers with a bounded wait: a warp that gave up must not leave the others waiting)
            __threadfence();
            mbar_arrive_warp(&ctl.part_done);
            if (q == 0) {
                if (!mbar_wait_warp(&ctl.part_done, np & 1, wc)) { ok = false; break; }
                if (lane == 0) {
                    *reinterpret_cast<volatile int*>(&ctl.last) =
                        atomicAdd(a.counts + static_cast<size_t>(x.part) * a.Hkv + x.head, 1) == x.ns - 1;
                    mbar_arrive(&ctl.last_known);
                }
                __syncwarp();
            }
            // the flag is set again only after all four warps' next arrival on part_done
            if (!mbar_wait_warp(&ctl.last_known, np & 1, wc)) { ok = false; break; }
            ++np;
            if (*reinterpret_cast<volatile int*>(&ctl.last) == 0) continue;
            __threadfence();
            // join the splits: a warp takes kJoin rows at a time (their loads in flight
            // together), D / 32 columns a lane
            constexpr int CPL = D / 32;
            const size_t stride = static_cast<size_t>(a.Hkv) * kBM;   // rows between the splits of a tile
            const int rows = x.ntok * a.G;
            const size_t base = (static_cast<size_t>(x.part) * a.Hkv + x.head) * kBM;
            for (int r0 = q; r0 < rows; r0 += 4 * kJoin) {
                float M[kJoin], L[kJoin], acc[kJoin][CPL];
#pragma unroll
                for (int k = 0; k < kJoin; ++k) {
                    M[k] = -CUDART_INF_F;
                    L[k] = 0.f;
#pragma unroll
                    for (int e = 0; e < CPL; ++e) acc[k][e] = 0.f;
                }
                // rows past the last repeat it: loaded, not stored
                for (int s = lane; s < x.ns; s += 32) {
#pragma unroll
                    for (int k = 0; k < kJoin; ++k)
                        M[k] = fmaxf(M[k], __ldcg(a.part_ml + base + min(r0 + 4 * k, rows - 1) + s * stride).x);
                }
#pragma unroll
                for (int k = 0; k < kJoin; ++k)
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1) M[k] = fmaxf(M[k], __shfl_xor_sync(0xffffffffu, M[k], o));
                for (int s0 = 0; s0 < x.ns; s0 += 32) {
                    float wgt[kJoin];
#pragma unroll
                    for (int k = 0; k < kJoin; ++k) {
                        wgt[k] = 0.f;
                        if (s0 + static_cast<int>(lane) < x.ns) {
                            const float2 ml = __ldcg(a.part_ml + base + min(r0 + 4 * k, rows - 1) + (s0 + lane) * stride);
                            wgt[k] = ml.x == -CUDART_INF_F ? 0.f : fast_exp2(ml.x - M[k]);
                            L[k] = fmaf(wgt[k], ml.y, L[k]);
                        }
                    }
                    const int cnt = min(32, x.ns - s0);
#pragma unroll 1
                    for (int s = 0; s < cnt; ++s) {
                        const float* src = a.part_o + (base + (s0 + s) * stride) * D + lane * CPL;
                        float v[kJoin][CPL];
#pragma unroll
                        for (int k = 0; k < kJoin; ++k) {
                            const float* at = src + static_cast<size_t>(min(r0 + 4 * k, rows - 1)) * D;
                            if constexpr (CPL == 4) {
                                const float4 f = __ldcg(reinterpret_cast<const float4*>(at));
                                v[k][0] = f.x; v[k][1] = f.y; v[k][2] = f.z; v[k][3] = f.w;
                            } else {
                                const float2 f = __ldcg(reinterpret_cast<const float2*>(at));
                                v[k][0] = f.x; v[k][1] = f.y;
                            }
                        }
#pragma unroll
                        for (int k = 0; k < kJoin; ++k) {
                            const float ws = __shfl_sync(0xffffffffu, wgt[k], s);
                            if (ws != 0.f) {   // (a split in which the row sees no key does not count, whatever it holds)
#pragma unroll
                                for (int e = 0; e < CPL; ++e) acc[k][e] = fmaf(ws, v[k][e], acc[k][e]);
                            }
                        }
                    }
                }
#pragma unroll
                for (int k = 0; k < kJoin; ++k) {
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1) L[k] += __shfl_xor_sync(0xffffffffu, L[k], o);
                    const int rr = r0 + 4 * k;
                    if (rr >= rows) continue;
                    const float inv = 1.f / L[k];
                    const int tk = rr / a.G, h = rr - tk * a.G;
                    const size_t at = (static_cast<size_t>(x.tok0) + tk) * a.Hq + static_cast<size_t>(x.head) * a.G + h;
                    uint32_t* dst = reinterpret_cast<uint32_t*>(a.O + at * D) + lane * (CPL / 2);
#pragma unroll
                    for (int e = 0; e < CPL / 2; ++e) dst[e] = pack_bf16x2(acc[k][2 * e] * inv, acc[k][2 * e + 1] * inv);
                    if (lane == 0 && a.LSE != nullptr) a.LSE[at] = M[k] * kLn2 + logf(L[k]);
                }
            }
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
    const int R = kBM / a.G;
    CUtensorMap mq, mk, mv;
    const uint64_t rows = static_cast<uint64_t>(a.num_pages) * a.Hkv;
    if (make_tmap_bf16_box(&mq, a.Q, D, a.Hq, a.T, 64, a.G, R) != 0 ||
        make_tmap_bf16_3d(&mk, a.K_cache, D, kBN, rows, 64, kBN) != 0 ||
        make_tmap_bf16_3d(&mv, a.V_cache, D, kBN, rows, 64, kBN) != 0) {
        *err = "tensor map";
        return cudaErrorInvalidValue;
    }
    chunk_tiles_kernel<<<1, kPlanThreads, 0, env.stream>>>(a, R);
    e = cudaGetLastError();
    if (e != cudaSuccess) { *err = "chunk work list launch"; return e; }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2 * device_sm_count());
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = C::SMEM;
    cfg.stream = env.stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, chunk_attn_kernel<D>, mq, mk, mv, a, a.sm_scale * kLog2e, env.limit);
    if (e != cudaSuccess) *err = "chunk attention launch";
    return e;
}

}  // namespace

int chunk_target_items() { return 4 * device_sm_count(); }

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
