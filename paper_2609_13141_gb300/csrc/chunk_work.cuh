// How the attention of new tokens over a paged cache is cut into work, and the join of the
// splits: what its kernels share.
//
// A tile is R = 2^rl consecutive tokens of one sequence times the G query heads of one KV
// group; a unit is one tile of one KV group, its cost its pages and a constant.  All units, in
// the order (sequence, tile, group), are cut into equal ranges, one per block: no scheduling at
// run time, every block ends at about the same time however long the units are, and a block
// splits at most the first and the last unit of its range.  A split writes its (max, sum, O) in
// fp32, and chunk_join_kernel joins the splits of a unit in their order, so equal inputs give
// equal outputs.
#pragma once

#include <math_constants.h>

#include "serve.h"
#include "serve_ptx.cuh"

namespace sas {
namespace {

constexpr int kBM = 128;          // rows of a tile, at most
constexpr int kBN = 64;           // keys of a page
constexpr int kRangeThreads = 256;
constexpr float kLn2 = 0.69314718055994531f;
constexpr int kStatusBadInput = 1;
constexpr int kUnitCost = 4;      // what a unit costs beside its pages (its Q tile, its epilogue: 2 to 3 us), in pages
constexpr int kSnap = 4;          // pages: ranges do not cut this close to a unit's ends
// A block's range has this many pages at least, twice as many where units have kLongUnit
// pages on average and would go into many splits: 7 requests of 2 to 12 tokens over 2000
// to 16000, 2 heads of 128, 31.4 us with 4 and 27.3 with 8; 4 single tokens over 100 to
// 800, 8 KV groups of 128, 12.5 and 15.1.
constexpr int kMinShare = 4;
constexpr int kLongUnit = 64;
constexpr int kJoinThreads = 512;

// ------------------------------------------------------------------ shares

// Sequence b: its new tokens and its length, no new tokens if the length is wrong.
struct Seq {
    int c0, n, L;
    __device__ __forceinline__ Seq(const ChunkArgs& a, int b) {
        c0 = load(a.cu + b);
        n = load(a.cu + b + 1) - c0;
        L = load(a.kv_lens + b);
        if (L < n || L > 64LL * a.max_blocks) n = 0;
    }
    // R = 2^rl tokens a tile
    __device__ __forceinline__ int tiles(int rl) const { return (n + (1 << rl) - 1) >> rl; }
    // pages of tile t
    __device__ __forceinline__ int pages(int t, int rl) const { return ((L - n + min(n, (t + 1) << rl) - 1) >> 6) + 1; }
    // Cost of tiles 0 .. m - 1, all full: their pages are the sum over t = 1 .. m of floor((p + t R) / 64) + 1
    // with p = L - n - 1 = 64 q + r.  For R >= 64 the floor is q + t R / 64.  For R = 64 / k it
    // is q + floor((floor(r / R) + t) / k), and sums
    // of floor(u / k) over u = 0 .. x are k y (y - 1) / 2 + y (x % k + 1), y = floor(x / k).
    __device__ __forceinline__ long long before(int m, int rl) const {
        const int p = L - n - 1;
        const long long flat = static_cast<long long>(m) * ((p >> 6) + 1 + kUnitCost);
        if (rl >= 6) return flat + (static_cast<long long>(m) * (m + 1) / 2 << (rl - 6));
        const int kl = 6 - rl, x = ((p & 63) >> rl) + m;
        const long long y = x >> kl;
        return flat + ((y * (y - 1) / 2) << kl) + y * ((x & ((1 << kl) - 1)) + 1);
    }
    __device__ __forceinline__ long long all(int rl) const {
        const int nt = tiles(rl);
        return nt <= 0 ? 0 : before(nt - 1, rl) + pages(nt - 1, rl) + kUnitCost;
    }
};

// A boundary between two ranges: page `page` of unit (seq, tile, head) of nb pages; `at`
// is the unit's cost before it, of nb + kUnitCost, where the ranges cut it before kSnap.
struct Bound {
    int seq, tile, head, page, nb, at;
};

// How everything is cut: boundary k is at cost k share + min(k, rest).
struct Cut {
    long long share;
    int rest, ranges;
};

// Where a block's two boundaries are: a sequence, and the cost before them in it.
struct Shares {
    long long sum[kRangeThreads / 32], off[2];
    int tiles[kRangeThreads / 32], seq[2];
    bool last[2];   // the end of everything
    Cut cut;
};

// Finds the sequences of the block's range; false if it has none.  All threads call it (those
// past the first kRangeThreads have no sequences).
// Every block sums up all sequences itself (12 bytes each, from L2): no launch before
// this one, nothing to wait for.
__device__ __forceinline__ bool find_range(const ChunkArgs& a, int rl, Shares& sh) {
    const int t = threadIdx.x, lane = lane_id(), warp = warp_id();
    const int per = (a.B + kRangeThreads - 1) / kRangeThreads;   // neighbouring sequences of a thread
    const int b0 = min(a.B, t * per), b1 = min(a.B, b0 + per);
    long long cost = 0;
    int tiles = 0, bad = 0;
    for (int b = b0; b < b1; ++b) {
        const int c0 = load(a.cu + b), c1 = load(a.cu + b + 1);
        const Seq x(a, b);
        bad |= c0 < 0 || c1 < c0 || c1 > a.T;
        if (x.n != c1 - c0 && blockIdx.x == 0) atomicExch(a.status, kStatusBadInput);
        cost += x.all(rl);
        tiles += x.tiles(rl);
    }
    long long inc = cost;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long x = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += x;
    }
    tiles = __reduce_add_sync(0xffffffffu, tiles);
    if (lane == 31 && warp < kRangeThreads / 32) {
        sh.sum[warp] = inc;
        sh.tiles[warp] = tiles;
    }
    if (__syncthreads_or(bad)) {
        if (blockIdx.x == 0 && t == 0) atomicExch(a.status, kStatusBadInput);
        return false;
    }
    long long base = 0, total = 0, units = 0;
#pragma unroll
    for (int w = 0; w < kRangeThreads / 32; ++w) {
        if (w == warp) base = total;
        total += sh.sum[w];
        units += sh.tiles[w];
    }
    total *= a.Hkv;
    units *= a.Hkv;
    if (total == 0) return false;
    // as many ranges as blocks, fewer where they would be under the least share of pages or a unit
    const long long pages = total - units * kUnitCost;
    const int least = pages >= kLongUnit * units ? 2 * kMinShare : kMinShare;
    const long long want = max(units, (pages + least - 1) / least);
    const int ranges = static_cast<int>(min(static_cast<long long>(gridDim.x), want));
    if (static_cast<int>(blockIdx.x) >= ranges) return false;
    // ranges differ by one at most
    const long long share = (total >> 32) == 0 ? static_cast<unsigned>(total) / static_cast<unsigned>(ranges) : total / ranges;
    const int rest = static_cast<int>(total - share * ranges);
    if (t == 0) sh.cut = Cut{share, rest, ranges};
    const long long lo = (base + inc - cost) * a.Hkv, hi = (base + inc) * a.Hkv;   // this thread's sequences
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int c = blockIdx.x + k;
        const long long p = c * share + min(c, rest);
        // the end of the last range is the end of the last unit
        const long long q = p < total ? p : total - 1;
        if (q < lo || q >= hi) continue;
        long long off = q - lo;
        int b = b0;
        for (; b + 1 < b1; ++b) {
            const long long y = Seq(a, b).all(rl) * a.Hkv;
            if (off < y) break;
            off -= y;
        }
        sh.off[k] = off;
        sh.seq[k] = b;
        sh.last[k] = p >= total;
    }
    __syncthreads();
    return true;
}

// The boundaries themselves, by one warp: a half-warp searches the tile of one, 16 tiles
// at a time.
__device__ __forceinline__ void find_bounds(const ChunkArgs& a, int rl, const Shares& sh, Bound& from, Bound& to) {
    const int lane = lane_id(), k = lane >> 4, i = lane & 15;
    long long off = sh.off[k];
    const Seq x(a, sh.seq[k]);
    int tl = 0, th = x.tiles(rl), step;   // the last tile that starts at or before off is in [tl, th)
    do {
        step = (th - tl + 15) >> 4;
        const int m = tl + i * step;
        const unsigned at_or_before = __ballot_sync(0xffffffffu, m < th && x.before(m, rl) * a.Hkv <= off) >> (16 * k) & 0xffffu;
        tl += (__popc(at_or_before) - 1) * step;
        th = min(th, tl + step);
    } while (__any_sync(0xffffffffu, step > 1));
    off -= x.before(tl, rl) * a.Hkv;   // < Hkv (pages + kUnitCost) < 2^32
    Bound y;
    y.seq = sh.seq[k];
    y.tile = tl;
    y.nb = x.pages(tl, rl);
    y.head = static_cast<unsigned>(off) / static_cast<unsigned>(y.nb + kUnitCost);
    y.at = static_cast<int>(off - static_cast<long long>(y.head) * (y.nb + kUnitCost));
    const int page = y.at - kUnitCost;
    y.page = page < kSnap ? 0 : (y.nb - page < kSnap ? y.nb : page);
    if (sh.last[k]) y.page = y.nb;
    auto get = [&](Bound& z, int src) {
        z.seq = __shfl_sync(0xffffffffu, y.seq, src);
        z.tile = __shfl_sync(0xffffffffu, y.tile, src);
        z.head = __shfl_sync(0xffffffffu, y.head, src);
        z.page = __shfl_sync(0xffffffffu, y.page, src);
        z.nb = __shfl_sync(0xffffffffu, y.nb, src);
        z.at = __shfl_sync(0xffffffffu, y.at, src);
    };
    get(from, 0);
    get(to, 16);
}

// A work item as the roles read it: a unit, or a split of one.
struct Item {
    int head;                 // KV group, or -1: no more work
    int seq, tok0, ntok, pos0;
    int blk0, blk1, nb;       // its pages, of the unit's nb
    int part;                 // where a split's results go (-1: the whole unit)
};

// Row of the cache's [page][KV group] axis that holds logical page m + lane of the
// item's sequence (lanes past blk1: unused).
__device__ __forceinline__ int page_row(const ChunkArgs& a, const Item& x, int m, int lane) {
    if (m + lane >= x.blk1) return 0;
    int page = load(a.block_table + static_cast<size_t>(x.seq) * a.max_blocks + m + lane);
    if (page < 0 || page >= a.num_pages) {
        atomicExch(a.status, kStatusBadInput);
        return a.num_pages * a.Hkv;   // past the end: TMA fills with zero
    }
    return page * a.Hkv + x.head;
}

// The items of a block's range in the order it takes them, by one warp: its whole units, the
// split of the last one among them, and the split of the first one at the end.
struct Walk {
    Bound from, to;
    int seq, tile, head;   // the unit to look at next
    bool any, more, first;
    int late_lo, late_hi;  // the split of the first unit, left for the end
    __device__ __forceinline__ Walk(const ChunkArgs& a, int rl, const Shares& sh, bool any_) : from{}, to{}, any(any_) {
        if (any) find_bounds(a, rl, sh, from, to);
        seq = from.seq;
        tile = from.tile;
        head = from.head;
        more = any;
        first = true;
        late_lo = late_hi = 0;
    }
    __device__ __forceinline__ Item next(const ChunkArgs& a, int rl) {
        const int R = 1 << rl;
        Item x;
        x.head = -1;
        x.blk0 = x.blk1 = 0;
        while (more && x.head < 0) {
            const Seq q(a, seq);
            const int nb = q.pages(tile, rl);
            const bool last = seq == to.seq && tile == to.tile && head == to.head;
            const int lo = first ? from.page : 0, hi = last ? to.page : nb;
            if (first && lo < hi && (lo > 0 || hi < nb)) {
                late_lo = lo;
                late_hi = hi;
            } else if (lo < hi) {
                x = Item{head, seq, q.c0 + tile * R, min(R, q.n - tile * R), q.L - q.n + tile * R, lo, hi, nb,
                         hi < nb ? static_cast<int>(2 * blockIdx.x + 1) : -1};
            }
            first = false;
            more = !last;
            if (more && ++head == a.Hkv) {
                head = 0;
                if (++tile >= q.tiles(rl)) {
                    // the next sequence with new tokens; the range's end lies in one
                    tile = 0;
                    for (int b = seq + 1;; b += 32) {
                        const int y = b + static_cast<int>(lane_id());
                        const unsigned has = __ballot_sync(0xffffffffu, y <= to.seq && Seq(a, min(y, to.seq)).n > 0);
                        if (has != 0 || b >= to.seq) {
                            seq = has != 0 ? b + __ffs(has) - 1 : to.seq;
                            break;
                        }
                    }
                }
            }
        }
        if (x.head < 0 && late_lo < late_hi) {
            const Seq q(a, from.seq);
            x = Item{from.head, from.seq, q.c0 + from.tile * R, min(R, q.n - from.tile * R), q.L - q.n + from.tile * R,
                     late_lo, late_hi, from.nb, static_cast<int>(2 * blockIdx.x)};
            late_hi = 0;
        }
        return x;
    }
    // Off the block's critical path: what it has to join, if its range ends inside a unit (the
    // boundaries once more, rather than registers held all the way).
    __device__ __forceinline__ void record(const ChunkArgs& a, int rl, const Shares& sh) {
        const int R = 1 << rl;
        if (any) find_bounds(a, rl, sh, from, to);
        if (lane_id() != 0) return;
        int4 y = make_int4(0, 0, 0, 0);
        if (any && to.page > 0 && to.page < to.nb) {
            const long long share = sh.cut.share;
            const int rest = sh.cut.rest, here = blockIdx.x;
            auto cost = [&](int k) { return k * share + min(k, rest); };        // before boundary k
            auto last = [&](long long x) {                                      // the last boundary at x or before
                const long long longer = rest * (share + 1);
                return static_cast<int>(x < longer ? x / (share + 1) : rest + (x - longer) / share);
            };
            // the unit is cut at every boundary from kSnap pages after its start to kSnap before its end
            const long long start = cost(here + 1) - to.at;
            const int begin = last(start + kUnitCost + kSnap - 1);
            const int end = min(sh.cut.ranges, last(start + kUnitCost + to.nb - kSnap) + 1);
            const Seq q(a, to.seq);
            y = make_int4(end - begin, begin, to.head, q.c0 + to.tile * R);
            // the block that begins it has it in its first slot if it has no unit before
            a.joins[2 * here + 1] = make_int4(min(R, q.n - to.tile * R), here - begin, cost(begin) < start, 0);
        }
        a.joins[2 * blockIdx.x] = y;
    }
};

// ------------------------------------------------------------------ join

// The splits of a unit are block `begin`'s of the attention and the following blocks'
// first ones, up to its last page.  All of these blocks but the last join it here, each
// some of its columns.  Threads are (row, columns, share of the splits), each a power of
// two: few rows leave many threads for the splits of a row.  Latency-bound: a thread's
// loads are in flight together, and two blocks fit a multiprocessor, so that all run at
// once.  (A join that finds its splits itself before the wait saves one load's latency,
// and takes more from the attention blocks still at work: 117 against 113 us for a mixed
// batch at d = 128.)
// TILES: a tile's rows come 128 to a slot of the splits.
template <int D, int TILES = 1>
__global__ void __launch_bounds__(kJoinThreads, 2) chunk_join_kernel(ChunkArgs a) {
    constexpr int QUADS = D / 4;      // of columns
    constexpr int QB = 2, U = 4;      // quads and splits of a thread in flight together
    __shared__ float top[kJoinThreads], len[kJoinThreads];
    __shared__ float4 part[kJoinThreads];
    const int t = threadIdx.x;
    const int gl = 31 - __clz(a.G);   // G = 2^gl heads
    grid_dep_wait();                  // the splits
    const int4 u = load(a.joins + 2 * blockIdx.x), v = load(a.joins + 2 * blockIdx.x + 1);
    const int ns = u.x, rows = v.x << gl;
    if (ns == 0) return;
    // A split in which the row sees no key does not count, whatever its O holds.  Its sum tells: scores
    // that are all NaN leave a maximum of -infinity too, but a sum of NaN, which has to come through.
    auto nothing = [](float m, float l) { return m == -CUDART_INF_F && l == 0.f; };
    // split s: the first in its slot, the others in slot 0 of the following blocks
    auto slot = [&](int s) { return static_cast<size_t>(2 * (u.y + s) + (s == 0 ? v.z : 0)) * TILES; };
    constexpr int QL = D == 128 ? 5 : 4, TL = 9;
    static_assert(QUADS == 1 << QL && kJoinThreads == 1 << TL, "powers of two");
    const int rpl = max(2, 32 - __clz(rows - 1));       // rows, to a power of two (a clz of 0 is 32)
    // 2^wl blocks share the columns, as long as each has 64 (row, quad) pairs
    const int wl = min(min(31 - __clz(ns - 1), QL), max(0, rpl + QL - 6)), ql = QL - wl;
    if (v.y >> wl != 0) return;
    const int groupl = min(ql, TL - rpl);               // column groups, of `per` quads each
    const int per = 1 << (ql - groupl), spanl = rpl + groupl, span = 1 << spanl;
    const int shares = kJoinThreads >> spanl;           // of the splits; more than one only where per = 1
    const int row = t & ((1 << rpl) - 1), cg = (v.y << groupl) + (t >> rpl & ((1 << groupl) - 1)), mine = t >> spanl;
    const bool live = row < rows;
    const int at = live ? row : 0;
    const int tok = at >> gl, h = at & (a.G - 1);
    const size_t orow = (static_cast<size_t>(u.w) + tok) * a.Hq + static_cast<size_t>(u.z) * a.G + h;
    const int sub = TILES > 1 ? at >> 7 : 0, in = TILES > 1 ? at & 127 : at;
    const float4* const po = reinterpret_cast<const float4*>(a.part_o) + in;
    for (int q0 = 0; q0 < per; q0 += QB) {
        const int quad = cg * per + q0;
        float M = -CUDART_INF_F, L = 0.f;
        float4 o[QB];
#pragma unroll
        for (int k = 0; k < QB; ++k) o[k] = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int s0 = mine; s0 < ns; s0 += U * shares) {
            float2 ml[U];
            float4 x[U][QB];
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int s = s0 + i * shares;
                ml[i] = make_float2(-CUDART_INF_F, 0.f);
                if (s < ns) {
                    ml[i] = __ldcg(a.part_ml + (slot(s) + sub) * kBM + in);
#pragma unroll
                    for (int k = 0; k < QB; ++k)
                        if (k < per) x[i][k] = __ldcg(po + ((slot(s) + sub) * QUADS + quad + k) * kBM);
                }
            }
            float m2 = M;
#pragma unroll
            for (int i = 0; i < U; ++i) m2 = fmaxf(m2, ml[i].x);
            const float f = M == -CUDART_INF_F ? 0.f : fast_exp2(M - m2);
            M = m2;
            L *= f;
#pragma unroll
            for (int k = 0; k < QB; ++k) {
                o[k].x *= f; o[k].y *= f; o[k].z *= f; o[k].w *= f;
            }
#pragma unroll
            for (int i = 0; i < U; ++i) {
                if (nothing(ml[i].x, ml[i].y)) continue;
                const float g = fast_exp2(ml[i].x - M);
                L = fmaf(g, ml[i].y, L);
#pragma unroll
                for (int k = 0; k < QB; ++k) {
                    if (k < per) {
                        o[k].x = fmaf(g, x[i][k].x, o[k].x);
                        o[k].y = fmaf(g, x[i][k].y, o[k].y);
                        o[k].z = fmaf(g, x[i][k].z, o[k].z);
                        o[k].w = fmaf(g, x[i][k].w, o[k].w);
                    }
                }
            }
        }
        if (shares > 1) {
            top[t] = M;
            len[t] = L;
            part[t] = o[0];
            __syncthreads();
            if (mine != 0) return;
            float m2 = M;
            for (int k = 1; k < shares; ++k) m2 = fmaxf(m2, top[k * span + t]);
            const float f = M == -CUDART_INF_F ? 0.f : fast_exp2(M - m2);
            L *= f;
            o[0].x *= f; o[0].y *= f; o[0].z *= f; o[0].w *= f;
            for (int k = 1; k < shares; ++k) {
                const float mk = top[k * span + t];
                const float lk = len[k * span + t];
                if (nothing(mk, lk)) continue;
                const float g = fast_exp2(mk - m2);
                const float4 x = part[k * span + t];
                L = fmaf(g, lk, L);
                o[0].x = fmaf(g, x.x, o[0].x);
                o[0].y = fmaf(g, x.y, o[0].y);
                o[0].z = fmaf(g, x.z, o[0].z);
                o[0].w = fmaf(g, x.w, o[0].w);
            }
            M = m2;
        }
        if (!live) continue;
        const float inv = 1.f / L;
#pragma unroll
        for (int k = 0; k < QB; ++k)
            if (k < per)
                *reinterpret_cast<uint2*>(a.O + orow * D + (quad + k) * 4) =
                    make_uint2(pack_bf16x2(o[k].x * inv, o[k].y * inv), pack_bf16x2(o[k].z * inv, o[k].w * inv));
        if (quad == 0 && a.LSE != nullptr) a.LSE[orow] = M * kLn2 + logf(L);
    }
}

}  // namespace
}  // namespace sas
