// Per-head RMS norm of queries and keys with the rotary position rotation, in one
// pass over the fused projection, and its gradient.
//
// For a head row x (d elements) at position p, with weight w and r = 1 / sqrt(mean(x^2) + eps):
//   xh = x r,  z = w xh,  y = R_p z,
// where R_p turns each pair (z_a, z_b) by the angle whose cosine and sine the
// tables hold: y_a = z_a c - z_b s, y_b = z_b c + z_a s.  Pair i of the first R
// dims is (i, i + R/2), or (2i, 2i + 1) when interleaved; dims past R pass.
// Gradient: dz = R_p^T dy, dw = sum dz xh, u = w dz, dx = r (u - xh mean(u xh)).
// Everything is in fp32 from the bf16 inputs to the one rounding of the output;
// dw is summed and returned in fp32.
//
// Value rows pass through, so that the fused projection [token][Hq + 2 Hkv][d] is
// read once and leaves in the attention's layouts.
//
// Bound: HBM, and close behind it the issue slots (a row of d = 128 is 256 bytes and
// some 110 instructions of 16 lanes).  So: both kernels are persistent, a warp keeps
// the same heads for all its tokens (their kinds, weights and addresses are then
// fixed), rows stream through a ring in shared memory (cp.async, no registers held
// while they are in flight), and the arithmetic runs on packed fp32 pairs.  Measured:
// 6.4 TB/s forward (127 us for 32768 tokens of 32 + 2 x 8 heads of 128, and as much into
// cache pages), 5.5 TB/s for the gradient (206 to 211 us), where a row is read twice as much
// as written and the waits for shared memory and reductions show.  One or two more
// stages of the rings are slower (158 us forward with three): the warps drift apart and
// DRAM pages are opened more often.
#include <type_traits>

#include <cuda_fp16.h>

#include "serve.h"
#include "serve_ptx.cuh"

namespace sas {
namespace {

constexpr int kWarps = 8;
constexpr int kThreads = kWarps * 32;
constexpr int kStatusBadInput = 1;   // == SAS_ERR_INVALID_ARG

__device__ __forceinline__ uint64_t dup2(float v) { return f32x2(v, v); }
__device__ __forceinline__ float sum2(uint64_t v) {
    float lo, hi;
    f32x2_split(v, lo, hi);
    return lo + hi;
}

// A lane's 8 elements of a head row: two quads in memory (bf16), four fp32 pairs.
struct Quads {
    uint2 a, b;
    __device__ __forceinline__ void load(const bf16* row, int ia, int ib) {
        a = sas::load(reinterpret_cast<const uint2*>(row + ia));
        b = sas::load(reinterpret_cast<const uint2*>(row + ib));
    }
    __device__ __forceinline__ void read(const uint8_t* row, int ia, int ib) {   // shared memory
        a = *reinterpret_cast<const uint2*>(row + 2 * ia);
        b = *reinterpret_cast<const uint2*>(row + 2 * ib);
    }
    __device__ __forceinline__ void store(bf16* row, int ia, int ib) const {
        *reinterpret_cast<uint2*>(row + ia) = a;
        *reinterpret_cast<uint2*>(row + ib) = b;
    }
    __device__ __forceinline__ void unpack(uint64_t (&f)[4]) const {
        const uint32_t w[4] = {a.x, a.y, b.x, b.y};
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = f32x2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
    }
    __device__ __forceinline__ void pack(const uint64_t (&f)[4]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float lo, hi;
            f32x2_split(f[i], lo, hi);
            w[i] = pack_bf16x2(lo, hi);
        }
        a = make_uint2(w[0], w[1]);
        b = make_uint2(w[2], w[3]);
    }
};

// Whether a lane's dims are turned.  The others pass, as they are: a turn by (1, 0) would take a
// NaN or an infinity of one dim to another.
__device__ __forceinline__ bool turned(const RopeArgs& a, int l) { return l < (a.rot >> 3); }

// Where a lane's two quads sit in a row, and its share of the rotation at one
// position.  A lane always holds whole pairs, so the rotation needs no exchange:
// half-split pairs put the second quad R / 2 past the first; interleaved pairs, and
// dims past R, take 8 neighbours.  Either way the lane's four pairs are 4 l .. 4 l + 3.
template <bool INTER>
struct Place {
    int ia, ib;
    __device__ __forceinline__ Place(const RopeArgs& a, int l) {
        const bool split = !INTER && turned(a, l);
        ia = split ? 4 * l : 8 * l;
        ib = split ? 4 * l + (a.rot >> 1) : 8 * l + 4;
    }
};

// The cosines and sines of a token, 16 bytes a lane each, in a ring stage.  Lanes past
// the rotated dims have none.
template <int D>
struct Table {
    static constexpr int BYTES = 2 * (D / 8) * 16;
    __device__ __forceinline__ static void fetch(uint8_t* at, const RopeArgs& a, int pos, int l) {
        if (!turned(a, l)) return;
        const size_t from = static_cast<size_t>(pos) * (a.rot >> 1) + 4 * l;
        cp_async16(at + l * 16, a.cos + from);
        cp_async16(at + BYTES / 2 + l * 16, a.sin + from);
    }
};

// BACK: the transposed rotation (the sine's sign flips).  PART: some lanes' dims pass.  Whole
// rotations have kernels without that choice: at 32768 tokens of 32 + 2 x 8 heads of 128 it
// costs them 2 us (129 against 127 forward, 212 against 209 back).
template <bool INTER, bool BACK, bool PART>
struct Turn {
    uint64_t c[INTER ? 4 : 2], s[INTER ? 4 : 2], t[INTER ? 1 : 2];
    __device__ __forceinline__ Turn(const uint8_t* cos, const uint8_t* sin) {
        const struct { float4 c, s; } g{*reinterpret_cast<const float4*>(cos), *reinterpret_cast<const float4*>(sin)};
        if constexpr (INTER) {   // per pair (c, c) and (-s, s)
            const float cs[4] = {g.c.x, g.c.y, g.c.z, g.c.w}, sn[4] = {g.s.x, g.s.y, g.s.z, g.s.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                c[i] = dup2(cs[i]);
                s[i] = BACK ? f32x2(sn[i], -sn[i]) : f32x2(-sn[i], sn[i]);
            }
        } else {   // first quad: a c + b s', second: b c + a t'
            c[0] = f32x2(g.c.x, g.c.y);
            c[1] = f32x2(g.c.z, g.c.w);
            const uint64_t p0 = f32x2(g.s.x, g.s.y), p1 = f32x2(g.s.z, g.s.w);
            const uint64_t n0 = f32x2(-g.s.x, -g.s.y), n1 = f32x2(-g.s.z, -g.s.w);
            s[0] = BACK ? p0 : n0;
            s[1] = BACK ? p1 : n1;
            t[0] = BACK ? n0 : p0;
            t[1] = BACK ? n1 : p1;
        }
    }
    __device__ __forceinline__ void apply(uint64_t (&z)[4], bool turns) const {
        if constexpr (INTER) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float lo, hi;
                f32x2_split(z[i], lo, hi);
                const uint64_t y = fma_f32x2(f32x2(hi, lo), s[i], mul_f32x2(z[i], c[i]));
                z[i] = !PART || turns ? y : z[i];
            }
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint64_t x = z[i], y = z[i + 2];
                const uint64_t u = fma_f32x2(y, s[i], mul_f32x2(x, c[i])), v = fma_f32x2(x, t[i], mul_f32x2(y, c[i]));
                z[i] = !PART || turns ? u : x;
                z[i + 2] = !PART || turns ? v : y;
            }
        }
    }
};

// kRows: rows of a lane group per token.
template <int D, int kRows>
struct Rows {
    static constexpr int LPR = D / 8, GPW = 32 / LPR, RPU = kRows * GPW;   // lanes a row, groups and rows a warp
    __host__ __device__ __forceinline__ static int parts(const RopeArgs& a) { return (a.Hq + 2 * a.Hkv + RPU - 1) / RPU; }
    // Sum over the lanes of a row (groups may be in different branches).
    __device__ __forceinline__ static float sum(float v, unsigned group) {
#pragma unroll
        for (int o = LPR / 2; o > 0; o >>= 1) v += __shfl_xor_sync(group, v, o);
        return v;
    }
    __device__ __forceinline__ static unsigned group_mask(int g) { return ((1u << LPR) - 1u) << (g * LPR); }
};

// How the warps share the work: a part (RPU neighbouring heads of the fused row) per
// warp, tokens t0, t0 + step, ...  With more parts than warps a warp takes several.
struct Share {
    int part, part_step;
    long long t0, step;
    __device__ __forceinline__ explicit Share(int parts, int block, int blocks) {
        const int warps = blocks * kWarps, w = block * kWarps + warp_id();
        part_step = min(parts, warps);
        part = w % part_step;
        step = warps / part_step;
        t0 = w / part_step;
        if (t0 >= step) part = parts;   // left over: nothing
    }
};

// A token's place: batch row b and index n there.
struct Where {
    long long b;
    int n;
    __device__ __forceinline__ Where(const RopeArgs& a, long long t) {
        b = 0;
        n = static_cast<int>(t);
        if (a.T != a.N) {   // batches: 32-bit division (T <= 2^31)
            const unsigned q = static_cast<unsigned>(t) / static_cast<unsigned>(a.N);
            b = q;
            n = static_cast<int>(static_cast<unsigned>(t) - q * static_cast<unsigned>(a.N));
        }
    }
};

// PAGED: keys and values go to the cache pages that `slots` names and the queries
// to [token][Hq][d]; else all three go to [batch][head][N][d].
constexpr int kFwdRows = 4, kFwdStages = 2, kFwdBlocks = 2;   // blocks: per multiprocessor
template <int D>
constexpr int rope_fwd_unit() { return kFwdRows * 32 * 16 + Table<D>::BYTES; }   // bytes of a token in a warp's ring
template <int D>
constexpr int rope_fwd_smem() { return kWarps * kFwdStages * rope_fwd_unit<D>(); }

// The block-th of `blocks` blocks' share; sm: rope_fwd_smem<D>() bytes.
template <int D, bool INTER, bool PAGED, bool PART>
__device__ __forceinline__ void rope_fwd(const RopeArgs& a, int block, int blocks, uint8_t* sm) {
    constexpr int kRows = kFwdRows;
    using R = Rows<D, kRows>;
    constexpr int UNIT = rope_fwd_unit<D>(), TAB = kRows * 512;
    const int lane = lane_id(), l = lane % R::LPR, g = lane / R::LPR;
    const unsigned group = R::group_mask(g);
    const int H = a.Hq + 2 * a.Hkv, HN = a.Hq + a.Hkv, parts = R::parts(a);
    uint8_t* const ring = sm + warp_id() * kFwdStages * UNIT;
    const int mine = g * (R::LPR * 16);   // the group's row within 512 bytes
    const Place<INTER> pl(a, l);
    const bool turns = turned(a, l);
    const Share sh(parts, block, blocks);
    grid_dep_wait();
    for (int part = sh.part; part < parts; part += sh.part_step) {
        const int h0 = part * R::RPU + g;   // row u of the group is head h0 + u GPW
        bf16* out[kRows];
        Quads w[kRows];
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            const int h = h0 + u * R::GPW;
            const bool isq = h < a.Hq, isv = h >= HN;
            const int hk = isq ? h : (isv ? h - HN : h - a.Hq);
            const long long rows = PAGED ? (isq ? 1 : 64) : a.N;   // rows of a head before the next head's
            out[u] = (isq ? a.Q : (isv ? a.V : a.K)) + hk * rows * D;
            w[u].load(isq ? a.wq : a.wk, pl.ia, pl.ib);
        }
        // the next token to fetch, its position and slot (read a token early)
        long long tf = sh.t0, slot_f = 0, slot = 0, slot1 = 0;
        int pos_f = 0;
        unsigned good = 0;   // per fetched token, the latest in bit 0: it has outputs
        auto locate = [&] {
            if (tf >= a.T) return;
            pos_f = a.pos != nullptr ? load(a.pos + tf) : Where(a, tf).n;
            if constexpr (PAGED) slot_f = load(a.slots + tf);
        };
        auto fetch = [&](int st) {
            good <<= 1;
            if (tf < a.T) {
                uint8_t* const dst = ring + st * UNIT;
                const bf16* const src = a.qkv + tf * a.ld + h0 * D + l * 8;
#pragma unroll
                for (int u = 0; u < kRows; ++u)
                    if (h0 + u * R::GPW < H) cp_async16(dst + u * 512 + mine + l * 16, src + u * R::GPW * D);
                const bool ok = pos_f >= 0 && pos_f < a.max_pos && (!PAGED || (slot_f >= 0 && slot_f < a.n_slots));
                if (ok && g == 0) Table<D>::fetch(dst + TAB, a, pos_f, l);
                if (!ok && !(PAGED && slot_f == -1) && lane == 0) atomicExch(a.status, kStatusBadInput);   // -1: padding
                good |= ok;
            }
            cp_async_commit();
            tf += sh.step;
            locate();
        };
        locate();
        for (int i = 0; i < kFwdStages - 1; ++i) fetch(i);
        // warps come in whole blocks: the last ones may have no token at all
        if (PAGED && sh.t0 < a.T) slot1 = load(a.slots + sh.t0);
        int st = 0;
        for (long long t = sh.t0; t < a.T; t += sh.step) {
            slot = slot1;
            if (PAGED && t + sh.step < a.T) slot1 = load(a.slots + t + sh.step);
            cp_async_wait<kFwdStages - 2>();
            __syncwarp();   // the lanes' copies of this token have landed; the stage refilled next has been read
            fetch(st == 0 ? kFwdStages - 1 : st - 1);
            const uint8_t* const stage = ring + st * UNIT;
            st = st + 1 == kFwdStages ? 0 : st + 1;
            if (!((good >> (kFwdStages - 1)) & 1u)) continue;
            const Turn<INTER, false, PART> turn(stage + TAB + l * 16, stage + TAB + Table<D>::BYTES / 2 + l * 16);
            long long at_q, at_kv;   // the token's offset in Q, and in K and V
            if constexpr (PAGED) {
                at_q = t * a.Hq * D;
                at_kv = ((slot >> 6) * a.Hkv * 64 + (slot & 63)) * D;
            } else {
                const Where at(a, t);
                at_q = (at.b * a.Hq * a.N + at.n) * D;
                at_kv = (at.b * a.Hkv * a.N + at.n) * D;
            }
#pragma unroll
            for (int u = 0; u < kRows; ++u) {
                const int h = h0 + u * R::GPW;
                const uint8_t* const row = stage + u * 512 + mine;
                if (h < HN) {
                    Quads q;
                    uint64_t z[4], wf[4];
                    q.read(row, pl.ia, pl.ib);
                    q.unpack(z);
                    w[u].unpack(wf);
                    uint64_t ss = mul_f32x2(z[0], z[0]);
#pragma unroll
                    for (int i = 1; i < 4; ++i) ss = fma_f32x2(z[i], z[i], ss);
                    const uint64_t r = dup2(rsqrtf(R::sum(sum2(ss), group) * (1.f / D) + a.eps));
#pragma unroll
                    for (int i = 0; i < 4; ++i) z[i] = mul_f32x2(mul_f32x2(z[i], r), wf[i]);
                    turn.apply(z, turns);
                    q.pack(z);
                    q.store(out[u] + (h < a.Hq ? at_q : at_kv), pl.ia, pl.ib);
                } else if (h < H) {   // values pass through
                    *reinterpret_cast<uint4*>(out[u] + at_kv + l * 8) = *reinterpret_cast<const uint4*>(row + l * 16);
                }
            }
        }
        cp_async_wait<0>();
        __syncwarp();
    }
}

template <int D, bool INTER, bool PAGED, bool PART>
__global__ void __launch_bounds__(kThreads, kFwdBlocks) rope_fwd_kernel(RopeArgs a) {
    extern __shared__ __align__(16) uint8_t sm[];
    rope_fwd<D, INTER, PAGED, PART>(a, blockIdx.x, gridDim.x, sm);
}

// A lane keeps its columns of dw in registers, per row of its group, and adds them to
// its warp's sums at the end; a block adds its warps' sums into one row of `part`,
// and the last block to finish adds those in their order: equal inputs give equal
// sums.
//
// Values cost no arithmetic.  Where neighbouring rows would give some warps nothing else,
// which end early, a warp's rows come half from the front of the fused row and half from
// its back (32768 tokens of 32 + 2 x 8 heads: 209 against 216 us; 58701 of 2 + 2 x 2: 52
// against 58), elsewhere in one piece (46113 of 4 + 2 x 1: 51.5 against 53.1).  The forward
// kernel reads its row better in one piece (by 3% at 32768 tokens).
constexpr int kBwdRows = 2, kBwdStages = 3, kBwdBlocks = 2;
template <int D>
constexpr int rope_bwd_unit() { return 2 * kBwdRows * 32 * 16 + Table<D>::BYTES; }
template <int D>
constexpr int rope_bwd_smem() { return kWarps * (kBwdStages * rope_bwd_unit<D>() + 2 * D * 4); }

template <int D, bool INTER, bool PART>
__global__ void __launch_bounds__(kThreads, kBwdBlocks) rope_bwd_kernel(RopeArgs a) {
    constexpr int kRows = kBwdRows;
    using R = Rows<D, kRows>;
    constexpr int UNIT = rope_bwd_unit<D>(), DY = kRows * 512, TAB = 2 * DY;   // rows of x, rows of dy, the table's row
    extern __shared__ __align__(16) uint8_t sm[];
    __shared__ int last;
    const int lane = lane_id(), warp = warp_id(), l = lane % R::LPR, g = lane / R::LPR;
    const unsigned group = R::group_mask(g);
    const int H = a.Hq + 2 * a.Hkv, HN = a.Hq + a.Hkv, parts = R::parts(a);
    const bool spread = (parts - 1) * R::RPU >= HN;
    const int hp = spread ? R::GPW : R::RPU, hs = spread ? parts * R::GPW : R::GPW;   // heads from part to part, row to row
    uint8_t* const ring = sm + warp * kBwdStages * UNIT;
    const int mine = g * (R::LPR * 16);
    float* const sums = reinterpret_cast<float*>(sm + kWarps * kBwdStages * UNIT);   // [kWarps][2 D]
    float* const sum = sums + warp * 2 * D;
    for (int i = lane; i < 2 * D; i += 32) sum[i] = 0.f;
    const Place<INTER> pl(a, l);
    const bool turns = turned(a, l);
    const Share sh(parts, blockIdx.x, gridDim.x);
    grid_dep_wait();
    for (int part = sh.part; part < parts; part += sh.part_step) {
        const int h0 = part * hp + g;   // row u of the group is head h0 + u hs
        const bf16* grad[kRows];
        Quads w[kRows];
        uint64_t acc[kRows][4];
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            const int h = h0 + u * hs;
            const bool isq = h < a.Hq, isv = h >= HN;
            const int hk = isq ? h : (isv ? h - HN : h - a.Hq);
            grad[u] = (isq ? a.Q : (isv ? a.V : a.K)) + static_cast<long long>(hk) * a.N * D + l * 8;
            w[u].load(isq ? a.wq : a.wk, pl.ia, pl.ib);
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[u][i] = 0;
        }
        long long tf = sh.t0;   // the next token to fetch and its position (read a token early)
        int pos_f = 0;
        unsigned good = 0;      // per fetched token, the latest in bit 0: its position is in the tables
        auto locate = [&] {
            if (tf < a.T) pos_f = a.pos != nullptr ? load(a.pos + tf) : Where(a, tf).n;
        };
        auto fetch = [&](int st) {
            good <<= 1;
            if (tf < a.T) {
                const bf16* const src = a.qkv + tf * a.ld + h0 * D + l * 8;
                const Where at(a, tf);
                const long long at_q = (at.b * a.Hq * a.N + at.n) * D, at_kv = (at.b * a.Hkv * a.N + at.n) * D;
                uint8_t* const dst = ring + st * UNIT;
#pragma unroll
                for (int u = 0; u < kRows; ++u) {
                    const int h = h0 + u * hs;
                    if (h < HN) cp_async16(dst + u * 512 + mine + l * 16, src + u * hs * D);
                    if (h < H) cp_async16(dst + DY + u * 512 + mine + l * 16, grad[u] + (h < a.Hq ? at_q : at_kv));
                }
                const bool ok = pos_f >= 0 && pos_f < a.max_pos;
                if (ok && g == 0) Table<D>::fetch(dst + TAB, a, pos_f, l);
                if (!ok && lane == 0) atomicExch(a.status, kStatusBadInput);
                good |= ok;
            }
            cp_async_commit();
            tf += sh.step;
            locate();
        };
        locate();
        for (int i = 0; i < kBwdStages - 1; ++i) fetch(i);
        int st = 0;
        for (long long t = sh.t0; t < a.T; t += sh.step) {
            cp_async_wait<kBwdStages - 2>();
            __syncwarp();   // the lanes' copies of this token have landed; the stage refilled next has been read
            fetch(st == 0 ? kBwdStages - 1 : st - 1);
            const uint8_t* const stage = ring + st * UNIT;
            st = st + 1 == kBwdStages ? 0 : st + 1;
            if (!((good >> (kBwdStages - 1)) & 1u)) continue;
            const Turn<INTER, true, PART> turn(stage + TAB + l * 16, stage + TAB + Table<D>::BYTES / 2 + l * 16);
            bf16* const dst = a.dqkv + t * a.ld_d + h0 * D;
#pragma unroll
            for (int u = 0; u < kRows; ++u) {
                const int h = h0 + u * hs;
                const uint8_t* const row = stage + u * 512 + mine;
                if (h < HN) {
                    Quads q;
                    uint64_t xf[4], z[4], wf[4];
                    q.read(row, pl.ia, pl.ib);
                    q.unpack(xf);
                    q.read(row + DY, pl.ia, pl.ib);
                    q.unpack(z);
                    w[u].unpack(wf);
                    uint64_t ss = mul_f32x2(xf[0], xf[0]);
#pragma unroll
                    for (int i = 1; i < 4; ++i) ss = fma_f32x2(xf[i], xf[i], ss);
                    const uint64_t r = dup2(rsqrtf(R::sum(sum2(ss), group) * (1.f / D) + a.eps));
                    turn.apply(z, turns);
                    uint64_t dot = 0;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        xf[i] = mul_f32x2(xf[i], r);   // xh
                        const uint64_t p = mul_f32x2(z[i], xf[i]);
                        acc[u][i] = add_f32x2(acc[u][i], p);
                        dot = fma_f32x2(p, wf[i], dot);
                    }
                    const uint64_t m = dup2(R::sum(sum2(dot), group) * (-1.f / D));
#pragma unroll
                    for (int i = 0; i < 4; ++i) z[i] = mul_f32x2(r, fma_f32x2(m, xf[i], mul_f32x2(z[i], wf[i])));
                    q.pack(z);
                    q.store(dst + u * hs * D, pl.ia, pl.ib);
                } else if (h < H) {   // values pass through
                    *reinterpret_cast<uint4*>(dst + u * hs * D + l * 8) = *reinterpret_cast<const uint4*>(row + DY + l * 16);
                }
            }
        }
        cp_async_wait<0>();
        // the part's sums, one lane group after the other
        for (int gg = 0; gg < R::GPW; ++gg) {
            __syncwarp();
            if (g != gg) continue;
#pragma unroll
            for (int u = 0; u < kRows; ++u) {
                const int h = h0 + u * hs;
                if (h >= HN) continue;
                float* const col = sum + (h < a.Hq ? 0 : D);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float lo, hi;
                    f32x2_split(acc[u][i], lo, hi);
                    const int at = i < 2 ? pl.ia + 2 * i : pl.ib + 2 * (i - 2);
                    col[at] += lo;
                    col[at + 1] += hi;
                }
            }
        }
        __syncwarp();
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * D; i += kThreads) {
        float v = 0.f;
#pragma unroll
        for (int k = 0; k < kWarps; ++k) v += sums[k * 2 * D + i];
        a.part[static_cast<size_t>(blockIdx.x) * 2 * D + i] = v;
    }
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) last = atomicAdd(a.counter, 1) == static_cast<int>(gridDim.x) - 1;
    __syncthreads();
    if (!last) return;
    __threadfence();
    if (threadIdx.x == 0) *a.counter = 0;   // zero again for the next launch
    constexpr int QUADS = 2 * D / 4, SL = kThreads / QUADS;   // 16-byte columns, slices of the rows
    const int qd = threadIdx.x % QUADS, sl = threadIdx.x / QUADS;
    float4 v4 = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 16
    for (int i = sl; i < static_cast<int>(gridDim.x); i += SL) {
        const float4 v = __ldcg(reinterpret_cast<const float4*>(a.part + static_cast<size_t>(i) * 2 * D) + qd);
        v4.x += v.x; v4.y += v.y; v4.z += v.z; v4.w += v.w;
    }
    float4* const slices = reinterpret_cast<float4*>(sm);   // the rings are drained
    slices[sl * QUADS + qd] = v4;
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * D; i += kThreads) {
        float v = 0.f;
#pragma unroll
        for (int k = 0; k < SL; ++k) v += reinterpret_cast<const float*>(slices)[k * 2 * D + i];
        (i < D ? a.dwq : a.dwk)[i < D ? i : i - D] = v;
    }
}

// Blocks for all (token, part) pairs at `tokens` a warp, at most `most` (the kernels are
// persistent).
template <int D, int kRows>
int blocks_for(const RopeArgs& a, int most, int tokens) {
    const long long need = (a.T * Rows<D, kRows>::parts(a) + kWarps * tokens - 1) / (kWarps * tokens);
    return static_cast<int>(need < most ? need : most);
}

template <int D, bool INTER, bool PAGED, bool PART>
cudaError_t launch_fwd(const RopeArgs& a, const KernelEnv& env) {
    const cudaError_t e = ensure_smem_attr(reinterpret_cast<const void*>(rope_fwd_kernel<D, INTER, PAGED, PART>), rope_fwd_smem<D>(), true);
    if (e != cudaSuccess) return e;
    return launch_early(rope_fwd_kernel<D, INTER, PAGED, PART>, dim3(blocks_for<D, kFwdRows>(a, kFwdBlocks * device_sm_count(), 1)), kThreads,
                        rope_fwd_smem<D>(), env.stream, a);
}

template <int D, bool INTER, bool PART>
cudaError_t launch_bwd(const RopeArgs& a, const KernelEnv& env) {
    const cudaError_t e = ensure_smem_attr(reinterpret_cast<const void*>(rope_bwd_kernel<D, INTER, PART>), rope_bwd_smem<D>(), true);
    if (e != cudaSuccess) return e;
    return launch_early(rope_bwd_kernel<D, INTER, PART>, dim3(blocks_for<D, kBwdRows>(a, rope_bwd_max_blocks(), 4)), kThreads,
                        rope_bwd_smem<D>(), env.stream, a);
}

template <int D, bool INTER>
cudaError_t launch_any_fwd(const RopeArgs& a, const KernelEnv& env) {
    if (a.rot < D) return a.slots != nullptr ? launch_fwd<D, INTER, true, true>(a, env) : launch_fwd<D, INTER, false, true>(a, env);
    return a.slots != nullptr ? launch_fwd<D, INTER, true, false>(a, env) : launch_fwd<D, INTER, false, false>(a, env);
}

template <int D, bool INTER>
cudaError_t launch_any_bwd(const RopeArgs& a, const KernelEnv& env) {
    return a.rot < D ? launch_bwd<D, INTER, true>(a, env) : launch_bwd<D, INTER, false>(a, env);
}

// ------------------------------------------------------------------ into pages of 8 bits
//
// A page of a KV head holds e4m3 numbers under one scale, a power of two s with max |x| <=
// 448 s.  A page whose row 0 is new starts a scale; otherwise the scale only grows, and where
// it does the rows that stay are rounded again under the larger one.  So the maximum of a
// page's new rows has to be known before any of them is written: the tokens of a page stand
// next to each other, and a run of them of one page and head is one piece of work, whose rows
// wait in registers.  A block has the runs of a head that begin in a window of neighbouring
// tokens: the ones of up to 8 tokens a warp each, the longer ones all together, 8 tokens a warp.
//
// Bound: HBM, a read of the fused rows and a write of the queries and of half as many bytes for
// keys and values.  15232 tokens of 32 + 2 x 8 heads of 128 take 81.5 us (4.3 TB/s, 64%): the
// queries' blocks 41, at HBM's rate, the windows' as long, as a block waits for slots, rows,
// tables, the joint maximum and its stores one after the other, with two blocks of 118 registers
// a thread at a time (106 to 118 by form; three, with their rows in local memory, 100 us).  96
// tokens: 6.1 us in a captured row of calls, 10 from the host.
constexpr int kRunRows = 8;                       // of a warp
constexpr int kMaxWindow = 64;                    // tokens; runs have 64 at most
static_assert(kWarps * kRunRows >= 64, "a block's longest run is a page");

// Least power of two s with amax <= 448 s, 448 = 1.75 * 2^8, within 2^-64 .. 2^120.
__device__ __forceinline__ float page_scale(float amax) {
    const uint32_t b = __float_as_uint(amax);
    int k = static_cast<int>(b >> 23) - 127 - 8 + ((b & 0x7fffffu) > 0x600000u);
    k = max(-64, min(120, k));
    return __uint_as_float(static_cast<uint32_t>(k + 127) << 23);
}
// Two numbers as e4m3, to nearest; NaN stays, infinities become the largest number.
__device__ __forceinline__ uint32_t pack_e4m3x2(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float finite_or(float x, float other) { return fabsf(x) < __uint_as_float(0x7f800000u) ? x : other; }
// Four numbers times inv; NaN (there is no infinity) for what is not finite, where any may be.
__device__ __forceinline__ uint32_t pack_quad(uint64_t a, uint64_t b, float inv, bool odd) {
    const uint64_t i2 = dup2(inv);
    float x0, x1, x2, x3;
    f32x2_split(mul_f32x2(a, i2), x0, x1);
    f32x2_split(mul_f32x2(b, i2), x2, x3);
    if (odd) {
        const float nan = __uint_as_float(0x7fc00000u);
        x0 = finite_or(x0, nan);
        x1 = finite_or(x1, nan);
        x2 = finite_or(x2, nan);
        x3 = finite_or(x3, nan);
    }
    return pack_e4m3x2(x0, x1) | (pack_e4m3x2(x2, x3) << 16);
}
// Four numbers under a larger scale.
__device__ __forceinline__ uint32_t shrink_quad(uint32_t w, float ratio) {
    uint32_t out = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t f;
        asm("{\n\t.reg .b16 x;\n\tcvt.u16.u32 x, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, x;\n\t}" : "=r"(f) : "r"((w >> (16 * h)) & 0xffffu));
        const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&f));
        out |= pack_e4m3x2(v.x * ratio, v.y * ratio) << (16 * h);
    }
    return out;
}

// A run as its warps know it: tokens first .. first + n - 1 of the window.
struct Run {
    int first, n, page;
    unsigned lo, hi;   // its rows of the page
};

__device__ __forceinline__ void prefetch_line(const void* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p) : "memory"); }

template <int D, bool INTER>
__device__ __forceinline__ void append8_window(const RopeArgs& a, const Cache8& c, int window, unsigned block) {
    using R = Rows<D, 1>;
    constexpr int P = kRunRows / R::GPW;   // passes: a group's rows
    __shared__ int pages[kMaxWindow + 65], rows[kMaxWindow + 64], spots[kMaxWindow + 64];   // pages: of the token before, too
    __shared__ float tops[2][2][kWarps];
    const int lane = lane_id(), warp = warp_id(), l = lane % R::LPR, g = lane / R::LPR;
    const unsigned at_window = block / static_cast<unsigned>(a.Hkv);
    const int head = static_cast<int>(block - at_window * a.Hkv);
    const long long t0 = static_cast<long long>(at_window) * window;
    const Place<INTER> pl(a, l);
    const bool turns = turned(a, l);
    grid_dep_wait();
    // what the window's tokens have for the head is on its way while their slots are read (85.5 -> 81.5 us)
    if (static_cast<int>(threadIdx.x) < 4 * window && t0 + (threadIdx.x >> 2) < a.T) {
        const int h = a.Hq + head + (threadIdx.x & 1) * a.Hkv;
        prefetch_line(a.qkv + (t0 + (threadIdx.x >> 2)) * a.ld + static_cast<long long>(h) * D + (threadIdx.x >> 1 & 1) * (D / 2));
    }
    Quads w;
    w.load(a.wk, pl.ia, pl.ib);
    // the window's tokens, and as many after it as its last run may have: page (-1: none), row of the page (64: no
    // place in the tables) and position
    for (int i = threadIdx.x; i < window + 65; i += kThreads) {
        const long long t = t0 + i - 1;
        const long long slot = t >= 0 && t < a.T ? load(a.slots + t) : -1;
        const bool there = slot >= 0 && slot < a.n_slots;
        pages[i] = there ? static_cast<int>(slot >> 6) : -1;
        if (i == 0) continue;
        const int p = t < a.T ? load(a.pos + t) : 0;
        const bool placed = p >= 0 && p < a.max_pos;
        rows[i - 1] = placed ? static_cast<int>(slot & 63) : 64;
        spots[i - 1] = p;
        // slots that name no row of the cache (-1: padding), positions outside the tables
        if (head == 0 && i <= window && ((!there && slot != -1) || (there && !placed))) atomicExch(a.status, kStatusBadInput);
    }
    __syncthreads();
    // The warp's tokens i0 .. i0 + 7 of a run; JOINT: with the block's other warps.
    int turn_of = 0;
    auto work = [&](const Run& run, int i0, auto joint) {
        constexpr bool JOINT = decltype(joint)::value;
        const size_t at_scale = static_cast<size_t>(run.page) * a.Hkv + head;
        const float old_k = load(c.k_scale + at_scale), old_v = load(c.v_scale + at_scale);
        Quads kq[P];
        uint4 v[P];
        int row[P];
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int i = i0 + p * R::GPW + g;
            row[p] = i < run.n ? rows[run.first + i] : 64;
            kq[p].a = kq[p].b = make_uint2(0, 0);
            v[p] = make_uint4(0, 0, 0, 0);
            if (row[p] < 64) {
                const bf16* const src = a.qkv + (t0 + run.first + i) * a.ld + static_cast<long long>(a.Hq + head) * D;
                kq[p].load(src, pl.ia, pl.ib);
                v[p] = load(reinterpret_cast<const uint4*>(src + static_cast<long long>(a.Hkv) * D + l * 8));
            }
        }
        uint64_t y[P][4];
#pragma unroll
        for (int p = 0; p < P; ++p) {
            uint64_t wf[4];
            kq[p].unpack(y[p]);
            w.unpack(wf);
            uint64_t ss = mul_f32x2(y[p][0], y[p][0]);
#pragma unroll
            for (int i = 1; i < 4; ++i) ss = fma_f32x2(y[p][i], y[p][i], ss);
            const uint64_t r = dup2(rsqrtf(R::sum(sum2(ss), 0xffffffffu) * (1.f / D) + a.eps));
#pragma unroll
            for (int i = 0; i < 4; ++i) y[p][i] = mul_f32x2(mul_f32x2(y[p][i], r), wf[i]);
            if (row[p] < 64) {
                if (turns) {
                    const size_t from = static_cast<size_t>(spots[run.first + i0 + p * R::GPW + g]) * (a.rot >> 1) + 4 * l;
                    const Turn<INTER, false, false> turn(reinterpret_cast<const uint8_t*>(a.cos + from),
                                                         reinterpret_cast<const uint8_t*>(a.sin + from));
                    turn.apply(y[p], true);
                }
            }
        }
        auto value = [&](int p, uint64_t (&f)[4]) {
            Quads q;
            q.a = make_uint2(v[p].x, v[p].y);
            q.b = make_uint2(v[p].z, v[p].w);
            q.unpack(f);
        };
        // The run's largest numbers: infinities among them, and where there are, without what is not finite (which
        // has no say in the scale).  Maxima pass over NaN.
        float top_k, top_v;
        auto largest = [&](bool finite) {
            top_k = top_v = 0.f;
#pragma unroll
            for (int p = 0; p < P; ++p) {
                if (row[p] == 64) continue;
                uint64_t f[4];
                value(p, f);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float a0, a1, b0, b1;
                    f32x2_split(y[p][i], a0, a1);
                    f32x2_split(f[i], b0, b1);
                    if (finite) {
                        a0 = finite_or(a0, 0.f);
                        a1 = finite_or(a1, 0.f);
                        b0 = finite_or(b0, 0.f);
                        b1 = finite_or(b1, 0.f);
                    }
                    top_k = max3f(top_k, fabsf(a0), fabsf(a1));
                    top_v = max3f(top_v, fabsf(b0), fabsf(b1));
                }
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                top_k = fmaxf(top_k, __shfl_xor_sync(0xffffffffu, top_k, o));
                top_v = fmaxf(top_v, __shfl_xor_sync(0xffffffffu, top_v, o));
            }
            if constexpr (JOINT) {
                if (lane == 0) {
                    tops[turn_of][0][warp] = top_k;
                    tops[turn_of][1][warp] = top_v;
                }
                __syncthreads();   // and the old scales have been read
#pragma unroll
                for (int i = 0; i < kWarps; ++i) {
                    top_k = fmaxf(top_k, tops[turn_of][0][i]);
                    top_v = fmaxf(top_v, tops[turn_of][1][i]);
                }
                turn_of ^= 1;      // the next maxima do not wait for these to be read
            }
        };
        largest(false);
        const bool odd = fmaxf(top_k, top_v) == __uint_as_float(0x7f800000u);
        if (odd) largest(true);
        __syncwarp();
        const bool fresh = (run.lo & 1u) != 0;
        const float sk = fresh ? page_scale(top_k) : fmaxf(old_k, page_scale(top_k));
        const float sv = fresh ? page_scale(top_v) : fmaxf(old_v, page_scale(top_v));
        if (lane == 0 && (!JOINT || warp == 0)) {
            c.k_scale[at_scale] = sk;
            c.v_scale[at_scale] = sv;
        }
        const size_t base = at_scale * (64 * D);
        const float ik = 1.f / sk, iv = 1.f / sv;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            if (row[p] == 64) continue;
            uint8_t* const k8 = c.K + base + row[p] * D;
            *reinterpret_cast<uint32_t*>(k8 + pl.ia) = pack_quad(y[p][0], y[p][1], ik, odd);
            *reinterpret_cast<uint32_t*>(k8 + pl.ib) = pack_quad(y[p][2], y[p][3], ik, odd);
            uint64_t vf[4];
            value(p, vf);
            *reinterpret_cast<uint2*>(c.V + base + row[p] * D + l * 8) =
                make_uint2(pack_quad(vf[0], vf[1], iv, odd), pack_quad(vf[2], vf[3], iv, odd));
        }
        // rows that stay, under a scale that grew
        auto shrink = [&](uint8_t* page8, float ratio) {
            constexpr int CH = D / 16;   // 16-byte chunks of a row
            for (int i = JOINT ? static_cast<int>(threadIdx.x) : lane; i < 64 * CH; i += JOINT ? kThreads : 32) {
                const int r = i / CH;
                if (((r < 32 ? run.lo >> r : run.hi >> (r - 32)) & 1u) != 0) continue;
                uint4* const p = reinterpret_cast<uint4*>(page8) + i;
                const uint4 x = load(p);
                *p = make_uint4(shrink_quad(x.x, ratio), shrink_quad(x.y, ratio), shrink_quad(x.z, ratio), shrink_quad(x.w, ratio));
            }
        };
        if (!fresh && sk > old_k) shrink(c.K + base, old_k / sk);
        if (!fresh && sv > old_v) shrink(c.V + base, old_v / sv);
    };
    // The runs that begin in the window, in every warp.
    unsigned begins[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int i = h * 32 + lane;
        begins[h] = __ballot_sync(0xffffffffu, i < window && pages[i + 1] >= 0 && pages[i] != pages[i + 1]);
    }
    auto find = [&](int first) {
        Run run;
        run.first = first;
        run.page = pages[first + 1];
        const unsigned m0 = __ballot_sync(0xffffffffu, pages[first + 1 + lane] == run.page);
        const unsigned m1 = __ballot_sync(0xffffffffu, pages[first + 33 + lane] == run.page);
        run.n = ~m0 != 0 ? __ffs(~m0) - 1 : 32 + (~m1 != 0 ? __ffs(~m1) - 1 : 32);
        const int r0 = lane < run.n ? rows[first + lane] : 64, r1 = lane + 32 < run.n ? rows[first + 32 + lane] : 64;
        run.lo = __reduce_or_sync(0xffffffffu, (r0 < 32 ? 1u << r0 : 0u) | (r1 < 32 ? 1u << r1 : 0u));
        run.hi = __reduce_or_sync(0xffffffffu, (r0 >= 32 && r0 < 64 ? 1u << (r0 - 32) : 0u) | (r1 >= 32 && r1 < 64 ? 1u << (r1 - 32) : 0u));
        return run;
    };
    int k = 0;
    for (int h = 0; h < 2; ++h) {
        for (unsigned m = begins[h]; m != 0; m &= m - 1, ++k) {
            const Run run = find(h * 32 + __ffs(m) - 1);
            if ((run.lo | run.hi) == 0) continue;   // no token of it has a place
            if (run.n > kRunRows) work(run, warp * kRunRows, std::true_type());
            else if (k % kWarps == warp) work(run, 0, std::false_type());
        }
    }
}

// One grid for both: first the blocks of the queries, which are rows of the fused projection's first heads (q: without
// the others), then the windows, which take their places as they end.  Two launches take 12.1 us instead of 10.0 where
// the host is the limit (96 tokens); taking turns, so that a multiprocessor has both kinds at a time, 96 to 134 us
// instead of 85 at 15232 tokens of 32 + 2 x 8 heads of 128: the queries' rows come slower than one after the other.
template <int D, bool INTER, bool PART>
__global__ void __launch_bounds__(kThreads, 2) append8_kernel(RopeArgs a, RopeArgs q, Cache8 c, int window, unsigned q_blocks) {
    extern __shared__ __align__(16) uint8_t sm[];
    if (blockIdx.x < q_blocks) rope_fwd<D, INTER, true, PART>(q, blockIdx.x, q_blocks, sm);
    else append8_window<D, INTER>(a, c, window, blockIdx.x - q_blocks);
}

// Tokens of a window: as few as give every warp a token, more where there are blocks enough
// (eight a multiprocessor: an empty window costs a block 2 us).
int append8_tokens(const RopeArgs& a) {
    const long long w = a.T * a.Hkv / (8LL * device_sm_count());
    return w < kWarps ? kWarps : (w > kMaxWindow ? kMaxWindow : static_cast<int>(w));
}

template <int D, bool INTER, bool PART>
cudaError_t launch_append8(const RopeArgs& a, const Cache8& c, const KernelEnv& env) {
    const void* const kernel = reinterpret_cast<const void*>(append8_kernel<D, INTER, PART>);
    const cudaError_t e = ensure_smem_attr(kernel, rope_fwd_smem<D>(), true);
    if (e != cudaSuccess) return e;
    RopeArgs q = a;
    q.Hkv = 0;
    const int window = append8_tokens(a);
    const unsigned kv_blocks = static_cast<unsigned>((a.T + window - 1) / window * a.Hkv);
    const unsigned q_blocks = static_cast<unsigned>(blocks_for<D, kFwdRows>(q, kFwdBlocks * device_sm_count(), 1));
    return launch_early(append8_kernel<D, INTER, PART>, dim3(kv_blocks + q_blocks), kThreads, rope_fwd_smem<D>(), env.stream, a, q, c, window, q_blocks);
}

template <int D>
cudaError_t launch_append8(const RopeArgs& a, const Cache8& c, const KernelEnv& env) {
    if (a.rot < D) return a.interleaved ? launch_append8<D, true, true>(a, c, env) : launch_append8<D, false, true>(a, c, env);
    return a.interleaved ? launch_append8<D, true, false>(a, c, env) : launch_append8<D, false, false>(a, c, env);
}

template <int D>
cudaError_t prepare_fwd() {
    const void* kernels[] = {reinterpret_cast<const void*>(rope_fwd_kernel<D, true, true, true>),
                             reinterpret_cast<const void*>(rope_fwd_kernel<D, true, true, false>),
                             reinterpret_cast<const void*>(rope_fwd_kernel<D, false, true, true>),
                             reinterpret_cast<const void*>(rope_fwd_kernel<D, false, true, false>),
                             reinterpret_cast<const void*>(append8_kernel<D, true, true>),
                             reinterpret_cast<const void*>(append8_kernel<D, true, false>),
                             reinterpret_cast<const void*>(append8_kernel<D, false, true>),
                             reinterpret_cast<const void*>(append8_kernel<D, false, false>)};
    cudaError_t e = cudaSuccess;
    for (const void* k : kernels)
        if (e == cudaSuccess) e = ensure_smem_attr(k, rope_fwd_smem<D>(), true);
    return e;
}

}  // namespace

const char* rope_check(int rot, int interleaved, int max_pos, float eps, long long heads, int d, long long ld) {
    if (rot < 16 || rot > d || rot % 16 != 0) return "rot must be a multiple of 16 from 16 to d";
    if (interleaved != 0 && interleaved != 1) return "interleaved must be 0 or 1";
    if (max_pos < 1) return "max_pos must be positive";
    if (heads * d > (1 << 30)) return "a token's heads must not exceed 2^30 elements";
    if (!(eps >= 0.f) || eps > 3.0e38f) return "eps must be finite and not negative";
    if (ld < heads * d || ld % 8 != 0) return "a token's row stride must hold all its heads and be a multiple of 8";
    return nullptr;
}

// Tokens are counted in 32 bits where a batch row is found by division.
bool rope_supported(const RopeArgs& a) { return a.T <= 0x7fffffffLL; }

bool append8_supported(const RopeArgs& a) { return (a.T + kWarps - 1) / kWarps * a.Hkv <= 0x70000000LL; }

int rope_bwd_max_blocks() { return kBwdBlocks * device_sm_count(); }   // all resident

cudaError_t rope_paged_prepare(int d) {
    cudaError_t e = d == 128 ? prepare_fwd<128>() : prepare_fwd<64>();
    return e;
}

cudaError_t launch_rope_fwd(const RopeArgs& a, int d, const KernelEnv& env) {
    if (d == 128) return a.interleaved ? launch_any_fwd<128, true>(a, env) : launch_any_fwd<128, false>(a, env);
    if (d == 64) return a.interleaved ? launch_any_fwd<64, true>(a, env) : launch_any_fwd<64, false>(a, env);
    return cudaErrorInvalidValue;
}

cudaError_t launch_append8(const RopeArgs& a, const Cache8& c, int d, const KernelEnv& env) {
    return d == 128 ? launch_append8<128>(a, c, env) : launch_append8<64>(a, c, env);
}

cudaError_t launch_rope_bwd(const RopeArgs& a, int d, const KernelEnv& env) {
    if (d == 128) return a.interleaved ? launch_any_bwd<128, true>(a, env) : launch_any_bwd<128, false>(a, env);
    if (d == 64) return a.interleaved ? launch_any_bwd<64, true>(a, env) : launch_any_bwd<64, false>(a, env);
    return cudaErrorInvalidValue;
}

}  // namespace sas
