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
// Bound: HBM.  A row is a group of d / 8 lanes with 8 elements each; a warp takes
// kRows rows per group of one token, all in flight before any is used, and reads the
// table's row once.
#include "internal.h"
#include "ptx.cuh"

namespace sas {
namespace {

constexpr int kWarps = 8;
constexpr int kThreads = kWarps * 32;
constexpr int kRows = 4;          // rows in flight per lane group
constexpr int kStatusBadInput = 1;   // == SAS_ERR_INVALID_ARG

// A lane's 8 elements of a head row, as two quads (bf16 in memory).
struct Quads {
    uint2 a, b;
    __device__ __forceinline__ void load(const bf16* row, int ia, int ib) {
        a = __ldg(reinterpret_cast<const uint2*>(row + ia));
        b = __ldg(reinterpret_cast<const uint2*>(row + ib));
    }
    __device__ __forceinline__ void read(const uint8_t* row, int ia, int ib) {   // shared memory
        a = *reinterpret_cast<const uint2*>(row + 2 * ia);
        b = *reinterpret_cast<const uint2*>(row + 2 * ib);
    }
    __device__ __forceinline__ void store(bf16* row, int ia, int ib) const {
        *reinterpret_cast<uint2*>(row + ia) = a;
        *reinterpret_cast<uint2*>(row + ib) = b;
    }
    __device__ __forceinline__ void unpack(float (&f)[8]) const {
        const uint32_t w[4] = {a.x, a.y, b.x, b.y};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    __device__ __forceinline__ void pack(const float (&f)[8]) {
        a = make_uint2(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]));
        b = make_uint2(pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
    }
};

// Sum over the LPR lanes of a row.
template <int LPR>
__device__ __forceinline__ float row_sum(float v) {
#pragma unroll
    for (int o = LPR / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// Where a lane's two quads sit in a row, and its share of the rotation at one
// position.  A lane always holds whole pairs, so the rotation needs no exchange:
// half-split pairs put the second quad R / 2 past the first; interleaved pairs, and
// dims past R, take 8 neighbours.  Either way the lane's four pairs are 4 l .. 4 l + 3.
template <bool INTER>
struct Turn {
    int ia, ib;
    float c[4], s[4];

    __device__ __forceinline__ void place(const RopeArgs& a, int l) {
        const bool split = !INTER && l < (a.rot >> 3);
        ia = split ? 4 * l : 8 * l;
        ib = split ? 4 * l + (a.rot >> 1) : 8 * l + 4;
    }
    __device__ __forceinline__ void load(const RopeArgs& a, int pos, int l) {
        float4 cv = make_float4(1.f, 1.f, 1.f, 1.f), sv = make_float4(0.f, 0.f, 0.f, 0.f);
        if (l < (a.rot >> 3)) {
            const size_t at = static_cast<size_t>(pos) * (a.rot >> 1) + 4 * l;
            cv = __ldg(reinterpret_cast<const float4*>(a.cos + at));
            sv = __ldg(reinterpret_cast<const float4*>(a.sin + at));
        }
        c[0] = cv.x; c[1] = cv.y; c[2] = cv.z; c[3] = cv.w;
        s[0] = sv.x; s[1] = sv.y; s[2] = sv.z; s[3] = sv.w;
    }
    // BACK: the transposed rotation (the sine's sign flips).
    template <bool BACK>
    __device__ __forceinline__ void apply(float (&z)[8]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int p = INTER ? 2 * i : i, q = INTER ? 2 * i + 1 : i + 4;
            const float za = z[p], zb = z[q], sn = BACK ? -s[i] : s[i];
            z[p] = fmaf(-zb, sn, za * c[i]);
            z[q] = fmaf(za, sn, zb * c[i]);
        }
    }
};

// A warp's unit: RPU = kRows rows per lane group of one token, any kinds (queries,
// keys, values).  Row u of group g is head part * RPU + u * groups + g, so that one
// load of the warp covers neighbouring rows.
template <int D>
struct Unit {
    static constexpr int LPR = D / 8, GPW = 32 / LPR, RPU = kRows * GPW;
    __host__ __device__ __forceinline__ static int parts(const RopeArgs& a) { return (a.Hq + 2 * a.Hkv + RPU - 1) / RPU; }
    unsigned t, b, n;   // token, its batch row, its index there
    int h0;             // the group's first head
    __device__ __forceinline__ Unit(const RopeArgs& a, unsigned unit, int parts, int g) {
        t = unit / parts;
        h0 = (unit - t * parts) * RPU + g;
        b = t / static_cast<unsigned>(a.N);
        n = t - b * a.N;
    }
    __device__ __forceinline__ int head(int u) const { return h0 + u * GPW; }
};

// PAGED: keys and values go to the cache pages that `slots` names and the queries
// to [token][Hq][d]; else all three go to [batch][head][N][d].
template <int D, bool INTER, bool PAGED>
__global__ void __launch_bounds__(kThreads) rope_fwd_kernel(RopeArgs a, unsigned units) {
    using U = Unit<D>;
    const unsigned unit = blockIdx.x * kWarps + warp_id();
    if (unit >= units) return;
    const int lane = lane_id(), l = lane % U::LPR;
    const U w(a, unit, U::parts(a), lane / U::LPR);
    const int H = a.Hq + 2 * a.Hkv;
    Turn<INTER> turn;
    turn.place(a, l);
    Quads x[kRows];
    const bf16* const xrow = a.qkv + static_cast<long long>(w.t) * a.ld;
#pragma unroll
    for (int u = 0; u < kRows; ++u) x[u].load(xrow + min(w.head(u), H - 1) * D, turn.ia, turn.ib);   // past the last: unused
    const int pos = a.pos != nullptr ? __ldg(a.pos + w.t) : static_cast<int>(w.n);
    long long slot = 0;
    if constexpr (PAGED) {
        slot = __ldg(a.slots + w.t);
        if (slot == -1) return;   // padding
    }
    if (pos < 0 || pos >= a.max_pos || (PAGED && (slot < 0 || slot >= a.n_slots))) {
        if (lane == 0) atomicExch(a.status, kStatusBadInput);
        return;
    }
    turn.load(a, pos, l);
    Quads wq, wk;
    wq.load(a.wq, turn.ia, turn.ib);
    wk.load(a.wk, turn.ia, turn.ib);
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
        const int h = w.head(u);
        const bool isq = h < a.Hq, isv = h >= a.Hq + a.Hkv;
        float z[8], wf[8];
        x[u].unpack(z);
        (isq ? wq : wk).unpack(wf);
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fmaf(z[e], z[e], ss);
        const float r = rsqrtf(row_sum<U::LPR>(ss) * (1.f / D) + a.eps);
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] = z[e] * r * wf[e];
        turn.template apply<false>(z);
        if (h >= H) continue;
        if (!isv) x[u].pack(z);   // values pass through
        const int hk = isq ? h : (isv ? h - a.Hq - a.Hkv : h - a.Hq);
        bf16* dst;
        if constexpr (PAGED)
            dst = isq ? a.Q + (static_cast<size_t>(w.t) * a.Hq + hk) * D
                      : (isv ? a.V : a.K) + ((static_cast<size_t>(slot >> 6) * a.Hkv + hk) * 64 + (slot & 63)) * D;
        else
            dst = (isq ? a.Q : (isv ? a.V : a.K)) + ((static_cast<size_t>(w.b) * (isq ? a.Hq : a.Hkv) + hk) * a.N + w.n) * D;
        x[u].store(dst, turn.ia, turn.ib);
    }
}

// Persistent.  A warp streams its units through its own ring in shared memory
// (cp.async of 16 bytes a lane, kStages - 1 units ahead, no registers held) and keeps
// its lanes' columns of dwq and dwk in registers.  A block adds its warps' sums into
// one row of `part`, and the last block to finish adds those in their order: equal
// inputs give equal sums.
constexpr int kStages = 3;
template <int D>
constexpr int rope_bwd_smem() { return kWarps * (kStages * 2 * kRows * 32 * 16 + 2 * D * 4); }

template <int D, bool INTER>
__global__ void __launch_bounds__(kThreads, 2) rope_bwd_kernel(RopeArgs a, unsigned units) {
    using U = Unit<D>;
    constexpr int LPR = U::LPR;
    constexpr int UNIT = 2 * kRows * 32 * 16;   // bytes: kRows rows of x and of dy per group
    extern __shared__ __align__(16) uint8_t sm[];
    __shared__ int last;
    const int lane = lane_id(), warp = warp_id(), l = lane % LPR, g = lane / LPR;
    const int H = a.Hq + 2 * a.Hkv, HN = a.Hq + a.Hkv, parts = U::parts(a);
    uint8_t* const ring = sm + warp * kStages * UNIT;
    float* const sums = reinterpret_cast<float*>(sm + kWarps * kStages * UNIT);   // [kWarps][2 D]
    const unsigned step = gridDim.x * kWarps;
    unsigned long long next = blockIdx.x * kWarps + warp;

    // row u of the lane's group, x (0) or dy (1), in stage st
    auto slot = [&](int st, int which, int u) { return ring + st * UNIT + ((which * kRows + u) * 32 + g * LPR) * 16; };
    auto fetch = [&](int st) {
        if (next < units) {
            const U w(a, static_cast<unsigned>(next), parts, g);
#pragma unroll
            for (int u = 0; u < kRows; ++u) {
                const int h = w.head(u);
                if (h < H) {
                    const bool isq = h < a.Hq, isv = h >= HN;
                    const int hk = isq ? h : (isv ? h - HN : h - a.Hq);
                    if (!isv) cp_async16(slot(st, 0, u) + l * 16, a.qkv + static_cast<long long>(w.t) * a.ld + h * D + l * 8);
                    cp_async16(slot(st, 1, u) + l * 16,
                               (isq ? a.Q : (isv ? a.V : a.K)) +
                                   ((static_cast<size_t>(w.b) * (isq ? a.Hq : a.Hkv) + hk) * a.N + w.n) * D + l * 8);
                }
            }
        }
        cp_async_commit();
        next += step;
    };
    for (int i = 0; i < kStages - 1; ++i) fetch(i);

    Turn<INTER> turn;
    turn.place(a, l);
    Quads wq, wk;
    wq.load(a.wq, turn.ia, turn.ib);
    wk.load(a.wk, turn.ia, turn.ib);
    float aq[8], ak[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) aq[e] = ak[e] = 0.f;
    int st = 0;
    for (unsigned long long unit = blockIdx.x * kWarps + warp; unit < units; unit += step) {
        const U w(a, static_cast<unsigned>(unit), parts, g);
        const int pos = a.pos != nullptr ? __ldg(a.pos + w.t) : static_cast<int>(w.n);
        const bool ok = pos >= 0 && pos < a.max_pos;
        if (ok) turn.load(a, pos, l);
        else if (lane == 0) atomicExch(a.status, kStatusBadInput);
        cp_async_wait<kStages - 2>();
        __syncwarp();   // the lanes' copies of this unit have landed; the stage refilled next has been read
        fetch(st == 0 ? kStages - 1 : st - 1);
        if (ok) {
#pragma unroll
            for (int u = 0; u < kRows; ++u) {
                const int h = w.head(u);
                const bool isq = h < a.Hq, isk = !isq && h < HN;
                Quads q;
                float xf[8], z[8], wf[8];
                q.read(slot(st, 0, u), turn.ia, turn.ib);
                q.unpack(xf);
                q.read(slot(st, 1, u), turn.ia, turn.ib);
                q.unpack(z);
                (isq ? wq : wk).unpack(wf);
                float ss = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) ss = fmaf(xf[e], xf[e], ss);
                const float r = rsqrtf(row_sum<LPR>(ss) * (1.f / D) + a.eps);
                turn.template apply<true>(z);
                float dot = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    xf[e] *= r;   // xh
                    const float p = z[e] * xf[e];
                    if (isq) aq[e] += p;
                    if (isk) ak[e] += p;
                    dot = fmaf(p, wf[e], dot);
                }
                const float m = row_sum<LPR>(dot) * (1.f / D);
#pragma unroll
                for (int e = 0; e < 8; ++e) z[e] = r * fmaf(-m, xf[e], z[e] * wf[e]);
                if (isq || isk) q.pack(z);   // values pass through
                if (h < H) q.store(a.dqkv + static_cast<long long>(w.t) * a.ld_d + h * D, turn.ia, turn.ib);
            }
        }
        st = st + 1 == kStages ? 0 : st + 1;
    }
    cp_async_wait<0>();
    // the warp's groups, then the block's warps
#pragma unroll
    for (int e = 0; e < 8; ++e) {
#pragma unroll
        for (int o = LPR; o < 32; o <<= 1) {
            aq[e] += __shfl_xor_sync(0xffffffffu, aq[e], o);
            ak[e] += __shfl_xor_sync(0xffffffffu, ak[e], o);
        }
        if (g == 0) {
            const int at = warp * 2 * D + (e < 4 ? turn.ia + e : turn.ib + e - 4);
            sums[at] = aq[e];
            sums[at + D] = ak[e];
        }
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

template <int D>
long long units_of(const RopeArgs& a) { return a.T * Unit<D>::parts(a); }

template <int D, bool INTER>
cudaError_t launch_fwd(const RopeArgs& a, const KernelEnv& env) {
    const unsigned units = static_cast<unsigned>(units_of<D>(a)), blocks = (units + kWarps - 1) / kWarps;
    if (a.slots != nullptr) rope_fwd_kernel<D, INTER, true><<<blocks, kThreads, 0, env.stream>>>(a, units);
    else rope_fwd_kernel<D, INTER, false><<<blocks, kThreads, 0, env.stream>>>(a, units);
    return cudaGetLastError();
}

template <int D, bool INTER>
cudaError_t launch_bwd(const RopeArgs& a, const KernelEnv& env) {
    const cudaError_t e = ensure_smem_attr(reinterpret_cast<const void*>(rope_bwd_kernel<D, INTER>), rope_bwd_smem<D>(), true);
    if (e != cudaSuccess) return e;
    const unsigned units = static_cast<unsigned>(units_of<D>(a));
    const long long need = (static_cast<long long>(units) + kWarps - 1) / kWarps;
    const int blocks = static_cast<int>(need < rope_bwd_max_blocks() ? need : rope_bwd_max_blocks());
    rope_bwd_kernel<D, INTER><<<blocks, kThreads, rope_bwd_smem<D>(), env.stream>>>(a, units);
    return cudaGetLastError();
}

}  // namespace

const char* rope_check(int rot, int interleaved, int max_pos, float eps, long long heads, int d, long long ld) {
    if (rot < 16 || rot > d || rot % 16 != 0) return "rot must be a multiple of 16 from 16 to d";
    if (interleaved != 0 && interleaved != 1) return "interleaved must be 0 or 1";
    if (max_pos < 1) return "max_pos must be positive";
    if (!(eps >= 0.f) || eps > 3.0e38f) return "eps must be finite and not negative";
    if (ld < heads * d || ld % 8 != 0) return "a token's row stride must hold all its heads and be a multiple of 8";
    return nullptr;
}

// Units are counted in 32 bits, so that the kernels divide 32-bit numbers.
bool rope_supported(const RopeArgs& a, int d) { return (d == 128 ? units_of<128>(a) : units_of<64>(a)) <= 0x7fffffffLL; }

int rope_bwd_max_blocks() { return 2 * device_sm_count(); }   // two a multiprocessor, all resident

cudaError_t launch_rope_fwd(const RopeArgs& a, int d, const KernelEnv& env) {
    if (d == 128) return a.interleaved ? launch_fwd<128, true>(a, env) : launch_fwd<128, false>(a, env);
    if (d == 64) return a.interleaved ? launch_fwd<64, true>(a, env) : launch_fwd<64, false>(a, env);
    return cudaErrorInvalidValue;
}

cudaError_t launch_rope_bwd(const RopeArgs& a, int d, const KernelEnv& env) {
    if (d == 128) return a.interleaved ? launch_bwd<128, true>(a, env) : launch_bwd<128, false>(a, env);
    if (d == 64) return a.interleaved ? launch_bwd<64, true>(a, env) : launch_bwd<64, false>(a, env);
    return cudaErrorInvalidValue;
}

}  // namespace sas
