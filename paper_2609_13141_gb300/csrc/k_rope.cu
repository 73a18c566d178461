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
// Bound: HBM.  A row is d / 8 lanes of 16 bytes; a warp takes kRows rows per
// group of lanes of ONE token, all loaded before any is used, so the table's row
// is read once per unit and stays in registers.
#include "internal.h"
#include "ptx.cuh"

namespace sas {
namespace {

constexpr int kWarps = 8;
constexpr int kThreads = kWarps * 32;
constexpr int kRows = 4;          // rows in flight per lane group
constexpr int kStatusBadInput = 1;   // == SAS_ERR_INVALID_ARG

__device__ __forceinline__ void unpack8(const uint4& v, float (&f)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}

__device__ __forceinline__ uint4 pack8(const float (&f)[8]) {
    return make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]),
                      pack_bf16x2(f[6], f[7]));
}

// Sum over the LPR lanes of a row.
template <int LPR>
__device__ __forceinline__ float row_sum(float v) {
#pragma unroll
    for (int o = LPR / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// A lane's share of the rotation at one position: element e of the lane becomes
// z_e c[e] + partner(z)_e s[e], the sign of the sine included.
template <int D, bool INTER>
struct Turn {
    float c[8], s[8];
    int src;   // half-split pairs: the warp lane that holds the partners

    __device__ __forceinline__ void load(const RopeArgs& a, int pos, int l, int lane) {
        const int rl = a.rot >> 3, hl = rl >> 1;   // lanes that hold rotated dims, and half of them
        src = lane;
        if (l >= rl) {
#pragma unroll
            for (int e = 0; e < 8; ++e) { c[e] = 1.f; s[e] = 0.f; }
            return;
        }
        const size_t row = static_cast<size_t>(pos) * (a.rot >> 1);
        if constexpr (INTER) {
            const float4 cv = __ldg(reinterpret_cast<const float4*>(a.cos + row) + l);
            const float4 sv = __ldg(reinterpret_cast<const float4*>(a.sin + row) + l);
            const float cs[4] = {cv.x, cv.y, cv.z, cv.w}, sn[4] = {sv.x, sv.y, sv.z, sv.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                c[2 * i] = c[2 * i + 1] = cs[i];
                s[2 * i] = -sn[i];
                s[2 * i + 1] = sn[i];
            }
        } else {
            const bool first = l < hl;
            src = first ? lane + hl : lane - hl;
            const int at = 2 * (first ? l : l - hl);   // in float4
            const float4 c0 = __ldg(reinterpret_cast<const float4*>(a.cos + row) + at);
            const float4 c1 = __ldg(reinterpret_cast<const float4*>(a.cos + row) + at + 1);
            const float4 s0 = __ldg(reinterpret_cast<const float4*>(a.sin + row) + at);
            const float4 s1 = __ldg(reinterpret_cast<const float4*>(a.sin + row) + at + 1);
            const float sg = first ? -1.f : 1.f;
            c[0] = c0.x; c[1] = c0.y; c[2] = c0.z; c[3] = c0.w; c[4] = c1.x; c[5] = c1.y; c[6] = c1.z; c[7] = c1.w;
            s[0] = sg * s0.x; s[1] = sg * s0.y; s[2] = sg * s0.z; s[3] = sg * s0.w;
            s[4] = sg * s1.x; s[5] = sg * s1.y; s[6] = sg * s1.z; s[7] = sg * s1.w;
        }
    }

    // BACK: the transposed rotation (the sine's sign flips).
    template <bool BACK>
    __device__ __forceinline__ void apply(float (&z)[8]) const {
        float p[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = INTER ? z[e ^ 1] : __shfl_sync(0xffffffffu, z[e], src);
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] = fmaf(p[e], BACK ? -s[e] : s[e], z[e] * c[e]);
    }
};

template <int D>
__device__ __forceinline__ int units_per_token(const RopeArgs& a) {
    constexpr int RPU = kRows * 32 / (D / 8);
    return (a.Hq + 2 * a.Hkv + RPU - 1) / RPU;
}

// PAGED: keys and values go to the cache pages that `slots` names and the queries
// to [token][Hq][d]; else all three go to [batch][head][N][d].
template <int D, bool INTER, bool PAGED>
__global__ void __launch_bounds__(kThreads) rope_fwd_kernel(RopeArgs a) {
    constexpr int LPR = D / 8, GPW = 32 / LPR, RPU = kRows * GPW;
    const int parts = units_per_token<D>(a);
    const unsigned unit = blockIdx.x * kWarps + warp_id();
    if (unit >= static_cast<unsigned>(a.T) * static_cast<unsigned>(parts)) return;
    const unsigned t = unit / parts;
    const int part = unit - t * parts;
    const int lane = lane_id(), l = lane % LPR, g = lane / LPR;
    const int H = a.Hq + 2 * a.Hkv;

    uint4 x[kRows];
    const bf16* xrow = a.qkv + static_cast<long long>(t) * a.ld + l * 8;
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
        const int h = part * RPU + u * GPW + g;
        x[u] = h < H ? __ldg(reinterpret_cast<const uint4*>(xrow + h * D)) : make_uint4(0, 0, 0, 0);
    }
    unsigned b = 0, n = t;
    if constexpr (!PAGED) {
        b = t / a.N;
        n = t - b * a.N;
    }
    const int pos = a.pos != nullptr ? __ldg(a.pos + t) : static_cast<int>(n);
    long long slot = 0;
    if constexpr (PAGED) {
        slot = __ldg(a.slots + t);
        if (slot == -1) return;   // padding
    }
    if (pos < 0 || pos >= a.max_pos || (PAGED && (slot < 0 || slot >= a.n_slots))) {
        if (lane == 0) atomicExch(a.status, kStatusBadInput);
        return;
    }
    Turn<D, INTER> turn;
    turn.load(a, pos, l, lane);
    float wq[8], wk[8];
    unpack8(__ldg(reinterpret_cast<const uint4*>(a.wq) + l), wq);
    unpack8(__ldg(reinterpret_cast<const uint4*>(a.wk) + l), wk);
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
        const int h = part * RPU + u * GPW + g;
        float z[8];
        unpack8(x[u], z);
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fmaf(z[e], z[e], ss);
        const float r = rsqrtf(row_sum<LPR>(ss) * (1.f / D) + a.eps);
        const bool isq = h < a.Hq;
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] = z[e] * r * (isq ? wq[e] : wk[e]);
        turn.template apply<false>(z);
        if (h >= H) continue;
        const bool isv = h >= a.Hq + a.Hkv;
        const uint4 y = isv ? x[u] : pack8(z);
        const int hk = isq ? h : (isv ? h - a.Hq - a.Hkv : h - a.Hq);
        bf16* dst;
        if constexpr (PAGED) {
            dst = isq ? a.Q + (static_cast<size_t>(t) * a.Hq + hk) * D
                      : (isv ? a.V : a.K) + ((static_cast<size_t>(slot >> 6) * a.Hkv + hk) * 64 + (slot & 63)) * D;
        } else {
            dst = (isq ? a.Q : (isv ? a.V : a.K)) +
                  ((static_cast<size_t>(b) * (isq ? a.Hq : a.Hkv) + hk) * a.N + n) * D;
        }
        *reinterpret_cast<uint4*>(dst + l * 8) = y;
    }
}

// Persistent: a lane keeps its 8 columns of dwq and dwk over all its rows, a
// block adds its lanes' into one row of `part`, and the last block to finish
// adds the rows in their order, so equal inputs give equal sums.
template <int D, bool INTER>
__global__ void __launch_bounds__(kThreads) rope_bwd_kernel(RopeArgs a) {
    constexpr int LPR = D / 8, GPW = 32 / LPR, RPU = kRows * GPW;
    __shared__ __align__(16) float sum[kWarps][2 * D];
    __shared__ int last;
    const int parts = units_per_token<D>(a);
    const unsigned units = static_cast<unsigned>(a.T) * static_cast<unsigned>(parts);
    const int lane = lane_id(), warp = warp_id(), l = lane % LPR, g = lane / LPR;
    const int H = a.Hq + 2 * a.Hkv, HN = a.Hq + a.Hkv;
    float wq[8], wk[8], aq[8], ak[8];
    unpack8(__ldg(reinterpret_cast<const uint4*>(a.wq) + l), wq);
    unpack8(__ldg(reinterpret_cast<const uint4*>(a.wk) + l), wk);
#pragma unroll
    for (int e = 0; e < 8; ++e) aq[e] = ak[e] = 0.f;

    for (unsigned long long unit = blockIdx.x * kWarps + warp; unit < units; unit += gridDim.x * kWarps) {
        const unsigned t = static_cast<unsigned>(unit) / parts;
        const int part = static_cast<unsigned>(unit) - t * parts;
        const unsigned b = t / a.N, n = t - b * a.N;
        const int pos = a.pos != nullptr ? __ldg(a.pos + t) : static_cast<int>(n);
        if (pos < 0 || pos >= a.max_pos) {
            if (lane == 0) atomicExch(a.status, kStatusBadInput);
            continue;
        }
        uint4 x[kRows], dy[kRows];
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            const int h = part * RPU + u * GPW + g;
            const bool isq = h < a.Hq, isv = h >= HN;
            const int hk = isq ? h : (isv ? h - HN : h - a.Hq);
            x[u] = dy[u] = make_uint4(0, 0, 0, 0);
            if (h < HN) x[u] = __ldg(reinterpret_cast<const uint4*>(a.qkv + static_cast<long long>(t) * a.ld + h * D) + l);
            if (h < H) {
                const bf16* src = (isq ? a.Q : (isv ? a.V : a.K)) +
                                  ((static_cast<size_t>(b) * (isq ? a.Hq : a.Hkv) + hk) * a.N + n) * D;
                dy[u] = __ldg(reinterpret_cast<const uint4*>(src) + l);
            }
        }
        Turn<D, INTER> turn;
        turn.load(a, pos, l, lane);
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            const int h = part * RPU + u * GPW + g;
            const bool isq = h < a.Hq, normed = h < HN;   // value rows only pass through
            float xf[8], z[8];
            unpack8(x[u], xf);
            unpack8(dy[u], z);
            float ss = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) ss = fmaf(xf[e], xf[e], ss);
            const float r = rsqrtf(row_sum<LPR>(ss) * (1.f / D) + a.eps);
            turn.template apply<true>(z);
            float dot = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                xf[e] *= r;   // xh
                const float p = normed ? z[e] * xf[e] : 0.f;
                aq[e] += isq ? p : 0.f;
                ak[e] += isq ? 0.f : p;
                z[e] *= isq ? wq[e] : wk[e];
                dot = fmaf(z[e], xf[e], dot);
            }
            const float m = row_sum<LPR>(dot) * (1.f / D);
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] = r * fmaf(-m, xf[e], z[e]);
            if (h < H)
                *(reinterpret_cast<uint4*>(a.dqkv + static_cast<long long>(t) * a.ld_d + h * D) + l) =
                    normed ? pack8(z) : dy[u];
        }
    }
    // the warp's groups, then the block's warps
#pragma unroll
    for (int e = 0; e < 8; ++e) {
#pragma unroll
        for (int o = LPR; o < 32; o <<= 1) {
            aq[e] += __shfl_xor_sync(0xffffffffu, aq[e], o);
            ak[e] += __shfl_xor_sync(0xffffffffu, ak[e], o);
        }
        if (g == 0) {
            sum[warp][l * 8 + e] = aq[e];
            sum[warp][D + l * 8 + e] = ak[e];
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * D; i += kThreads) {
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) v += sum[w][i];
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
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 16
    for (int i = sl; i < static_cast<int>(gridDim.x); i += SL) {
        const float4 v = __ldcg(reinterpret_cast<const float4*>(a.part + static_cast<size_t>(i) * 2 * D) + qd);
        acc.x += v.x; acc.y += v.y; acc.z += v.z; acc.w += v.w;
    }
    reinterpret_cast<float4*>(sum[sl])[qd] = acc;
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * D; i += kThreads) {
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < SL; ++w) v += sum[w][i];
        (i < D ? a.dwq : a.dwk)[i < D ? i : i - D] = v;
    }
}

long long units(const RopeArgs& a, int d) {
    const int rpu = kRows * 32 / (d / 8);
    return a.T * ((a.Hq + 2LL * a.Hkv + rpu - 1) / rpu);
}

template <int D, bool INTER>
cudaError_t launch_fwd(const RopeArgs& a, const KernelEnv& env) {
    const unsigned blocks = static_cast<unsigned>((units(a, D) + kWarps - 1) / kWarps);
    if (a.slots != nullptr) rope_fwd_kernel<D, INTER, true><<<blocks, kThreads, 0, env.stream>>>(a);
    else rope_fwd_kernel<D, INTER, false><<<blocks, kThreads, 0, env.stream>>>(a);
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

bool rope_supported(const RopeArgs& a, int d) { return units(a, d) <= 0x7fffffffLL; }

int rope_bwd_max_blocks() { return 4 * device_sm_count(); }

cudaError_t launch_rope_fwd(const RopeArgs& a, int d, const KernelEnv& env) {
    if (d == 128) return a.interleaved ? launch_fwd<128, true>(a, env) : launch_fwd<128, false>(a, env);
    if (d == 64) return a.interleaved ? launch_fwd<64, true>(a, env) : launch_fwd<64, false>(a, env);
    return cudaErrorInvalidValue;
}

cudaError_t launch_rope_bwd(const RopeArgs& a, int d, const KernelEnv& env) {
    const long long need = (units(a, d) + kWarps - 1) / kWarps;
    const int blocks = static_cast<int>(need < rope_bwd_max_blocks() ? need : rope_bwd_max_blocks());
    if (d == 128) {
        if (a.interleaved) rope_bwd_kernel<128, true><<<blocks, kThreads, 0, env.stream>>>(a);
        else rope_bwd_kernel<128, false><<<blocks, kThreads, 0, env.stream>>>(a);
    } else if (d == 64) {
        if (a.interleaved) rope_bwd_kernel<64, true><<<blocks, kThreads, 0, env.stream>>>(a);
        else rope_bwd_kernel<64, false><<<blocks, kThreads, 0, env.stream>>>(a);
    } else {
        return cudaErrorInvalidValue;
    }
    return cudaGetLastError();
}

}  // namespace sas
