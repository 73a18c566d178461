// Device primitives of the norm + rotation and the serving-step kernels, beside ptx.cuh.
#pragma once

#include "ptx.cuh"

namespace sas {

// Whether the phase has completed, without waiting at all (try_wait may hold the
// thread for microseconds, whatever its time hint).
__device__ __forceinline__ bool mbar_test_wait(uint64_t* bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(smem_u32(bar)), "r"(parity)
        : "memory");
    return ok != 0;
}

// mbar_wait_warp by polling: for rare waits whose budget must be noticed as soon
// as it has run out.
__device__ __forceinline__ bool mbar_poll_warp(uint64_t* bar, uint32_t parity, const WaitCtl& w) {
    bool ok = mbar_test_wait(bar, parity);
    const long long t0 = clock64();
    while (!ok) {
        ok = mbar_test_wait(bar, parity);
        if (ok || *w.abort_flag) break;
        if (clock64() - t0 > w.limit) {
            *w.abort_flag = 1;
            atomicExch(w.status, kStatusTimeout);
            break;
        }
    }
    return __all_sync(0xffffffffu, ok);
}

// Waits until the kernel ahead in the stream has ended; lets the next one's blocks come
// in as places open up (they wait the same way).
__device__ __forceinline__ void grid_dep_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void grid_dep_launch() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// A load of what an earlier kernel may have written.  Not through the read-only path: its
// data must not change while the kernel runs, which begins ahead of the wait, and a load
// by it may be moved there.
template <class T>
__device__ __forceinline__ T load(const T* p) { return *p; }

// Launches a kernel that may set up while the kernel ahead of it is still at work: its
// every thread calls grid_dep_wait before its first access to global memory.
template <class... P, class... A>
cudaError_t launch_early(void (*kernel)(P...), dim3 grid, int threads, int smem, cudaStream_t stream, A... args) {
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// 16-byte asynchronous copy global -> shared, past L1 (both addresses 16-byte aligned).
__device__ __forceinline__ void cp_async16(void* smem_dst, const void* gsrc) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(smem_dst)), "l"(gsrc) : "memory");
}

// The box that tma_load_3d would load, into L2 only.
__device__ __forceinline__ void tma_prefetch_3d(const CUtensorMap* map, int c0, int c1, int c2) {
    asm volatile("cp.async.bulk.prefetch.tensor.3d.L2.global.tile [%0, {%1, %2, %3}];" ::"l"(
                     reinterpret_cast<uint64_t>(map)),
                 "r"(c0), "r"(c1), "r"(c2)
                 : "memory");
}

__device__ __forceinline__ uint64_t mul_f32x2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}

}  // namespace sas
