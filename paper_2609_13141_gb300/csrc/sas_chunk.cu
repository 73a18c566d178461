// C ABI of the serving step over the paged cache: page plan, norm + rotation +
// append, attention of the new tokens, verification of drafts.  Argument checks,
// workspace ownership, launches on the caller's stream, event timing and the
// device status word; the arithmetic is in k_serve.cu, k_rope.cu and k_chunk.cu.
#include <cmath>
#include <new>
#include <string>
#include <vector>

#include "../../include/sas.h"
#include "serve.h"

namespace {

constexpr long long kChunkWaitLimit = 4000000000LL;   // ~2 s of SM clock per wait

struct ChunkTimeRec {
    int kind;
    cudaEvent_t a, b;
};

}  // namespace

struct sas_chunk_handle {
    sas_chunk_config cfg;
    int G = 1, device = 0;
    float sm_scale = 0.f;
    int blocks = 0;
    // workspace
    int4* joins = nullptr;
    float* part_o = nullptr;
    float2* part_ml = nullptr;
    unsigned long long* vkey = nullptr;
    int* vcount = nullptr;
    int* status = nullptr;
    // timing
    bool timing = false;
    std::vector<ChunkTimeRec> recs;
    std::vector<cudaEvent_t> events;
    size_t events_used = 0;
    int64_t launches = 0;
    long long limit = kChunkWaitLimit;
    std::string last_error;
};

namespace {

sas_status cfail(sas_chunk_handle* h, sas_status s, const char* msg) {
    try {
        if (h) h->last_error = msg;
    } catch (...) {   // no memory for the text: the code alone
    }
    return s;
}

sas_status ccuda_fail(sas_chunk_handle* h, cudaError_t e, const char* what) {
    const sas_status s = e == cudaErrorMemoryAllocation ? SAS_ERR_OOM : SAS_ERR_CUDA;
    try {
        h->last_error = std::string(what) + ": " + cudaGetErrorString(e);
    } catch (...) {
    }
    return s;
}

bool al16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool al8(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 7u) == 0; }
bool al4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

template <class T>
cudaError_t calloc_dev(T** p, size_t count) {
    void* v = nullptr;
    const size_t bytes = count * sizeof(T) < 16 ? 16 : count * sizeof(T);
    cudaError_t e = cudaMalloc(&v, bytes);
    *p = static_cast<T*>(v);
    return e;
}

cudaEvent_t cnext_event(sas_chunk_handle* h) {
    if (h->events_used == h->events.size()) {
        cudaEvent_t e;
        if (cudaEventCreate(&e) != cudaSuccess) return nullptr;
        h->events.push_back(e);
    }
    return h->events[h->events_used++];
}

// Runs one entry point's launches, bracketed by events when timing is on (as
// external event nodes while the stream is captured).
template <class Fn>
cudaError_t ctimed(sas_chunk_handle* h, int kind, int launches, cudaStream_t s, Fn&& fn) {
    cudaEvent_t a = nullptr, b = nullptr;
    unsigned flags = cudaEventRecordDefault;
    if (h->timing) {
        a = cnext_event(h);
        b = cnext_event(h);
        cudaStreamCaptureStatus cs = cudaStreamCaptureStatusNone;
        if (cudaStreamIsCapturing(s, &cs) == cudaSuccess && cs == cudaStreamCaptureStatusActive)
            flags = cudaEventRecordExternal;
        if (a && cudaEventRecordWithFlags(a, s, flags) != cudaSuccess) a = nullptr;
    }
    const cudaError_t e = fn();
    if (e == cudaSuccess) h->launches += launches;
    if (h->timing && a && b && cudaEventRecordWithFlags(b, s, flags) == cudaSuccess) h->recs.push_back({kind, a, b});
    return e;
}

// The workspace lives on the device the handle was made on.
sas_status on_device(sas_chunk_handle* h) {
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess) return cfail(h, SAS_ERR_CUDA, "cudaGetDevice");
    if (dev != h->device) return cfail(h, SAS_ERR_INVALID_ARG, "the current device is not the handle's");
    return SAS_OK;
}

// No C++ exception leaves a C entry point.
template <class Fn>
sas_status guarded(sas_chunk_handle* h, Fn&& fn) {
    try {
        return fn();
    } catch (const std::bad_alloc&) {
        return cfail(h, SAS_ERR_OOM, "out of host memory");
    } catch (...) {
        return cfail(h, SAS_ERR_CUDA, "internal error");
    }
}

}  // namespace

extern "C" {

sas_status sas_chunk_create(const sas_chunk_config* cfg, sas_chunk_handle** out) {
    if (out == nullptr || cfg == nullptr) return SAS_ERR_INVALID_ARG;
    *out = nullptr;
    const sas_chunk_config& c = *cfg;
    if (c.max_seqs < 1 || c.Hq < 1 || c.Hkv < 1 || c.max_blocks < 1 || c.num_pages < 1 || c.max_tokens < 1)
        return SAS_ERR_INVALID_ARG;
    if (c.Hq % c.Hkv != 0) return SAS_ERR_INVALID_ARG;
    const int G = c.Hq / c.Hkv;
    if (G != 1 && G != 2 && G != 4 && G != 8) return SAS_ERR_UNSUPPORTED;
    if (c.block != 64) return SAS_ERR_UNSUPPORTED;
    if (c.d != 64 && c.d != 128) return SAS_ERR_UNSUPPORTED;
    if (c.Hq > 65536 || c.max_seqs > 8192 || c.max_blocks > 32768 || c.max_tokens > (1 << 26)) return SAS_ERR_UNSUPPORTED;
    if (!(c.sm_scale >= 0.f) || !std::isfinite(c.sm_scale)) return SAS_ERR_INVALID_ARG;
    // (page, KV head) pairs are TMA coordinates, one past the last included
    if (static_cast<long long>(c.num_pages) * c.Hkv > 0x7fffffffLL) return SAS_ERR_UNSUPPORTED;
    int dev = 0, major = 0, minor = 0;
    if (cudaGetDevice(&dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&minor, cudaDevAttrComputeCapabilityMinor, dev) != cudaSuccess)
        return SAS_ERR_CUDA;
    if (major != 10 || minor != 3) return SAS_ERR_UNSUPPORTED;
    sas_chunk_handle* h = new (std::nothrow) sas_chunk_handle();
    if (h == nullptr) return SAS_ERR_OOM;
    h->cfg = c;
    h->G = G;
    h->device = dev;
    h->blocks = sas::chunk_blocks();
    h->sm_scale = c.sm_scale > 0.f ? c.sm_scale : 1.0f / std::sqrt(static_cast<float>(c.d));
    const size_t parts = 2 * static_cast<size_t>(h->blocks);
    cudaError_t e = calloc_dev(&h->joins, parts);
    if (e == cudaSuccess) e = calloc_dev(&h->part_o, parts * 128 * c.d);
    if (e == cudaSuccess) e = calloc_dev(&h->part_ml, parts * 128);
    if (e == cudaSuccess) e = calloc_dev(&h->vkey, c.max_seqs);
    if (e == cudaSuccess) e = calloc_dev(&h->vcount, c.max_seqs);
    if (e == cudaSuccess) e = calloc_dev(&h->status, 4);
    if (e == cudaSuccess) e = cudaMemset(h->vkey, 0, static_cast<size_t>(c.max_seqs) * 8);
    if (e == cudaSuccess) e = cudaMemset(h->vcount, 0, static_cast<size_t>(c.max_seqs) * 4);
    if (e == cudaSuccess) e = cudaMemset(h->status, 0, 16);
    // shared-memory limits now, so that a captured call sets nothing
    if (e == cudaSuccess) e = sas::plan_prepare(c.max_seqs);
    if (e == cudaSuccess) e = sas::rope_paged_prepare(c.d);
    if (e == cudaSuccess) e = sas::chunk_attn_prepare(c.d);
    if (e == cudaSuccess) e = cudaDeviceSynchronize();
    if (e != cudaSuccess) {
        const sas_status s = e == cudaErrorMemoryAllocation ? SAS_ERR_OOM : SAS_ERR_CUDA;
        sas_chunk_destroy(h);
        return s;
    }
    *out = h;
    return SAS_OK;
}

void sas_chunk_destroy(sas_chunk_handle* h) {
    if (h == nullptr) return;
    cudaDeviceSynchronize();
    cudaFree(h->joins);
    cudaFree(h->part_o);
    cudaFree(h->part_ml);
    cudaFree(h->vkey);
    cudaFree(h->vcount);
    cudaFree(h->status);
    for (cudaEvent_t ev : h->events) cudaEventDestroy(ev);
    delete h;
}

sas_status sas_chunk_plan(sas_chunk_handle* h, int32_t num_seqs, int32_t T, const int32_t* seq_lens,
                          const int32_t* new_lens, const int32_t* held_lens, const int32_t* free_pages, int32_t num_free,
                          const int32_t* free_begin, int32_t* block_table, int32_t* kv_lens, int32_t* cu_new,
                          int32_t* positions, int64_t* slots, int32_t* free_end, void* stream) {
    if (h == nullptr) return SAS_ERR_INVALID_ARG;
    return guarded(h, [&]() -> sas_status {
        if (sas_status st = on_device(h); st != SAS_OK) return st;
        const sas_chunk_config& c = h->cfg;
        if (num_seqs < 1 || num_seqs > c.max_seqs)
            return cfail(h, SAS_ERR_INVALID_ARG, "num_seqs must be 1 .. max_seqs");
        if (T < 1 || T > c.max_tokens) return cfail(h, SAS_ERR_INVALID_ARG, "T must be 1 .. max_tokens");
        if (num_free < 0) return cfail(h, SAS_ERR_INVALID_ARG, "num_free must not be negative");
        if (!seq_lens || !new_lens || (!free_pages && num_free > 0) || !free_begin || !block_table || !kv_lens || !cu_new ||
            !positions || !slots || !free_end)
            return cfail(h, SAS_ERR_INVALID_ARG, "a required argument is NULL");
        if (!al4(seq_lens) || !al4(new_lens) || !al4(held_lens) || !al4(free_pages) || !al4(free_begin) || !al4(block_table) ||
            !al4(kv_lens) || !al4(cu_new) || !al4(positions) || !al8(slots) || !al4(free_end))
            return cfail(h, SAS_ERR_INVALID_ARG, "misaligned pointer");
        // every block reads the inputs while others write
        if (kv_lens == seq_lens || kv_lens == new_lens || kv_lens == held_lens || free_end == free_begin)
            return cfail(h, SAS_ERR_INVALID_ARG, "outputs must not be the inputs' memory");
        sas::PlanArgs a{};
        a.B = num_seqs; a.T = T; a.max_blocks = c.max_blocks; a.num_pages = c.num_pages; a.num_free = num_free;
        a.seq_lens = seq_lens; a.new_lens = new_lens; a.held_lens = held_lens; a.free_pages = free_pages; a.free_begin = free_begin;
        a.block_table = block_table; a.kv_lens = kv_lens; a.cu_new = cu_new; a.positions = positions; a.slots = slots;
        a.free_end = free_end; a.status = h->status;
        cudaStream_t s = static_cast<cudaStream_t>(stream);
        const sas::KernelEnv env{s, h->status, h->limit};
        const cudaError_t e = ctimed(h, 0, 1, s, [&] { return sas::launch_plan(a, env); });
        return e == cudaSuccess ? SAS_OK : ccuda_fail(h, e, "page plan");
    });
}

sas_status sas_chunk_append(sas_chunk_handle* h, const sas_rope_config* rope, int32_t T, const void* qkv, int64_t ld,
                            const void* wq, const void* wk, const float* cos, const float* sin,
                            const int32_t* positions, const int64_t* slots, void* Q, void* K_cache, void* V_cache,
                            void* stream) {
    if (h == nullptr) return SAS_ERR_INVALID_ARG;
    return guarded(h, [&]() -> sas_status {
        if (sas_status st = on_device(h); st != SAS_OK) return st;
        const sas_chunk_config& c = h->cfg;
        if (T < 1 || T > c.max_tokens) return cfail(h, SAS_ERR_INVALID_ARG, "T must be 1 .. max_tokens");
        if (!rope || !qkv || !wq || !wk || !cos || !sin || !positions || !slots || !Q || !K_cache || !V_cache)
            return cfail(h, SAS_ERR_INVALID_ARG, "a required argument is NULL");
        if (!al16(qkv) || !al16(wq) || !al16(wk) || !al16(cos) || !al16(sin) || !al4(positions) || !al8(slots) || !al16(Q) ||
            !al16(K_cache) || !al16(V_cache))
            return cfail(h, SAS_ERR_INVALID_ARG, "misaligned pointer");
        if (const char* why = sas::rope_check(rope->rot, rope->interleaved, rope->max_pos, rope->eps,
                                              c.Hq + 2LL * c.Hkv, c.d, ld))
            return cfail(h, SAS_ERR_INVALID_ARG, why);
        sas::RopeArgs a{};
        a.qkv = static_cast<const sas::bf16*>(qkv); a.ld = ld;
        a.wq = static_cast<const sas::bf16*>(wq); a.wk = static_cast<const sas::bf16*>(wk);
        a.cos = cos; a.sin = sin; a.pos = positions;
        a.max_pos = rope->max_pos; a.rot = rope->rot; a.interleaved = rope->interleaved; a.eps = rope->eps;
        a.Hq = c.Hq; a.Hkv = c.Hkv; a.T = T; a.N = T;
        a.Q = static_cast<sas::bf16*>(Q); a.K = static_cast<sas::bf16*>(K_cache); a.V = static_cast<sas::bf16*>(V_cache);
        a.slots = slots; a.n_slots = 64LL * c.num_pages; a.status = h->status;
        if (!sas::rope_supported(a)) return cfail(h, SAS_ERR_UNSUPPORTED, "too many tokens");
        cudaStream_t s = static_cast<cudaStream_t>(stream);
        const sas::KernelEnv env{s, h->status, h->limit};
        const cudaError_t e = ctimed(h, 1, 1, s, [&] { return sas::launch_rope_fwd(a, c.d, env); });
        return e == cudaSuccess ? SAS_OK : ccuda_fail(h, e, "norm + rotation + append");
    });
}

sas_status sas_chunk_attention(sas_chunk_handle* h, int32_t num_seqs, int32_t T, const void* Q, const void* K_cache,
                               const void* V_cache, const int32_t* block_table, const int32_t* cu_new,
                               const int32_t* kv_lens, void* O, float* LSE, void* stream) {
    if (h == nullptr) return SAS_ERR_INVALID_ARG;
    return guarded(h, [&]() -> sas_status {
        if (sas_status st = on_device(h); st != SAS_OK) return st;
        const sas_chunk_config& c = h->cfg;
        if (num_seqs < 1 || num_seqs > c.max_seqs)
            return cfail(h, SAS_ERR_INVALID_ARG, "num_seqs must be 1 .. max_seqs");
        if (T < 1 || T > c.max_tokens) return cfail(h, SAS_ERR_INVALID_ARG, "T must be 1 .. max_tokens");
        if (!Q || !K_cache || !V_cache || !block_table || !cu_new || !kv_lens || !O)
            return cfail(h, SAS_ERR_INVALID_ARG, "a required argument is NULL");
        if (!al16(Q) || !al16(K_cache) || !al16(V_cache) || !al4(block_table) || !al4(cu_new) || !al4(kv_lens) || !al16(O) ||
            !al4(LSE))
            return cfail(h, SAS_ERR_INVALID_ARG, "misaligned pointer");
        sas::ChunkArgs a{};
        a.B = num_seqs; a.T = T; a.Hq = c.Hq; a.Hkv = c.Hkv; a.G = h->G; a.d = c.d; a.max_blocks = c.max_blocks;
        a.num_pages = c.num_pages; a.sm_scale = h->sm_scale;
        a.Q = static_cast<const sas::bf16*>(Q);
        a.K_cache = static_cast<const sas::bf16*>(K_cache); a.V_cache = static_cast<const sas::bf16*>(V_cache);
        a.block_table = block_table; a.cu = cu_new; a.kv_lens = kv_lens;
        a.O = static_cast<sas::bf16*>(O); a.LSE = LSE;
        a.blocks = h->blocks; a.joins = h->joins; a.part_o = h->part_o; a.part_ml = h->part_ml;
        a.status = h->status;
        cudaStream_t s = static_cast<cudaStream_t>(stream);
        const sas::KernelEnv env{s, h->status, h->limit};
        const char* err = "chunk attention";
        const cudaError_t e = ctimed(h, 2, 2, s, [&] { return sas::launch_chunk_attn(a, env, &err); });
        return e == cudaSuccess ? SAS_OK : ccuda_fail(h, e, err);
    });
}

sas_status sas_chunk_verify(sas_chunk_handle* h, int32_t num_seqs, int32_t num_drafts, int32_t max_draft, int32_t V,
                            const int32_t* tokens, const int32_t* cu_draft, const float* target, int64_t ld_target,
                            const float* draft, int64_t ld_draft, const float* u, const float* noise, int64_t ld_noise,
                            int32_t* accepted, int32_t* out_tokens, void* stream) {
    if (h == nullptr) return SAS_ERR_INVALID_ARG;
    return guarded(h, [&]() -> sas_status {
        if (sas_status st = on_device(h); st != SAS_OK) return st;
        const sas_chunk_config& c = h->cfg;
        if (num_seqs < 1 || num_seqs > c.max_seqs)
            return cfail(h, SAS_ERR_INVALID_ARG, "num_seqs must be 1 .. max_seqs");
        if (num_drafts < 0 || max_draft < 0 || max_draft >= (1 << 20) || V < 1 || V > (1 << 30))
            return cfail(h, SAS_ERR_INVALID_ARG, "num_drafts, max_draft or V out of range");
        if (!cu_draft || !target || !noise || !accepted || !out_tokens || (num_drafts > 0 && (!tokens || !u)))
            return cfail(h, SAS_ERR_INVALID_ARG, "a required argument is NULL");
        if (!al4(tokens) || !al4(cu_draft) || !al4(target) || !al4(draft) || !al4(u) || !al4(noise) || !al4(accepted) ||
            !al4(out_tokens))
            return cfail(h, SAS_ERR_INVALID_ARG, "misaligned pointer");
        if (ld_target < V || (draft && ld_draft < V) || ld_noise < V)
            return cfail(h, SAS_ERR_INVALID_ARG, "a row stride is below V");
        sas::VerifyArgs a{};
        a.B = num_seqs; a.Td = num_drafts; a.V = V; a.W = max_draft;
        a.tokens = tokens; a.cu = cu_draft; a.target = target; a.draft = draft; a.u = u; a.noise = noise;
        a.ldp = ld_target; a.ldq = draft ? ld_draft : 0; a.lde = ld_noise;
        a.accepted = accepted; a.out = out_tokens; a.key = h->vkey; a.count = h->vcount; a.status = h->status;
        cudaStream_t s = static_cast<cudaStream_t>(stream);
        const sas::KernelEnv env{s, h->status, h->limit};
        const cudaError_t e = ctimed(h, 3, 1, s, [&] { return sas::launch_verify(a, env); });
        return e == cudaSuccess ? SAS_OK : ccuda_fail(h, e, "draft verification");
    });
}

const char* sas_chunk_last_error(const sas_chunk_handle* h) { return h ? h->last_error.c_str() : ""; }

sas_status sas_chunk_get_device_status(sas_chunk_handle* h, int32_t* out_status) {
    if (h == nullptr || out_status == nullptr) return SAS_ERR_INVALID_ARG;
    cudaError_t e = cudaDeviceSynchronize();
    if (e != cudaSuccess) return ccuda_fail(h, e, "synchronize");
    int v = 0;
    e = cudaMemcpy(&v, h->status, sizeof(int), cudaMemcpyDeviceToHost);
    if (e == cudaSuccess) e = cudaMemset(h->status, 0, sizeof(int));
    if (e != cudaSuccess) return ccuda_fail(h, e, "status word");
    *out_status = v;
    return SAS_OK;
}

sas_status sas_chunk_set_wait_limit(sas_chunk_handle* h, int64_t cycles) {
    if (h == nullptr || cycles < 0) return SAS_ERR_INVALID_ARG;
    h->limit = cycles == 0 ? kChunkWaitLimit : cycles;
    return SAS_OK;
}

sas_status sas_chunk_set_timing(sas_chunk_handle* h, int32_t enable) {
    if (h == nullptr) return SAS_ERR_INVALID_ARG;
    cudaDeviceSynchronize();
    h->timing = enable != 0;
    if (h->timing) {   // a new recording starts; stopping keeps the records
        h->recs.clear();
        h->events_used = 0;
    }
    return SAS_OK;
}

sas_status sas_chunk_get_timings(sas_chunk_handle* h, int64_t* launches, double* total_ms, int32_t n_kinds) {
    if (h == nullptr || launches == nullptr || total_ms == nullptr || n_kinds < 0 || n_kinds > SAS_CHUNK_NUM_KERNEL_KINDS)
        return SAS_ERR_INVALID_ARG;
    cudaError_t e = cudaDeviceSynchronize();
    if (e != cudaSuccess) return ccuda_fail(h, e, "synchronize");
    for (int k = 0; k < n_kinds; ++k) {
        launches[k] = 0;
        total_ms[k] = 0.0;
    }
    for (const ChunkTimeRec& r : h->recs) {
        if (r.kind >= n_kinds) continue;
        float ms = 0.f;
        if (cudaEventElapsedTime(&ms, r.a, r.b) == cudaSuccess) {
            launches[r.kind] += 1;
            total_ms[r.kind] += ms;
        }
    }
    return SAS_OK;
}

int64_t sas_chunk_launch_count(const sas_chunk_handle* h) { return h ? h->launches : 0; }

}  // extern "C"
