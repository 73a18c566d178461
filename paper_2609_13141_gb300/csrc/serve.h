// Host-side declarations of the norm + rotation and the serving-step kernels.
#pragma once

#include "internal.h"

namespace sas {

// make_tmap_bf16_3d with a (box_inner x box_rows x box_outer) box.
int make_tmap_bf16_box(CUtensorMap* map, const void* base, uint64_t inner, uint64_t rows, uint64_t outer,
                       uint32_t box_inner, uint32_t box_rows, uint32_t box_outer);

// ---- per-head RMS norm of queries and keys + rotation (forward, into cache pages, gradient).
struct RopeArgs {
    const bf16* qkv;            // [T] rows of (Hq + 2 Hkv) d elements, ld elements apart
    long long ld;
    const bf16* wq;             // [d]
    const bf16* wk;
    const float* cos;           // [max_pos][rot / 2]
    const float* sin;
    const int32_t* pos;         // [T] or null (token index within its batch row)
    int max_pos, rot, interleaved;
    float eps;
    int Hq, Hkv;
    long long T;                // tokens, all batch rows together
    int N;                      // tokens of a batch row
    // forward: outputs; gradient: dQ, dK, dV (read)
    bf16* Q;
    bf16* K;
    bf16* V;
    const int64_t* slots;       // [T] cache slots (page * 64 + row, -1: skip), K and V then the cache pages; or null
    long long n_slots;
    // gradient
    bf16* dqkv;                 // rows ld_d elements apart
    long long ld_d;
    float* dwq;                 // [d]
    float* dwk;
    float* part;                // [rope_bwd_max_blocks()][2 d]
    int* counter;               // zero between launches
    int* status;
};
// What is wrong with a rotation of rows of `heads` heads, ld elements apart, or null.
const char* rope_check(int rot, int interleaved, int max_pos, float eps, long long heads, int d, long long ld);
bool rope_supported(const RopeArgs& a);   // the kernels can count this many tokens
int rope_bwd_max_blocks();
cudaError_t rope_paged_prepare(int d);    // shared-memory limit of the form into cache pages (before any capture)
cudaError_t launch_rope_fwd(const RopeArgs& a, int d, const KernelEnv& env);
cudaError_t launch_rope_bwd(const RopeArgs& a, int d, const KernelEnv& env);

// ---- page plan of a serving step.
struct PlanArgs {
    int B, T, max_blocks, num_pages, num_free;
    const int32_t* seq_lens;    // [B]
    const int32_t* new_lens;    // [B]
    const int32_t* held_lens;   // [B] tokens whose pages are held, or null (seq_lens)
    const int32_t* free_pages;  // [num_free]
    const int32_t* free_begin;  // [1]
    int32_t* block_table;       // [B][max_blocks]
    int32_t* kv_lens;           // [B]
    int32_t* cu_new;            // [B + 1]
    int32_t* positions;         // [T]
    int64_t* slots;             // [T]
    int32_t* free_end;          // [1]
    int* status;
};
size_t plan_smem(int B);
cudaError_t plan_prepare(int max_seqs);   // shared-memory limit (before any capture)
cudaError_t launch_plan(const PlanArgs& a, const KernelEnv& env);

// ---- verification of drafted tokens.
struct VerifyArgs {
    int B, Td, V, W;            // requests, drafts of all requests, columns, most drafts of one request
    const int32_t* tokens;      // [Td]
    const int32_t* cu;          // [B + 1]
    const float* target;        // [Td + B] rows, ldp apart: request b's n + 1 rows from row cu[b] + b
    const float* draft;         // [Td] rows, ldq apart, or null (certain drafts)
    const float* u;             // [Td]
    const float* noise;         // [B] rows, lde apart
    long long ldp, ldq, lde;
    int32_t* accepted;          // [B]
    int32_t* out;               // [B][W + 1]
    unsigned long long* key;    // [B] zero between launches
    int* count;                 // [B] zero between launches
    int chunk;                  // columns of a block (set by the launch)
    int* status;
};
cudaError_t launch_verify(VerifyArgs a, const KernelEnv& env);

// ---- attention of a chunk of new tokens over a paged cache.
struct ChunkArgs {
    int B, T, Hq, Hkv, G, d, max_blocks, num_pages;
    float sm_scale;
    const bf16* Q;              // [T][Hq][d]
    const bf16* K_cache;        // [num_pages][Hkv][64][d]
    const bf16* V_cache;
    const int32_t* block_table; // [B][max_blocks]
    const int32_t* cu;          // [B + 1] first new token of each sequence
    const int32_t* kv_lens;     // [B] tokens of each sequence, the new ones included
    bf16* O;                    // [T][Hq][d]
    float* LSE;                 // [T][Hq] or null
    // workspace
    int blocks;                 // chunk_blocks()
    int4* joins;                // [blocks][2] {splits (0: nothing to join), first one's block, KV group, first token},
                                // {tokens, which of the joining blocks, first one's slot, 0}
    float* part_o;              // [2 blocks][d / 4][128][4]
    float2* part_ml;            // [2 blocks][128] (max, sum)
    int* status;
};
int chunk_blocks();             // blocks of the attention; each writes at most two splits
cudaError_t chunk_attn_prepare(int d);   // shared-memory limit (before any capture)
cudaError_t launch_chunk_attn(const ChunkArgs& a, const KernelEnv& env, const char** err);

}  // namespace sas
