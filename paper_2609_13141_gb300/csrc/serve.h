// Host-side declarations of the norm + rotation and the serving-step kernels.
#pragma once

#include "internal.h"

namespace sas {

// make_tmap_bf16_3d with a (box_inner x box_rows x box_outer) box.
int make_tmap_bf16_box(CUtensorMap* map, const void* base, uint64_t inner, uint64_t rows, uint64_t outer,
                       uint32_t box_inner, uint32_t box_rows, uint32_t box_outer);

// 3-D map of bytes [outer][rows][inner] with an (inner x rows x 1) box, swizzled over its rows of 64
// or 128 bytes.
int make_tmap_u8_3d(CUtensorMap* map, const void* base, uint64_t inner, uint64_t rows, uint64_t outer);

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
// Cache of e4m3 numbers, a scale for each page and KV head.
struct Cache8 {
    uint8_t* K;                 // [num_pages][Hkv][64][d]
    uint8_t* V;
    float* k_scale;             // [num_pages][Hkv]
    float* v_scale;
};
// What is wrong with a rotation of rows of `heads` heads, ld elements apart, or null.
const char* rope_check(int rot, int interleaved, int max_pos, float eps, long long heads, int d, long long ld);
bool rope_supported(const RopeArgs& a);   // the kernels can count this many tokens
int rope_bwd_max_blocks();
cudaError_t rope_paged_prepare(int d);    // shared-memory limit of the form into cache pages (before any capture)
cudaError_t launch_rope_fwd(const RopeArgs& a, int d, const KernelEnv& env);
bool append8_supported(const RopeArgs& a);   // blocks of windows: at most one for a head and 8 tokens
// Queries to a.Q, keys and values into an 8-bit cache (a.K and a.V are not used): one launch.
cudaError_t launch_append8(const RopeArgs& a, const Cache8& c, int d, const KernelEnv& env);
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
    const uint8_t* K8;          // the 8-bit form: [num_pages][Hkv][64][d] and [num_pages][Hkv]
    const uint8_t* V8;
    const float* k_scale;
    const float* v_scale;
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
cudaError_t chunk8_prepare(int d);
cudaError_t chunk8_tile_prepare(int d);
cudaError_t launch_chunk8_tile(const ChunkArgs& a, const KernelEnv& env, const char** err);
cudaError_t launch_chunk8(ChunkArgs a, const KernelEnv& env, const char** err);   // over an 8-bit cache

// ---- log probabilities of given tokens, entropy and likeliest columns; their gradient.
struct LogpArgs {
    int rows, V, is_bf16;
    const void* logits;         // [rows] rows of V, ld apart, bf16 or fp32
    long long ld;
    const int32_t* tokens;      // [rows], -1: the row does not count
    float* logprob;             // [rows]
    float* entropy;
    float* lse;
    int k;                      // likeliest columns, 0 .. logp_max_top()
    int32_t* top_index;         // [rows][k]
    float* top_logprob;
    // workspace of rows in several parts; rows x parts <= logp_max_splits()
    float4* part;               // [splits] (max, sum, weighted sum)
    unsigned long long* part_top;   // [splits][logp_max_top()]
    int* count;                 // [splits] zero between launches
    int parts, chunk;           // set by the launch
    int* status;
};
struct LogpBwdArgs {
    int rows, V, is_bf16;
    const void* logits;
    long long ld;
    const int32_t* tokens;
    const float* lse;           // [rows]
    const float* entropy;
    const float* dlogprob;
    const float* dentropy;      // or null
    void* dlogits;              // the logits' type, rows ld_d apart
    long long ld_d;
    int parts, chunk;           // set by the launch
    int* status;
};
// What is wrong with logits of V columns, rows ld elements of type `dtype` apart, or null.
const char* logp_check(int V, int dtype, const void* logits, long long ld);
int logp_max_splits();
int logp_max_top();
cudaError_t launch_logp(const LogpArgs& a, const KernelEnv& env);
cudaError_t launch_logp_bwd(const LogpBwdArgs& a, const KernelEnv& env);

}  // namespace sas
