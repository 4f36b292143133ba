// Internal declarations of the operators over a KV cache in 8 bits (include/gllm_cache8.h).
#pragma once
#include "../../include/gllm_stage.h"
#include "common.h"

constexpr float kCodeMax = 448.0f;                 // the largest e4m3 value
constexpr float kScaleMin = 0x1p-100f, kScaleMax = 0x1p100f;

struct Attn8Args {
    const bf16_t* q;             // [num_rows][ld_q]
    int64_t ld_q;
    const uint8_t* k_pool;       // this layer
    const uint8_t* v_pool;
    const f32x2* scales;         // [num_blocks][n_kv] of keys and values
    int32_t num_blocks;
    const int32_t* block_tables; // [num_seqs][table_stride]
    int32_t table_stride;
    const int32_t* cached_len;   // [num_seqs]
    const int32_t* row_start;    // [num_seqs + 1]
    int32_t num_seqs, num_rows, max_new;
    int32_t window, sinks;       // window 0: none
    bf16_t* out;                 // [num_rows][ld_o]
    int64_t ld_o;
    int32_t n_q, n_kv, d;
    float scale_log2;            // scale * log2(e)
    void* workspace;             // attention8_workspace_bytes()
};
constexpr int kMaxAttn8Seqs = 1 << 20;
size_t attention8_workspace_bytes(int n_q, int n_kv, int d, int max_new);
// GLLM_E_CAPACITY, with nothing enqueued, for more work than a launch takes; GLLM_E_HIP for errors of the runtime.
gllm_status launch_attention8(const Attn8Args& a, hipStream_t stream);
