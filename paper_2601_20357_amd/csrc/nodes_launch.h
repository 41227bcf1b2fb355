// Operators on trees given by parents: layouts of their workspaces, and the launchers (arguments are checked by the caller).
#pragma once
#include "internal.h"

namespace tabed {

hipError_t launch_append_nodes(const tabed_cache_paged& c, int layer, int rows, int N, int dtype, const void* k, const void* v, int64_t kv_row,
                               int64_t kv_tok, int q_heads, const void* q, int64_t q_row, int64_t q_tok, void* q_out, int64_t out_row, int64_t out_tok,
                               const int32_t* ctx_len, const int32_t* parents, const int32_t* n_nodes, float rope_theta, hipStream_t s);
hipError_t launch_keep_nodes(const tabed_cache_paged& c, int rows, int N, const int32_t* ctx_base, const int32_t* path, const int32_t* n_path,
                             int32_t* ctx_len, hipStream_t s);
struct NodesAttnLayout {
    size_t off_ml;       // float4 [slots, kv_heads, tiles][queries of a tile] maxima and sums of ranges; before it the ranges of every row
    size_t off_o;        // float [slots, kv_heads, tiles][queries of a tile][head_dim] their sums of values
};
NodesAttnLayout nodes_attn_layout(const tabed_cache_paged& c, int rows, int N, int q_heads);
size_t nodes_attn_bytes(const tabed_cache_paged& c, int rows, int N, int q_heads);
int64_t nodes_attn_workgroups(const tabed_cache_paged& c, int rows, int N, int q_heads);
hipError_t launch_nodes_attn_init(char* ws, hipStream_t s);
hipError_t launch_attention_nodes(const tabed_cache_paged& c, int layer, char* ws, int rows, int N, int q_heads, const uint16_t* q, int64_t q_row,
                                  int64_t q_tok, const int32_t* ctx_len, const int32_t* parents, const int32_t* n_nodes, float scale, uint16_t* out,
                                  int64_t out_row, int64_t out_tok, float* lse, hipStream_t s);
struct NodesVerifyLayout {
    int G;               // workgroups of a sequence
    size_t off_rec;      // uint64 [B][N][G][4] what a workgroup found at a step of the walk
    size_t off_dev;      // uint64 [B][gamma][G][n][2] its sums of the distances
    size_t off_state;    // uint64 [B] what has come of a row
    size_t total;
};
NodesVerifyLayout nodes_verify_layout(const tabed_cfg& c, int N);
hipError_t launch_nodes_verify_init(const tabed_cfg& c, int N, char* ws, hipStream_t s);
hipError_t launch_verify_nodes(const tabed_cfg& c, char* ws, uint64_t round, int N, const float* target_logits, const float* draft_logits,
                               const double* draft_lse, const int32_t* tokens, const float* node_q, const int32_t* parents, const int32_t* n_nodes,
                               const float* weights, const float* temperature, const float* u_acc, const float* u_res, int32_t* path, int32_t* n_path,
                               int32_t* out_tokens, uint8_t* flags, float* dev, int32_t* n_valid, hipStream_t s, int spins = 0, int late = -1);      // (the last two: for tests)

}  // namespace tabed
