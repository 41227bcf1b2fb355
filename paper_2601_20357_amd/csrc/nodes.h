// Shared by the operators on trees of drafted tokens: who is above whom, and where the cache holds a token.
#pragma once
#include "body_utils.h"
#include "device_utils.h"

namespace tabed {

constexpr int kNodeWords = TABED_MAX_NODES / 64;

// A row's positions before its tree, and its nodes.
__device__ __forceinline__ int context_of(const int32_t* ctx_len, int r) { return max(ctx_len[r], 0); }
__device__ __forceinline__ int nodes_of(const int32_t* n_nodes, int r, int N) { return n_nodes != nullptr ? min(max(n_nodes[r], 0), N) : N; }
// The node that node j follows, -1 for a root.  (Whatever stands there instead of a node before j makes j a root.)
__device__ __forceinline__ int parent_of(const int32_t* parents, int r, int j, int N) {
    if (parents == nullptr) return j - 1;
    const int p = parents[(size_t)r * N + j];
    return p >= 0 && p < j ? p : -1;
}

// Where (layer, head) of a token lies, and its scale.  The block is -1 where the position is in none.
struct PagedView {
    int kv_heads, blocks, max_blocks, layer;
    int64_t layer_stride, block_stride, head_stride, tok_stride;
    char* k;
    char* v;
    float* kscale;
    float* vscale;
    const int32_t* table;
    __device__ __forceinline__ int block_of(int r, int64_t pos) const {
        const int64_t e = pos / TABED_CACHE_BLOCK;
        if (e >= max_blocks) return -1;
        const int b = table[(int64_t)r * max_blocks + e];
        return b >= 0 && b < blocks ? b : -1;
    }
    __device__ __forceinline__ int block_at(int r, int entry) const {
        const int b = table[(int64_t)r * max_blocks + min(entry, max_blocks - 1)];
        return entry < max_blocks && b >= 0 && b < blocks ? b : -1;
    }
    __device__ __forceinline__ int64_t entry(int layer_, int block, int head, int slot) const {      // in elements
        return layer_ * layer_stride + block * block_stride + head * head_stride + slot * tok_stride;
    }
    __device__ __forceinline__ int64_t scale_entry(int layer_, int block, int head, int slot) const {
        return (((int64_t)layer_ * blocks + block) * kv_heads + head) * TABED_CACHE_BLOCK + slot;
    }
};
inline PagedView paged_view(const tabed_cache_paged& c, int layer) {
    return PagedView{c.kv_heads, c.blocks, c.max_blocks, layer, c.layer_stride, c.block_stride, c.head_stride, c.tok_stride,
                     static_cast<char*>(c.k), static_cast<char*>(c.v), c.kscale, c.vscale, c.table};
}

}  // namespace tabed
