// Attention of a tree's nodes over the paged cache.
#include <hip/hip_runtime.h>

#include "internal.h"
#include "nodes.h"

namespace tabed {

struct NodesAttnArgs {
    PagedView c;
    int N, q_heads, group, hd;
    const uint16_t* q;
    uint16_t* out;
    float* lse;
    int64_t q_row, q_tok, out_row, out_tok;
    const int32_t* ctx_len;
    const int32_t* parents;
    const int32_t* n_nodes;
    float scale;
};

__device__ __forceinline__ float bf16_value(uint16_t b) { return __builtin_bit_cast(float, (uint32_t)b << 16); }
template <bool F8>
__device__ __forceinline__ float cache_value(const char* base, int64_t at) {
    if constexpr (F8) return __builtin_amdgcn_cvt_f32_fp8((int)(unsigned char)base[at], 0);
    else return bf16_value(reinterpret_cast<const uint16_t*>(base)[at]);
}

// The simple kernel: a wave takes one query; a lane a position for the scores, dims for the sums.
template <bool F8>
__global__ __launch_bounds__(256) void k_attention_nodes_simple(NodesAttnArgs a) {
    const int r = blockIdx.y, wave = threadIdx.x / 64, lane = threadIdx.x % 64, unit = blockIdx.x * 4 + wave;
    __shared__ float s_q[4][256];
    __shared__ uint64_t s_mask[4][kNodeWords];
    const int node = unit / a.q_heads, head = unit % a.q_heads, n = nodes_of(a.n_nodes, r, a.N);
    if (node >= n) return;                                               // (no barrier below: waves are on their own)
    const int ctx = context_of(a.ctx_len, r), kvh = head / a.group;
    const uint16_t* q = a.q + r * a.q_row + node * a.q_tok + (int64_t)head * a.hd;
    for (int d = lane; d < a.hd; d += 64) s_q[wave][d] = bf16_value(q[d]);
    if (lane < kNodeWords) s_mask[wave][lane] = 0;
    if (lane == 0)
        for (int j = node; j >= 0; j = parent_of(a.parents, r, j, a.N)) s_mask[wave][j / 64] |= 1ull << (j % 64);
    __builtin_amdgcn_wave_barrier();
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    float m = -INFINITY, l = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
    for (int64_t p0 = 0; p0 < (int64_t)ctx + n; p0 += 64) {
        const int block = a.c.block_of(r, p0);
        if (block < 0) continue;
        const int64_t pos = p0 + lane;
        const int64_t j = pos - ctx;
        const bool seen = j < 0 || (j < n && (s_mask[wave][j / 64] >> (j % 64) & 1));
        float s = 0.f, vs = 1.f;
        if (seen) {
            const int64_t at = a.c.entry(a.c.layer, block, kvh, lane);
            for (int d = 0; d < a.hd; ++d) s = fmaf(s_q[wave][d], cache_value<F8>(a.c.k, at + d), s);
            if (F8) {
                const int64_t se = a.c.scale_entry(a.c.layer, block, kvh, lane);
                s *= a.c.kscale[se];
                vs = a.c.vscale[se];
            }
            s *= a.scale;
        } else {
            s = -INFINITY;
        }
        const float top = fmaxf(m, wave_max(s));
        const bool bad = __any(seen && !(s <= top));                     // a NaN
        const float p = seen ? (s == -INFINITY && top == -INFINITY ? 0.f : __expf(s - top)) : 0.f;
        const float fade = m == -INFINITY ? 0.f : __expf(m - top);
        (void)bad;
        l = l * fade + wave_sum(p);
        for (int i = 0; i < 4; ++i) acc[i] *= fade;
        uint64_t who = __ballot(seen);
        while (who) {
            const int t = __ffsll((long long)who) - 1;
            who &= who - 1;
            const float pt = lane_f32(p, t) * lane_f32(vs, t);
            const int64_t at = a.c.entry(a.c.layer, block, kvh, t);
            for (int i = 0; i < 4; ++i)
                if (i * 64 + lane < a.hd) acc[i] = fmaf(pt, cache_value<F8>(a.c.v, at + i * 64 + lane), acc[i]);
        }
        m = top;
    }
    uint16_t* out = a.out + r * a.out_row + node * a.out_tok + (int64_t)head * a.hd;
    for (int i = 0; i < 4; ++i)
        if (i * 64 + lane < a.hd) out[i * 64 + lane] = f32_to_bf16_bits(l == 0.f ? 0.f : acc[i] / l);
    if (a.lse != nullptr && lane == 0) a.lse[((int64_t)r * a.N + node) * a.q_heads + head] = l == 0.f ? -INFINITY : m + logf(l);
}

NodesAttnLayout nodes_attn_layout(const tabed_cache_paged&, int, int, int) { return NodesAttnLayout{256}; }
hipError_t launch_nodes_attn_init(char*, hipStream_t) { return hipSuccess; }

hipError_t launch_attention_nodes(const tabed_cache_paged& c, int layer, char* ws, int rows, int N, int q_heads, const uint16_t* q, int64_t q_row,
                                  int64_t q_tok, const int32_t* ctx_len, const int32_t* parents, const int32_t* n_nodes, float scale, uint16_t* out,
                                  int64_t out_row, int64_t out_tok, float* lse, hipStream_t s) {
    (void)ws;
    ProfScope prof(TABED_K_BODY, s);
    NodesAttnArgs a{paged_view(c, layer), N, q_heads, q_heads / c.kv_heads, c.head_dim, q, out, lse, q_row, q_tok, out_row, out_tok,
                    ctx_len, parents, n_nodes, scale};
    const dim3 grid((unsigned)((N * q_heads + 3) / 4), rows);
    if (c.type == 2) launch(&prof, k_attention_nodes_simple<true>, grid, dim3(256), 0, s, a);
    else launch(&prof, k_attention_nodes_simple<false>, grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace tabed
