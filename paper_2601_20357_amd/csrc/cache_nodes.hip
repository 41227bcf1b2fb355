// A tree's nodes into the paged cache (rotated, in bf16 or e4m3), and the accepted path's entries to where the context ends.
#include <hip/hip_runtime.h>

#include <cmath>

#include "nodes.h"
#include "nodes_launch.h"
#include "q8_utils.h"

namespace tabed {

constexpr int kAppendThreads = 256;

// ---------------------------------------------------------------- append
// x' = R(pos) x for queries and keys: pairs (i, i + hd/2) turn by pos * theta^(-2i/hd).  The angle is formed in 64 bits in revolutions, of
// which the fraction alone is kept: exact up to any position, and sine and cosine are then fp32's own.
// One workgroup a node: it finds the node's depth in the row's parents, makes the hd/2 sines and cosines once for all heads, and
// a thread then takes 8 dims from either half of a head.  Memory bounds it with many nodes (64 rows of 256 nodes, 32 / 8 heads of 128: 74 us, 5.4 TB/s;
// into e4m3 73), the trips length -> page -> entry with few: 64 rows of 24 8.4 us, one row of 6 3.4, of which the launch is most.
struct AppendArgs {
    PagedView c;
    int N, q_heads, hd;
    const void* k;
    const void* v;
    const void* q;
    uint16_t* q_out;
    int64_t kv_row, kv_tok, q_row, q_tok, out_row, out_tok;
    const int32_t* ctx_len;
    const int32_t* parents;
    const int32_t* n_nodes;
    double log2_theta;
    int rotate;
};

__device__ __forceinline__ void store_bf16x8(uint16_t* p, const float (&x)[8]) {
    const uint2 a = pack_bf16x4(x[0], x[1], x[2], x[3]), b = pack_bf16x4(x[4], x[5], x[6], x[7]);
    *reinterpret_cast<u32x4_e2*>(p) = u32x4_e2{a.x, a.y, b.x, b.y};
}

// Eight values in steps of e4m3, the largest 448: the division as fp32 rounds it, then to even.
__device__ __forceinline__ uint2 to_e4m3x8(const float (&x)[8], float scale) {
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = scale > 0.f ? fminf(fmaxf(x[e] / scale, -448.f), 448.f) : 0.f;
    uint2 w;
    int lo = 0, hi = 0;
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], lo, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], hi, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], hi, true);
    w.x = (uint32_t)lo;
    w.y = (uint32_t)hi;
    return w;
}

// The scale of a token in a head (e4m3): 1/448 of its largest magnitude, as scale_of for int8.
__device__ __forceinline__ float scale_e4m3(uint32_t bits) {
    const float most = __builtin_bit_cast(float, bits);
    return bits >= kInfBits ? __builtin_nanf("") : most >= kTiny ? most / 448.f : 0.f;
}

template <bool F8, bool BF16>
__global__ __launch_bounds__(kAppendThreads) void k_append_nodes(AppendArgs a) {
    const int j = blockIdx.x, r = blockIdx.y, tid = threadIdx.x;
    __shared__ int s_parent[TABED_MAX_NODES];
    __shared__ float2 s_turn[128];                                       // cos, sin of the hd/2 angles
    if (j >= nodes_of(a.n_nodes, r, a.N)) return;
    const int ctx = context_of(a.ctx_len, r);
    const int half = a.hd / 2;
    if (a.rotate) {
        int depth = j;
        if (a.parents != nullptr) {
            for (int i = tid; i <= j; i += kAppendThreads) s_parent[i] = parent_of(a.parents, r, i, a.N);
            __syncthreads();
            depth = 0;
            for (int p = s_parent[j]; p >= 0; p = s_parent[p]) ++depth;
        }
        if (tid < half) {
            const double turns = ((double)ctx + depth) * exp2(-2.0 * tid / a.hd * a.log2_theta) * 0.15915494309189533577;
            const float part = (float)(2.0 * (turns - rint(turns)));
            float sn, cs;
            sincospif(part, &sn, &cs);
            s_turn[tid] = make_float2(cs, sn);
        }
        __syncthreads();
    }
    const int per = half / 8, lanes = per <= 2 ? 2 : per <= 4 ? 4 : per <= 8 ? 8 : 16;     // threads of a head (96 dims: 6 of 8)
    const int part = tid % lanes;
    const int64_t pos = (int64_t)ctx + j;
    const int block = a.c.block_of(r, pos), slot = (int)(pos % TABED_CACHE_BLOCK);
    for (int h = tid / lanes; h < a.q_heads + 2 * a.c.kv_heads; h += kAppendThreads / lanes) {
        const bool is_q = h < a.q_heads, is_v = h >= a.q_heads + a.c.kv_heads;
        const int head = is_q ? h : is_v ? h - a.q_heads - a.c.kv_heads : h - a.q_heads;
        const void* src = is_q ? a.q : is_v ? a.v : a.k;
        const int64_t at = (is_q ? r * a.q_row + j * a.q_tok : r * a.kv_row + j * a.kv_tok) + (int64_t)head * a.hd + part * 8;
        float x[8], y[8];
        const bool live = part < per;
        uint32_t most = 0;
        if (live) {
            load_values<8, BF16>(src, at, x);
            load_values<8, BF16>(src, at + half, y);
            if (!is_v && a.rotate) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float2 t = s_turn[part * 8 + e];
                    const float lo = x[e] * t.x - y[e] * t.y, hi = x[e] * t.y + y[e] * t.x;
                    x[e] = lo;
                    y[e] = hi;
                }
            }
            if (is_q) {
                uint16_t* to = a.q_out + r * a.out_row + j * a.out_tok + (int64_t)head * a.hd + part * 8;
                store_bf16x8(to, x);
                store_bf16x8(to + half, y);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) most = max(most, max(magnitude(x[e]), magnitude(y[e])));
        }
        char* pool = is_v ? a.c.v : a.c.k;
        if constexpr (!F8) {
            if (live && !is_q && block >= 0) {
                uint16_t* to = reinterpret_cast<uint16_t*>(pool) + a.c.entry(a.c.layer, block, head, slot) + part * 8;
                store_bf16x8(to, x);
                store_bf16x8(to + half, y);
            }
        } else {
            // (all threads of a head's group are here: a group is 2 to 16 lanes of one wave)
            for (int m = 1; m < lanes; m <<= 1) most = max(most, (uint32_t)__shfl_xor((int)most, m));
            if (live && !is_q && block >= 0) {
                const float scale = scale_e4m3(most);
                char* to = pool + a.c.entry(a.c.layer, block, head, slot) + part * 8;
                *reinterpret_cast<uint2*>(to) = to_e4m3x8(x, scale);
                *reinterpret_cast<uint2*>(to + half) = to_e4m3x8(y, scale);
                if (part == 0) (is_v ? a.c.vscale : a.c.kscale)[a.c.scale_entry(a.c.layer, block, head, slot)] = scale;
            }
        }
    }
}

hipError_t launch_append_nodes(const tabed_cache_paged& c, int layer, int rows, int N, int dtype, const void* k, const void* v, int64_t kv_row,
                               int64_t kv_tok, int q_heads, const void* q, int64_t q_row, int64_t q_tok, void* q_out, int64_t out_row, int64_t out_tok,
                               const int32_t* ctx_len, const int32_t* parents, const int32_t* n_nodes, float rope_theta, hipStream_t s) {
    ProfScope prof(TABED_K_BODY, s);
    AppendArgs a{paged_view(c, layer), N, q != nullptr ? q_heads : 0, c.head_dim, k, v, q, static_cast<uint16_t*>(q_out), kv_row, kv_tok, q_row, q_tok,
                 out_row, out_tok, ctx_len, parents, n_nodes, rope_theta > 0.f ? std::log2((double)rope_theta) : 0.0, rope_theta > 0.f};
    const dim3 grid(N, rows), block(kAppendThreads);
    if (c.type == 2) {
        if (dtype == 1) launch(&prof, k_append_nodes<true, true>, grid, block, 0, s, a);
        else launch(&prof, k_append_nodes<true, false>, grid, block, 0, s, a);
    } else {
        if (dtype == 1) launch(&prof, k_append_nodes<false, true>, grid, block, 0, s, a);
        else launch(&prof, k_append_nodes<false, false>, grid, block, 0, s, a);
    }
    return hipGetLastError();
}

// ---------------------------------------------------------------- keep
// Path entries ascend, so path[i] >= i: no entry comes from a place that an earlier one went to.  A workgroup moves one row's entries in one
// layer and head, as many at a time as its threads hold; those are read before the first of them is written, and later ones come from behind.  All layers go in one
// launch, as the path is known when the round is over: 32 rows, 12 layers of 8 heads of 128, up to 7 entries 4.9 us; one row of 2 layers 2.6; the trips path -> page ->
// entry are what it takes.
constexpr int kKeepThreads = 256;

struct KeepArgs {
    PagedView c;
    int N, piece;                                                        // 16-byte pieces of an entry
    const int32_t* ctx_base;
    const int32_t* path;
    const int32_t* n_path;
    int32_t* ctx_len;
};

template <bool F8>
__global__ __launch_bounds__(kKeepThreads) void k_keep_nodes(KeepArgs a) {
    const int h = blockIdx.x % a.c.kv_heads, layer = blockIdx.x / a.c.kv_heads, r = blockIdx.y, tid = threadIdx.x;
    __shared__ int s_path[TABED_MAX_NODES], s_count;
    __shared__ int64_t s_from[TABED_MAX_NODES], s_to[TABED_MAX_NODES];   // entries, -1: not moved
    __shared__ int64_t s_sfrom[TABED_MAX_NODES], s_sto[TABED_MAX_NODES]; // and their scales
    const int ctx = context_of(a.ctx_base, r), said = min(max(a.n_path[r], 0), a.N);
    if (tid == 0) s_count = said;
    if (tid < said) s_path[tid] = a.path[(size_t)r * a.N + tid];
    __syncthreads();
    if (tid < said) {
        const int p = s_path[tid];
        if (p < 0 || p >= a.N || (tid > 0 && p <= s_path[tid - 1])) atomicMin(&s_count, tid);
    }
    __syncthreads();
    const int count = s_count;
    if (blockIdx.x == 0 && tid == 0) a.ctx_len[r] = ctx + count;
    if (tid < count) {
        const int64_t from = (int64_t)ctx + s_path[tid], to = (int64_t)ctx + tid;
        const int bf = a.c.block_of(r, from), bt = a.c.block_of(r, to);
        const bool moves = from != to && bf >= 0 && bt >= 0;
        s_from[tid] = moves ? a.c.entry(layer, bf, h, (int)(from % TABED_CACHE_BLOCK)) : -1;
        s_to[tid] = moves ? a.c.entry(layer, bt, h, (int)(to % TABED_CACHE_BLOCK)) : -1;
        if constexpr (F8) {
            s_sfrom[tid] = moves ? a.c.scale_entry(layer, bf, h, (int)(from % TABED_CACHE_BLOCK)) : -1;
            s_sto[tid] = moves ? a.c.scale_entry(layer, bt, h, (int)(to % TABED_CACHE_BLOCK)) : -1;
        }
    }
    __syncthreads();
    constexpr int kBytes = F8 ? 1 : 2;
    const int at_once = kKeepThreads / a.piece;                          // entries: 256 threads hold 8 of 512 bytes, 128 of 32
    for (int i0 = 0; i0 < count; i0 += at_once) {
        const int i = i0 + tid / a.piece, part = tid % a.piece;
        const bool mine = tid / a.piece < at_once && i < count && s_from[i] >= 0;
        u32x4b k, v;
        float ks = 0.f, vs = 0.f;
        if (mine) {
            k = *reinterpret_cast<const u32x4b*>(a.c.k + s_from[i] * kBytes + part * 16);
            v = *reinterpret_cast<const u32x4b*>(a.c.v + s_from[i] * kBytes + part * 16);
            if (F8 && part == 0) { ks = a.c.kscale[s_sfrom[i]]; vs = a.c.vscale[s_sfrom[i]]; }
        }
        publish_barrier();                                               // all loads have arrived
        if (mine) {
            *reinterpret_cast<u32x4b*>(a.c.k + s_to[i] * kBytes + part * 16) = k;
            *reinterpret_cast<u32x4b*>(a.c.v + s_to[i] * kBytes + part * 16) = v;
            if (F8 && part == 0) { a.c.kscale[s_sto[i]] = ks; a.c.vscale[s_sto[i]] = vs; }
        }
    }
}

hipError_t launch_keep_nodes(const tabed_cache_paged& c, int rows, int N, const int32_t* ctx_base, const int32_t* path, const int32_t* n_path,
                             int32_t* ctx_len, hipStream_t s) {
    ProfScope prof(TABED_K_BODY, s);
    KeepArgs a{paged_view(c, 0), N, c.head_dim * (c.type == 2 ? 1 : 2) / 16, ctx_base, path, n_path, ctx_len};
    const dim3 grid((unsigned)(c.kv_heads * c.layers), rows), block(kKeepThreads);
    if (c.type == 2) launch(&prof, k_keep_nodes<true>, grid, block, 0, s, a);
    else launch(&prof, k_keep_nodes<false>, grid, block, 0, s, a);
    return hipGetLastError();
}

}  // namespace tabed
