// Attention of a tree's nodes over the paged cache: the kernel, for one head dimension, and the launch of its variants.
//
//   s_t = scale q k_t,  o = sum_t exp(s_t - m) v_t / sum_t exp(s_t - m)     over the context, the nodes above and the node itself
//
// One pass over the keys and values with the running maximum m and sum.  The queries of a row that read one key / value head, N * group of them, go
// together: every entry of the cache then comes from memory once for up to 64 * WQ queries.
//
// Products are of 16 x 16 x 32 (bf16), turned so that nothing has to be transposed in registers: S^T = K Q^T has a query in a lane's column and four
// tokens in its rows, which is, two 16-token tiles side by side, how P^T is taken as the column operand of O^T = V^T P^T; the 32 tokens of that product are
// numbered (group of 16 lanes, tile, row), and V's fragments are read in that order, transposed on the way out of LDS.
//
// Tiles of KT tokens go from memory straight to LDS, where a row's 16-byte pieces lie in another order in every row, so that fragments are
// read without conflicts.  With few queries (WQ = 1) a wave has tiles, and LDS, of its own: four waves take every fourth tile of the range, nothing in
// the loop waits for another wave, and their results meet in LDS at the end.  With many, WQ waves share a tile, one barrier a tile.
//
// The cache's bytes bound it with few queries, the matrix cores and the softmax between the products with many.
#pragma once
#include <algorithm>
#include <mutex>
#include <type_traits>

#include "internal.h"
#include "lmhead_store.h"
#include "nodes.h"
#include "q8_utils.h"

namespace tabed {

struct NodesAttnArgs {
    PagedView c;
    int rows, N, q_heads, group, tiles;                                  // tiles of queries of a row and key / value head
    int slots, split, target, min_tiles;                                 // ranges of keys: see k_attention_nodes
    const uint16_t* q;
    uint16_t* out;
    float* lse;
    int64_t q_row, q_tok, out_row, out_tok;
    const int32_t* ctx_len;
    const int32_t* parents;
    const int32_t* n_nodes;
    float scale2;                                                        // scale * log2(e)
    int2* ranges;                                                        // [rows] first slot and number of ranges
    float2* ml;
    float* o;
};

// The 16-byte pieces of a tile's row stand in the order piece ^ turn(row).  Read are, in one go, 16 rows' pieces of one number (keys), and the pairs of
// pieces that hold 16 dims of 8 rows (values); e4m3: the pieces of 16 rows, rows 8 to 15 of a tile being tokens 16 on for the values.
template <int HD, bool F8>
__device__ __forceinline__ int turn_k(int row) {
    constexpr int kPieces = HD * (F8 ? 1 : 2) / 16;
    if constexpr (kPieces >= 16) return row & 15;
    else if constexpr (kPieces == 8) return row >> 1 & 7;
    else if constexpr (kPieces == 4 || kPieces == 12) return row >> 2 & 3;
    else return row >> 3 & 1;                                            // 2, 6
}
template <int HD, bool F8>
__device__ __forceinline__ int turn_v(int row) {
    constexpr int kPieces = HD * (F8 ? 1 : 2) / 16;
    if constexpr (!F8) {
        if constexpr (kPieces >= 16) return (row & 7) * 2;
        else if constexpr (kPieces == 8) return (row >> 1 & 3) * 2;
        else return (row >> 2 & 1) * 2;                                  // 4, 12
    } else {
        if constexpr (kPieces == 16) return (row & 7) | (row >> 4 & 1) * 8;
        else if constexpr (kPieces == 8) return (row >> 1 & 3) | (row >> 4 & 1) * 4;
        else if constexpr (kPieces == 4) return (row >> 2 & 1) | (row >> 4 & 1) * 2;
        else return row >> 4 & 1;                                        // 2, 6
    }
}

// N loads of a wave, 1024 bytes of LDS each, from `lds` on.
template <int N>
__device__ __forceinline__ void dma_pieces(const char* base, const uint32_t (&off)[N], uint32_t lds) {
    if constexpr (N == 1 || N == 2 || N == 4) {
        dma_lines(base, off, lds, 1024u);
    } else {
        constexpr int H = N >= 8 ? 4 : N > 4 ? 4 : 2;
        uint32_t a[H], b[N - H];
#pragma unroll
        for (int i = 0; i < H; ++i) a[i] = off[i];
#pragma unroll
        for (int i = H; i < N; ++i) b[i - H] = off[i];
        dma_lines(base, a, lds, 1024u);
        dma_pieces(base, b, lds + H * 1024u);
    }
}
// 64 words, one from each lane's address.
__device__ __forceinline__ void dma_words(const float* from, uint32_t lds) {
    uint32_t m0;
    asm volatile("s_mov_b32 %0, m0\n\ts_nop 4\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %2, off\n\ts_mov_b32 m0, %0"
                 : "=&s"(m0) : "s"(lds), "v"(from) : "memory");
}

// An address that all lanes have, in scalar registers.
__device__ __forceinline__ const char* uniform(const char* p) {
    const uint64_t v = (uint64_t)(uintptr_t)p;
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
    return reinterpret_cast<const char*>((uintptr_t)((uint64_t)hi << 32 | lo));
}

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));

__device__ __forceinline__ bf16x8 widen_e4m3(uint32_t lo, uint32_t hi) {
    union {
        bf16x8 v;
        bf16x2v p[4];
    } u;
    u.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false);
    u.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true);
    u.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false);
    u.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true);
    return u.v;
}

template <int HD_, bool F8_, int QW_, int WQ_, int WK_, int KT_, int NST_>
struct NodesVariant {
    static constexpr int HD = HD_, QW = QW_, WQ = WQ_, WK = WK_, KT = KT_, NST = NST_;
    static constexpr bool F8 = F8_;
    static constexpr int kWaves = WQ * WK, kThreads = kWaves * 64, kQueries = QW * 16 * WQ;
    static constexpr int kRow = HD * (F8 ? 1 : 2), kPieces = kRow / 16, kTile = KT * kRow;        // bytes of a row, its pieces, bytes of a tile
    static constexpr int kScales = F8 ? KT * 8 : 0;                                               // of keys and values
    static constexpr int kStage = 2 * kTile + (F8 ? (kScales + 1023) / 1024 * 1024 : 0);
    static constexpr int kLoads = kTile / 1024 / WQ;                                              // of a wave, for keys and for values each
    static constexpr int kAll = 2 * kLoads + (F8 ? KT / 32 : 0);
    static_assert(kTile % (1024 * WQ) == 0 && (KT == 32 || KT == 64) && NST <= 3);
    static constexpr size_t kJoin = WK > 1 ? (size_t)WK * kQueries * (HD + 4) * 4 + WK * kQueries * 8 : 0;
    static constexpr size_t kLds = std::max((size_t)WK * NST * kStage, kJoin) + TABED_MAX_NODES * 8 * kNodeWords;
};

// What a partial result (its maximum and sum) counts for in one with maximum m.  One that has seen something counts, so that an infinite value in it stays;
// one that has seen a NaN and nothing else has no maximum.
__device__ __forceinline__ float share(float2 ml, float m) {
    if (ml.x == -INFINITY) return ml.y == ml.y ? 0.f : 1.f;
    const float f = __builtin_amdgcn_exp2f(ml.x - m);
    return f < 1e-37f ? 1e-37f : f;
}

// Ranges of keys.  Where there are fewer (row, head, tile of queries) than workgroups that run at a time, every row's keys are cut into ranges of about the
// same number of tiles for all rows, as many as there is room for: all workgroups work this out from the rows' lengths, and each takes the range
// its number falls on.  A row of one range is finished by its workgroup; others' results are joined by a second launch.
template <class T>
__global__ __launch_bounds__(T::kThreads, 2) void k_attention_nodes(NodesAttnArgs a) {
    constexpr int HD = T::HD, QW = T::QW, WQ = T::WQ, WK = T::WK, KT = T::KT, NST = T::NST, RT = KT / 16, KS = HD / 32, DT = HD / 16;
    constexpr bool F8 = T::F8;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    uint64_t(*const s_mask)[kNodeWords] = reinterpret_cast<uint64_t(*)[kNodeWords]>(lds + T::kLds - TABED_MAX_NODES * 8 * kNodeWords);
    __shared__ int s_pick[4], s_sum[T::kWaves], s_up[TABED_MAX_NODES];
    __shared__ double s_whole[T::kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, grp = lane >> 4;
    const int wq = wave % WQ, wk = wave / WQ;

    // Workgroup w goes to XCD w % 8: the tiles of queries that read the same keys run back to back on one.
    const int xcd = blockIdx.x & 7, at = blockIdx.x >> 3, tile_q = at % a.tiles, unit = at / a.tiles * 8 + xcd;
    const int kvh = unit % a.c.kv_heads, slot = unit / a.c.kv_heads;
    if (slot >= a.slots) return;                                         // uniform: the grid is padded to whole rounds of XCDs
    int r = slot, range = 0, ranges = 1;
    auto tiles_of = [&](int row) {
        const int n = nodes_of(a.n_nodes, row, a.N);
        const int64_t end = min((int64_t)context_of(a.ctx_len, row) + n, (int64_t)a.c.max_blocks * TABED_CACHE_BLOCK);
        return n > 0 ? (int)((end + KT - 1) / KT) : 0;
    };
    if (a.split) {
        double whole = 0.0;
        for (int row = tid; row < a.rows; row += T::kThreads) whole += tiles_of(row);
        whole = wave_sum(whole);
        if (lane == 0) s_whole[wave] = whole;
        if (tid < 4) s_pick[tid] = -1;
        __syncthreads();
        whole = 0.0;
#pragma unroll
        for (int w = 0; w < T::kWaves; ++w) whole += s_whole[w];
        const int per = max(a.min_tiles, (int)fmin(ceil(whole / a.target), 1e9));
        auto ranges_of = [&](int row) { return max(1, (tiles_of(row) + per - 1) / per); };
        int before = 0;                                                  // of the rows before those of this round
        for (int r0 = 0; r0 < a.rows; r0 += T::kThreads) {
            const int row = r0 + tid, n = row < a.rows ? ranges_of(row) : 0;
            const int incl = (int)wave_inclusive_scan((double)n);
            __syncthreads();
            if (lane == 63) s_sum[wave] = incl;
            __syncthreads();
            int base = before;
#pragma unroll
            for (int w = 0; w < T::kWaves; ++w) {
                if (w < wave) base += s_sum[w];
                before += s_sum[w];
            }
            const int first = base + incl - n;
            if (n > 0 && slot >= first && slot < first + n) {
                s_pick[0] = row;
                s_pick[1] = slot - first;
                s_pick[2] = n;
            }
        }
        __syncthreads();
        r = __builtin_amdgcn_readfirstlane(s_pick[0]);
        if (r < 0) return;
        range = __builtin_amdgcn_readfirstlane(s_pick[1]);
        ranges = __builtin_amdgcn_readfirstlane(s_pick[2]);
        if (range == 0 && kvh == 0 && tile_q == 0 && tid == 0) a.ranges[r] = make_int2(slot, ranges);
    }
    const int nodes = __builtin_amdgcn_readfirstlane(nodes_of(a.n_nodes, r, a.N)), queries = nodes * a.group, q0 = tile_q * T::kQueries + wq * QW * 16;
    if (tile_q * T::kQueries >= queries) return;
    const int ctx = __builtin_amdgcn_readfirstlane(context_of(a.ctx_len, r)), all_tiles = __builtin_amdgcn_readfirstlane(tiles_of(r));
    const int t_begin = (int)((int64_t)all_tiles * range / ranges), t_end = (int)((int64_t)all_tiles * (range + 1) / ranges);

    // ---- tiles of keys and values into LDS
    unsigned char* const area = lds + wk * NST * T::kStage;
    const uint32_t area0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)area;
    uint32_t ko[T::kLoads], vo[T::kLoads];
#pragma unroll
    for (int i = 0; i < T::kLoads; ++i) {
        const int p = (wq * T::kLoads + i) * 64 + lane, row = p / T::kPieces, piece = p % T::kPieces;
        const uint32_t line = (uint32_t)(row * a.c.tok_stride * (F8 ? 1 : 2));
        ko[i] = line + (uint32_t)(piece ^ turn_k<HD, F8>(row)) * 16;
        vo[i] = line + (uint32_t)(piece ^ turn_v<HD, F8>(row)) * 16;
    }
    // (A tile whose block is not there is read from block 0, and not seen.)
    // The table is read through the scalar cache: a vector load's wait would be one for the tiles on their way too.
    typedef const __attribute__((address_space(4))) int32_t* ScalarInts;
    const ScalarInts row_table = (ScalarInts)(uintptr_t)(a.c.table + (int64_t)r * a.c.max_blocks);
    auto block_of_tile = [&](int t) { return row_table[min(t * KT / TABED_CACHE_BLOCK, a.c.max_blocks - 1)]; };      // (tiles end with the table)
    uint32_t there = 0;                                                  // a bit a stage: its tile's block is one
    auto request = [&](int t, int stage, int entry) {
        const bool is = entry >= 0 && entry < a.c.blocks;
        const int block = is ? entry : 0, first = t * KT % TABED_CACHE_BLOCK;
        there = is ? there | 1u << stage : there & ~(1u << stage);
        const int64_t from = a.c.entry(a.c.layer, block, kvh, first) * (F8 ? 1 : 2);
        const uint32_t to = area0 + (uint32_t)(stage * T::kStage) + (uint32_t)(wq * T::kLoads * 1024);
        dma_pieces(uniform(a.c.k + from), ko, __builtin_amdgcn_readfirstlane(to));
        dma_pieces(uniform(a.c.v + from), vo, __builtin_amdgcn_readfirstlane(to + T::kTile));
        if constexpr (F8) {
            const int64_t se = a.c.scale_entry(a.c.layer, block, kvh, first);
            const uint32_t sc = area0 + (uint32_t)(stage * T::kStage + 2 * T::kTile);
            if constexpr (KT == 32) {
                dma_words((lane < 32 ? a.c.kscale : a.c.vscale) + se + (lane & 31), __builtin_amdgcn_readfirstlane(sc));
            } else {
                dma_words(a.c.kscale + se + lane, __builtin_amdgcn_readfirstlane(sc));
                dma_words(a.c.vscale + se + lane, __builtin_amdgcn_readfirstlane(sc + 256));
            }
        }
    };
    const int step = WK;
    const int t0 = t_begin + wk;
#pragma unroll
    for (int i = 0; i < NST - 1; ++i)
        if (t0 + i * step < t_end) request(t0 + i * step, i, block_of_tile(t0 + i * step));
    int entry = block_of_tile(t0 + (NST - 1) * step);                    // of the tile that is requested next

    // ---- while they come: the queries, and who sees whom
    bf16x8 qf[QW][KS];
    int my_node[QW];
#pragma unroll
    for (int b = 0; b < QW; ++b) {
        const int i = q0 + b * 16 + col;
        const bool live = i < queries;
        my_node[b] = live ? i / a.group : 0;
        const int head = kvh * a.group + (live ? i % a.group : 0);
        const uint16_t* from = a.q + r * a.q_row + my_node[b] * a.q_tok + (int64_t)head * HD + grp * 8;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const u32x4_e2 w = *reinterpret_cast<const u32x4_e2*>(from + ks * 32);
            u32x4b x;
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = live ? w[e] : 0u;
            qf[b][ks] = __builtin_bit_cast(bf16x8, x);
        }
    }
    // Who sees whom, by doubling: a node's mask takes in that of the first node above that it has not looked through, log2 of the depth times.
    if (a.parents == nullptr) {
        for (int j = tid; j < nodes; j += T::kThreads)
#pragma unroll
            for (int w = 0; w < kNodeWords; ++w) s_mask[j][w] = j >= 64 * w + 63 ? ~0ull : j < 64 * w ? 0ull : (2ull << (j - 64 * w)) - 1;
    } else {
        constexpr int PN = (TABED_MAX_NODES + T::kThreads - 1) / T::kThreads;
        uint64_t m[PN][kNodeWords], more[PN][kNodeWords];
        int up[PN], next[PN];
#pragma unroll
        for (int p = 0; p < PN; ++p) {
            const int j = p * T::kThreads + tid;
            up[p] = j < nodes ? parent_of(a.parents, r, j, a.N) : -1;
#pragma unroll
            for (int w = 0; w < kNodeWords; ++w) m[p][w] = j / 64 == w ? 1ull << (j & 63) : 0ull;
        }
        for (int left = nodes - 1;; left >>= 1) {
#pragma unroll
            for (int p = 0; p < PN; ++p) {
                const int j = p * T::kThreads + tid;
                if (j < nodes) {
                    s_up[j] = up[p];
#pragma unroll
                    for (int w = 0; w < kNodeWords; ++w) s_mask[j][w] = m[p][w];
                }
            }
            lds_barrier();
            if (left == 0) break;
#pragma unroll
            for (int p = 0; p < PN; ++p) {
                const int from = max(up[p], 0);
                next[p] = up[p] >= 0 ? s_up[from] : -1;
#pragma unroll
                for (int w = 0; w < kNodeWords; ++w) more[p][w] = up[p] >= 0 ? s_mask[from][w] : 0ull;
            }
            lds_barrier();
#pragma unroll
            for (int p = 0; p < PN; ++p) {
                up[p] = next[p];
#pragma unroll
                for (int w = 0; w < kNodeWords; ++w) m[p][w] |= more[p][w];
            }
        }
    }
    lds_barrier();

    f32x4b acc[QW][DT];
    float m_run[QW], l_run[QW];
#pragma unroll
    for (int b = 0; b < QW; ++b) {
        m_run[b] = -INFINITY;
        l_run[b] = 0.f;
#pragma unroll
        for (int d = 0; d < DT; ++d) acc[b][d] = f32x4b{0.f, 0.f, 0.f, 0.f};
    }

    const bool idle = q0 >= queries;                                     // a wave without queries only helps with the tiles
    bool odd_any = false;
    auto compute = [&](int t, int stage, auto masked) {
        if (idle) return;
        const unsigned char* const sk = area + stage * T::kStage;
        const unsigned char* const sv = sk + T::kTile;
        const float* const ss = reinterpret_cast<const float*>(sv + T::kTile);
        f32x4b s[QW][RT];
        // ---- S^T = K Q^T
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            const int row = i * 16 + col;
            const unsigned char* const line = sk + row * T::kRow;
            const int turn = turn_k<HD, F8>(row);
#pragma unroll
            for (int b = 0; b < QW; ++b) s[b][i] = f32x4b{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                bf16x8 kf;
                if constexpr (F8) {
                    const uint2 w = *reinterpret_cast<const uint2*>(line + ((ks * 2 + (grp >> 1)) ^ turn) * 16 + (grp & 1) * 8);
                    kf = widen_e4m3(w.x, w.y);
                } else {
                    kf = *reinterpret_cast<const bf16x8*>(line + ((ks * 4 + grp) ^ turn) * 16);
                }
#pragma unroll
                for (int b = 0; b < QW; ++b) s[b][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[b][ks], s[b][i], 0, 0, 0);
            }
        }
        // ---- scores in units of log2, what is not seen -inf
        uint64_t seen[QW];
        if constexpr (masked.value) {
            const int64_t j0 = (int64_t)t * KT - ctx;                    // the node that the tile's first token is
#pragma unroll
            for (int b = 0; b < QW; ++b) {
                uint64_t m = 0;
                const uint64_t* const mask = s_mask[my_node[b]];
                if (j0 <= -64) m = ~0ull;
                else if (j0 < 0) m = (mask[0] << -j0) | ((1ull << -j0) - 1);
                else if (j0 < TABED_MAX_NODES) {
                    const int w = (int)j0 >> 6, f = (int)j0 & 63;
                    m = mask[w] >> f;
                    if (f && w + 1 < kNodeWords) m |= mask[w + 1] << (64 - f);
                }
                seen[b] = there >> stage & 1 ? m : 0ull;
            }
        }
        float ps[QW][RT][4];
        f32x4b vs[RT];
        if constexpr (F8) {
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                const f32x4b k4 = *reinterpret_cast<const f32x4b*>(ss + i * 16 + grp * 4);
                vs[i] = *reinterpret_cast<const f32x4b*>(ss + KT + i * 16 + grp * 4);
#pragma unroll
                for (int b = 0; b < QW; ++b)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[b][i][e] = s[b][i][e] * k4[e];
            }
        }
#pragma unroll
        for (int b = 0; b < QW; ++b) {
            float top = -INFINITY;
#pragma unroll
            for (int i = 0; i < RT; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float x = s[b][i][e] * a.scale2;
                    if constexpr (masked.value) x = seen[b] >> (i * 16 + grp * 4 + e) & 1 ? x : -INFINITY;
                    s[b][i][e] = x;
                    top = fmaxf(top, x);
                }
            top = max_lanes16_32(top);
            // The maximum is raised only where it would be by more than 2^6: probabilities are relative to the one they were taken with, and no less exact.
            if (__any(top > m_run[b] + 6.f)) {
                const float next = fmaxf(m_run[b], top), fade = next == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run[b] - next);
                m_run[b] = next;
                l_run[b] *= fade;
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[b][d][e] *= fade;
            }
            const float base = m_run[b] == -INFINITY ? 0.f : m_run[b];
#pragma unroll
            for (int i = 0; i < RT; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float p = __builtin_amdgcn_exp2f(s[b][i][e] - base);
                    l_run[b] += p;
                    if constexpr (F8) {
                        p *= vs[i][e];
                        if constexpr (masked.value) p = seen[b] >> (i * 16 + grp * 4 + e) & 1 ? p : 0.f;
                    }
                    ps[b][i][e] = p;
                }
        }
        // ---- O^T += V^T P^T
        bool odd = false;                                                // values that are not finite: left out here, see below
#pragma unroll
        for (int h = 0; h < KT / 32; ++h) {
            bf16x8 pf[QW];
#pragma unroll
            for (int b = 0; b < QW; ++b) {
                const uint2 lo = pack_bf16x4(ps[b][2 * h][0], ps[b][2 * h][1], ps[b][2 * h][2], ps[b][2 * h][3]);
                const uint2 hi = pack_bf16x4(ps[b][2 * h + 1][0], ps[b][2 * h + 1][1], ps[b][2 * h + 1][2], ps[b][2 * h + 1][3]);
                pf[b] = __builtin_bit_cast(bf16x8, u32x4b{lo.x, lo.y, hi.x, hi.y});
            }
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                bf16x8 vf;
                if constexpr (F8) {
                    const int k = col >> 1, row = h * 32 + (k < 4 ? grp * 4 + k : 12 + grp * 4 + k);
                    auto from = (__attribute__((address_space(3))) i32x2*)(sv + row * T::kRow + (d ^ turn_v<HD, F8>(row)) * 16 + (col & 1) * 8);
                    i32x2 w = __builtin_amdgcn_ds_read_tr8_b64_v2i32(from);
                    if constexpr (masked.value) {
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const uint32_t x = (uint32_t)w[i], nan = ((x & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;     // bytes 0x7f and 0xff
                            odd |= nan != 0;
                            w[i] = (int)(x & ~((nan >> 7) * 255u));
                        }
                    }
                    vf = widen_e4m3((uint32_t)w[0], (uint32_t)w[1]);
                } else {
                    u32x4b x;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int row = h * 32 + i * 16 + grp * 4 + (col >> 2);
                        auto from = (__attribute__((address_space(3))) s16x4*)(sv + row * T::kRow + ((d * 2 + ((col & 3) >> 1)) ^ turn_v<HD, F8>(row)) * 16 + (col & 1) * 8);
                        const uint2 w = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(from));
                        x[2 * i] = w.x;
                        x[2 * i + 1] = w.y;
                    }
                    if constexpr (masked.value) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const bool lo = (x[i] & 0x7f80u) == 0x7f80u, hi = (x[i] & 0x7f800000u) == 0x7f800000u;
                            odd |= lo | hi;
                            x[i] &= (lo ? 0u : 0xffffu) | (hi ? 0u : 0xffff0000u);
                        }
                    }
                    vf = __builtin_bit_cast(bf16x8, x);
                }
#pragma unroll
                for (int b = 0; b < QW; ++b) acc[b][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[b], acc[b][d], 0, 0, 0);
            }
        }
        if constexpr (masked.value) odd_any |= odd;
    };

    // Tiles that all queries see to their end come first; from the first other one on (nodes, the end of the row, a block that is not there) every tile
    // goes by what is seen.  (One loop with both kinds in it has two sets of sums, and takes twice the registers for them.)
    int stage = 0, t = t0;
    auto arrive_tile = [&] {
        const int ahead = t + (NST - 1) * step;
        const bool more = ahead < t_end;
        const int to = stage == 0 ? NST - 1 : stage - 1;
        if constexpr (WQ == 1) {
            // (what was read of the stage that is filled now has arrived)
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            if (more) request(ahead, to, entry);
            entry = block_of_tile(ahead + step);
        }
        // This tile is there once no more is outstanding than was asked for behind it.
        constexpr int kBehind = WQ == 1 ? NST - 1 : NST - 2;
        const int left = min(kBehind, (t_end - 1 - t) / step);
        if (left <= 0) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        else if (left == 1) asm volatile("s_waitcnt vmcnt(%0)" :: "n"(T::kAll) : "memory");
        else asm volatile("s_waitcnt vmcnt(%0)" :: "n"(2 * T::kAll) : "memory");
        if constexpr (WQ > 1) {
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
            if (more) request(ahead, to, entry);
            entry = block_of_tile(ahead + step);
        }
    };
    auto next_tile = [&] {
        stage = stage + 1 == NST ? 0 : stage + 1;
        t += step;
    };
    while (t < t_end && (int64_t)(t + 1) * KT <= ctx && (there >> stage & 1)) {
        arrive_tile();
        compute(t, stage, std::false_type{});
        next_tile();
    }
    const int first_masked = t;
    // (Waves that share tiles meet once a tile, so all groups of them go on for as long as the first.)
    while (t - (WQ > 1 ? wk : 0) < t_end) {
        arrive_tile();
        if (t < t_end) compute(t, stage, std::true_type{});
        next_tile();
    }

    // ---- values that are not finite
    // 0 times such a value is NaN, so the products of tiles that not everybody sees are without them, and nodes that do see one get it added by itself at the end,
    // by a second look at those tiles.
    if (tid == 0) s_pick[3] = 0;
    __syncthreads();
    if (wq == 0 && lane == 0) s_sum[wk] = first_masked;
    if (odd_any) s_pick[3] = 1;
    __syncthreads();
    const bool odd_tiles = s_pick[3] != 0;
    auto add_odd = [&](int node, int dim, float (&o)[4]) {
        for (int t = t_begin; t < t_end; ++t) {
            const int entry = block_of_tile(t);
            if (t < s_sum[(t - t_begin) % WK] || entry < 0 || entry >= a.c.blocks) continue;
            for (int k = 0; k < KT; ++k) {
                const int64_t j = (int64_t)t * KT + k - ctx;
                if (j >= nodes || (j >= 0 && !(s_mask[node][j >> 6] >> (j & 63) & 1))) continue;
                const int64_t from = a.c.entry(a.c.layer, entry, kvh, t * KT % TABED_CACHE_BLOCK + k) + dim;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if constexpr (F8) {
                        if ((a.c.v[from + e] & 0x7f) == 0x7f) o[e] = __builtin_nanf("");
                    } else {
                        const uint16_t w = reinterpret_cast<const uint16_t*>(a.c.v)[from + e];
                        if ((w & 0x7f80) == 0x7f80) o[e] += __builtin_bit_cast(float, (uint32_t)w << 16);
                    }
                }
            }
        }
    };

    // ---- the waves' results, or this one's
#pragma unroll
    for (int b = 0; b < QW; ++b) l_run[b] = add_lanes16_32(l_run[b]);
    const int64_t place = ((int64_t)slot * a.c.kv_heads + kvh) * a.tiles + tile_q;
    auto finish = [&](int i, int dim, float m, float l, float (&o)[4], bool first) {             // i: query of the tile; four dims of it
        const int qi = tile_q * T::kQueries + i;
        if (qi >= queries) return;
        if (odd_tiles) add_odd(qi / a.group, dim, o);
        if (ranges > 1) {
            *reinterpret_cast<f32x4b*>(a.o + (place * T::kQueries + i) * HD + dim) = f32x4b{o[0], o[1], o[2], o[3]};
            if (first) a.ml[place * T::kQueries + i] = make_float2(m, l);
            return;
        }
        const int node = qi / a.group, head = kvh * a.group + qi % a.group;
        const float inv = l == 0.f ? 0.f : 1.f / l;
        const uint2 w = pack_bf16x4(o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
        typedef uint32_t u32x2_e2 __attribute__((ext_vector_type(2), aligned(2)));
        *reinterpret_cast<u32x2_e2*>(a.out + r * a.out_row + node * a.out_tok + (int64_t)head * HD + dim) = u32x2_e2{w.x, w.y};
        if (first && a.lse != nullptr)
            a.lse[((int64_t)r * a.N + node) * a.q_heads + head] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994530942f;
    };
    if constexpr (WK == 1) {
#pragma unroll
        for (int b = 0; b < QW; ++b)
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                float o[4] = {acc[b][d][0], acc[b][d][1], acc[b][d][2], acc[b][d][3]};
                finish(wq * QW * 16 + b * 16 + col, d * 16 + grp * 4, m_run[b], l_run[b], o, d == 0 && grp == 0);
            }
    } else {
        constexpr int kLine = HD + 4;
        __syncthreads();                                                 // all tiles have been read, none is on its way
        float* const s_o = reinterpret_cast<float*>(lds);
        float2* const s_ml = reinterpret_cast<float2*>(lds + (size_t)WK * T::kQueries * kLine * 4);
#pragma unroll
        for (int b = 0; b < QW; ++b) {
#pragma unroll
            for (int d = 0; d < DT; ++d) *reinterpret_cast<f32x4b*>(s_o + (size_t)(wk * T::kQueries + (wq * QW + b) * 16 + col) * kLine + d * 16 + grp * 4) = acc[b][d];
            if (grp == 0) s_ml[wk * T::kQueries + (wq * QW + b) * 16 + col] = make_float2(m_run[b], l_run[b]);
        }
        __syncthreads();
        for (int p = tid; p < T::kQueries * (HD / 4); p += T::kThreads) {
            const int i = p / (HD / 4), dim = p % (HD / 4) * 4;
            float m = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < WK; ++w) m = fmaxf(m, s_ml[w * T::kQueries + i].x);
#pragma unroll
            for (int w = 0; w < WK; ++w) {
                const float2 ml = s_ml[w * T::kQueries + i];
                const f32x4b x = *reinterpret_cast<const f32x4b*>(s_o + (size_t)(w * T::kQueries + i) * kLine + dim);
                const float f = share(ml, m);
                l += f == 0.f ? 0.f : ml.y * f;
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] += f == 0.f ? 0.f : x[e] * f;
            }
            finish(i, dim, m, l, o, dim == 0);
        }
    }
}

// Ranges joined: a wave a query, a lane every 64th pair of dims.
template <int HD>
__global__ __launch_bounds__(256) void k_attention_nodes_join(NodesAttnArgs a, int per_tile) {
    const int r = blockIdx.y, unit = blockIdx.x * 4 + threadIdx.x / 64, lane = threadIdx.x & 63;
    const int nodes = nodes_of(a.n_nodes, r, a.N), node = unit / a.q_heads, head = unit % a.q_heads;
    if (node >= nodes) return;
    const int2 got = a.ranges[r];
    const int ranges = got.y;
    if (ranges <= 1) return;
    const int kvh = head / a.group, qi = node * a.group + head % a.group, tile = qi / per_tile, i = qi % per_tile;
    auto place = [&](int s) { return (((int64_t)(got.x + s) * a.c.kv_heads + kvh) * a.tiles + tile) * per_tile + i; };
    float m = -INFINITY;
    for (int s = lane; s < ranges; s += 64) m = fmaxf(m, a.ml[place(s)].x);
    m = wave_max(m);
    constexpr int PL = (HD / 2 + 63) / 64;
    const bool mine = lane < HD / 2;
    float l = 0.f, o[PL][2] = {};
    for (int s0 = 0; s0 < ranges; s0 += 64) {
        float f = 0.f, lw = 0.f;
        if (s0 + lane < ranges) {
            const float2 ml = a.ml[place(s0 + lane)];
            f = share(ml, m);
            lw = f == 0.f ? 0.f : ml.y * f;
        }
        l += wave_sum(lw);
        const int some = min(64, ranges - s0);
        for (int s = 0; s < some; s += 8) {                              // (eight at a time in flight; past the last one its sums again, times 0)
            float2 x[8][PL];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float* from = a.o + place(s0 + min(s + i, some - 1)) * HD;
#pragma unroll
                for (int p = 0; p < PL; ++p) x[i][p] = *reinterpret_cast<const float2*>(from + (mine ? (p * 64 + lane) * 2 : 0));
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float fs = s + i < some ? lane_f32(f, s + i) : 0.f;
#pragma unroll
                for (int p = 0; p < PL; ++p) {
                    o[p][0] += fs == 0.f ? 0.f : x[i][p].x * fs;
                    o[p][1] += fs == 0.f ? 0.f : x[i][p].y * fs;
                }
            }
        }
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    uint16_t* out = a.out + r * a.out_row + node * a.out_tok + (int64_t)head * HD;
    if (mine) {
#pragma unroll
        for (int p = 0; p < PL; ++p) {
            out[(p * 64 + lane) * 2] = f32_to_bf16_bits(o[p][0] * inv);
            out[(p * 64 + lane) * 2 + 1] = f32_to_bf16_bits(o[p][1] * inv);
        }
    }
    if (lane == 0 && a.lse != nullptr)
        a.lse[((int64_t)r * a.N + node) * a.q_heads + head] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994530942f;
}

// ---------------------------------------------------------------- host side
struct NodesPlan {
    int queries, tiles, slots, split, target, min_tiles;                 // queries of a workgroup
};

template <class T>
hipError_t launch_nodes_variant(const ProfScope* prof, NodesAttnArgs a, hipStream_t s) {
    static std::once_flag once[kMaxDevices];
    static hipError_t rc[kMaxDevices];
    const hipError_t e = raise_on_device(&k_attention_nodes<T>, T::kLds, once, rc);
    if (e != hipSuccess) return e;
    const int64_t units = (int64_t)a.slots * a.c.kv_heads;
    launch(prof, k_attention_nodes<T>, dim3((unsigned)((units + 7) / 8 * 8 * a.tiles)), dim3(T::kThreads), T::kLds, s, a);
    if (a.split) hipLaunchKernelGGL((k_attention_nodes_join<T::HD>), dim3((unsigned)((a.N * a.q_heads + 3) / 4), a.rows), dim3(256), 0, s, a, T::kQueries);
    return hipGetLastError();
}

// The variants: 16 and 32 queries with tiles of their own for four waves, 64 with tiles that pairs of waves share, 128 and 256 with ones that four and eight share.
template <int HD, bool F8, typename F>
inline auto with_nodes_variant(int queries, F&& f) {
    constexpr bool kBig = HD == 256 && !F8;                              // (LDS)
    if (queries <= 16) return f(NodesVariant<HD, F8, 1, 1, kBig ? 2 : 4, 32, 2>{});
    if (queries <= 32) return f(NodesVariant<HD, F8, 2, 1, kBig ? 2 : 4, 32, 2>{});
    if constexpr (HD * (F8 ? 1 : 2) % 64 == 0) {
        if (queries <= 64) return f(NodesVariant<HD, F8, 2, 2, HD == 256 ? 2 : 4, 32, 2>{});
        if (queries <= 128 || HD * (F8 ? 1 : 2) % 128 != 0) return f(NodesVariant<HD, F8, 2, 4, 1, 64, kBig ? 2 : 3>{});
        return f(NodesVariant<HD, F8, 2, HD * (F8 ? 1 : 2) % 128 == 0 ? 8 : 4, 1, 64, kBig ? 2 : 3>{});
    } else {
        return f(NodesVariant<HD, F8, 2, 2, 4, 64, 2>{});
    }
}

#define TABED_NODES_HD(HD_)                                                                                                   \
    template <>                                                                                                               \
    hipError_t launch_nodes_hd<HD_>(bool f8, int queries, const ProfScope* prof, const NodesAttnArgs& a, hipStream_t s) {     \
        auto go = [&](auto v) { return launch_nodes_variant<decltype(v)>(prof, a, s); };                                      \
        return f8 ? with_nodes_variant<HD_, true>(queries, go) : with_nodes_variant<HD_, false>(queries, go);                 \
    }
template <int HD>
hipError_t launch_nodes_hd(bool f8, int queries, const ProfScope* prof, const NodesAttnArgs& a, hipStream_t s);

}  // namespace tabed
