// Attention of a tree's nodes over the paged cache: the kernels, for one head dimension, and the launch of their variants.
//
//   s_t = scale q k_t,  o = sum_t exp(s_t - m) v_t / sum_t exp(s_t - m)     over the context, the nodes above and the node itself
//
// One pass over the keys and values with the running maximum m and sum.  The queries of a row that read one key / value head, N * group of them, go
// together: an entry of the cache comes from memory once for up to 128 queries.
//
// Products are of 16 x 16 x 32, turned so that nothing has to be transposed in registers: S^T = K Q^T has a query in a lane's column and four
// tokens in its rows, which is, two 16-token halves side by side, how P^T is taken as the column operand of O^T = V^T P^T; the 32 tokens of that product are
// numbered (group of 16 lanes, half, row), and V's fragments are read in that order, transposed on the way out of LDS.
//
// Keys and values go from memory straight to LDS, where a row's 16-byte pieces lie in another order in every row, so that fragments are
// read without conflicts.  Up to 32 queries (k_attention_nodes): a wave has tiles of 32 tokens, and LDS, of its own: the waves take every WK-th tile of a range,
// nothing in the loop waits for another wave, and their results meet in LDS at the end.  More (k_attention_nodes_wide): four waves share a tile, one
// barrier a tile; 1, 2 or 4 of them, as the row's own number of nodes has it, take different queries, and those with the same ones take turns at steps of 64 tokens.
//
// The cache's bytes bound it with few queries: 1 row of 120011 tokens, 32 / 8 heads of 128, one node 93 us (5.3 TB/s), 16 nodes 110; 64 rows of 256 to 768, 12 heads of
// 64, 16 nodes 25 (4.2 TB/s).  With many the matrix cores and the softmax between the products do: 8 rows of 10000 tokens, 256 nodes, 32 / 8 heads of 128 434 us
// (780 TFLOP/s; matrix cores 46 % of the cycles, vector instructions nearly all others, which two waves a SIMD overlap little), in e4m3 527 (every wave widens the
// tile's values for its own queries: 300 more vector instructions a step of 64 tokens).
#pragma once
#include <algorithm>
#include <mutex>
#include <type_traits>

#include "launch_utils.h"
#include "lmhead_store.h"
#include "nodes.h"
#include "nodes_launch.h"
#include "q8_utils.h"

namespace tabed {

struct NodesAttnArgs {
    PagedView c;
    int rows, N, q_heads, group, tiles, per_tile;                        // tiles of queries of a row and key / value head, queries of a tile
    int slots, split, fill, min_tiles, whole_tiles;                      // ranges of keys, see find_range
    const uint16_t* q;
    uint16_t* out;
    float* lse;
    int64_t q_row, q_tok, out_row, out_tok;
    const int32_t* ctx_len;
    const int32_t* parents;
    const int32_t* n_nodes;
    float scale2;                                                        // scale * log2(e)
    int2* ranges;                                                        // [rows] first slot and number of ranges
    float4* ml;
    float* o;
};

constexpr int kNodesTile = 32;                                           // tokens of a step of a wave
constexpr int kMaskBytes = TABED_MAX_NODES * 8 * kNodeWords;

// The 16-byte pieces of a row in LDS stand in the order piece ^ turn(row).  Read are, in one go, 16 rows' pieces of one number (keys), and the pairs of
// pieces that hold 16 dims of 8 rows (values); e4m3: the pieces of 16 rows, rows 8 to 15 of which are 16 tokens on for the values.
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
        constexpr int H = N > 4 ? 4 : 2;
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
__device__ __forceinline__ uint32_t lds_address(const void* p) { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p; }

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2v __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2v __attribute__((ext_vector_type(2)));

// Eight e4m3 values, which both 16-bit types hold exactly.
__device__ __forceinline__ bf16x8 widen_bf16(uint32_t lo, uint32_t hi) {
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
__device__ __forceinline__ f16x8 widen_f16(uint32_t lo, uint32_t hi) {
    union {
        f16x8 v;
        f16x2v p[4];
    } u;
    u.p[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, false);
    u.p[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, true);
    u.p[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, false);
    u.p[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, true);
    return u.v;
}

// The 64 nodes from j0 on of a mask, what comes before the nodes seen by all.
__device__ __forceinline__ uint64_t window(const uint64_t* mask, int64_t j0) {
    if (j0 <= -64) return ~0ull;
    if (j0 < 0) return (mask[0] << -j0) | ((1ull << -j0) - 1);
    if (j0 >= TABED_MAX_NODES) return 0ull;
    const int w = (int)j0 >> 6, f = (int)j0 & 63;
    uint64_t m = mask[w] >> f;
    if (f > 0 && w + 1 < kNodeWords) m |= mask[w + 1] << (64 - f);
    return m;
}

// What a step of 32 or 64 tokens is: kWhole, all queries see all of them; kMasked, who sees them is in a mask; kFar (e4m3), kWhole with products that fp16 does not hold.
enum NodesStep { kWhole, kFar, kMasked };
template <NodesStep MODE>
using NodesMode = std::integral_constant<NodesStep, MODE>;

// ---------------------------------------------------------------- a wave's queries, 16 * QW of them, and what they have seen
template <int HD, bool F8, int QW>
struct NodesWave {
    static constexpr int KS = HD / 32, DT = HD / 16, kRow = HD * (F8 ? 1 : 2);
    bf16x8 qf[QW][KS];
    int node[QW];
    f32x4b acc[QW][DT];
    f32x4b rounded[QW];                                                  // bf16: sums of the probabilities as they are rounded
    float m[QW], l[QW];                                                  // what probabilities are relative to (log2), and their sums
    bool odd;                                                            // some value was not finite, and left out

    __device__ __forceinline__ void begin(const NodesAttnArgs& a, int r, int kvh, int q0, int queries) {
        const int col = threadIdx.x & 15, grp = threadIdx.x >> 4 & 3;
#pragma unroll
        for (int b = 0; b < QW; ++b) {
            const int i = q0 + b * 16 + col;
            const bool live = i < queries;
            node[b] = live ? i / a.group : 0;
            const int head = kvh * a.group + (live ? i % a.group : 0);
            const uint16_t* from = a.q + r * a.q_row + node[b] * a.q_tok + (int64_t)head * HD + grp * 8;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const u32x4_e2 w = *reinterpret_cast<const u32x4_e2*>(from + ks * 32);
                u32x4b x;
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = live ? w[e] : 0u;
                qf[b][ks] = __builtin_bit_cast(bf16x8, x);
            }
            m[b] = -INFINITY;
            l[b] = 0.f;
            rounded[b] = f32x4b{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int d = 0; d < DT; ++d) acc[b][d] = f32x4b{0.f, 0.f, 0.f, 0.f};
        }
        odd = false;
    }

    // RT halves of 16 tokens: their rows of keys and values, and scales.  seen: a bit a token for each query, of kMasked steps.
    // False, with nothing taken, where a step is not kWhole but kFar.
    template <NodesStep MODE, int RT, typename Seen>
    __device__ __forceinline__ bool step(const unsigned char* sk, const unsigned char* sv, const float* kscale, const float* vscale, float scale2,
                                         const Seen (&seen)[QW]) {
        constexpr bool MASKED = MODE == kMasked, F16 = F8 && MODE != kFar;
        static_assert(F8 || MODE != kFar);
        static_assert(!MASKED || sizeof(Seen) * 8 >= RT * 16);
        const int col = threadIdx.x & 15, grp = threadIdx.x >> 4 & 3;
        f32x4b s[QW][RT];
        __builtin_amdgcn_s_setprio(1);                                   // (the other wave's softmax fills what the products leave: 1 to 3 % with many queries)
        // ---- S^T = K Q^T
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            if (i > 0 && i % 2 == 0) __builtin_amdgcn_sched_barrier(0);          // (64 tokens' fragments at once are more than there are registers)
            const unsigned char* const line = sk + col * kRow + i * 16 * kRow;    // (a row's turn goes by its number in 16, or 32, alone)
            const int turn = turn_k<HD, F8>(col);
#pragma unroll
            for (int b = 0; b < QW; ++b) s[b][i] = f32x4b{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                bf16x8 kf;
                if constexpr (F8) {
                    const uint2 w = *reinterpret_cast<const uint2*>(line + ((ks * 2 + (grp >> 1)) ^ turn) * 16 + (grp & 1) * 8);
                    kf = widen_bf16(w.x, w.y);
                } else {
                    kf = *reinterpret_cast<const bf16x8*>(line + ((ks * 4 + grp) ^ turn) * 16);
                }
#pragma unroll
                for (int b = 0; b < QW; ++b) s[b][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[b][ks], s[b][i], 0, 0, 0);
            }
        }
        __builtin_amdgcn_s_setprio(0);
        f32x4b vs[RT], ks2[RT], size[RT];
        auto sees = [&](int b, int i, int e) { return (seen[b] >> (i * 16 + grp * 4 + e) & 1) != 0; };
        // e4m3: what is multiplied with the values is probability times scale, and scales can be anything.  So what probabilities are relative to is a power of two that follows
        // the largest of these products, for every query by what it sees itself: 2^8 when it is chosen and up to 2^15 before it is chosen anew.  fp16 then holds products to 2^-11 of
        // themselves down to 2^-14 and to 2^-8 down to 2^-17.  A step with smaller ones, or with a scale outside 2^-38 to 2^38, is kFar: products in bf16, to 2^-8 whatever they are.
        // From there on a wave's steps are, up to the kMasked ones: in these, what others see must not count, and each product goes by itself, in fp16 or in bf16.
        // (One power of two a wave, by the largest scale that any of its queries saw, let a sibling's entry, or one that hardly counts, take all precision from the others.  It was
        // a little faster: 16 ragged trees of up to 33 nodes 78.5 us for 79.0; with scores of four times the spread, where steps are kFar, 80 for 84; heads of 256 dims, 4 rows of 3000, 64
        // nodes, 32 / 8 heads 72 for 76.)
        // For that choice scales count as 2^-40 to 2^38, so that the largest probability is in 2^-32 to 2^65: the sum of them is none of tiny ones, and products with tiny scales are there.
        constexpr float kRaise = MODE == kFar ? 25.f : 15.f, kLow = -16.9f;      // (fp16 ends at 2^15.99)
        bool apart = false;                                              // kMasked: there may be products for bf16; kWhole: the step is kFar
        float big = 0.f, little = 0.f;                                   // kWhole: log2 of the largest and the smallest scale of this lane's tokens
        // log2 of a scale, at most 0.09 too low: the exponent, and the mantissa as if it were linear, from the bits as 2^23 + bits / 2^9.
        auto log2_of = [](float v) {
            return fmaf(__builtin_bit_cast(float, __builtin_amdgcn_alignbit(0x96u, __builtin_bit_cast(uint32_t, v), 9u)), 0x1p-14f, -639.f);
        };
        if constexpr (F8) {
            float most = 0.f, least = MODE == kWhole ? INFINITY : 0.f;
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                ks2[i] = *reinterpret_cast<const f32x4b*>(kscale + i * 16 + grp * 4);
                vs[i] = *reinterpret_cast<const f32x4b*>(vscale + i * 16 + grp * 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    ks2[i][e] *= scale2;
                    const float v = vs[i][e];                            // (a bit cast of a vector's element reads element 0)
                    if constexpr (MODE == kWhole) {
                        most = fmaxf(most, fabsf(v));
                        least = fminf(least, fabsf(v));
                    } else {
                        const float lg = log2_of(v);
                        if constexpr (MASKED) most = fmaxf(most, lg), least = fminf(least, v == 0.f ? 0.f : lg);
                        size[i][e] = __builtin_amdgcn_fmed3f(lg, -40.f, 38.f);
                    }
                }
            }
            if constexpr (MASKED) apart = most > 38.f || least < -40.f;
            if constexpr (MODE == kWhole) {
                big = __builtin_amdgcn_logf(most);
                little = __builtin_amdgcn_logf(least);
                if (__any(big > 38.f || little < -38.f)) return false;
            }
        }
        // ---- the softmax, in units of log2.  Scores are taken relative to the maximum so far before the new one is known: it is raised only where it would be by
        // more than 2^8 (probabilities are relative to the one they were taken with, and no less exact), and then they are made again.
        float p[QW][RT][4];
#pragma unroll
        for (int b = 0; b < QW; ++b) {
            auto relative_to = [&](float base) {
#pragma unroll
                for (int i = 0; i < RT; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float x = s[b][i][e];
                        if constexpr (MASKED) x = sees(b, i, e) ? x : -INFINITY;
                        if constexpr (F8 && MASKED) x = fmaf(x, sees(b, i, e) ? ks2[i][e] : 1.f, -base);
                        else if constexpr (F8) x = fmaf(x, ks2[i][e], -base);
                        else x = fmaf(x, scale2, -base);
                        p[b][i][e] = x;
                    }
            };
            const float base = m[b] == -INFINITY ? 0.f : m[b];
            relative_to(base);
            if constexpr (F8) {
                auto log2_product = [&](int i, int e) {
                    const float v = vs[i][e];
                    return p[b][i][e] + (MODE == kWhole ? log2_of(v) : size[i][e]);
                };
                float top = -INFINITY, low = MODE == kWhole ? INFINITY : 0.f;
#pragma unroll
                for (int i = 0; i < RT; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float y = MODE == kWhole ? p[b][i][e] : log2_product(i, e);
                        top = fmaxf(top, y);
                        if constexpr (MODE == kWhole) low = fminf(low, y);
                        if constexpr (MASKED) low = fminf(low, sees(b, i, e) ? y : 0.f);
                    }
                // (kWhole: bounds first, of the largest and the smallest score and scale)
                if (__any(MODE == kWhole ? top + big > kRaise || low + little < kLow || m[b] == -INFINITY : top > kRaise || (m[b] == -INFINITY && top > -INFINITY))) {
                    if constexpr (MODE == kWhole) {
                        top = -INFINITY;
                        low = INFINITY;
#pragma unroll
                        for (int i = 0; i < RT; ++i)
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                top = fmaxf(top, log2_product(i, e));
                                low = fminf(low, log2_product(i, e));
                            }
                    }
                    top = max_lanes16_32(top);
                    const bool mine = top > kRaise || (m[b] == -INFINITY && top > -INFINITY);
                    const float next = ceilf(base + top) - 8.f, change = mine ? next - base : 0.f;
                    const int fade = m[b] == -INFINITY ? 0 : (int)fmaxf(-change, -1000.f);
                    m[b] = mine ? next : m[b];
                    l[b] = ldexpf(l[b], fade);
#pragma unroll
                    for (int d = 0; d < DT; ++d)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[b][d][e] = ldexpf(acc[b][d][e], fade);
                    low -= change;
#pragma unroll
                    for (int i = 0; i < RT; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) p[b][i][e] -= change;
                    if constexpr (MODE == kWhole) apart |= low < kLow;
                }
                if constexpr (MASKED) apart |= low < kLow;
                continue;
            }
            float top = -INFINITY;
#pragma unroll
            for (int i = 0; i < RT; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) top = fmaxf(top, p[b][i][e]);
            top = max_lanes16_32(top);
            if (__any(top > 8.f || (m[b] == -INFINITY && top > -INFINITY))) {
                // (A query whose own maximum does not ask for it stays as it is, to the bit: others' scores are those of entries that it may not see.)
                const bool mine = top > 8.f || m[b] == -INFINITY;
                const float next = mine ? fmaxf(m[b], base + top) : m[b], fade = next == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[b] - next);
                m[b] = next;
                l[b] *= fade;
#pragma unroll
                for (int e = 0; e < 4; ++e) rounded[b][e] *= fade;
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[b][d][e] *= fade;
                relative_to(next == -INFINITY ? 0.f : next);
            }
        }
        if constexpr (F8 && MODE == kWhole)
            if (__any(apart)) return false;
        // ---- O^T += V^T P^T
        bool left_out = false;
        const int k8 = col >> 1, vrow = F8 ? (k8 < 4 ? grp * 4 + k8 : 12 + grp * 4 + k8) : grp * 4 + (col >> 2);      // of 32, or of 16
        auto values8 = [&](int h, int d) {                               // e4m3: eight tokens' values of a dim
            auto from = (__attribute__((address_space(3))) i32x2*)(sv + vrow * kRow + (d ^ turn_v<HD, F8>(vrow)) * 16 + (col & 1) * 8 + h * 32 * kRow);
            i32x2 w = __builtin_amdgcn_ds_read_tr8_b64_v2i32(from);
            if constexpr (MASKED) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint32_t x = (uint32_t)w[i], nan = ((x & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;     // bytes 0x7f and 0xff
                    left_out |= nan != 0;
                    w[i] = (int)(x & ~((nan >> 7) * 255u));
                }
            }
            return w;
        };
        if constexpr (F8 && MASKED) {
            if (__any(apart)) {                                          // products that fp16 does not hold, in bf16 into the same sums
#pragma unroll
                for (int h = 0; h < RT / 2; ++h) {
                    bf16x8 rest[QW];
#pragma unroll
                    for (int b = 0; b < QW; ++b) {
                        float x[8];
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            const int i = 2 * h + k / 4, e = k % 4;
                            const float one = __builtin_amdgcn_exp2f(p[b][i][e]);
                            float w = one * vs[i][e];
                            w = sees(b, i, e) ? w : 0.f;
                            const bool held = (int)(fabsf(w) >= 0x1p-17f) & (int)(fabsf(w) <= 65504.f);
                            x[k] = held ? 0.f : w;
                            l[b] += held ? 0.f : one;
                            p[b][i][e] = held ? p[b][i][e] : -INFINITY;
                        }
                        const uint2 lo = pack_bf16x4(x[0], x[1], x[2], x[3]), hi = pack_bf16x4(x[4], x[5], x[6], x[7]);
                        rest[b] = __builtin_bit_cast(bf16x8, u32x4b{lo.x, lo.y, hi.x, hi.y});
                    }
#pragma unroll
                    for (int d = 0; d < DT; ++d) {
                        const i32x2 w = values8(h, d);
                        const bf16x8 vf = widen_bf16((uint32_t)w[0], (uint32_t)w[1]);
#pragma unroll
                        for (int b = 0; b < QW; ++b) acc[b][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, rest[b], acc[b][d], 0, 0, 0);
                    }
                }
#pragma unroll
                for (int i = 0; i < RT; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) vs[i][e] = fabsf(vs[i][e]) < INFINITY ? vs[i][e] : 0.f;
            }
        }
#pragma unroll
        for (int b = 0; b < QW; ++b)
#pragma unroll
            for (int i = 0; i < RT; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float x = __builtin_amdgcn_exp2f(p[b][i][e]);
                    l[b] += x;
                    if constexpr (F8) {
                        x *= vs[i][e];
                        if constexpr (MASKED) x = sees(b, i, e) ? x : 0.f;
                    }
                    p[b][i][e] = x;
                }
        __builtin_amdgcn_s_setprio(1);
        using Frag = std::conditional_t<F16, f16x8, bf16x8>;
#pragma unroll
        for (int h = 0; h < RT / 2; ++h) {
            if (h > 0) __builtin_amdgcn_sched_barrier(0);
            Frag pf[QW];
#pragma unroll
            for (int b = 0; b < QW; ++b) {
                if constexpr (F16) {
                    union {
                        f16x8 v;
                        f16x2v h[4];
                    } u;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        u.h[2 * i] = __builtin_convertvector(f32x2v{p[b][2 * h + i][0], p[b][2 * h + i][1]}, f16x2v);
                        u.h[2 * i + 1] = __builtin_convertvector(f32x2v{p[b][2 * h + i][2], p[b][2 * h + i][3]}, f16x2v);
                    }
                    pf[b] = u.v;
                } else {
                    const uint2 lo = pack_bf16x4(p[b][2 * h][0], p[b][2 * h][1], p[b][2 * h][2], p[b][2 * h][3]), hi = pack_bf16x4(p[b][2 * h + 1][0], p[b][2 * h + 1][1], p[b][2 * h + 1][2], p[b][2 * h + 1][3]);
                    pf[b] = __builtin_bit_cast(bf16x8, u32x4b{lo.x, lo.y, hi.x, hi.y});
                    // Results are divided by the sum of what was multiplied: with few tokens the rounding of the largest would show in all dims.
                    if constexpr (!F8) {
                        const bf16x8 ones = __builtin_bit_cast(bf16x8, u32x4b{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u});
                        rounded[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pf[b], rounded[b], 0, 0, 0);
                    }
                }
            }
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                Frag vf;
                if constexpr (F8) {
                    const i32x2 w = values8(h, d);
                    if constexpr (F16) vf = widen_f16((uint32_t)w[0], (uint32_t)w[1]);
                    else vf = widen_bf16((uint32_t)w[0], (uint32_t)w[1]);
                } else {
                    u32x4b x;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        auto from = (__attribute__((address_space(3))) s16x4*)(sv + vrow * kRow + ((d * 2 + ((col & 3) >> 1)) ^ turn_v<HD, F8>(vrow)) * 16 + (col & 1) * 8 +
                                                                               (h * 32 + i * 16) * kRow);
                        const uint2 w = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(from));
                        x[2 * i] = w.x;
                        x[2 * i + 1] = w.y;
                    }
                    if constexpr (MASKED) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const bool lo = (x[i] & 0x7f80u) == 0x7f80u, hi = (x[i] & 0x7f800000u) == 0x7f800000u;
                            left_out |= lo | hi;
                            x[i] &= (lo ? 0u : 0xffffu) | (hi ? 0u : 0xffff0000u);
                        }
                    }
                    vf = __builtin_bit_cast(bf16x8, x);
                }
#pragma unroll
                for (int b = 0; b < QW; ++b) {
                    if constexpr (F16) acc[b][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, pf[b], acc[b][d], 0, 0, 0);
                    else acc[b][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[b], acc[b][d], 0, 0, 0);
                }
            }
        }
        __builtin_amdgcn_s_setprio(0);
        if constexpr (MASKED) odd |= left_out;
        return true;
    }

    // What probabilities are relative to, their sum, and the sum that results are divided by, of this wave's query b (in a lane of any group of 16).
    __device__ __forceinline__ float4 sums(int b) const {
        const float whole = add_lanes16_32(l[b]);
        return make_float4(m[b], whole, F8 ? whole : rounded[b][0], 0.f);
    }
};

// What a partial result, relative to its m, counts for in one relative to m.  What is not finite stays whatever it counts for; a part that has seen a NaN and nothing else has no m.
__device__ __forceinline__ float share(float4 ml, float m) {
    return ml.x == -INFINITY ? (ml.y == ml.y ? 0.f : 1.f) : __builtin_amdgcn_exp2f(ml.x - m);
}
__device__ __forceinline__ float counted(float x, float f) { return fabsf(x) < INFINITY ? x * f : x; }

// ---------------------------------------------------------------- what a workgroup takes
struct NodesRange {
    int row, slot, ranges, t_begin, t_end, nodes, ctx;                   // (tiles of `tokens` tokens)
};
struct NodesShared {
    int pick[4], sum[8], up[TABED_MAX_NODES], first_masked[8];
    double whole[8];
    int lengths[64];
};

__device__ __forceinline__ int tiles_of(const NodesAttnArgs& a, int row, int tokens) {
    const int n = nodes_of(a.n_nodes, row, a.N);
    const int64_t end = min((int64_t)context_of(a.ctx_len, row) + n, (int64_t)a.c.max_blocks * TABED_CACHE_BLOCK);
    return n > 0 ? (int)((end + tokens - 1) / tokens) : 0;
}

// A row's length, for its share of the ranges.  UNIT: queries of a wave of four that share e4m3 tiles, 0 elsewhere.  Waves that have no queries of their own take turns
// with others, so a tile of one or two units of queries takes about half the time of one with three or four (16 rows of 300 to 5000 tokens and 4 to 132 queries, head_dim
// 128: 80 us against 96 with equal lengths; 8 rows of 4000 to 16000: 95 against 123).  With bf16, whose tiles take a step each and twice the bytes, longer ranges of such rows
// cost more than they give (78 against 72 us, 102 against 93).
template <int UNIT>
__device__ __forceinline__ int length_of(const NodesAttnArgs& a, int row, int tokens) {
    const int t = tiles_of(a, row, tokens);
    if constexpr (UNIT == 0) return t;
    const int q = min(nodes_of(a.n_nodes, row, a.N) * a.group, a.per_tile);
    return min(a.N * a.group, a.per_tile) <= 2 * UNIT || q > 2 * UNIT ? t : (int)(((int64_t)t * (q > UNIT ? 5 : 4) + 7) / 8);
}

// Ranges of keys.  Where there are fewer (row, head, tile of queries) than workgroups that run at a time, or rows are long and of unequal lengths, rows are cut
// into ranges of no more than `per` tiles, the same for all rows and as small as leaves no more than `fill` ranges: all workgroups work that out from the
// rows' lengths, and each takes the range its slot falls on.  A short row is not cut.  A row of one range is finished by its workgroup; others' results are joined by a
// second launch.  False: there is no such range.
template <int THREADS, int UNIT>
__device__ __forceinline__ bool find_range(const NodesAttnArgs& a, NodesShared& s, int slot, int tokens, bool tell, NodesRange& g) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    constexpr int W = THREADS / 64;
    int row = slot, range = 0, ranges = 1;
    auto ranges_of = [&](int length, int each) { return length <= a.whole_tiles ? 1 : (length + each - 1) / each; };
    if (a.split) {
        double whole = 0.0;
        for (int i = tid; i < a.rows; i += THREADS) {
            const int t = length_of<UNIT>(a, i, tokens);
            if (i < 64) s.lengths[i] = t;
            whole += t;
        }
        whole = wave_sum(whole);
        if (lane == 0) s.whole[wave] = whole;
        if (tid < 4) s.pick[tid] = -1;
        __syncthreads();
        whole = 0.0;
#pragma unroll
        for (int w = 0; w < W; ++w) whole += s.whole[w];
        // sum ceil(t / per) is at most whole / per + rows
        const int least = max(a.min_tiles, (int)fmin(ceil(whole / a.fill), 1e9));
        int per = max(least, (int)fmin(ceil(whole / max(a.fill - a.rows, 1)), 1e9));
        if (a.rows <= 64 && a.fill > a.rows) {                           // a candidate a thread, between the two
            const int mine = least + (int)((int64_t)(per - least) * tid / THREADS);
            int count = 0;
            for (int i = 0; i < a.rows; ++i) count += ranges_of(s.lengths[i], mine);
            const uint64_t good = __ballot(count <= a.fill);
            const int best = good ? __builtin_amdgcn_readlane(mine, __ffsll((long long)good) - 1) : 0x7fffffff;
            if (lane == 0) s.sum[wave] = best;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < W; ++w) per = min(per, s.sum[w]);
            __syncthreads();
        }
        int before = 0;                                                  // ranges of the rows before those of this round
        for (int r0 = 0; r0 < a.rows; r0 += THREADS) {
            const int i = r0 + tid, n = i < a.rows ? ranges_of(length_of<UNIT>(a, i, tokens), per) : 0;
            const int incl = (int)wave_inclusive_scan((double)n);
            __syncthreads();
            if (lane == 63) s.sum[wave] = incl;
            __syncthreads();
            int base = before;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                if (w < wave) base += s.sum[w];
                before += s.sum[w];
            }
            const int first = base + incl - n;
            if (n > 0 && slot >= first && slot < first + n) {
                s.pick[0] = i;
                s.pick[1] = slot - first;
                s.pick[2] = n;
            }
        }
        __syncthreads();
        row = __builtin_amdgcn_readfirstlane(s.pick[0]);
        if (row < 0) return false;
        range = __builtin_amdgcn_readfirstlane(s.pick[1]);
        ranges = __builtin_amdgcn_readfirstlane(s.pick[2]);
        if (tell && range == 0 && tid == 0) a.ranges[row] = make_int2(slot, ranges);
    }
    const int all = __builtin_amdgcn_readfirstlane(tiles_of(a, row, tokens));
    g.row = row;
    g.slot = slot;
    g.ranges = ranges;
    g.nodes = __builtin_amdgcn_readfirstlane(nodes_of(a.n_nodes, row, a.N));
    g.ctx = __builtin_amdgcn_readfirstlane(context_of(a.ctx_len, row));
    g.t_begin = (int)((int64_t)all * range / ranges);
    g.t_end = (int)((int64_t)all * (range + 1) / ranges);
    return true;
}

// Who sees whom, by doubling: a node's mask takes in that of the first node above that it has not looked through, log2 of the depth times.
template <int THREADS>
__device__ __forceinline__ void find_masks(const NodesAttnArgs& a, int r, int nodes, int* s_up, uint64_t (*s_mask)[kNodeWords]) {
    const int tid = threadIdx.x;
    if (a.parents == nullptr) {
        for (int j = tid; j < nodes; j += THREADS)
#pragma unroll
            for (int w = 0; w < kNodeWords; ++w) s_mask[j][w] = j >= 64 * w + 63 ? ~0ull : j < 64 * w ? 0ull : (2ull << (j - 64 * w)) - 1;
        lds_barrier();
        return;
    }
    constexpr int PN = (TABED_MAX_NODES + THREADS - 1) / THREADS;
    uint64_t m[PN][kNodeWords], more[PN][kNodeWords];
    int up[PN], next[PN];
#pragma unroll
    for (int p = 0; p < PN; ++p) {
        const int j = p * THREADS + tid;
        up[p] = j < nodes ? parent_of(a.parents, r, j, a.N) : -1;
#pragma unroll
        for (int w = 0; w < kNodeWords; ++w) m[p][w] = j / 64 == w ? 1ull << (j & 63) : 0ull;
    }
    for (int left = nodes - 1;; left >>= 1) {
#pragma unroll
        for (int p = 0; p < PN; ++p) {
            const int j = p * THREADS + tid;
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

// The table is read through the scalar cache: a vector load's wait would be one for the tiles on their way too.
typedef const __attribute__((address_space(4))) int32_t* ScalarInts;

// Values that are not finite.  0 times such a value is NaN, so the products of tiles that not everybody sees are without them, and nodes that do see one get
// it added by itself at the end, by a second look: masked(t): tile t (of 32 tokens) was one of those.
template <int HD, bool F8, typename Masked>
__device__ __forceinline__ void add_odd(const NodesAttnArgs& a, const NodesRange& g, int t_begin, int t_end, int kvh, const uint64_t* mask, int dim, Masked masked,
                                        float (&o)[4]) {
    for (int t = t_begin; t < t_end; ++t) {
        const int first = t * kNodesTile, entry = a.c.block_at(g.row, first / TABED_CACHE_BLOCK);
        if (!masked(t) || entry < 0) continue;
        const uint32_t seen = (uint32_t)window(mask, (int64_t)first - g.ctx);
        for (int k = 0; k < kNodesTile; ++k) {
            if (!(seen >> k & 1)) continue;
            const int64_t from = a.c.entry(a.c.layer, entry, kvh, first % TABED_CACHE_BLOCK + k) + dim;
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
}

// What was left out may be what nobody sees: slots behind the row's end or nodes that are not there, in a pool that was never cleared, or the block read in place of one that is not there.
// The workgroup goes once over the row's tokens in those tiles, all at a time (add_odd goes one by one: with 6000 tokens behind a hole 40 nodes took 576 us for 26), and only
// if one of them has such a value is there something to add.
template <int HD, bool F8, int THREADS, typename Masked>
__device__ __forceinline__ bool odd_is_seen(const NodesAttnArgs& a, const NodesRange& g, int t_begin, int t_end, int kvh, int* found, Masked masked) {
    constexpr int kPieces = HD * (F8 ? 1 : 2) / 16;
    __syncthreads();
    if (threadIdx.x == 0) *found = 0;
    __syncthreads();
    const int64_t first = (int64_t)t_begin * kNodesTile, end = min((int64_t)t_end * kNodesTile, (int64_t)g.ctx + g.nodes);
    for (int64_t i = first * kPieces + threadIdx.x; i < end * kPieces; i += THREADS) {
        const int64_t pos = i / kPieces;
        if (!masked((int)(pos / kNodesTile))) continue;
        const int block = a.c.block_of(g.row, pos);
        if (block < 0) continue;
        const int64_t from = a.c.entry(a.c.layer, block, kvh, (int)(pos % TABED_CACHE_BLOCK)) * (F8 ? 1 : 2) + i % kPieces * 16;
        const u32x4b x = *reinterpret_cast<const u32x4b*>(a.c.v + from);
        bool odd = false;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (F8) odd |= (((x[e] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) != 0;
            else odd |= (x[e] & 0x7f80u) == 0x7f80u || (x[e] & 0x7f800000u) == 0x7f800000u;
        }
        if (odd) *found = 1;
    }
    __syncthreads();
    return *found != 0;
}

// Four dims of query qi of (row, head): the result, or a range's part of it.
template <int HD>
__device__ __forceinline__ void store_result(const NodesAttnArgs& a, const NodesRange& g, int kvh, int tile_q, int qi, int dim, float4 ml, const float (&o)[4]) {
    if (g.ranges > 1) {
        const int64_t place = (((int64_t)g.slot * a.c.kv_heads + kvh) * a.tiles + tile_q) * a.per_tile + (qi - tile_q * a.per_tile);
        *reinterpret_cast<f32x4b*>(a.o + place * HD + dim) = f32x4b{o[0], o[1], o[2], o[3]};
        if (dim == 0) a.ml[place] = ml;
        return;
    }
    const int node = qi / a.group, head = kvh * a.group + qi % a.group;
    const float inv = ml.z == 0.f ? 0.f : 1.f / ml.z;
    const uint2 w = pack_bf16x4(o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
    typedef uint32_t u32x2_e2 __attribute__((ext_vector_type(2), aligned(2)));
    *reinterpret_cast<u32x2_e2*>(a.out + g.row * a.out_row + node * a.out_tok + (int64_t)head * HD + dim) = u32x2_e2{w.x, w.y};
    if (dim == 0 && a.lse != nullptr)
        a.lse[((int64_t)g.row * a.N + node) * a.q_heads + head] = ml.y == 0.f ? -INFINITY : (ml.x + __builtin_amdgcn_logf(ml.y)) * 0.69314718055994530942f;
}

// Results of `parts` waves with the same query, their lines in s_o and sums in s_ml `apart` queries apart, as one.
template <int LINE>
__device__ __forceinline__ float4 join_parts(const float* s_o, const float4* s_ml, int parts, int apart, int i, int dim, float (&o)[4]) {
    float4 ml = make_float4(-INFINITY, 0.f, 0.f, 0.f);
    for (int w = 0; w < parts; ++w) ml.x = fmaxf(ml.x, s_ml[w * apart + i].x);
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = 0.f;
    for (int w = 0; w < parts; ++w) {
        const float4 part = s_ml[w * apart + i];
        const f32x4b x = *reinterpret_cast<const f32x4b*>(s_o + (size_t)(w * apart + i) * LINE + dim);
        const float f = share(part, ml.x);
        ml.y += part.y * f;
        ml.z += part.z * f;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += counted(x[e], f);
    }
    return ml;
}

// ---------------------------------------------------------------- up to 32 queries: every wave has tiles of its own
// QW groups of 16 queries a wave: one for up to 16 (6 queries, one row of 600 tokens, heads of 64: 7.8 us, with two groups 9.0, by four waves; 64 rows of 256 to 768, 16 queries: 25.1 and
// 27.6), two for up to 32 (16 rows of 300 to 5000, 8 heads of 128, e4m3: 35 us, with waves that share tiles 47; 64 rows of 2000, 12 heads of 64: 77 and 91).  Four waves
// (with two 42, 81 and 97 us for 35, 77 and 92, one row of 120011 tokens), two where four would need more LDS than there is.
template <int HD_, bool F8_, int QW_, int WK_>
struct NodesNarrow {
    static constexpr int HD = HD_, QW = QW_, WK = WK_, kThreads = WK * 64, kQueries = QW * 16, kUnit = kQueries, kTokens = kNodesTile;
    static constexpr bool F8 = F8_;
    static constexpr int kRow = HD * (F8 ? 1 : 2), kPieces = kRow / 16, kTile = kNodesTile * kRow;      // bytes of a row, its pieces, bytes of a tile
    static constexpr int kStage = 2 * kTile + (F8 ? 256 : 0), kLoads = kTile / 1024, kAll = 2 * kLoads + (F8 ? 1 : 0);
    static constexpr int kLine = HD + 4;
    static constexpr size_t kJoin = (size_t)WK * kQueries * (kLine * 4 + 16);
    static constexpr size_t kLds = std::max((size_t)WK * 2 * kStage, kJoin) + kMaskBytes;
    static_assert(kTile % 1024 == 0);
};

template <class T>
__global__ __launch_bounds__(T::kThreads, 2) void k_attention_nodes(NodesAttnArgs a) {
    constexpr int HD = T::HD, QW = T::QW, WK = T::WK;
    constexpr bool F8 = T::F8;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    uint64_t(*const s_mask)[kNodeWords] = reinterpret_cast<uint64_t(*)[kNodeWords]>(lds + T::kLds - kMaskBytes);
    __shared__ NodesShared sh;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int kvh = blockIdx.x % a.c.kv_heads, slot = blockIdx.x / a.c.kv_heads;                   // (one tile of queries)
    NodesRange g;
    if (!find_range<T::kThreads, 0>(a, sh, slot, kNodesTile, kvh == 0, g)) return;
    const int queries = g.nodes * a.group;
    if (queries == 0) return;

    // ---- tiles of keys and values into LDS
    unsigned char* const area = lds + wave * 2 * T::kStage;
    const uint32_t area0 = __builtin_amdgcn_readfirstlane(lds_address(area));
    uint32_t ko[T::kLoads], vo[T::kLoads];
#pragma unroll
    for (int i = 0; i < T::kLoads; ++i) {
        const int p = i * 64 + lane, row = p / T::kPieces, piece = p % T::kPieces;
        const uint32_t line = (uint32_t)(row * a.c.tok_stride * (F8 ? 1 : 2));
        ko[i] = line + (uint32_t)(piece ^ turn_k<HD, F8>(row)) * 16;
        vo[i] = line + (uint32_t)(piece ^ turn_v<HD, F8>(row)) * 16;
    }
    const ScalarInts table = (ScalarInts)(uintptr_t)(a.c.table + (int64_t)g.row * a.c.max_blocks);
    auto block_of_tile = [&](int t) { return table[min(t * kNodesTile / TABED_CACHE_BLOCK, a.c.max_blocks - 1)]; };      // (tiles end with the table)
    uint32_t there = 0;                                                  // a bit a stage: its tile's block is one
    // (A tile whose block is not there is read from block 0, and not seen.)
    auto request = [&](int t, int stage, int entry) {
        const bool is = entry >= 0 && entry < a.c.blocks;
        const int block = is ? entry : 0, first = t * kNodesTile % TABED_CACHE_BLOCK;
        there = is ? there | 1u << stage : there & ~(1u << stage);
        const int64_t from = a.c.entry(a.c.layer, block, kvh, first) * (F8 ? 1 : 2);
        const uint32_t to = area0 + (uint32_t)(stage * T::kStage);
        dma_pieces(uniform(a.c.k + from), ko, to);
        dma_pieces(uniform(a.c.v + from), vo, to + T::kTile);
        if constexpr (F8) dma_words((lane < 32 ? a.c.kscale : a.c.vscale) + a.c.scale_entry(a.c.layer, block, kvh, first) + (lane & 31), to + 2 * T::kTile);
    };
    const int t0 = g.t_begin + wave;
    if (t0 < g.t_end) request(t0, 0, block_of_tile(t0));
    int entry = block_of_tile(t0 + WK);                                  // of the tile that is requested next

    // ---- while they come: the queries, and who sees whom
    NodesWave<HD, F8, QW> w;
    w.begin(a, g.row, kvh, 0, queries);
    find_masks<T::kThreads>(a, g.row, g.nodes, sh.up, s_mask);

    // Tiles that all queries see to their end come first; from the first other one on (nodes, the end of the row, a block that is not there) every tile
    // goes by what is seen.  (One loop with both kinds in it has two sets of sums, and takes twice the registers for them.)
    int stage = 0, t = t0;
    bool far = false;                                                    // uniform
    auto arrive_tile = [&] {
        const bool more = t + WK < g.t_end;
        // (what was read of the stage that is filled now has arrived)
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (more) request(t + WK, stage ^ 1, entry);
        entry = block_of_tile(t + 2 * WK);
        // This tile is there once no more is outstanding than was asked for behind it.
        if (more) asm volatile("s_waitcnt vmcnt(%0)" :: "n"(T::kAll) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    };
    auto take = [&](auto mode) {
        const unsigned char* const sk = area + stage * T::kStage;
        const unsigned char* const sv = sk + T::kTile;
        const float* const sc = reinterpret_cast<const float*>(sv + T::kTile);
        uint32_t seen[QW];
#pragma unroll
        for (int b = 0; b < QW; ++b) {
            seen[b] = ~0u;
            if constexpr (mode.value == kMasked) seen[b] = there >> stage & 1 ? (uint32_t)window(s_mask[w.node[b]], (int64_t)t * kNodesTile - g.ctx) : 0u;
        }
        if constexpr (F8 && mode.value == kWhole) {
            // (In the same loop: a loop of its own for what is kFar costs this kernel 170 registers that spill.)
            if (far || !w.template step<kWhole, 2>(sk, sv, sc, sc + 32, a.scale2, seen)) {
                far = true;
                w.template step<kFar, 2>(sk, sv, sc, sc + 32, a.scale2, seen);
            }
        } else {
            w.template step<mode.value, 2>(sk, sv, sc, sc + 32, a.scale2, seen);
        }
        stage ^= 1;
        t += WK;
    };
    while (t < g.t_end && (int64_t)(t + 1) * kNodesTile <= g.ctx && (there >> stage & 1)) {
        arrive_tile();
        take(NodesMode<kWhole>{});
    }
    const int first_masked = t;
    while (t < g.t_end) {
        arrive_tile();
        take(NodesMode<kMasked>{});
    }

    // ---- the waves' results as one
    if (tid == 0) sh.pick[3] = 0;
    __syncthreads();                                                     // all tiles have been read, none is on its way
    float* const s_o = reinterpret_cast<float*>(lds);
    float4* const s_ml = reinterpret_cast<float4*>(lds + (size_t)WK * T::kQueries * T::kLine * 4);
    const int col = lane & 15, grp = lane >> 4;
#pragma unroll
    for (int b = 0; b < QW; ++b) {
        const int i = wave * T::kQueries + b * 16 + col;
#pragma unroll
        for (int d = 0; d < HD / 16; ++d) *reinterpret_cast<f32x4b*>(s_o + (size_t)i * T::kLine + d * 16 + grp * 4) = w.acc[b][d];
        const float4 ml = w.sums(b);
        if (grp == 0) s_ml[i] = ml;
    }
    if (lane == 0) sh.first_masked[wave] = first_masked;
    if (w.odd) sh.pick[3] = 1;
    __syncthreads();
    auto masked = [&](int tile) { return tile >= sh.first_masked[(tile - g.t_begin) % WK]; };
    const bool odd = sh.pick[3] != 0 && odd_is_seen<HD, F8, T::kThreads>(a, g, g.t_begin, g.t_end, kvh, &sh.pick[3], masked);
    for (int p = tid; p < queries * (HD / 4); p += T::kThreads) {
        const int i = p / (HD / 4), dim = p % (HD / 4) * 4;
        float o[4];
        const float4 ml = join_parts<T::kLine>(s_o, s_ml, WK, T::kQueries, i, dim, o);
        if (odd)
            add_odd<HD, F8>(a, g, g.t_begin, g.t_end, kvh, s_mask[i / a.group], dim, masked, o);
        store_result<HD>(a, g, kvh, 0, i, dim, ml, o);
    }
}

// ---------------------------------------------------------------- more: four waves share tiles
// 32 queries a wave (256 dims: 16, for the registers), so that a fragment of keys or values read from LDS serves two products: with 48 a wave, and one wave a SIMD, 771 us where
// this takes 477 (8 rows of 4000 to 16000 tokens, 256 nodes, 32 / 8 heads of 128).  Steps of 64 tokens: one test of the maximum, and one pass of the softmax, for
// twice the products (515 us with 32).  Tiles of 16 KB of keys, two of them: two workgroups a CU.
template <int HD_, bool F8_>
struct NodesWide {
    static constexpr int HD = HD_, QW = HD == 256 ? 1 : 2, RT = 4, kWaves = 4, kThreads = kWaves * 64, kUnit = QW * 16, kQueries = kWaves * kUnit;
    static constexpr bool F8 = F8_;
    static constexpr int kRow = HD * (F8 ? 1 : 2), kPieces = kRow / 16;
    static constexpr int kTokens = std::min(256, std::max(64, 16384 / kRow / 64 * 64)), kPages = kTokens / TABED_CACHE_BLOCK;      // of a tile
    static constexpr int kTile = kTokens * kRow, kStage = 2 * kTile + (F8 ? kTokens * 8 : 0);
    static constexpr int kLoads = kTile / 1024 / kWaves;                 // of a wave, for keys and for values each: all in one page
    static constexpr int kLine = HD + 4;
    static constexpr size_t kJoin = (size_t)kQueries * (kLine * 4 + 16);
    static constexpr size_t kLds = std::max((size_t)2 * kStage, kJoin) + kMaskBytes;
    static_assert(kTile % (1024 * kWaves) == 0 && TABED_CACHE_BLOCK * kRow % (1024 * kLoads) == 0 && kLds <= 155 * 1024);
};

template <class T>
__global__ __launch_bounds__(T::kThreads, 2) void k_attention_nodes_wide(NodesAttnArgs a) {
    constexpr int HD = T::HD, QW = T::QW;
    constexpr bool F8 = T::F8;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    uint64_t(*const s_mask)[kNodeWords] = reinterpret_cast<uint64_t(*)[kNodeWords]>(lds + T::kLds - kMaskBytes);
    __shared__ NodesShared sh;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // Workgroup w goes to XCD w % 8: the tiles of queries that read the same keys run back to back on one.  The last tile, which may have less to do, is another one for each
    // 32 workgroups, so that no CU has all of them (two tiles of 96 and 36 queries: 90 us against 104).
    const int xcd = blockIdx.x & 7, at = blockIdx.x >> 3, tile_q = (at % a.tiles + at / a.tiles * a.tiles / 32) % a.tiles, unit = at / a.tiles * 8 + xcd;
    const int kvh = unit % a.c.kv_heads, slot = unit / a.c.kv_heads;
    if (slot >= a.slots) return;                                         // uniform: the grid is padded to whole rounds of XCDs
    NodesRange g;
    if (!find_range<T::kThreads, F8 ? T::kUnit : 0>(a, sh, slot, T::kTokens, kvh == 0 && tile_q == 0, g)) return;
    const int queries = min(g.nodes * a.group, (tile_q + 1) * a.per_tile), here = queries - tile_q * a.per_tile;
    if (here <= 0) return;
    // As many waves as there are units of queries, 1, 2 or 4, take different ones; the 64-token steps are dealt to the WK waves that have the same.
    const int units = (here + T::kUnit - 1) / T::kUnit, WQ = units > 2 ? 4 : units, WK = 4 / WQ, wq = wave % WQ, wk = wave / WQ;
    const int q0 = tile_q * a.per_tile + wq * T::kUnit;

    const uint32_t area0 = __builtin_amdgcn_readfirstlane(lds_address(lds));
    constexpr int kPageLoads = TABED_CACHE_BLOCK * T::kRow / 1024;       // of a page, keys or values
    const int my_page = wave * T::kLoads / kPageLoads;
    uint32_t ko[T::kLoads], vo[T::kLoads];
#pragma unroll
    for (int i = 0; i < T::kLoads; ++i) {
        const int p = (wave * T::kLoads % kPageLoads + i) * 64 + lane, row = p / T::kPieces, piece = p % T::kPieces;      // in the page
        const uint32_t line = (uint32_t)(row * a.c.tok_stride * (F8 ? 1 : 2));
        ko[i] = line + (uint32_t)(piece ^ turn_k<HD, F8>(row)) * 16;
        vo[i] = line + (uint32_t)(piece ^ turn_v<HD, F8>(row)) * 16;
    }
    const ScalarInts table = (ScalarInts)(uintptr_t)(a.c.table + (int64_t)g.row * a.c.max_blocks);
    auto entry_at = [&](int t, int page) {                               // (pages past the table: none)
        const int64_t e = (int64_t)t * T::kPages + page;
        return e < a.c.max_blocks ? table[e] : -1;
    };
    auto is_block = [&](int e) { return e >= 0 && e < a.c.blocks; };
    // Entries of the tile that is requested next: they are asked for a tile before that, so that no request waits for them.
    int entries[T::kPages];
    auto look_up = [&](int t) {
#pragma unroll
        for (int p = 0; p < T::kPages; ++p) entries[p] = entry_at(t, p);
    };
    auto block_of = [&](int page) {
        int e = entries[0];
#pragma unroll
        for (int p = 1; p < T::kPages; ++p) e = page == p ? entries[p] : e;
        return is_block(e) ? e : 0;
    };
    auto request = [&](int stage) {
        const int64_t from = a.c.entry(a.c.layer, block_of(my_page), kvh, 0) * (F8 ? 1 : 2);
        const uint32_t to = area0 + (uint32_t)(stage * T::kStage + wave * T::kLoads * 1024);
        dma_pieces(uniform(a.c.k + from), ko, to);
        dma_pieces(uniform(a.c.v + from), vo, to + T::kTile);
        if constexpr (F8) {
#pragma unroll
            for (int i = 0; i < (T::kPages * 2 + T::kWaves - 1) / T::kWaves; ++i) {      // a page's scales of keys, or of values: 64 words
                const int part = i * T::kWaves + wave;
                if (part >= T::kPages * 2) break;
                dma_words((part & 1 ? a.c.vscale : a.c.kscale) + a.c.scale_entry(a.c.layer, block_of(part >> 1), kvh, lane),
                          area0 + (uint32_t)(stage * T::kStage + 2 * T::kTile + ((part & 1) * T::kTokens + (part >> 1) * 64) * 4));
            }
        }
    };
    auto bits = [&] {                                                    // a bit a page of that tile: it is there
        uint32_t x = 0;
#pragma unroll
        for (int p = 0; p < T::kPages; ++p) x |= is_block(entries[p]) ? 1u << p : 0u;
        return x;
    };
    look_up(g.t_begin);
    uint32_t pages = bits(), pages_ahead = 0;
    if (g.t_begin < g.t_end) request(0);
    look_up(g.t_begin + 1);

    NodesWave<HD, F8, QW> w;
    w.begin(a, g.row, kvh, q0, queries);
    find_masks<T::kThreads>(a, g.row, g.nodes, sh.up, s_mask);
    const bool idle = q0 >= queries;                                     // a wave without queries only helps with the tiles

    int stage = 0, t = g.t_begin;
    auto arrive_tile = [&] {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (t + 1 < g.t_end) request(stage ^ 1);
        pages_ahead = bits();
        look_up(t + 2);
    };
    auto next_tile = [&] {
        pages = pages_ahead;
        stage ^= 1;
        ++t;
    };
    constexpr int kStep = T::RT * 16;                                    // tokens of a wave's step
    constexpr int kSteps = T::kTokens / kStep;
    auto take = [&](auto mode, int from) {                               // the tile's steps from `from` on; how far that came
        if (idle) return kSteps;
        const unsigned char* const base = lds + stage * T::kStage;
#pragma unroll 1
        for (int step = from; step < kSteps; ++step) {
            if (((t * kSteps + step) & (WK - 1)) != wk) continue;
            const int64_t j0 = (int64_t)t * T::kTokens + step * kStep - g.ctx;
            if constexpr (mode.value == kMasked)
                if (j0 >= g.nodes) break;                                // (past the row's end)
            const unsigned char* const sk = base + step * kStep * T::kRow;
            const float* const sc = reinterpret_cast<const float*>(base + 2 * T::kTile) + step * kStep;
            uint64_t seen[QW];
#pragma unroll
            for (int b = 0; b < QW; ++b) {
                seen[b] = ~0ull;
                if constexpr (mode.value == kMasked) seen[b] = pages >> (step * kStep / TABED_CACHE_BLOCK) & 1 ? window(s_mask[w.node[b]], j0) : 0ull;
            }
            if constexpr (mode.value == kMasked && F8) {                 // (in halves: with 64 tokens, of which some are not seen, registers spill in all steps' way, 16 ragged trees 80 us for 79)
#pragma unroll 1
                for (int half = 0; half < 2; ++half) {
                    uint32_t some[QW];
#pragma unroll
                    for (int b = 0; b < QW; ++b) some[b] = (uint32_t)(seen[b] >> half * 32);
                    const unsigned char* const row = sk + half * kNodesTile * T::kRow;
                    w.template step<kMasked, 2>(row, row + T::kTile, sc + half * kNodesTile, sc + T::kTokens + half * kNodesTile, a.scale2, some);
                }
            } else if (!w.template step<mode.value, T::RT>(sk, sk + T::kTile, sc, sc + T::kTokens, a.scale2, seen)) {
                return step;
            }
        }
        return kSteps;
    };
    auto whole = [&] { return t < g.t_end && (int64_t)(t + 1) * T::kTokens <= g.ctx && pages == (1u << T::kPages) - 1; };
    int came = kSteps;
    while (whole()) {
        arrive_tile();
        came = take(NodesMode<kWhole>{}, 0);
        if (came < kSteps) break;
        next_tile();
    }
    if constexpr (F8) {
        if (came < kSteps) {                                             // (in a tile that is there; all waves meet as often as there are tiles, whichever loop they are in)
            take(NodesMode<kFar>{}, came);
            next_tile();
            while (whole()) {
                arrive_tile();
                take(NodesMode<kFar>{}, 0);
                next_tile();
            }
        }
    }
    const int first_masked = t;
    while (t < g.t_end) {
        arrive_tile();
        take(NodesMode<kMasked>{}, 0);
        next_tile();
    }

    // ---- the waves' results as one
    if (tid == 0) sh.pick[3] = 0;
    __syncthreads();
    if (w.odd) sh.pick[3] = 1;
    float* const s_o = reinterpret_cast<float*>(lds);
    float4* const s_ml = reinterpret_cast<float4*>(lds + (size_t)T::kQueries * T::kLine * 4);
    const int col = lane & 15, grp = lane >> 4, apart = WQ * T::kUnit;
#pragma unroll
    for (int b = 0; b < QW; ++b) {
        const int i = wk * apart + wq * T::kUnit + b * 16 + col;
#pragma unroll
        for (int d = 0; d < HD / 16; ++d) *reinterpret_cast<f32x4b*>(s_o + (size_t)i * T::kLine + d * 16 + grp * 4) = w.acc[b][d];
        const float4 ml = w.sums(b);
        if (grp == 0) s_ml[i] = ml;
    }
    __syncthreads();
    auto masked = [](int) { return true; };                              // from the first one on
    const int odd_from = first_masked * (T::kTokens / kNodesTile), odd_to = g.t_end * (T::kTokens / kNodesTile);
    const bool odd = sh.pick[3] != 0 && odd_is_seen<HD, F8, T::kThreads>(a, g, odd_from, odd_to, kvh, &sh.pick[3], masked);
    for (int p = tid; p < here * (HD / 4); p += T::kThreads) {
        const int i = p / (HD / 4), dim = p % (HD / 4) * 4, qi = tile_q * a.per_tile + i;
        float o[4];
        const float4 ml = join_parts<T::kLine>(s_o, s_ml, WK, apart, i, dim, o);
        if (odd) add_odd<HD, F8>(a, g, odd_from, odd_to, kvh, s_mask[qi / a.group], dim, masked, o);
        store_result<HD>(a, g, kvh, tile_q, qi, dim, ml, o);
    }
}

// Ranges joined: PARTS waves a query, a lane every 64th pair of dims.  (Four where a row has 16 ranges or more: 64 of them read by one wave take 12 us; with four ranges
// a row and 8192 queries four waves a query take 13 us longer.)
template <int HD, int PARTS>
__global__ __launch_bounds__(256) void k_attention_nodes_join(NodesAttnArgs a) {
    constexpr int PL = (HD / 2 + 63) / 64;
    __shared__ float2 s_o[PARTS > 1 ? PARTS : 1][PL * 64];
    const int r = blockIdx.y, wave = threadIdx.x / 64, lane = threadIdx.x & 63, part = wave % PARTS, unit = blockIdx.x * (4 / PARTS) + wave / PARTS;
    const int nodes = nodes_of(a.n_nodes, r, a.N), node = unit / a.q_heads, head = unit % a.q_heads;
    if (node >= nodes) return;                                           // (all waves of a query)
    const int2 got = a.ranges[r];
    const int ranges = got.y;
    if (ranges <= 1) return;
    const int kvh = head / a.group, qi = node * a.group + head % a.group, tile = qi / a.per_tile, i = qi % a.per_tile;
    auto place = [&](int s) { return (((int64_t)(got.x + s) * a.c.kv_heads + kvh) * a.tiles + tile) * a.per_tile + i; };
    float m = -INFINITY;
    for (int s = lane; s < ranges; s += 64) m = fmaxf(m, a.ml[place(s)].x);
    m = wave_max(m);
    const bool mine = lane < HD / 2;
    float l = 0.f, lr = 0.f, o[PL][2] = {};
    for (int s0 = 0; s0 < ranges; s0 += 64) {
        float f = 0.f, lw = 0.f, lrw = 0.f;
        if (s0 + lane < ranges) {
            const float4 ml = a.ml[place(s0 + lane)];
            f = share(ml, m);
            lw = ml.y * f;
            lrw = ml.z * f;
        }
        l += wave_sum(lw);
        lr += wave_sum(lrw);
        const int some = min(64, ranges - s0);
        for (int s = part; s < some; s += 8 * PARTS) {                   // (eight at a time in flight; past the last one its sums again, times 0)
            float2 x[8][PL];
#pragma unroll
            for (int i8 = 0; i8 < 8; ++i8) {
                const float* from = a.o + place(s0 + min(s + i8 * PARTS, some - 1)) * HD;
#pragma unroll
                for (int p = 0; p < PL; ++p) x[i8][p] = *reinterpret_cast<const float2*>(from + (mine ? (p * 64 + lane) * 2 : 0));
            }
#pragma unroll
            for (int i8 = 0; i8 < 8; ++i8) {
                const float fs = s + i8 * PARTS < some ? lane_f32(f, s + i8 * PARTS) : 0.f;
#pragma unroll
                for (int p = 0; p < PL; ++p) {
                    o[p][0] += counted(x[i8][p].x, fs);
                    o[p][1] += counted(x[i8][p].y, fs);
                }
            }
        }
    }
    if constexpr (PARTS > 1) {
#pragma unroll
        for (int p = 0; p < PL; ++p) s_o[part][p * 64 + lane] = make_float2(o[p][0], o[p][1]);
        __syncthreads();
        if (part > 0) return;
#pragma unroll
        for (int p = 0; p < PL; ++p)
#pragma unroll
            for (int w = 1; w < PARTS; ++w) {
                o[p][0] += s_o[w][p * 64 + lane].x;
                o[p][1] += s_o[w][p * 64 + lane].y;
            }
    }
    const float inv = lr == 0.f ? 0.f : 1.f / lr;
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
// The variant for a row and head's number of queries, handed to `go`; few: rows and heads leave half of the CUs without a workgroup, and eight waves share what one has (LDS
// holds their stages where a row of keys has 128 bytes at most): 4 rows of 900 tokens, 6 nodes, 12 heads of 64 8.8 us, with four waves 10.1; 8 rows of 1000, 4 nodes, 32 / 8
// heads of 128, e4m3 11.7 and 14.2; with more of them they only hold each other up (16 rows of 900 12.5 and 12.3, 16 of 300 to 5000 in e4m3 29.9 and 28.6).
inline bool few_units(int64_t rows, int kv_heads) { return rows * kv_heads < 128; }
template <int HD, bool F8, typename F>
inline auto with_nodes_variant(int queries, bool few, F&& go) {
    constexpr int kRow = HD * (F8 ? 1 : 2), WK = kRow >= 512 ? 2 : 4;    // (LDS)
    if constexpr (kRow <= 128) {
        if (few && queries <= 16) return go(NodesNarrow<HD, F8, 1, 8>{});
        if (few && queries <= 32) return go(NodesNarrow<HD, F8, 2, 8>{});
    }
    if (queries <= 16) return go(NodesNarrow<HD, F8, 1, WK>{});
    if constexpr (HD < 256)
        if (queries <= 32) return go(NodesNarrow<HD, F8, 2, WK>{});
    return go(NodesWide<HD, F8>{});
}
template <class T>
struct IsWide : std::false_type {};
template <int HD, bool F8>
struct IsWide<NodesWide<HD, F8>> : std::true_type {};

template <class T>
hipError_t launch_nodes_variant(const ProfScope* prof, const NodesAttnArgs& a, hipStream_t s) {
    static std::once_flag once[kMaxDevices];
    static hipError_t rc[kMaxDevices];
    const int64_t units = (int64_t)a.slots * a.c.kv_heads;
    hipError_t e;
    if constexpr (IsWide<T>::value) {
        e = raise_on_device(&k_attention_nodes_wide<T>, T::kLds, once, rc);
        if (e != hipSuccess) return e;
        launch(prof, k_attention_nodes_wide<T>, dim3((unsigned)((units + 7) / 8 * 8 * a.tiles)), dim3(T::kThreads), T::kLds, s, a);
    } else {
        e = raise_on_device(&k_attention_nodes<T>, T::kLds, once, rc);
        if (e != hipSuccess) return e;
        launch(prof, k_attention_nodes<T>, dim3((unsigned)units), dim3(T::kThreads), T::kLds, s, a);
    }
    if (a.split && a.slots >= 16 * a.rows)
        hipLaunchKernelGGL((k_attention_nodes_join<T::HD, 4>), dim3((unsigned)(a.N * a.q_heads), a.rows), dim3(256), 0, s, a);
    else if (a.split)
        hipLaunchKernelGGL((k_attention_nodes_join<T::HD, 1>), dim3((unsigned)((a.N * a.q_heads + 3) / 4), a.rows), dim3(256), 0, s, a);
    return hipGetLastError();
}

#define TABED_NODES_HD(HD_)                                                                                                   \
    template <>                                                                                                               \
    hipError_t launch_nodes_hd<HD_>(bool f8, const ProfScope* prof, const NodesAttnArgs& a, hipStream_t s) {                  \
        auto go = [&](auto v) { return launch_nodes_variant<decltype(v)>(prof, a, s); };                                      \
        const bool few = few_units(a.rows, a.c.kv_heads);                                                                     \
        return f8 ? with_nodes_variant<HD_, true>(a.N * a.group, few, go) : with_nodes_variant<HD_, false>(a.N * a.group, few, go); \
    }
template <int HD>
hipError_t launch_nodes_hd(bool f8, const ProfScope* prof, const NodesAttnArgs& a, hipStream_t s);

}  // namespace tabed
