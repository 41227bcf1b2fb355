// The 8-bit key / value cache: appending tokens (tabed_cache_append_q8) and attention over it (tabed_attention_q8).
//
// A block holds 64 tokens of one head in int8 with one scale for its keys and one for its values, in the order in which the
// matrix instructions take them, so that a wave's 16-byte loads are whole lines:
//   keys    [token / 4 % 4][dim / 16][token / 16][token % 4][dim % 16]
//   values  [dim / 16][token / 16][dim % 16][token % 16]
#include <algorithm>
#include <cmath>

#include "body_utils.h"
#include "q8_utils.h"

namespace tabed {

constexpr int kCB = TABED_CACHE_BLOCK;
static_assert(kCB == 64, "a block is one k-step of v_mfma_i32_16x16x64_i8");

struct CacheView {
    int kv_heads, hd, blocks, max_blocks;
    int8_t* k;
    int8_t* v;
    float* kscale;
    float* vscale;
    const int32_t* table;
};
static CacheView view_of(const tabed_cache_q8& c) {
    return CacheView{c.kv_heads, c.head_dim, c.blocks, c.max_blocks, static_cast<int8_t*>(c.k), static_cast<int8_t*>(c.v), c.kscale, c.vscale, c.table};
}
__device__ __forceinline__ int row_tokens(const int32_t* n_new, int row, int T) {
    return n_new == nullptr ? T : min(max(n_new[row], 0), T);
}

// ---------------------------------------------------------------- append
// The keys, or the values, of one head in one block of a row's new tokens are one task: largest magnitude, scale, steps.  Tokens that a
// begun block keeps are read only where its scale grows; they are rounded again then.
struct AppendArgs {
    CacheView c;
    int rows, T, nb;
    const void* k;
    const void* v;
    int64_t row_stride, tok_stride;
    const int32_t* ctx_len;
    const int32_t* n_new;
};

struct AppendTask {
    bool values;
    int off, count;          // the first `off` tokens of the block are kept, `count` new ones go behind them
    int64_t from;            // the first new token's, in k or v (elements)
    int64_t ph;              // block and head: scale (open_task)
    int page, h;
};
// Task number w; false: there is nothing to do.  The new tokens can be requested before the block's page is there (open_task).
__device__ __forceinline__ bool append_task(const AppendArgs& a, int w, AppendTask& t) {
    t.values = w & 1;
    w >>= 1;
    const int h = w % a.c.kv_heads;
    w /= a.c.kv_heads;
    const int j = w % a.nb, row = w / a.nb;
    if (row >= a.rows) return false;
    const int n = row_tokens(a.n_new, row, a.T), ctx = max(a.ctx_len[row], 0);
    const int64_t slot = (int64_t)(ctx / kCB) + j, first = slot * kCB;         // (64 bits: a position may be near 2^31)
    if (slot >= a.c.max_blocks) return false;
    t.off = (int)max(ctx - first, (int64_t)0);
    const int64_t t0 = first + t.off - ctx;
    if (t0 >= n) return false;
    t.count = (int)min((int64_t)(kCB - t.off), n - t0);
    t.page = a.c.table[(int64_t)row * a.c.max_blocks + slot];
    t.h = h;
    t.from = row * a.row_stride + t0 * a.tok_stride + (int64_t)h * a.c.hd;
    return true;
}
__device__ __forceinline__ bool open_task(const AppendArgs& a, AppendTask& t) {
    if (t.page < 0 || t.page >= a.c.blocks) return false;
    t.ph = (int64_t)t.page * a.c.kv_heads + t.h;
    return true;
}
__device__ __forceinline__ float grown_scale(float before, uint32_t most) {
    const float fresh = scale_of(most);
    return (before != before || fresh != fresh) ? __builtin_nanf("") : fmaxf(before, fresh);
}
// A kept token's step, in steps of the new scale.
__device__ __forceinline__ int step_again(int q, float before, float scale) { return scale > 0.f ? to_step((float)q * before / scale) : 0; }
__device__ __forceinline__ uint32_t word_again(uint32_t w, int keep /* of its four steps, the first ones */, float before, float scale) {
    int s[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int q = (int8_t)(w >> (8 * e));
        s[e] = e < keep ? step_again(q, before, scale) : q;
    }
    return pack_i8(s[0], s[1], s[2], s[3]);
}
__device__ __forceinline__ u32x4_e4 pack_steps(const int (&s)[16]) {
    return u32x4_e4{pack_i8(s[0], s[1], s[2], s[3]), pack_i8(s[4], s[5], s[6], s[7]), pack_i8(s[8], s[9], s[10], s[11]), pack_i8(s[12], s[13], s[14], s[15])};
}
__device__ __forceinline__ int key_piece(int at, int c, int chunks) { return ((at / 4 % 4) * chunks + c) * 16 + at / 16 * 4 + at % 4; }      // 16 dims of a token
__device__ __forceinline__ int value_piece(int g, int dim) { return (dim / 16 * 4 + g) * 16 + dim % 16; }                                     // 16 tokens of a dim

// Up to FEW new tokens a row: a wave a task, a lane for every 64th dim, a byte stored for each value.  Latency bounds it: positions
// -> page -> scale; the new values are on their way meanwhile (64 rows x 12 heads of 64 dims, four tokens: 4.35 -> 3.95 us; a workgroup a task gains nothing by it).
template <bool BF16, int hd, int FEW>
__global__ __launch_bounds__(kBlock) void k_cache_append_few(AppendArgs a) {
    constexpr int chunks = hd / 16, kDims = (hd + 63) / 64;           // kDims: of a lane
    AppendTask t;
    if (!append_task(a, blockIdx.x * kWavesPerBlock + (threadIdx.x >> 6), t)) return;      // uniform for the wave; no barriers
    const int lane = threadIdx.x & 63;
    const void* const src = t.values ? a.v : a.k;
    float x[FEW][kDims];
    uint32_t most = 0;
#pragma unroll
    for (int n = 0; n < FEW; ++n)
#pragma unroll
        for (int i = 0; i < kDims; ++i)                                // (past the last token or dim: that again)
            x[n][i] = load_value<BF16>(src, t.from + min(n, t.count - 1) * a.tok_stride + min(i * 64 + lane, hd - 1));
    __builtin_amdgcn_sched_barrier(0);
    if (!open_task(a, t)) return;
    int8_t* const block = (t.values ? a.c.v : a.c.k) + t.ph * kCB * hd;
    float* const scale_at = (t.values ? a.c.vscale : a.c.kscale) + t.ph;
    const float before = t.off > 0 ? *scale_at : 0.f;
#pragma unroll
    for (int n = 0; n < FEW; ++n)
#pragma unroll
        for (int i = 0; i < kDims; ++i) most = max(most, magnitude(x[n][i]));
    const float scale = grown_scale(before, wave_max_u32(most));
    const bool live = scale > 0.f;
    if (t.off > 0 && !(scale == before)) {                             // pieces with kept tokens, a lane each
        for (int p = lane; p < (t.values ? (t.off + 15) / 16 * hd : t.off * chunks); p += 64) {
            const int piece = t.values ? value_piece(p / hd, p % hd) : key_piece(p / chunks, p % chunks, chunks);
            const int keep = t.values ? t.off - p / hd * 16 : 16;      // of its 16 steps
            u32x4_e4* const at = reinterpret_cast<u32x4_e4*>(block) + piece;
            u32x4_e4 w = *at;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = word_again(w[i], keep - 4 * i, before, scale);
            *at = w;
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");              // the new tokens' bytes, which share pieces with them, come after
    }
#pragma unroll
    for (int n = 0; n < FEW; ++n)
#pragma unroll
        for (int i = 0; i < kDims; ++i) {
            const int dim = i * 64 + lane, at = t.off + n;
            if (n < t.count && dim < hd)
                block[t.values ? value_piece(at / 16, dim) * 16 + at % 16 : key_piece(at, dim / 16, chunks) * 16 + dim % 16] =
                    (int8_t)(live ? (int)rintf(x[n][i] / scale) : 0);
        }
    if (lane == 0) *scale_at = scale;
}

// Four words of four bytes, transposed.
__device__ __forceinline__ void transpose_bytes(const uint32_t (&r)[4], uint32_t (&out)[4]) {
    const uint32_t a = __builtin_amdgcn_perm(r[1], r[0], 0x05010400u), b = __builtin_amdgcn_perm(r[1], r[0], 0x07030602u);
    const uint32_t c = __builtin_amdgcn_perm(r[3], r[2], 0x05010400u), d = __builtin_amdgcn_perm(r[3], r[2], 0x07030602u);
    out[0] = __builtin_amdgcn_perm(c, a, 0x05040100u);
    out[1] = __builtin_amdgcn_perm(c, a, 0x07060302u);
    out[2] = __builtin_amdgcn_perm(d, b, 0x05040100u);
    out[3] = __builtin_amdgcn_perm(d, b, 0x07060302u);
}

// More: a workgroup a task, a thread for pieces of 16 dims of a token.  Keys are stored as such a piece, values go through LDS, from
// where a thread takes 16 tokens of four dims and transposes them.  Memory bounds a prompt: 12000 tokens x 8 heads of 128 dims in 16 rows,
// 74 MB, 23 us, 3.2 TB/s (a workgroup asks for its tokens once, waits for its largest and stores: nothing overlaps within it).
template <bool BF16, int hd>
__global__ __launch_bounds__(kBlock) void k_cache_append(AppendArgs a) {
    constexpr int chunks = hd / 16, row_bytes = hd + 16, kPer = (kCB * chunks + kBlock - 1) / kBlock;      // kPer: pieces of a thread
    __shared__ uint32_t s_most[kWavesPerBlock];
    __shared__ __attribute__((aligned(16))) unsigned char s_t[kCB * row_bytes];       // values: [token][hd] steps
    AppendTask t;
    if (!append_task(a, blockIdx.x, t) || !open_task(a, t)) return;    // uniform
    const int tid = threadIdx.x;
    int8_t* const block = (t.values ? a.c.v : a.c.k) + t.ph * kCB * hd;
    float* const scale_at = (t.values ? a.c.vscale : a.c.kscale) + t.ph;
    const float before = t.off > 0 ? *scale_at : 0.f;
    const void* const src = t.values ? a.v : a.k;
    float x[kPer][16];
    uint32_t most = 0;
#pragma unroll
    for (int p = 0; p < kPer; ++p) {
        const int idx = p * kBlock + tid;
        if (idx < t.count * chunks) {
            load_values<16, BF16>(src, t.from + (int64_t)(idx / chunks) * a.tok_stride + idx % chunks * 16, x[p]);
#pragma unroll
            for (int e = 0; e < 16; ++e) most = max(most, magnitude(x[p][e]));
        }
    }
    most = wave_max_u32(most);
    if ((tid & 63) == 0) s_most[tid >> 6] = most;
    __syncthreads();
    most = max(max(s_most[0], s_most[1]), max(s_most[2], s_most[3]));
    const float scale = grown_scale(before, most), inv = scale > 0.f ? 1.f / scale : 0.f;
    const bool grown = t.off > 0 && !(scale == before);                // uniform
    if (tid == 0) *scale_at = scale;
#pragma unroll
    for (int p = 0; p < kPer; ++p) {
        const int idx = p * kBlock + tid, at = t.off + idx / chunks, c = idx % chunks;
        if (idx < t.count * chunks) {
            int s[16];
            if (scale > 0.f) {
                steps_of(x[p], scale, inv, s);
            } else {
#pragma unroll
                for (int e = 0; e < 16; ++e) s[e] = 0;
            }
            if (t.values) *reinterpret_cast<u32x4_e4*>(s_t + at * row_bytes + c * 16) = pack_steps(s);
            else reinterpret_cast<u32x4_e4*>(block)[key_piece(at, c, chunks)] = pack_steps(s);
        }
    }
    if (!t.values) {
        if (grown)
            for (int idx = tid; idx < t.off * chunks; idx += kBlock) {
                u32x4_e4* const at = reinterpret_cast<u32x4_e4*>(block) + key_piece(idx / chunks, idx % chunks, chunks);
                u32x4_e4 w = *at;
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = word_again(w[i], 4, before, scale);
                *at = w;
            }
        return;
    }
    __syncthreads();
    const int end = t.off + t.count, g0 = grown ? 0 : t.off / 16, g1 = (end + 15) / 16;       // groups of 16 tokens that change
    for (int idx = tid; idx < (g1 - g0) * (hd / 4); idx += kBlock) {
        const int g = g0 + idx / (hd / 4), dim0 = idx % (hd / 4) * 4, keep = t.off - g * 16;   // of its tokens, the first `keep` are kept
        u32x4_e4 w[4];                                                 // [dim]: words of four tokens
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t r[4], c[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) r[e] = *reinterpret_cast<const uint32_t*>(s_t + (g * 16 + 4 * i + e) * row_bytes + dim0);      // (not new: replaced below)
            transpose_bytes(r, c);
#pragma unroll
            for (int d = 0; d < 4; ++d) w[d][i] = c[d];
        }
        const bool some_stay = keep > 0 || (g + 1) * 16 > end;
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            u32x4_e4* const at = reinterpret_cast<u32x4_e4*>(block) + value_piece(g, dim0 + d);
            if (some_stay) {
                const u32x4_e4 old = *at;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t kept = grown ? word_again(old[i], keep - 4 * i, before, scale) : old[i];
                    uint32_t mask = 0;                                 // bytes of tokens that are not new
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (4 * i + e < keep || g * 16 + 4 * i + e >= end) mask |= 255u << (8 * e);
                    w[d][i] = (w[d][i] & ~mask) | (kept & mask);
                }
            }
            *at = w[d];
        }
    }
}

static int append_blocks(int T) { return (T + kCB - 2) / kCB + 1; }

int64_t append_workgroups(const tabed_cache_q8& c, int rows, int T) { return 2ll * c.kv_heads * rows * append_blocks(T); }

template <int hd>
static void launch_append(const ProfScope* prof, int kv_dtype, unsigned tasks, const AppendArgs& a, hipStream_t s) {
    // A wave's own time grows with tokens times dims, a workgroup's hardly; but four times as many workgroups start.  Six tokens of 64 rows
    // x 8 heads: 4.8 us against 7.2 with 64 dims, 6.8 against 7.5 with 128, 11.7 against 9.8 with 256; 16 rows 4.2 - 5.3, 5.8 - 5.2, 8.6 - 5.5.
    const unsigned quarter = (tasks + kWavesPerBlock - 1) / kWavesPerBlock;
    auto go = [&](auto kernel, unsigned workgroups) { launch(prof, kernel, dim3(workgroups), dim3(kBlock), 0, s, a); };
    if (a.T <= 4) kv_dtype == 1 ? go(k_cache_append_few<true, hd, 4>, quarter) : go(k_cache_append_few<false, hd, 4>, quarter);
    else if (hd <= 64 && a.T <= 8) kv_dtype == 1 ? go(k_cache_append_few<true, std::min(hd, 64), 8>, quarter) : go(k_cache_append_few<false, std::min(hd, 64), 8>, quarter);
    else kv_dtype == 1 ? go(k_cache_append<true, hd>, tasks) : go(k_cache_append<false, hd>, tasks);
}

hipError_t launch_cache_append(const tabed_cache_q8& c, int rows, int T, int kv_dtype, const void* k, const void* v, int64_t row_stride,
                               int64_t tok_stride, const int32_t* ctx_len, const int32_t* n_new, hipStream_t s) {
    const AppendArgs a{view_of(c), rows, T, append_blocks(T), k, v, row_stride, tok_stride, ctx_len, n_new};
    ProfScope prof(TABED_K_BODY, s);
    const unsigned tasks = (unsigned)append_workgroups(c, rows, T);
    switch (c.head_dim) {
        case 32: launch_append<32>(&prof, kv_dtype, tasks, a, s); break;
        case 64: launch_append<64>(&prof, kv_dtype, tasks, a, s); break;
        case 96: launch_append<96>(&prof, kv_dtype, tasks, a, s); break;
        case 128: launch_append<128>(&prof, kv_dtype, tasks, a, s); break;
        case 256: launch_append<256>(&prof, kv_dtype, tasks, a, s); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

// ---------------------------------------------------------------- attention
// A query is one new token and one of the `group` heads that share a key / value head.  One wave walks over blocks of a row and key / value
// head: scores S^T = K Q^T, outputs O^T = V^T P^T, the cache as the row operand of both products, softmax with a running maximum and sum.  The
// lane that holds the scores of tokens 16 g .. 16 g + 15 (g = lane / 16) for a column (lane % 16) is the one that has to hold their
// probabilities for the second product: they never leave it.  K of the next block is requested when the scores are there, V when
// the outputs are.
// Cached bytes go into the products as they are or exactly converted; queries and probabilities with 22 bits and more:
//   * scores: v_mfma_i32_16x16x64_i8.  A query is integers relative to its largest, in digits of base 256 (-128 .. 127) that are multiplied
//     one by one; the products and their sums are exact.
//   * up to four queries (a step's token, up to four heads a group): four digits stand in four columns, lane 4 query + digit adds them up,
//     and the probabilities (2^30 for 1) go the same way into v_mfma_i32_16x16x64_i8.  Nothing is converted.
//   * more queries: sixteen, a column each; three digits are three products.  Probabilities (2^14 for 1) are the sum of two halves, for
//     v_mfma_f32_16x16x32_f16, and the values' bytes become halves on the way, five vector instructions for four of them.  Digits
//     would take half as many instructions again for the sixteen, and four times as many with the layout above.  Vector instructions
//     bound this form from about 1000 tokens a row on: 380 a block of 128 dims, of which converting the values is 160.
// With few queries the bytes bound it: 120000 tokens x 8 heads of 128 dims, 246 MB, take 50 us, 4.9 TB/s; 64 rows x 12 heads of 64 dims and 500
// tokens, 50 MB, 13.6 us, of which about 4 are the launch and the chain length -> page -> keys -> values.
// The waves of a workgroup take blocks in turn and meet in LDS; a row's blocks are cut into S ranges where the rows and heads do
// not fill the chip, and the last of its workgroups to arrive joins them (in range order: results do not depend on who is last).
struct AttnArgs {
    CacheView c;
    int rows, T, group;          // group: query heads of a key / value head
    int tiles;                   // workgroups of one row and key / value head (and range)
    int S;                       // ranges of blocks
    int q_bf16, out_bf16;
    const void* q;
    int64_t q_row, q_tok;
    void* out;
    int64_t out_row, out_tok;
    float* lse;                  // [rows,T,q_heads] or null
    const int32_t* ctx_len;
    const int32_t* n_new;
    float scale2;                // scale * log2(e)
    uint32_t* arrivals;          // [rows, kv_heads, tiles], where there are several ranges
    float* po;                   // [rows, kv_heads, tiles, S][queries][hd]: sums of p v, at the range's own maximum
    float* pml;                  // the same [2][queries]: maxima (base 2), sums of p
};

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4v __attribute__((ext_vector_type(4)));
typedef float f32x4v __attribute__((ext_vector_type(4)));
typedef float f32x2_any __attribute__((ext_vector_type(2), aligned(4)));
typedef uint32_t u32_e2 __attribute__((aligned(2)));

constexpr int kMaxRanges = 64;
constexpr int kCutUnits = 256;   // rows x heads x tiles that are cut into ranges: fewer than this
constexpr int attn_queries(bool wide) { return wide ? 16 : 4; }        // of a workgroup

// The four lanes of a query add the same four products, each in its own order, and have to come to the same sum: they give the digits of one
// probability.  A product that is fused into the addition in one lane, and rounded in the others, gave digits of different numbers.
__device__ __forceinline__ float rounded_product(float a, float b) {
#pragma clang fp contract(off)
    return a * b;
}

// Eight steps (two words of four bytes) as halves: 0x6400 + u is 1024 + u, and u = step + 128.
__device__ __forceinline__ f16x8 halves_of(int lo, int hi) {
    u32x4v r;
    const uint32_t w[2] = {(uint32_t)lo ^ 0x80808080u, (uint32_t)hi ^ 0x80808080u};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const f16x2 shift = {(_Float16)1152.f, (_Float16)1152.f};
        r[2 * i] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, w[i], 0x04010400u)) - shift);
        r[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, w[i], 0x04030402u)) - shift);
    }
    return __builtin_bit_cast(f16x8, r);
}
// x as the sum of two halves.  (`one` is 1 in a way that the compiler does not see: a product and a sum with a half among their operands
// are one instruction that rounds to a half, v_fma_mixlo_f16; the sum alone takes three.)
__device__ __forceinline__ void split_halves(const float* x, float one, f16x8& hi, f16x8& lo) {
#pragma unroll
    for (int e = 0; e < 8; ++e) hi[e] = (_Float16)x[e];
#pragma unroll
    for (int e = 0; e < 8; ++e) lo[e] = (_Float16)fmaf(x[e], one, -(float)hi[e]);
}
__device__ __forceinline__ void publish_pair(float* p, float a, float b) {          // 8-byte aligned
    publish_store(reinterpret_cast<double*>(p), __builtin_bit_cast(double, make_float2(a, b)));
}
__device__ __forceinline__ float2 published_pair(const float* p) {
    return __builtin_bit_cast(float2, published_load(reinterpret_cast<const double*>(p)));
}
// A lane's value and that of the lane 16 (32) away, in either order: over the four lanes of a column without going through LDS.
__device__ __forceinline__ uint2 with_16(uint32_t v) {
    const auto p = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return make_uint2(p[0], p[1]);
}
__device__ __forceinline__ uint2 with_32(uint32_t v) {
    const auto p = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return make_uint2(p[0], p[1]);
}
template <typename F>
__device__ __forceinline__ uint32_t over_groups(uint32_t v, F&& f) {
    const uint2 a = with_16(v);
    const uint2 b = with_32(f(a.x, a.y));
    return f(b.x, b.y);
}
__device__ __forceinline__ float max_groups(float v) {
    return __builtin_bit_cast(float, over_groups(__builtin_bit_cast(uint32_t, v), [](uint32_t x, uint32_t y) {
        return __builtin_bit_cast(uint32_t, fmaxf(__builtin_bit_cast(float, x), __builtin_bit_cast(float, y)));
    }));
}
__device__ __forceinline__ float sum_groups(float v) {
    return __builtin_bit_cast(float, over_groups(__builtin_bit_cast(uint32_t, v), [](uint32_t x, uint32_t y) {
        return __builtin_bit_cast(uint32_t, __builtin_bit_cast(float, x) + __builtin_bit_cast(float, y));
    }));
}
// Byte `b` of four words side by side (sel: attn_byte(b)).
__device__ __forceinline__ uint32_t attn_byte(int b) { return (uint32_t)b | (uint32_t)(4 + b) << 8 | 0x0c0c0000u; }
__device__ __forceinline__ uint32_t bytes_of(const uint32_t (&z)[4], uint32_t sel) {
    return __builtin_amdgcn_perm(z[1], z[0], sel) | __builtin_amdgcn_perm(z[3], z[2], sel) << 16;
}

// (Two waves a SIMD: up to 256 registers, all of them vector registers.  With more at hand the products' results go through accumulation
// registers, an instruction each to get them back.  With 256 dims and few queries the kernel would take 260, and 64 rows x 8 heads then have
// half of their workgroups waiting: 250 tokens 22.7 us against 18.3, 1000 tokens 49.2 against 43.9.  Many queries need 370.)
template <int HD, bool WIDE, int NW>
__global__ __launch_bounds__(NW * 64, HD <= 128 || !WIDE ? 2 : 1) void k_attn_q8(AttnArgs a) {
    constexpr int NQ = attn_queries(WIDE), KS = (HD + 63) / 64, H16 = HD / 16, OT = HD / 16, DG = WIDE ? 3 : 1;
    constexpr int RD = !WIDE ? HD : (HD % 64 == 0 ? 64 : 32);          // dims that meet in LDS at a time
    __shared__ __attribute__((aligned(16))) float s_o[NW][NQ][RD + 4];
    __shared__ float s_m[NW][NQ], s_l[NW][NQ], s_M[NQ], s_L[NQ];
    __shared__ int64_t s_out[NQ];                                     // where a query's output begins; -1: it has none
    __shared__ float s_f[kMaxRanges][NQ];                             // shares of the waves, later of the ranges
    __shared__ int s_last;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = lane >> 4, c = lane & 15, dig = c & 3, my_q = WIDE ? c : c >> 2;
    // Workgroup w goes to XCD w % 8: the tiles of a row and head, which read the same blocks, run back to back on one.  The first
    // ranges come first: short rows have no others.
    const int tile = (int)(blockIdx.x >> 3) % a.tiles;
    int w = ((int)(blockIdx.x >> 3) / a.tiles) * 8 + (int)(blockIdx.x & 7);
    const int h = w % a.c.kv_heads;
    w /= a.c.kv_heads;
    const int row = w % a.rows, sp = w / a.rows;
    if (sp >= a.S) return;                                             // uniform: the grid is padded to whole rounds of XCDs
    const int q0 = tile * NQ, most = a.T * a.group;
    const int32_t* const table = a.c.table + (int64_t)row * a.c.max_blocks;

    // What does not wait for anything else is requested first: this lane's query (past the last: the last, whose result is not stored
    // twice), and the first blocks' pages where the range is not yet to be worked out.
    const int qi = min(q0 + my_q, most - 1), tok = qi / a.group;
    u32x4_e4 raw[KS][4];                                               // (bf16: two of the four)
    {
        const int64_t base = row * a.q_row + tok * a.q_tok + (int64_t)(h * a.group + qi % a.group) * HD;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const int64_t from = base + (HD % 64 == 0 ? (ks * 4 + g) * 16 : min((ks * 4 + g) * 16, HD - 16));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (!a.q_bf16) raw[ks][i] = *reinterpret_cast<const u32x4_e4*>(static_cast<const float*>(a.q) + from + 4 * i);
                else if (i < 2) raw[ks][i] = u32x4_e4(*reinterpret_cast<const u32x4_e2*>(static_cast<const uint16_t*>(a.q) + from + 8 * i));
            }
        }
    }
    int page_l = -1;                                                   // of this wave's blocks, one a lane; -1: none
    if (a.S == 1) page_l = table[min(wave + NW * lane, a.c.max_blocks - 1)];
    __builtin_amdgcn_sched_barrier(0);

    // ---- blocks of this workgroup's range
    const int n = row_tokens(a.n_new, row, a.T), queries = n * a.group;
    if (q0 >= queries) return;                                         // uniform
    const int64_t cap = (int64_t)a.c.max_blocks * kCB;
    const int ctx = (int)min((int64_t)max(a.ctx_len[row], 0), cap);
    const int t_first = q0 / a.group, t_last = min(n - 1, (q0 + NQ - 1) / a.group);
    const int NB = (int)((min((int64_t)ctx + t_last + 1, cap) + kCB - 1) / kCB);       // that some query of the tile sees
    const int ranges = min(a.S, max(1, NB / NW));                      // (a block for every wave, where there are several)
    if (sp >= ranges) return;
    const int per = (NB + ranges - 1) / ranges, b_begin = min(sp * per, NB), b_end = min(b_begin + per, NB);

    float m_run = -INFINITY, l_run = 0.f;
    f32x4v o[OT];
#pragma unroll
    for (int ot = 0; ot < OT; ++ot) o[ot] = f32x4v{0.f, 0.f, 0.f, 0.f};
    const uint32_t sel = attn_byte(dig);
    const uint32_t flip = dig == 3 ? 0u : 0x80808080u;
    float one = 1.f;
    asm("" : "+s"(one));

    i32x4 kf[4][KS], vf[OT];                                           // the block that is on its way
    // Requests are never predicated, so that their number in flight is known: where there is no further block (mask 0 instead of ~0) all lanes
    // read the first 16 bytes of pieces of some block.
    const uint32_t at_lane = (uint32_t)lane * 16u, at_ragged = (HD % 64 == 0 || (KS - 1) * 4 + g < H16) ? at_lane : (uint32_t)c * 16u;     // (past a ragged
    auto request_k = [&](int page, uint32_t mask) {                                                          // end: for zeros of the query)
        const int8_t* const kb = a.c.k + ((int64_t)page * a.c.kv_heads + h) * (kCB * HD);
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
                kf[t][ks] = *reinterpret_cast<const i32x4*>(kb + ((ks + 1 < KS ? at_lane : at_ragged) & mask) + t * H16 * 256 + ks * 1024);
    };
    auto request_v = [&](int page, uint32_t mask) {
        const int8_t* const vb = a.c.v + ((int64_t)page * a.c.kv_heads + h) * (kCB * HD);
#pragma unroll
        for (int ot = 0; ot < OT; ++ot) vf[ot] = *reinterpret_cast<const i32x4*>(vb + (at_lane & mask) + ot * 1024);
    };

    // This wave's blocks are b_begin + wave + NW i; 64 of them are opened at a time, one a lane: pages, scales, and the request of the first.
    float ks_l = 0.f, vs_l = 0.f;
    unsigned long long there = 0;                                      // lanes whose blocks have not been requested
    int left = 0, at = 0;                                              // blocks that have not been used; the lane of the requested one
    auto open = [&](int i0) {
        const int b_lane = b_begin + wave + NW * (i0 + lane);
        if (a.S > 1 || i0 > 0) page_l = table[min(b_lane, a.c.max_blocks - 1)];
        if (b_lane >= b_end || page_l >= a.c.blocks) page_l = -1;
        ks_l = vs_l = 0.f;
        if (page_l >= 0) {
            ks_l = a.c.kscale[(int64_t)page_l * a.c.kv_heads + h];
            vs_l = a.c.vscale[(int64_t)page_l * a.c.kv_heads + h];
        }
        there = __ballot(page_l >= 0);
        left = __builtin_amdgcn_readfirstlane(__builtin_popcountll(there));
        if (left == 0) return;
        at = __builtin_ctzll(there);
        there &= there - 1;
        request_k(__builtin_amdgcn_readlane(page_l, at), ~0u);
        request_v(__builtin_amdgcn_readlane(page_l, at), ~0u);
    };
    open(0);
    __builtin_amdgcn_sched_barrier(0);

    // ---- the query as it goes into the product
    i32x4 qd[DG][KS];
    float worth;                                                       // what a step of it, times one of the keys', adds to a score
    {
        float x[KS][16];
        uint32_t top = 0;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const uint32_t half = raw[ks][e / 8][e / 2 % 4];
                const uint32_t bits = !a.q_bf16 ? raw[ks][e / 4][e % 4] : (e & 1) ? half & 0xffff0000u : half << 16;
                x[ks][e] = (HD % 64 == 0 || (ks * 4 + g) * 16 < HD) ? __builtin_bit_cast(float, bits) : 0.f;
                top = max(top, magnitude(x[ks][e]));
            }
        }
        top = over_groups(top, [](uint32_t x, uint32_t y) { return max(x, y); });
        // The largest becomes 2^30, or 0x7f7f78 (0x7f7f7f is the most that three digits hold); below 2^-100 all are zeros.
        constexpr float kTop = WIDE ? 8355704.f : 0x1p30f;
        const float m = __builtin_bit_cast(float, top);
        const bool finite = top < kInfBits, some = finite && m >= kTiny;
        const float by = some ? kTop / m : 0.f;
        worth = finite ? (some ? m / kTop : 0.f) * a.scale2 : __builtin_nanf("");
        if constexpr (!WIDE) worth *= (float)(1 << (8 * dig));
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t z[4];                                         // bytes: digits + 128, the lowest first; the fourth is one as it is
#pragma unroll
                for (int e = 0; e < 4; ++e) z[e] = (uint32_t)(int)rintf(x[ks][4 * i + e] * by) + 0x00808080u;
#pragma unroll
                for (int d = 0; d < DG; ++d) qd[d][ks][i] = (int)(bytes_of(z, WIDE ? attn_byte(d) : sel) ^ (WIDE ? 0x80808080u : flip));
            }
    }

    // One block, whose K and V are on their way; those of `next` are requested in between.
    auto block = [&](int b, float ksc, float vsc, int next, uint32_t mask) {
        float s[16], step = worth * ksc, vs = vsc;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            i32x4 acc[DG];
#pragma unroll
            for (int d = 0; d < DG; ++d) acc[d] = i32x4{0, 0, 0, 0};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                for (int d = 0; d < DG; ++d) acc[d] = __builtin_amdgcn_mfma_i32_16x16x64_i8(kf[t][ks], qd[d][ks], acc[d], 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (WIDE) s[4 * t + i] = fmaf((float)acc[2][i], 65536.f, (float)(acc[1][i] * 256 + acc[0][i]));    // (a digit's sum: below 2^22)
                else s[4 * t + i] = rounded_product((float)acc[0][i], step);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        request_k(next, mask);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (!WIDE) {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] += dpp_f32<kDppXor1>(s[i]);
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] += dpp_f32<kDppXor2>(s[i]);
            step = 1.f;
        }
        // With many queries the maximum comes off a score in the addition that scales it: both roundings then are of the score's size, and past 2^25
        // or so they would take the largest probability out of a half's range.  Where scores can be as large as 2^20 they are scaled before.
        constexpr float kFar = 0x1p20f / (8355704.f * 127.f * HD);
        const bool far = WIDE && __any(step > kFar);
        if (far || b * kCB + kCB - 1 > ctx + t_first) {                // uniform: some query does not see all of the block
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = b * kCB + g * 16 + i > ctx + tok ? -INFINITY : s[i] * step;
            step = 1.f;
            vs = b * kCB > ctx + tok ? 0.f : vsc;                      // (a query that sees none of the block: 0 times a bad scale is not 0)
        }
        float mx = s[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[i]);
        mx = max_groups(mx) * step;                                    // (no step is negative: the largest before is the largest after)
        const float m_new = fmaxf(m_run, mx), base = (m_new > -INFINITY) ? m_new : 0.f;
        if (__any(m_new > m_run)) {                                    // seldom after the first blocks
            const float alpha = __builtin_amdgcn_exp2f(m_run - base);
            m_run = m_new;
            l_run *= alpha;
#pragma unroll
            for (int ot = 0; ot < OT; ++ot) o[ot] *= alpha;
        }
        constexpr float kOneExp = WIDE ? 14.f : 0.f;
        float off = kOneExp - base;
        if (far) {                                                     // uniform
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] -= base;
            off = kOneExp;
        }
        float p[16], sum = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            p[i] = __builtin_amdgcn_exp2f(fmaf(s[i], step, off));
            sum += p[i];
        }
        l_run += sum;
        if constexpr (!WIDE) {
            i32x4 pd;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t z[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) z[e] = (uint32_t)(int)fmaf(p[4 * i + e], 0x1p30f, 0.5f) + 0x00808080u;
                pd[i] = (int)(bytes_of(z, sel) ^ flip);
            }
#pragma unroll
            for (int ot = 0; ot < OT; ++ot) {
                const i32x4 acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(vf[ot], pd, i32x4{0, 0, 0, 0}, 0, 0, 0);
#pragma unroll
                for (int i = 0; i < 4; ++i) o[ot][i] = fmaf((float)acc[i], vs, o[ot][i]);
            }
        } else {
            f16x8 ph[2], pl[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) split_halves(&p[8 * u], one, ph[u], pl[u]);
            constexpr int kSide = OT < 4 ? OT : (OT % 4 == 0 ? 4 : 2);  // accumulators side by side: a chain of four products each
#pragma unroll
            for (int o0 = 0; o0 < OT; o0 += kSide) {
                f32x4v acc[kSide];
                f16x8 v[kSide];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
#pragma unroll
                    for (int i = 0; i < kSide; ++i) v[i] = halves_of(vf[o0 + i][2 * u], vf[o0 + i][2 * u + 1]);
#pragma unroll
                    for (int i = 0; i < kSide; ++i) acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v[i], pl[u], u == 0 ? f32x4v{0.f, 0.f, 0.f, 0.f} : acc[i], 0, 0, 0);
#pragma unroll
                    for (int i = 0; i < kSide; ++i) acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v[i], ph[u], acc[i], 0, 0, 0);
                }
#pragma unroll
                for (int i = 0; i < kSide; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[o0 + i][e] = fmaf(acc[i][e], vs, o[o0 + i][e]);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        request_v(next, mask);
        __builtin_amdgcn_sched_barrier(0);
    };

    for (int i0 = 0;;) {
        for (; left > 0; --left) {
            const int i = at;
            const uint32_t mask = there != 0 ? ~0u : 0u;
            if (there != 0) at = __builtin_ctzll(there);
            there &= there - 1;                                        // (0 stays 0)
            block(b_begin + wave + NW * (i0 + i), lane_f32(ks_l, i), lane_f32(vs_l, i), __builtin_amdgcn_readlane(page_l, at), mask);
        }
        i0 += 64;
        if (b_begin + wave + NW * i0 >= b_end) break;
        open(i0);
    }

    // ---- waves meet
    constexpr float kOne = WIDE ? 0x1p-14f : 0x1p-30f;                 // of the outputs; the sums of p are 2^14 times too large, or right
    const float l_all = sum_groups(l_run) * (WIDE ? kOne : 1.f);
    if (g == 0 && (WIDE || dig == 0)) {
        s_m[wave][my_q] = m_run;
        s_l[wave][my_q] = l_all;
    }
    lds_barrier();
    auto share_of = [](float l) { return (l > 0.f || l != l) ? 1.f / l : 0.f; };      // (nothing seen: zeros)
    auto store_lse = [&](int q, float m, float l) {
        if (a.lse != nullptr && q < queries)
            a.lse[((int64_t)row * a.T + q / a.group) * (a.c.kv_heads * a.group) + h * a.group + q % a.group] =
                (l > 0.f || l != l) ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
    };
    if (tid < NQ) {
        float m = s_m[0][tid], l = 0.f;
#pragma unroll
        for (int u = 1; u < NW; ++u) m = fmaxf(m, s_m[u][tid]);
        const float base = (m > -INFINITY) ? m : 0.f;
#pragma unroll
        for (int u = 0; u < NW; ++u) {
            const float f = __builtin_amdgcn_exp2f(s_m[u][tid] - base);
            s_f[u][tid] = f;
            l += s_l[u][tid] * f;
        }
        s_M[tid] = m;
        s_L[tid] = ranges == 1 ? share_of(l) : l;
        const int q = q0 + tid, t = q / a.group, head = h * a.group + q % a.group;
        s_out[tid] = q < queries ? row * a.out_row + t * a.out_tok + (int64_t)head * HD : -1;
        if (ranges == 1) store_lse(q, m, l);
    }
    const int64_t unit = ((int64_t)row * a.c.kv_heads + h) * a.tiles + tile;
    float* const my_po = a.po + (unit * a.S + sp) * (NQ * HD);
    // Two dims of query q0 + q from their sums.
    auto finish = [&](int q, int dim, float v0, float v1) {
        const int64_t at = s_out[q];
        if (at < 0) return;
        const float f = s_L[q], r0 = f != 0.f ? v0 * f : 0.f, r1 = f != 0.f ? v1 * f : 0.f;
        if (a.out_bf16) *reinterpret_cast<u32_e2*>(static_cast<uint16_t*>(a.out) + at + dim) = pack_bf16x4(r0, r1, 0.f, 0.f).x;
        else *reinterpret_cast<f32x2_any*>(static_cast<float*>(a.out) + at + dim) = f32x2_any{r0, r1};
    };
#pragma unroll
    for (int d0 = 0; d0 < HD; d0 += RD) {
        if (d0 > 0) lds_barrier();                                   // the last ones have been read
#pragma unroll
        for (int ot = 0; ot < RD / 16; ++ot) {
            f32x4v v = o[d0 / 16 + ot];
            if constexpr (!WIDE) {
                const float place = (float)(1 << (8 * dig)) * kOne;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v[i] *= place;
                    v[i] += dpp_f32<kDppXor1>(v[i]);
                    v[i] += dpp_f32<kDppXor2>(v[i]);
                }
                if (dig == 0) *reinterpret_cast<f32x4v*>(&s_o[wave][my_q][ot * 16 + g * 4]) = v;
            } else {
                *reinterpret_cast<f32x4v*>(&s_o[wave][my_q][ot * 16 + g * 4]) = v * kOne;
            }
        }
        lds_barrier();
        for (int e = tid; e < NQ * RD / 2; e += NW * 64) {
            const int q = e / (RD / 2), dim = e % (RD / 2) * 2;
            float v0 = 0.f, v1 = 0.f;
#pragma unroll
            for (int u = 0; u < NW; ++u) {
                const float2 x = *reinterpret_cast<const float2*>(&s_o[u][q][dim]);
                v0 += x.x * s_f[u][q];
                v1 += x.y * s_f[u][q];
            }
            if (ranges == 1) finish(q, d0 + dim, v0, v1);
            else publish_pair(my_po + q * HD + d0 + dim, v0, v1);
        }
    }
    if (ranges == 1) return;

    // ---- ranges meet
    float* const unit_ml = a.pml + unit * a.S * (2 * NQ);
    if (tid < NQ) {
        publish_store(unit_ml + sp * (2 * NQ) + tid, s_M[tid]);
        publish_store(unit_ml + sp * (2 * NQ) + NQ + tid, s_L[tid]);
    }
    publish_barrier();
    if (tid == 0) s_last = arrive(a.arrivals + unit, (uint32_t)ranges);
    __syncthreads();
    if (!s_last) return;
    // Everything that is read is requested at once: a wave has the maxima and sums of its queries, a lane for every range, a thread kE
    // pairs of dims, kFly ranges at a time.
    constexpr int kPairs = NQ * HD / 2, kE = (kPairs + NW * 64 - 1) / (NW * 64), kFly = 16 / kE;
    const float* const unit_po = a.po + unit * a.S * (NQ * HD);
    float2 x[kFly][kE];
    auto fetch = [&](int u0) {
#pragma unroll
        for (int u = 0; u < kFly; ++u)
#pragma unroll
            for (int i = 0; i < kE; ++i) x[u][i] = published_pair(unit_po + min(u0 + u, ranges - 1) * (NQ * HD) + 2 * min(i * NW * 64 + tid, kPairs - 1));
    };
    fetch(0);
    static_assert(kMaxRanges == 64, "a lane each");
    for (int q = wave; q < NQ; q += NW) {
        const float* const ml = unit_ml + min(lane, ranges - 1) * (2 * NQ) + q;
        const float mu = published_load(ml), lu = published_load(ml + NQ), m = wave_max(mu), base = (m > -INFINITY) ? m : 0.f;
        const float f = lane < ranges ? __builtin_amdgcn_exp2f(mu - base) : 0.f, l = wave_sum(lane < ranges ? lu * f : 0.f);
        s_f[lane][q] = f;
        if (lane == 0) {
            s_L[q] = share_of(l);
            store_lse(q0 + q, m, l);
        }
    }
    __syncthreads();
    float2 v[kE];
#pragma unroll
    for (int i = 0; i < kE; ++i) v[i] = make_float2(0.f, 0.f);
    for (int u0 = 0; u0 < ranges; u0 += kFly) {
        if (u0 > 0) fetch(u0);
#pragma unroll
        for (int u = 0; u < kFly; ++u) {
            if (u0 + u >= ranges) break;
#pragma unroll
            for (int i = 0; i < kE; ++i) {
                const float f = s_f[u0 + u][min(i * NW * 64 + tid, kPairs - 1) / (HD / 2)];
                v[i].x += x[u][i].x * f;
                v[i].y += x[u][i].y * f;
            }
        }
    }
#pragma unroll
    for (int i = 0; i < kE; ++i) {
        const int e = i * NW * 64 + tid;
        if (e < kPairs) finish(e / (HD / 2), e % (HD / 2) * 2, v[i].x, v[i].y);
    }
}

// How a call is cut up.  Units are rows x heads x tiles of queries.  Up to 256 of them have eight waves, whose shares meet in LDS (16 rows x 8 heads of
// 128 dims, 24 queries, 2600 tokens: 21 us, with four waves 24.4); more, or heads too large for two such waves a SIMD, have four (64 rows x 12 heads of
// 64, 500 tokens: 13.6 us, with eight 16.0).  Rows are cut into ranges until every compute unit has a workgroup and no further: a second round
// of workgroups and the joins cost more than evener shares give (512 instead of 256: 16 rows of 2600 tokens 29.6 us instead of 21, of 300 to 5000 tokens
// 37 instead of 30, one row of 120000 56 instead of 50).
struct AttnPlan {
    bool wide;
    int nw, tiles, S;
};
static AttnPlan attn_plan(const tabed_cache_q8& c, int rows, int T, int q_heads) {
    AttnPlan p;
    const int queries = T * (q_heads / c.kv_heads);
    p.wide = queries > 4;
    p.tiles = (queries + attn_queries(p.wide) - 1) / attn_queries(p.wide);
    const long units = (long)rows * c.kv_heads * p.tiles;
    p.nw = units <= 256 && c.head_dim <= 128 ? 8 : 4;
    const long want = (kCutUnits + units - 1) / units, most = std::max(1, c.max_blocks / p.nw);
    p.S = (int)std::min<long>({want, most, kMaxRanges});
    return p;
}

// All that a call expects to find is the arrival counters at 0, as the call before left them, and these are at the same place for all sizes: one
// workspace serves calls of different sizes one after the other.
AttnLayout attn_layout(const tabed_cache_q8& c, int rows, int T, int q_heads) {
    AttnLayout L;
    const AttnPlan p = attn_plan(c, rows, T, q_heads);
    const size_t nq = attn_queries(p.wide), units = (size_t)rows * c.kv_heads * p.tiles;
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    size_t off = sizeof(uint32_t) * kCutUnits;
    L.off_po = off;  off = up(off + (p.S > 1 ? sizeof(float) * units * p.S * nq * c.head_dim : 0));
    L.off_pml = off; off = up(off + (p.S > 1 ? sizeof(float) * units * p.S * nq * 2 : 0));
    L.total = off;
    return L;
}

int64_t attn_workgroups(const tabed_cache_q8& c, int rows, int T, int q_heads) {
    const AttnPlan p = attn_plan(c, rows, T, q_heads);
    return ((int64_t)rows * c.kv_heads * p.S + 7) / 8 * 8 * p.tiles;
}

__global__ void k_attn_init(uint32_t* arrivals) { arrivals[threadIdx.x] = 0u; }

hipError_t launch_attn_init(char* ws, hipStream_t s) {
    launch(nullptr, k_attn_init, dim3(1), dim3(kCutUnits), 0, s, reinterpret_cast<uint32_t*>(ws));
    return hipGetLastError();
}

template <int HD>
static void launch_attn(const ProfScope* prof, const AttnPlan& p, unsigned grid, const AttnArgs& a, hipStream_t s) {
    if constexpr (HD <= 128) {
        if (p.nw == 8) {
            if (p.wide) launch(prof, k_attn_q8<HD, true, 8>, dim3(grid), dim3(512), 0, s, a);
            else launch(prof, k_attn_q8<HD, false, 8>, dim3(grid), dim3(512), 0, s, a);
            return;
        }
    }
    if (p.wide) launch(prof, k_attn_q8<HD, true, 4>, dim3(grid), dim3(256), 0, s, a);
    else launch(prof, k_attn_q8<HD, false, 4>, dim3(grid), dim3(256), 0, s, a);
}

hipError_t launch_attention_q8(const tabed_cache_q8& c, char* ws, int rows, int T, int q_heads, int q_dtype, const void* q, int64_t q_row,
                               int64_t q_tok, const int32_t* ctx_len, const int32_t* n_new, float scale, int out_dtype, void* out,
                               int64_t out_row, int64_t out_tok, float* lse, hipStream_t s) {
    const AttnPlan p = attn_plan(c, rows, T, q_heads);
    const AttnLayout L = attn_layout(c, rows, T, q_heads);
    const AttnArgs a{view_of(c), rows, T, q_heads / c.kv_heads, p.tiles, p.S, q_dtype == 1, out_dtype == 1, q, q_row, q_tok, out, out_row, out_tok,
                     lse, ctx_len, n_new, scale * 1.4426950408889634f, reinterpret_cast<uint32_t*>(ws), reinterpret_cast<float*>(ws + L.off_po),
                     reinterpret_cast<float*>(ws + L.off_pml)};
    const unsigned grid = (unsigned)attn_workgroups(c, rows, T, q_heads);
    ProfScope prof(TABED_K_BODY, s);
    switch (c.head_dim) {
        case 32: launch_attn<32>(&prof, p, grid, a, s); break;
        case 64: launch_attn<64>(&prof, p, grid, a, s); break;
        case 96: launch_attn<96>(&prof, p, grid, a, s); break;
        case 128: launch_attn<128>(&prof, p, grid, a, s); break;
        case 256: launch_attn<256>(&prof, p, grid, a, s); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

}  // namespace tabed
