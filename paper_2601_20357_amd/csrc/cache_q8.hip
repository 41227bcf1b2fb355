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
// One workgroup: the keys, or the values, of one head in one block of one row's new tokens.  Reads the new tokens once;
// tokens that a begun block keeps are read only where its scale grows (they are rounded again then), values also where a group
// of 16 tokens is stored whole.  Latency bounds a decode step (positions -> page -> scale), memory a prompt.
struct AppendArgs {
    CacheView c;
    int rows, T, nb;
    const void* k;
    const void* v;
    int64_t row_stride, tok_stride;
    const int32_t* ctx_len;
    const int32_t* n_new;
};

template <bool BF16>
__global__ __launch_bounds__(kBlock) void k_cache_append(AppendArgs a) {
    __shared__ uint32_t s_most[kWavesPerBlock];
    extern __shared__ __attribute__((aligned(16))) unsigned char s_t[];       // values: [hd][64 + 4] new tokens' steps
    constexpr int kRow = kCB + 4;
    int w = blockIdx.x;
    const bool values = w & 1;
    w >>= 1;
    const int h = w % a.c.kv_heads;
    w /= a.c.kv_heads;
    const int j = w % a.nb, row = w / a.nb;
    const int tid = threadIdx.x, hd = a.c.hd, chunks = hd / 16;
    const int n = row_tokens(a.n_new, row, a.T), ctx = max(a.ctx_len[row], 0);
    const int64_t slot = (int64_t)(ctx / kCB) + j;
    if (slot >= a.c.max_blocks) return;
    const int b0 = (int)slot * kCB, off = max(ctx - b0, 0);                  // the first `off` tokens are kept
    const int t0 = b0 + off - ctx, count = min(kCB - off, n - t0);            // new tokens t0 .. t0 + count - 1 go behind them
    if (count <= 0) return;
    const int page = a.c.table[(int64_t)row * a.c.max_blocks + slot];
    if (page < 0 || page >= a.c.blocks) return;
    const int64_t ph = (int64_t)page * a.c.kv_heads + h;
    int8_t* const block = (values ? a.c.v : a.c.k) + ph * kCB * hd;
    float* const scales = values ? a.c.vscale : a.c.kscale;
    const float before = off > 0 ? scales[ph] : 0.f;
    const void* const src = values ? a.v : a.k;
    const int64_t base = row * a.row_stride + (int64_t)t0 * a.tok_stride + (int64_t)h * hd;

    constexpr int kPer = 4;                                                   // pieces of 16 dims a thread holds: 4 * 256 >= 64 * 256 / 16
    float x[kPer][16];
    uint32_t most = 0;
#pragma unroll
    for (int p = 0; p < kPer; ++p) {
        const int idx = p * kBlock + tid, tok = idx / chunks, c = idx % chunks;
        if (tok < count) {
            load_values<16, BF16>(src, base + (int64_t)tok * a.tok_stride + c * 16, x[p]);
#pragma unroll
            for (int e = 0; e < 16; ++e) most = max(most, magnitude(x[p][e]));
        }
    }
    most = wave_max_u32(most);
    if ((tid & 63) == 0) s_most[tid >> 6] = most;
    __syncthreads();
    most = max(max(s_most[0], s_most[1]), max(s_most[2], s_most[3]));
    const float fresh = scale_of(most);
    const float scale = (before != before || fresh != fresh) ? __builtin_nanf("") : fmaxf(before, fresh);
    const bool live = scale > 0.f, grown = off > 0 && !(scale == before);      // uniform
    if (tid == 0) scales[ph] = scale;
    auto again = [&](int q) { return live ? to_step((float)q * before / scale) : 0; };       // a kept token's step, in steps of the new scale

#pragma unroll
    for (int p = 0; p < kPer; ++p) {
        const int idx = p * kBlock + tid, tok = idx / chunks, c = idx % chunks;
        if (tok < count) {
            int s[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) s[e] = live ? to_step(x[p][e] / scale) : 0;
            const int at = off + tok;
            if (!values) {
                const u32x4_e4 out = {pack_i8(s[0], s[1], s[2], s[3]), pack_i8(s[4], s[5], s[6], s[7]), pack_i8(s[8], s[9], s[10], s[11]),
                                      pack_i8(s[12], s[13], s[14], s[15])};
                *reinterpret_cast<u32x4_e4*>(block + (((at / 4 % 4) * chunks + c) * 16 + at / 16 * 4 + at % 4) * 16) = out;
            } else {
#pragma unroll
                for (int e = 0; e < 16; ++e) s_t[(c * 16 + e) * kRow + at] = (unsigned char)s[e];
            }
        }
    }
    if (!values) {
        if (grown)
            for (int idx = tid; idx < off * chunks; idx += kBlock) {
                const int at = idx / chunks, c = idx % chunks;
                u32x4_e4* const p = reinterpret_cast<u32x4_e4*>(block + (((at / 4 % 4) * chunks + c) * 16 + at / 16 * 4 + at % 4) * 16);
                u32x4_e4 old = *p;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    old[i] = pack_i8(again((int8_t)old[i]), again((int8_t)(old[i] >> 8)), again((int8_t)(old[i] >> 16)), again((int8_t)(old[i] >> 24)));
                *p = old;
            }
        return;
    }
    __syncthreads();
    const int g0 = grown ? 0 : off / 16, g1 = (off + count - 1) / 16;          // groups of 16 tokens that change
    for (int idx = tid; idx < (g1 - g0 + 1) * hd; idx += kBlock) {
        const int g = g0 + idx / hd, dim = idx % hd;
        u32x4_e4* const p = reinterpret_cast<u32x4_e4*>(block + ((dim / 16 * 4 + g) * 16 + dim % 16) * 16);
        u32x4_e4 old = {0u, 0u, 0u, 0u};
        if (g * 16 < off || (g + 1) * 16 > off + count) old = *p;               // some of its tokens stay
        const unsigned char* const now = s_t + dim * kRow;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            int s[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int at = g * 16 + 4 * i + e, q = (int8_t)(old[i] >> (8 * e));
                s[e] = at < off ? (grown ? again(q) : q) : at < off + count ? (int8_t)now[at] : q;
            }
            old[i] = pack_i8(s[0], s[1], s[2], s[3]);
        }
        *p = old;
    }
}

static int append_blocks(int T) { return (T + kCB - 2) / kCB + 1; }

int64_t append_workgroups(const tabed_cache_q8& c, int rows, int T) { return 2ll * c.kv_heads * rows * append_blocks(T); }

hipError_t launch_cache_append(const tabed_cache_q8& c, int rows, int T, int kv_dtype, const void* k, const void* v, int64_t row_stride,
                               int64_t tok_stride, const int32_t* ctx_len, const int32_t* n_new, hipStream_t s) {
    const AppendArgs a{view_of(c), rows, T, append_blocks(T), k, v, row_stride, tok_stride, ctx_len, n_new};
    const dim3 grid((unsigned)append_workgroups(c, rows, T));
    const size_t lds = (size_t)c.head_dim * (kCB + 4);
    ProfScope prof(TABED_K_BODY, s);
    if (kv_dtype == 1) launch(&prof, k_cache_append<true>, grid, dim3(kBlock), lds, s, a);
    else launch(&prof, k_cache_append<false>, grid, dim3(kBlock), lds, s, a);
    return hipGetLastError();
}

// ---------------------------------------------------------------- attention
// One wave walks over blocks of one row and key / value head for CT column tiles of four queries (a query: one new token and one of
// the heads that share the key / value head).  Scores are S^T = K Q^T and outputs O^T = V^T P^T with v_mfma_i32_16x16x64_i8: the cache's
// bytes are operands as they are, and a query's 32-bit values stand in four columns, one for each digit of base 256:
//   q = max|q| 2^-30 (d3 256^3 + d2 256^2 + d1 256 + d0),  p 2^30 = the same,  digits -128 .. 127.
// Products and their sums are exact integers, and what fixed point costs is below fp32's own rounding: 2^-31 of the row's largest |q|, and
// of the largest probability.  (Converting the cache to bf16 instead is one and a half vector instructions a byte, at which a
// compute unit takes in less than memory delivers, and rounds p to 8 bits.)
// Lane (g = lane / 16, c = lane % 16) has column c = 4 query + digit.  Its 16 scores of a block are those of tokens 16 g .. 16 g + 15, which
// are also the 16 bytes that it gives to the second product: probabilities never leave the lane.
// The four waves of a workgroup take blocks in turn and meet in LDS; a row's blocks are cut into S ranges where the rows and heads do
// not fill the chip, and the last of its workgroups to arrive joins them (in range order: results do not depend on who is last).
struct AttnArgs {
    CacheView c;
    int rows, T, group;          // group: query heads of a key / value head
    int tiles;                   // workgroups of one row and key / value head: queries / (4 CT), rounded up
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
    uint32_t* arrivals;          // [rows, kv_heads, tiles]
    float* po;                   // [rows, kv_heads, tiles, S][4 CT][hd]: sums of p v, at the range's own maximum
    float* pml;                  // the same [2][4 CT]: maxima (base 2), sums of p
};

constexpr int kMinRange = 4;     // blocks: one for each wave

// The four lanes of a query add the same four products, each in its own order, and have to come to the same sum: they give the digits of one
// probability.  A product that is fused into the addition in one lane, and rounded in the others, gave digits of different numbers.
__device__ __forceinline__ float rounded_product(float a, float b) {
#pragma clang fp contract(off)
    return a * b;
}

template <int HD, int CT>
__global__ __launch_bounds__(kBlock) void k_attn_q8(AttnArgs a) {
    constexpr int KS = (HD + 63) / 64, H16 = HD / 16, OT = HD / 16, NQ = 4 * CT;
    __shared__ float s_o[kWavesPerBlock][NQ][HD + 4];
    __shared__ float s_m[kWavesPerBlock][NQ], s_l[kWavesPerBlock][NQ];
    __shared__ int s_last;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = lane >> 4, c = lane & 15, dig = c & 3;
    int w = blockIdx.x;
    const int tile = w % a.tiles;
    w /= a.tiles;
    const int h = w % a.c.kv_heads;
    w /= a.c.kv_heads;
    const int sp = w % a.S, row = w / a.S;
    const int n = row_tokens(a.n_new, row, a.T);
    const int queries = n * a.group, q0 = tile * NQ;
    if (q0 >= queries) return;                                         // uniform
    const int64_t cap = (int64_t)a.c.max_blocks * kCB;
    const int ctx = (int)min((int64_t)max(a.ctx_len[row], 0), cap);
    const int t_first = q0 / a.group, t_last = min(n - 1, (q0 + NQ - 1) / a.group);
    const int NB = (int)((min((int64_t)ctx + t_last + 1, cap) + kCB - 1) / kCB);       // blocks that some query of the tile sees
    const int ranges = min(a.S, max(1, NB / kMinRange));
    if (sp >= ranges) return;
    const int per = (NB + ranges - 1) / ranges, b_begin = min(sp * per, NB), b_end = min(b_begin + per, NB);

    // ---- queries: digits of this lane's columns, and what a step of them is worth
    i32x4 qd[CT][KS];
    float worth[CT];
    int limit[CT];                                                     // last position that the column's query sees
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        const int qi = min(q0 + ct * 4 + (c >> 2), queries - 1), t = qi / a.group, head = h * a.group + qi % a.group;
        limit[ct] = ctx + t;
        const int64_t base = row * a.q_row + t * a.q_tok + (int64_t)head * HD;
        float x[KS][16];
        uint32_t most = 0;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const int dim = (ks * 4 + g) * 16;
            if (HD % 64 == 0 || dim < HD) {
                if (a.q_bf16) load_values<16, true>(a.q, base + dim, x[ks]);
                else load_values<16, false>(a.q, base + dim, x[ks]);
            } else {
#pragma unroll
                for (int e = 0; e < 16; ++e) x[ks][e] = 0.f;
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) most = max(most, magnitude(x[ks][e]));
        }
        most = max(most, (uint32_t)__shfl_xor((int)most, 16));
        most = max(most, (uint32_t)__shfl_xor((int)most, 32));
        const float m = __builtin_bit_cast(float, most);
        const bool finite = most < kInfBits, some = finite && m >= kTiny;
        const float inv = some ? 0x1p30f / m : 0.f;
        worth[ct] = finite ? (some ? m * 0x1p-30f : 0.f) * a.scale2 * (float)(1 << (8 * dig)) : __builtin_nanf("");
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                int digits = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int xi = some ? (int)rintf(x[ks][4 * i + e] * inv) : 0;
                    const uint32_t z = ((uint32_t)xi + 0x00808080u) ^ 0x00808080u;
                    digits |= (int)(((z >> (8 * dig)) & 255u) << (8 * e));
                }
                qd[ct][ks][i] = digits;
            }
        }
    }

    float m_run[CT], l_run[CT];
    float o[CT][OT][4];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        m_run[ct] = -INFINITY;
        l_run[ct] = 0.f;
#pragma unroll
        for (int ot = 0; ot < OT; ++ot)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[ct][ot][i] = 0.f;
    }
    const uint32_t sel = (uint32_t)dig | (uint32_t)(4 + dig) << 8 | 0x0c0c0000u;       // byte `dig` of two words side by side
    const uint32_t flip = dig == 3 ? 0u : 0x80808080u;
    const int32_t* const table = a.c.table + (int64_t)row * a.c.max_blocks;

    for (int b = b_begin + wave; b < b_end; b += kWavesPerBlock) {
        const int page = table[b];
        if (page < 0 || page >= a.c.blocks) continue;                  // uniform
        const int64_t ph = (int64_t)page * a.c.kv_heads + h;
        const float ksc = a.c.kscale[ph], vsc = a.c.vscale[ph];
        const int8_t* const kb = a.c.k + ph * kCB * HD;
        const int8_t* const vb = a.c.v + ph * kCB * HD;
        i32x4 kf[4][KS], vf[OT];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const int piece = (ks * 4 + g < H16) ? ks * 4 + g : 0;
                kf[t][ks] = *reinterpret_cast<const i32x4*>(kb + ((t * H16 + piece) * 16 + c) * 16);
            }
#pragma unroll
        for (int ot = 0; ot < OT; ++ot) vf[ot] = *reinterpret_cast<const i32x4*>(vb + ot * 1024 + lane * 16);
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            const float step = worth[ct] * ksc;
            float s[16];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                i32x4 acc = {0, 0, 0, 0};
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(kf[t][ks], qd[ct][ks], acc, 0, 0, 0);
#pragma unroll
                for (int i = 0; i < 4; ++i) s[4 * t + i] = rounded_product((float)acc[i], step);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] += dpp_f32<kDppXor1>(s[i]);
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] += dpp_f32<kDppXor2>(s[i]);
            if (b * kCB + kCB - 1 > ctx + t_first) {                   // uniform: some query does not see all of the block
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (b * kCB + g * 16 + i > limit[ct]) s[i] = -INFINITY;
            }
            float mx = s[0];
#pragma unroll
            for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[i]);
            mx = fmaxf(mx, __shfl_xor(mx, 16));
            mx = fmaxf(mx, __shfl_xor(mx, 32));
            const float m_new = fmaxf(m_run[ct], mx), base = (m_new > -INFINITY) ? m_new : 0.f;
            const float alpha = __builtin_amdgcn_exp2f(m_run[ct] - base);
            m_run[ct] = m_new;
            uint32_t pz[16];
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float p = __builtin_amdgcn_exp2f(s[i] - base);
                sum += p;
                pz[i] = (uint32_t)(int)fmaf(p, 0x1p30f, 0.5f) + 0x00808080u;
            }
            l_run[ct] = l_run[ct] * alpha + sum;
            i32x4 pd;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t lo = __builtin_amdgcn_perm(pz[4 * i + 1], pz[4 * i], sel), hi = __builtin_amdgcn_perm(pz[4 * i + 3], pz[4 * i + 2], sel);
                pd[i] = (int)((lo | hi << 16) ^ flip);
            }
#pragma unroll
            for (int ot = 0; ot < OT; ++ot) {
                const i32x4 acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(vf[ot], pd, i32x4{0, 0, 0, 0}, 0, 0, 0);
#pragma unroll
                for (int i = 0; i < 4; ++i) o[ct][ot][i] = fmaf((float)acc[i], vsc, o[ct][ot][i] * alpha);
            }
        }
    }

    // ---- digits, then waves, then ranges meet
    const float place = (float)(1 << (8 * dig)) * 0x1p-30f;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        float l = l_run[ct];
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        const int q = ct * 4 + (c >> 2);
        if (g == 0 && dig == 0) { s_m[wave][q] = m_run[ct]; s_l[wave][q] = l; }
#pragma unroll
        for (int ot = 0; ot < OT; ++ot)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float v = o[ct][ot][i] * place;
                v += dpp_f32<kDppXor1>(v);
                v += dpp_f32<kDppXor2>(v);
                if (dig == i) s_o[wave][q][ot * 16 + g * 4 + i] = v;
            }
    }
    __syncthreads();
    auto finish = [&](int q, int dim, float m, float l, float v) {      // of query q0 + q
        const int qi = q0 + q;
        if (qi >= queries) return;
        const int t = qi / a.group, head = h * a.group + qi % a.group;
        const float r = (l > 0.f || l != l) ? v / l : 0.f;             // (nothing seen: zeros)
        const int64_t at = row * a.out_row + t * a.out_tok + (int64_t)head * HD + dim;
        if (a.out_bf16) static_cast<uint16_t*>(a.out)[at] = f32_to_bf16_bits(r);
        else static_cast<float*>(a.out)[at] = r;
        if (dim == 0 && a.lse != nullptr)
            a.lse[((int64_t)row * a.T + t) * (a.c.kv_heads * a.group) + head] =
                (l > 0.f || l != l) ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
    };
    const int64_t unit = ((int64_t)row * a.c.kv_heads + h) * a.tiles + tile;
    for (int e = tid; e < NQ * HD; e += kBlock) {
        const int q = e / HD, dim = e % HD;
        float m = -INFINITY, l = 0.f, v = 0.f;
#pragma unroll
        for (int u = 0; u < kWavesPerBlock; ++u) m = fmaxf(m, s_m[u][q]);
        const float base = (m > -INFINITY) ? m : 0.f;
#pragma unroll
        for (int u = 0; u < kWavesPerBlock; ++u) {
            const float f = __builtin_amdgcn_exp2f(s_m[u][q] - base);
            l += s_l[u][q] * f;
            v += s_o[u][q][dim] * f;
        }
        if (ranges == 1) {
            finish(q, dim, m, l, v);
        } else {
            publish_store(a.po + ((unit * a.S + sp) * NQ + q) * HD + dim, v);
            if (dim == 0) {
                publish_store(a.pml + ((unit * a.S + sp) * 2 + 0) * NQ + q, m);
                publish_store(a.pml + ((unit * a.S + sp) * 2 + 1) * NQ + q, l);
            }
        }
    }
    if (ranges == 1) return;
    publish_barrier();
    if (tid == 0) s_last = arrive(a.arrivals + unit, (uint32_t)ranges);
    __syncthreads();
    if (!s_last) return;
    for (int e = tid; e < NQ * HD; e += kBlock) {
        const int q = e / HD, dim = e % HD;
        float m = -INFINITY, l = 0.f, v = 0.f;
        for (int u = 0; u < ranges; ++u) {
            const float mu = published_load(a.pml + ((unit * a.S + u) * 2 + 0) * NQ + q), lu = published_load(a.pml + ((unit * a.S + u) * 2 + 1) * NQ + q);
            const float vu = published_load(a.po + ((unit * a.S + u) * NQ + q) * HD + dim);
            const float mn = fmaxf(m, mu), base = (mn > -INFINITY) ? mn : 0.f;
            const float fo = __builtin_amdgcn_exp2f(m - base), fn = __builtin_amdgcn_exp2f(mu - base);
            l = l * fo + lu * fn;
            v = v * fo + vu * fn;
            m = mn;
        }
        finish(q, dim, m, l, v);
    }
}

// Column tiles of a workgroup: as many as the queries fill, at most four (two where a head's 256 dims leave no registers).
static int attn_ct(int hd, int queries) { return queries <= 4 ? 1 : (queries <= 8 || hd > 128) ? 2 : 4; }
static int attn_tiles(int hd, int queries) { return (queries + 4 * attn_ct(hd, queries) - 1) / (4 * attn_ct(hd, queries)); }

// Ranges: enough workgroups for four on every compute unit, none shorter than kMinRange blocks of a full table.
static int attn_ranges(const tabed_cache_q8& c, int rows, int T, int q_heads) {
    const long units = (long)rows * c.kv_heads * attn_tiles(c.head_dim, T * (q_heads / c.kv_heads));
    const long want = (1024 + units - 1) / units, most = std::max(1, c.max_blocks / kMinRange);
    return (int)std::min<long>({want, most, 128});
}

AttnLayout attn_layout(const tabed_cache_q8& c, int rows, int T, int q_heads) {
    AttnLayout L;
    const int queries = T * (q_heads / c.kv_heads), nq = 4 * attn_ct(c.head_dim, queries);
    L.tiles = attn_tiles(c.head_dim, queries);
    L.S = attn_ranges(c, rows, T, q_heads);
    const size_t units = (size_t)rows * c.kv_heads * L.tiles;
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    size_t off = 0;
    L.units = units;
    off = up(off + sizeof(uint32_t) * units);
    L.off_po = off;  off = up(off + (L.S > 1 ? sizeof(float) * units * L.S * nq * c.head_dim : 0));
    L.off_pml = off; off = up(off + (L.S > 1 ? sizeof(float) * units * L.S * nq * 2 : 0));
    L.total = off;
    return L;
}

int64_t attn_workgroups(const tabed_cache_q8& c, int rows, int T, int q_heads) {
    const int64_t tiles = attn_tiles(c.head_dim, T * (q_heads / c.kv_heads));
    return (int64_t)rows * c.kv_heads * tiles * attn_ranges(c, rows, T, q_heads);
}

__global__ void k_attn_init(uint32_t* arrivals, size_t n) {
    const size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (i < n) arrivals[i] = 0u;
}

hipError_t launch_attn_init(const tabed_cache_q8& c, int rows, int T, int q_heads, char* ws, hipStream_t s) {
    const AttnLayout L = attn_layout(c, rows, T, q_heads);
    launch(nullptr, k_attn_init, dim3((unsigned)((L.units + 255) / 256)), dim3(256), 0, s, reinterpret_cast<uint32_t*>(ws), L.units);
    return hipGetLastError();
}

hipError_t launch_attention_q8(const tabed_cache_q8& c, char* ws, int rows, int T, int q_heads, int q_dtype, const void* q, int64_t q_row,
                               int64_t q_tok, const int32_t* ctx_len, const int32_t* n_new, float scale, int out_dtype, void* out,
                               int64_t out_row, int64_t out_tok, float* lse, hipStream_t s) {
    const AttnLayout L = attn_layout(c, rows, T, q_heads);
    const int group = q_heads / c.kv_heads, ct = attn_ct(c.head_dim, T * group);
    const AttnArgs a{view_of(c), rows, T, group, L.tiles, L.S, q_dtype == 1, out_dtype == 1, q, q_row, q_tok, out, out_row, out_tok, lse, ctx_len,
                     n_new, scale * 1.4426950408889634f, reinterpret_cast<uint32_t*>(ws), reinterpret_cast<float*>(ws + L.off_po),
                     reinterpret_cast<float*>(ws + L.off_pml)};
    const dim3 grid((unsigned)(L.units * L.S)), block(kBlock);
    ProfScope prof(TABED_K_BODY, s);
#define TABED_ATTN(HD_)                                                              \
    case HD_:                                                                        \
        if (ct == 1) launch(&prof, k_attn_q8<HD_, 1>, grid, block, 0, s, a);         \
        else if (ct == 2) launch(&prof, k_attn_q8<HD_, 2>, grid, block, 0, s, a);    \
        else if constexpr (HD_ <= 128) launch(&prof, k_attn_q8<HD_, 4>, grid, block, 0, s, a); \
        break;
    switch (c.head_dim) {
        TABED_ATTN(32)
        TABED_ATTN(64)
        TABED_ATTN(96)
        TABED_ATTN(128)
        TABED_ATTN(256)
        default: return hipErrorInvalidValue;
    }
#undef TABED_ATTN
    return hipGetLastError();
}

}  // namespace tabed
