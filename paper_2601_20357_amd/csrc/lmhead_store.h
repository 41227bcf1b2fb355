// What the LM head kernels of all operand types share: storing logits with their softmax partials, and loads straight to LDS.
#pragma once
#include <hip/hip_bf16.h>

#include "device_utils.h"
#include "internal.h"

namespace tabed {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));   // four floats that are only 4-byte aligned

__device__ __forceinline__ float inv_temperature(float T) { return (T > 0.f) ? 1.f / T : 1.f; }
__device__ __forceinline__ float row_inv_temperature(const float* temperature, int row, int n) { return inv_temperature(temperature[row / n]); }
// row / n for row < 65536 without an integer division: (row + 1/2) / n is at least 1 / 32 away from an integer (n <= 16),
// far more than the error of the reciprocal.
__device__ __forceinline__ int sequence_of(int row, int n) { return (int)(((float)row + 0.5f) * __builtin_amdgcn_rcpf((float)n)); }

// Four logits of a row, past L2 or, of more than 64 rows, through it.  Rows whose 64-byte sectors are shared by neighbouring tiles go through L2, which puts
// the sectors together, where there are so many logits that storing parts of sectors is what takes the time.  Draft steps in us,
// through / past L2: V = 100003, 255 rows, d = 1024 133 / 155, 128 rows, d = 640 68.8 / 78.4, V = 50004, 96 rows, d = 768 35.4 / 36.2,
// V = 32001, 480 rows, d = 72 49.3 / 59.9; but below 16 MB of logits, most of which would be left to the write-back at the end, V = 20001,
// 80 rows, d = 2048 36.1 / 31.3, V = 30001, 120 rows, d = 1160 36.8 / 35.9; up to 64 rows, whose stores go out beside the stream of W,
// V = 100003 60.3 / 57.8 at 64 rows, 52.4 / 50.6 at 32; and with whole sectors, V = 100000, 128 rows 61.9 / 54.9.
// The exception: W of about the last-level cache's size (256 MB) stays there from one draft step to the next, unless logits stored
// through L2 take its place, which costs more than the sectors where the logits are few beside W (the ratio of their bytes is 2 M / d).
// Steps back to back on the same buffers, through / past L2, us.  128 rows, d = 3000, W of 240 MB, V = 40001 98.6 / 75.2, 40008 96.8 / 74.3; of 205 MB,
// 34168 73.6 / 73.1, of 320 MB, 53329 104.7 / 107.5.  d = 1328, 225 MB, V = 84708 85.8 / 80.6, with 256 rows 130.6 / 135.8, V = 84705 86.5 / 83.9,
// 132.2 / 142.2; 205 MB 67.8 / 76.9.  66 rows, d = 520, 255 MB, V = 245192 112.8 / 100.5, 128 rows 142.5 / 138.9.  Whole lines lose less, later:
// 128 rows, d = 2048, 240 MB 54.5 / 56.8, 270 MB, V = 65908 98.8 / 91.7, 320 MB 119.4 / 126.7; 96 rows, d = 896, 255 MB 82.7 / 83.9.
[[maybe_unused]] static bool past_l2(int V, int d, int M) {
    if ((V & 15) == 0 || (long)M * V < (4l << 20)) return true;
    const bool lines = d % 64 == 0;
    const long w = 2l * V * d;
    return w > (lines ? 250000000l : 222000000l) && w < (lines ? 300000000l : 278000000l) && 2l * d >= (lines ? 28l : (V & 3) ? 22l : 15l) * M;
}
// (An instance each: a choice at run time between the two stores becomes one that goes through L2.)
template <bool PAST>
__device__ __forceinline__ void store_logits(float* p, f32x4u x) {
    if constexpr (PAST) __builtin_nontemporal_store(x, reinterpret_cast<f32x4u*>(p));
    else *reinterpret_cast<f32x4u*>(p) = x;
}

constexpr int kPatchBytes = 32 * 144;                  // LDS in which a wave turns 32 rows of 32 floats

// Epilogue of one 32x32 accumulator tile held TRANSPOSED: lane holds result row m_base + lane % 32 and the 16
// vocabulary entries v_base + 8*(r/4) + 4*(lane/32) + r%4.  The softmax partials of a row are then a
// 16-value in-register reduction plus one exchange between the two half-waves, and every lane stores four
// runs of four consecutive logits.  inv_t[m] = 1/T of row m (LDS table).  With `pstage` the partials go to an
// LDS table instead, from which the caller writes a workgroup's four tiles of a row as one 16-byte store.
template <bool PAST = true>
__device__ __forceinline__ void store_tile_32x32_t(const f32x16& acc, int m_base, int v_base, int M, int V, int NT,
                                                   const float* inv_t, float* __restrict__ L,
                                                   float* __restrict__ pm, float* __restrict__ ps,
                                                   unsigned char* tpatch, float* pstage = nullptr, int pslot = 0) {
    if (v_base >= V) return;
    const int lane = threadIdx.x & 63;
    const int col = lane & 31, half = lane >> 5;
    const int m = m_base + col;
    const bool live = (m < M);
    const float it = live ? inv_t[m] : 1.f;
    const bool full = v_base + 32 <= V;            // uniform: only the last tile of a row is ragged
    float x[16];
    float mx = -INFINITY;
#pragma unroll
    for (int r = 0; r < 16; ++r) x[r] = acc[r];            // (rows past the end: computed, not stored)
    if (!full) {
#pragma unroll
        for (int r = 0; r < 16; ++r)
            if (v_base + 8 * (r / 4) + 4 * half + (r % 4) >= V) x[r] = -INFINITY;
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) mx = fmaxf(mx, x[r]);
    mx = fmaxf(mx, __shfl_xor(mx, 32));
    mx = (mx > -INFINITY) ? mx * it : mx;                  // (the largest product: 1 / T is positive and rounding keeps the order)
    const float base = (mx > -INFINITY) ? mx : 0.f;        // a tile of -inf sums to 0
    float sum = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) sum += __expf(fmaf(x[r], it, -base));
    if (__any(sum != sum)) {                               // a NaN logit has no mass and does not take the tile's with it
        sum = 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) sum += (x[r] * it > -INFINITY) ? __expf(fmaf(x[r], it, -mx)) : 0.f;
    }
    sum += __shfl_xor(sum, 32);
    if (live && half == 0) {
        if (pstage != nullptr) {                    // collected per workgroup: [array][row][tile of the group]
            pstage[(0 * 64 + m) * 4 + pslot] = mx;
            pstage[(1 * 64 + m) * 4 + pslot] = sum;
        } else {
            pm[(size_t)m * NT + v_base / kTileV] = mx;
            ps[(size_t)m * NT + v_base / kTileV] = sum;
        }
    }
    if (full) {
        // Full tile: turn the block through the wave's LDS patch ([32 rows][32 v] floats, 144-byte rows) so
        // that 8 lanes store one whole 128-byte line of a row, and stream it past L2: the logits are next
        // read tens of megabytes later, and full-line streaming stores measured 1.9 us faster per launch
        // than leaving 8 MB of dirty partial lines to the end-of-kernel write-back.
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *reinterpret_cast<float4*>(tpatch + col * 144 + (8 * g + 4 * half) * 4) =
                make_float4(acc[4 * g], acc[4 * g + 1], acc[4 * g + 2], acc[4 * g + 3]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int mr = 8 * i + (lane >> 3), q = lane & 7;
            const float4 val = *reinterpret_cast<const float4*>(tpatch + mr * 144 + q * 16);
            if (m_base + mr < M)                   // (rows of an odd vocabulary are only 4-byte aligned)
                store_logits<PAST>(L + (size_t)(m_base + mr) * V + v_base + 4 * q, f32x4u{val.x, val.y, val.z, val.w});
        }
        return;
    }
    if (!live) return;
    float* row = L + (size_t)m * V;                // ragged last tile: element-wise
#pragma unroll
    for (int g = 0; g < 4; ++g)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int v = v_base + 8 * g + 4 * half + e;
            if (v < V) row[v] = acc[4 * g + e];
        }
}

// The other half-wave's value beside this one's: {lanes 0-31, lanes 0-31} and {lanes 32-63, lanes 32-63}.
__device__ __forceinline__ float2 both_halves(float v) {
    const auto p = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
    return make_float2(__builtin_bit_cast(float, (unsigned)p[0]), __builtin_bit_cast(float, (unsigned)p[1]));
}

// Epilogue of a wave's TV x TM accumulator tiles, none of which reaches past the vocabulary: the values, the operations and their
// order are those of store_tile_32x32_t.  The row tiles of a vocabulary tile go through each phase side by side, so that none waits for
// its own chain (maximum, exchange, exponentials, exchange), and the partials of the workgroup's rows are collected in LDS
// (part: [row][kPT tiles] maxima, kPS floats on the sums), from where a row's are stored 16 bytes at a time: a store of their own for
// every tile and row was two of three memory requests of the epilogue.
// rows: how many rows of the wave's block exist; patch: two of kPatchBytes.
template <bool PAST, int TV, int TM, int kPT, int kPS>
__device__ __forceinline__ void store_full_tiles(const f32x16 (&acc)[TV][TM], int rows, const float* s_it, float* part, float* L /* row, entry 0 of the block */,
                                                 int V, unsigned char* patch) {
    const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
    float it[TM];
#pragma unroll
    for (int b = 0; b < TM; ++b) it[b] = s_it[b * 32 + col];
#pragma unroll
    for (int a = 0; a < TV; ++a) {
        float mx[TM], base[TM], sum[TM];
#pragma unroll
        for (int b = 0; b < TM; ++b) {
            mx[b] = -INFINITY;
#pragma unroll
            for (int r = 0; r < 16; ++r) mx[b] = fmaxf(mx[b], acc[a][b][r]);
        }
#pragma unroll
        for (int b = 0; b < TM; ++b) {
            const float2 h = both_halves(mx[b]);
            mx[b] = fmaxf(h.x, h.y);
            mx[b] = (mx[b] > -INFINITY) ? mx[b] * it[b] : mx[b];
            base[b] = (mx[b] > -INFINITY) ? mx[b] : 0.f;
            sum[b] = 0.f;
        }
#pragma unroll
        for (int b = 0; b < TM; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) sum[b] += __expf(fmaf(acc[a][b][r], it[b], -base[b]));
        bool nan = false;
#pragma unroll
        for (int b = 0; b < TM; ++b) nan = nan || sum[b] != sum[b];
        if (__any(nan)) {                                  // a NaN logit has no mass and does not take the tile's with it
#pragma unroll
            for (int b = 0; b < TM; ++b) {
                if (!__any(sum[b] != sum[b])) continue;    // (tile by tile, as store_tile_32x32_t decides)
                sum[b] = 0.f;
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    sum[b] += (acc[a][b][r] * it[b] > -INFINITY) ? __expf(fmaf(acc[a][b][r], it[b], -mx[b])) : 0.f;
                }
            }
        }
#pragma unroll
        for (int b = 0; b < TM; ++b) {
            const float2 h = both_halves(sum[b]);
            if (half == 0) {
                part[(b * 32 + col) * kPT + a] = mx[b];
                part[(b * 32 + col) * kPT + a + kPS] = h.x + h.y;
            }
        }
#pragma unroll
        for (int b = 0; b < TM; ++b) {
            if (b * 32 >= rows) continue;                  // uniform
            unsigned char* const tp = patch + (b & 1) * kPatchBytes;
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<float4*>(tp + col * 144 + (8 * g + 4 * half) * 4) =
                    make_float4(acc[a][b][4 * g], acc[a][b][4 * g + 1], acc[a][b][4 * g + 2], acc[a][b][4 * g + 3]);
            const int q = lane & 7;
            float* const out = L + (size_t)(b * 32 + (lane >> 3)) * V + a * 32 + 4 * q;
            float4 val[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) val[i] = *reinterpret_cast<const float4*>(tp + (8 * i + (lane >> 3)) * 144 + q * 16);
            auto store = [&](int i) {
                store_logits<PAST>(out + (size_t)(8 * i) * V, f32x4u{val[i].x, val[i].y, val[i].z, val[i].w});
            };
            if ((b + 1) * 32 <= rows) {                    // uniform
#pragma unroll
                for (int i = 0; i < 4; ++i) store(i);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (b * 32 + 8 * i + (lane >> 3) < rows) store(i);
            }
        }
    }
}

// ---------------------------------------------------------------- loads straight to LDS
// Four (two, one) loads of 64 lanes x 16 bytes, from base + the lane's offset to LDS at `lds`, `step` further for each: lane l's bytes land at
// l * 16.  In assembly, since they have no destination register: with the builtin the compiler waits for LDS reads in flight.
// (M0 is put back: the compiler does not let it be named as clobbered, and keeps what it has in it.)
__device__ __forceinline__ void dma_lines(const char* base, const uint32_t (&off)[4], uint32_t lds, uint32_t step) {
    uint32_t m0;
    // (the waits: M0 written before an LDS load, and a scalar that may have come from a vector instruction)
    asm volatile("s_mov_b32 %0, m0\n\ts_nop 4\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %3, %7\n\ts_add_u32 m0, m0, %2\n\t"
                 "s_nop 0\n\tglobal_load_lds_dwordx4 %4, %7\n\ts_add_u32 m0, m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %5, %7\n\t"
                 "s_add_u32 m0, m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %6, %7\n\ts_mov_b32 m0, %0"
                 : "=&s"(m0) : "s"(lds), "s"(step), "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]), "s"(base) : "memory", "scc");
}
__device__ __forceinline__ void dma_lines(const char* base, const uint32_t (&off)[2], uint32_t lds, uint32_t step) {
    uint32_t m0;
    asm volatile("s_mov_b32 %0, m0\n\ts_nop 4\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %3, %5\n\ts_add_u32 m0, m0, %2\n\t"
                 "s_nop 0\n\tglobal_load_lds_dwordx4 %4, %5\n\ts_mov_b32 m0, %0"
                 : "=&s"(m0) : "s"(lds), "s"(step), "v"(off[0]), "v"(off[1]), "s"(base) : "memory", "scc");
}
__device__ __forceinline__ void dma_lines(const char* base, const uint32_t (&off)[1], uint32_t lds, uint32_t) {
    uint32_t m0;
    asm volatile("s_mov_b32 %0, m0\n\ts_nop 4\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3\n\ts_mov_b32 m0, %0"
                 : "=&s"(m0) : "s"(lds), "v"(off[0]), "s"(base) : "memory", "scc");
}

}  // namespace tabed
