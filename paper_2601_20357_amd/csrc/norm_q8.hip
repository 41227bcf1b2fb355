// Residual addition, RMSNorm and int8 rows with one scale each (tabed_norm_q8):
//   r = x + delta,  y = r / sqrt(mean r^2 + eps) * g,  scale = max |y| / 127,  q = round(y / scale).
// Without a gain the rows are quantised as they are (y = r): weights, or activations that another kernel left.
// One pass over memory: a row's threads keep its values in registers between the two reductions (sum of squares, largest
// magnitude), which are in fp32.  The norm is taken of the sum before it is rounded for storage.
#include "body_utils.h"
#include "q8_utils.h"

namespace tabed {

struct NormArgs {
    int rows, d;
    const void* x;
    int64_t ldx;
    const void* delta;
    int64_t ldd;
    void* sum;
    int64_t lds;
    const float* g;
    float eps;
    int8_t* q;
    int64_t ldq;
    float* scale;
    int32_t* advance;      // one entry a row that is counted up (the draft body's positions), or null
};

typedef uint32_t u32x2_e1 __attribute__((ext_vector_type(2), aligned(1)));

enum { kF32 = 0, kB16 = 1, kNone = 2 };

// TPR threads of a row, P pieces of 8 values each, as few as hold the row: 8192 rows of 4096 in bf16 with their deltas, 235 MB, took 58 us
// with room for four pieces, 46 with the two that there are, which is what a copy of as many bytes takes.  Few rows are bound by latency: x, two
// reductions, stores (4 rows of 768: 3.2 us, 1.5 of them between any two kernels; 333 rows of 2051: 4.8).  A wave a row needs no barrier, up to 2048
// values; longer rows have more threads so that a row's registers stay few.
template <int TPR, int P, int X, int D>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void k_norm_q8(NormArgs a) {
    constexpr int kWaves = TPR / 64;
    __shared__ float s_sum[kWaves];
    __shared__ uint32_t s_most[kWaves];
    const int t = threadIdx.x % TPR, d = a.d;
    const int64_t row = (TPR == 64) ? (int64_t)blockIdx.x * (blockDim.x / 64) + threadIdx.x / 64 : (int64_t)blockIdx.x;
    if (row >= a.rows) return;                                        // uniform for a wave, and for a workgroup that meets at a barrier
    float g[P][8];
    if (a.g != nullptr) {
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int at = (p * TPR + t) * 8;
            if (at + 8 <= d) {
                load_values<8, false>(a.g, at, g[p]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) g[p][e] = (at + e < d) ? a.g[at + e] : 0.f;
            }
        }
    }
    float v[P][8], ss = 0.f;
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const int at = (p * TPR + t) * 8;
        if (at + 8 <= d) {
            load_values<8, X == kB16>(a.x, row * a.ldx + at, v[p]);
            if constexpr (D != kNone) {
                float w[8];
                load_values<8, D == kB16>(a.delta, row * a.ldd + at, w);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[p][e] += w[e];
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[p][e] = 0.f;
                if (at + e < d) {
                    v[p][e] = load_value<X == kB16>(a.x, row * a.ldx + at + e);
                    if constexpr (D != kNone) v[p][e] += load_value<D == kB16>(a.delta, row * a.ldd + at + e);
                }
            }
        }
    }
    if constexpr (D != kNone) {
        if (a.sum != nullptr) {
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const int at = (p * TPR + t) * 8;
                if (at + 8 <= d) {
                    if constexpr (X == kB16) {
                        const uint2 lo = pack_bf16x4(v[p][0], v[p][1], v[p][2], v[p][3]), hi = pack_bf16x4(v[p][4], v[p][5], v[p][6], v[p][7]);
                        *reinterpret_cast<u32x4_e2*>(static_cast<uint16_t*>(a.sum) + row * a.lds + at) = u32x4_e2{lo.x, lo.y, hi.x, hi.y};
                    } else {
                        float* out = static_cast<float*>(a.sum) + row * a.lds + at;
                        *reinterpret_cast<f32x4_any*>(out) = f32x4_any{v[p][0], v[p][1], v[p][2], v[p][3]};
                        *reinterpret_cast<f32x4_any*>(out + 4) = f32x4_any{v[p][4], v[p][5], v[p][6], v[p][7]};
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (at + e < d) {
                            if constexpr (X == kB16) static_cast<uint16_t*>(a.sum)[row * a.lds + at + e] = f32_to_bf16_bits(v[p][e]);
                            else static_cast<float*>(a.sum)[row * a.lds + at + e] = v[p][e];
                        }
                }
            }
        }
    }
    if (a.g != nullptr) {
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int e = 0; e < 8; ++e) ss = fmaf(v[p][e], v[p][e], ss);
        ss = wave_sum(ss);
        if constexpr (kWaves > 1) {
            if ((t & 63) == 0) s_sum[t >> 6] = ss;
            __syncthreads();
            ss = 0.f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) ss += s_sum[w];
        }
        const float rms = 1.f / sqrtf(ss / (float)d + a.eps);
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[p][e] = v[p][e] * rms * g[p][e];
    }
    uint32_t most = (ss < INFINITY) ? 0u : kInfBits;               // (squares past fp32: the row is not finite either)
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
        for (int e = 0; e < 8; ++e) most = max(most, magnitude(v[p][e]));
    most = wave_max_u32(most);
    if constexpr (kWaves > 1) {
        if ((t & 63) == 0) s_most[t >> 6] = most;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) most = max(most, s_most[w]);
    }
    const float scale = scale_of(most);
    const float inv = (scale > 0.f) ? 1.f / scale : 0.f;
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const int at = (p * TPR + t) * 8;
        int s[8];
        if (scale > 0.f) {                                             // (uniform for a wave)
            steps_of(v[p], scale, inv, s);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) s[e] = 0;
        }
        int8_t* out = a.q + row * a.ldq + at;
        if (at + 8 <= d) {
            *reinterpret_cast<u32x2_e1*>(out) = u32x2_e1{pack_i8(s[0], s[1], s[2], s[3]), pack_i8(s[4], s[5], s[6], s[7])};
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (at + e < d) out[e] = (int8_t)s[e];
        }
    }
    if (t == 0) {
        a.scale[row] = scale;
        if (a.advance != nullptr) a.advance[row] += 1;
    }
}

template <int TPR, int P>
static void launch_norm_t(const ProfScope* prof, int xt, int dt, const NormArgs& a, hipStream_t s) {
    constexpr int per = (TPR == 64) ? 4 : 1;                           // rows of a workgroup, a wave each
    const dim3 grid((a.rows + per - 1) / per), block(TPR * per);
    auto go = [&](auto kernel) { launch(prof, kernel, grid, block, 0, s, a); };
    if (xt == kF32) {
        if (dt == kF32) go(k_norm_q8<TPR, P, kF32, kF32>);
        else if (dt == kB16) go(k_norm_q8<TPR, P, kF32, kB16>);
        else go(k_norm_q8<TPR, P, kF32, kNone>);
    } else {
        if (dt == kF32) go(k_norm_q8<TPR, P, kB16, kF32>);
        else if (dt == kB16) go(k_norm_q8<TPR, P, kB16, kB16>);
        else go(k_norm_q8<TPR, P, kB16, kNone>);
    }
}

hipError_t launch_norm_q8(int rows, int d, int x_dtype, const void* x, int64_t ldx, int delta_dtype, const void* delta, int64_t ldd, void* sum,
                          int64_t lds, const float* g, float eps, int8_t* q, int64_t ldq, float* scale, int32_t* advance, hipStream_t s) {
    const NormArgs a{rows, d, x, ldx, delta, ldd, sum, lds, g, eps, q, ldq, scale, advance};
    const int dt = delta == nullptr ? kNone : delta_dtype;
    ProfScope prof(TABED_K_BODY, s);
    if (d <= 64 * 8) launch_norm_t<64, 1>(&prof, x_dtype, dt, a, s);
    else if (d <= 64 * 16) launch_norm_t<64, 2>(&prof, x_dtype, dt, a, s);
    else if (d <= 64 * 32) launch_norm_t<64, 4>(&prof, x_dtype, dt, a, s);
    else if (d <= 256 * 16) launch_norm_t<256, 2>(&prof, x_dtype, dt, a, s);
    else if (d <= 256 * 32) launch_norm_t<256, 4>(&prof, x_dtype, dt, a, s);
    else if (d <= 1024 * 16) launch_norm_t<1024, 2>(&prof, x_dtype, dt, a, s);
    else launch_norm_t<1024, 4>(&prof, x_dtype, dt, a, s);
    return hipGetLastError();
}

}  // namespace tabed
