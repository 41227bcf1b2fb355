// Products of int8 rows with int8 weights (tabed_linear_q8): Y[m][n] = (sum_k X[m][k] W[n][k]) * sx[m] * sw[n], the sum in int32
// (exact for the K allowed), one rounding for each scale and one for storage.
#include "body_utils.h"
#include "q8_utils.h"

namespace tabed {

struct LinearArgs {
    int M, N, K;
    const int8_t* X;
    int64_t ldx;
    const float* sx;
    const int8_t* W;
    const float* sw;
    void* Y;
    int64_t ldy;
};

// One wave: 16 columns and 64 rows of the result.
template <bool BF16>
__global__ __launch_bounds__(kBlock) void k_linear_q8(LinearArgs a) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, c = lane & 15;
    const int n0 = (blockIdx.x * kWavesPerBlock + wave) * 16, m0 = blockIdx.y * 64;
    if (n0 >= a.N) return;
    const int8_t* const wrow = a.W + (int64_t)min(n0 + c, a.N - 1) * a.K;
    const int8_t* xrow[4];
    i32x4 acc[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        xrow[j] = a.X + (int64_t)min(m0 + 16 * j + c, a.M - 1) * a.ldx;
        acc[j] = i32x4{0, 0, 0, 0};
    }
    for (int k = 0; k < a.K; k += 64) {
        const int at = k + g * 16;
        const bool in = at < a.K;
        const i32x4 zero = {0, 0, 0, 0};
        const i32x4 w = in ? *reinterpret_cast<const i32x4*>(wrow + at) : zero;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const i32x4 x = in ? *reinterpret_cast<const i32x4*>(xrow[j] + at) : zero;
            acc[j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w, x, acc[j], 0, 0, 0);
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int m = m0 + 16 * j + c;
        if (m >= a.M) continue;
        const float sx = a.sx[m];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int n = n0 + 4 * g + i;
            if (n >= a.N) continue;
            const float y = (float)acc[j][i] * sx * a.sw[n];
            if constexpr (BF16) static_cast<uint16_t*>(a.Y)[m * a.ldy + n] = f32_to_bf16_bits(y);
            else static_cast<float*>(a.Y)[m * a.ldy + n] = y;
        }
    }
}

hipError_t launch_linear_q8(int M, int N, int K, const int8_t* X, int64_t ldx, const float* sx, const int8_t* W, const float* sw, int y_dtype,
                            void* Y, int64_t ldy, hipStream_t s) {
    const LinearArgs a{M, N, K, X, ldx, sx, W, sw, Y, ldy};
    ProfScope prof(TABED_K_LMHEAD, s);
    const dim3 grid((N + 63) / 64, (M + 63) / 64);
    if (y_dtype == 1) launch(&prof, k_linear_q8<true>, grid, dim3(kBlock), 0, s, a);
    else launch(&prof, k_linear_q8<false>, grid, dim3(kBlock), 0, s, a);
    return hipGetLastError();
}

}  // namespace tabed
