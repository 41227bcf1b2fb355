// Products of int8 rows with int8 weights (tabed_linear_q8): Y[m][n] = (sum_k X[m][k] W[n][k]) * sx[m] * sw[n], and the LM head in
// 8 bits, which is the same with softmax partials.  The sum is in int32 and exact for the K allowed, so the order of its terms is
// free: waves and k-steps share it as suits the memory; one rounding for the integer, one for each scale and one for storage.
// One kernel in tiles of several sizes: with few rows W's bytes bound it and small tiles give every compute unit some of them, with many
// the matrix cores do and tiles are as large as registers and LDS hold.
#include <algorithm>
#include <mutex>
#include <type_traits>

#include "body_utils.h"
#include "lmhead_store.h"
#include "q8_utils.h"

namespace tabed {

enum { kOutF32 = 0, kOutB16 = 1, kOutHead = 2 };      // kOutHead: fp32 logits and the softmax partials of every 32 columns

struct LinearArgs {
    int M, N, K;
    const int8_t* X;
    uint32_t ldx;
    const float* sx;
    const int8_t* W;
    const float* sw;
    void* Y;
    int64_t ldy;
    int n;                       // kOutHead: rows of a sequence
    const float* temperature;    //   [M / n]
    float* pm;                   //   [M][ceil(N / 32)]
    float* ps;
};

constexpr int kLine = 128;       // bytes of a row that a k-block takes
constexpr int kLinearThreads = 512;

// ---------------------------------------------------------------- the product
// Workgroup tile BM rows x BN columns, eight waves: KW of them share a block of it and take 128 bytes each of a k-block of 128 KW; the
// others split it, into 32x32 MFMA tiles with W as the row operand.  With KW = 1 a wave has up to 128 x 64 of the tile and its fragments are used
// again and again; small tiles have too little to split, and there KW > 1 makes a k-block long and the barriers few (32 x 64, K = 4096:
// 9.1 us with KW = 4 for 8192 columns, 64 x 128 with KW = 1 takes 14.3).  The KW integer sums of a block meet in LDS.
// Operands go from memory straight to LDS in SW stages of W and SH of X; a stage has lines of 128 bytes, row r with its
// 16-byte pieces in the order piece ^ (r / 2 % 8), which the lanes bring about by the address they load from: 16 rows' pieces lie in 64 different
// banks (with r % 8 two of them share theirs, and a read of fragments takes 8 cycles instead of 4).  One barrier per k-block, before the
// products of its last k-step: the next k-block's first fragments are read while those run.  Workgroup w goes to XCD w % 8:
// the row blocks that share a column block run back to back on one XCD, so W comes from memory once, and all XCDs have as many tiles but for one
// (4150 x 5659, K = 2048: 87 us; dealt out in whole column blocks to the last, 108).
// What bounds it: few rows W's bytes (64 x 32000, K = 768: 8.2 us for 33 MB; 16 x 32000, K = 8192 53 us, 4.95 TB/s), many rows the products at the
// clock that the power leaves (4096 x 8192, K = 8192: 247 us, 2.2 POP/s; 512 x 128256, K = 2048 with 263 MB of W and as many of results 166 us).
// K past the last whole k-block: loads re-read its last 16 bytes, and X's fragments are zeroed there.
template <int BM, int BN, int KW, int SW, int SH, int EPI, bool PAST>
__global__ __launch_bounds__(kLinearThreads, 2) void k_linear_tile(LinearArgs a, int mblocks, int whole, int share) {
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    constexpr int kStW = KW * BN * kLine, kStX = KW * BM * kLine, kRows = (BM == 32 || KW > 2) ? 1 : 2, kCols = 8 / KW / kRows;
    constexpr int TV = BN / (32 * kCols), TM = BM / (32 * kRows), WI = KW * BN / 64, XI = KW * BM / 64;
    constexpr uint32_t kNext = 8 * 8 * kLine;                         // LDS bytes from one of a wave's loads to its next
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int nn = lane & 31, half = lane >> 5;
    const int xcd = blockIdx.x & 7, slot = blockIdx.x >> 3, rest = slot - whole * mblocks, at = rest < 0 ? slot : xcd * share + rest;
    const int mb = at % mblocks, nb = rest < 0 ? at / mblocks * 8 + xcd : whole * 8 + at / mblocks;
    const int M = a.M, N = a.N, K = a.K, m0 = mb * BM, n0 = nb * BN;
    if (n0 >= N) return;                                              // uniform: the last XCD's share of the rest may be smaller
    const int wm = wave / kCols % kRows, wn = wave % kCols, kw = wave / (kCols * kRows);
    const float my_sx = a.sx[min(m0 + (tid & (BM - 1)), M - 1)], my_sw = a.sw[min(n0 + (tid & (BN - 1)), N - 1)];      // used after the loop
    float my_temp = 1.f;
    if constexpr (EPI == kOutHead) my_temp = a.temperature[min(m0 + (tid & (BM - 1)), M - 1) / a.n];
    const int KB = (K + KW * kLine - 1) / (KW * kLine), last_pieces = (K - (KB - 1) * KW * kLine) / 16;
    const char* const wbase = reinterpret_cast<const char*>(a.W) + (size_t)n0 * K;
    const char* const xbase = reinterpret_cast<const char*>(a.X) + (size_t)m0 * a.ldx;
    // Load i of a wave: lines (i * 8 + wave) * 8 .. + 8 of a stage, which holds KW times 128 bytes of every row, one after the other.
    const int line0 = wave * 8 + (lane >> 3), piece = (lane & 7) ^ (line0 >> 1 & 7);
    uint32_t wo[WI], xo[XI];                                          // rows past the end re-read the last one
#pragma unroll
    for (int i = 0; i < WI; ++i) wo[i] = (uint32_t)min((i * 64 + line0) % BN, N - 1 - n0) * (uint32_t)K + (i * 64 + line0) / BN * kLine + piece * 16;
#pragma unroll
    for (int i = 0; i < XI; ++i) xo[i] = (uint32_t)min((i * 64 + line0) % BM, M - 1 - m0) * a.ldx + (i * 64 + line0) / BM * kLine + piece * 16;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds + (uint32_t)wave * 8u * kLine;
    auto request = [&](const char* base, const auto& off, auto per, int kb, uint32_t to) {
        kb = min(kb, KB - 1);
        if (kb == KB - 1 && last_pieces < 8 * KW) {                        // uniform
            std::remove_cv_t<std::remove_reference_t<decltype(off)>> o;
#pragma unroll
            for (size_t i = 0; i < sizeof(o) / 4; ++i) o[i] = off[i] - (uint32_t)max(((int)i * 64 + line0) / per.value * 8 + piece - (last_pieces - 1), 0) * 16u;
            dma_lines(base + (size_t)kb * (KW * kLine), o, to, kNext);
        } else {
            dma_lines(base + (size_t)kb * (KW * kLine), off, to, kNext);
        }
    };
    auto request_w = [&](int kb, int stage) { request(wbase, wo, std::integral_constant<int, BN>{}, kb, lds0 + (uint32_t)(stage * kStW)); };
    auto request_x = [&](int kb, int stage) { request(xbase, xo, std::integral_constant<int, BM>{}, kb, lds0 + (uint32_t)(SW * kStW + stage * kStX)); };

    i32x16 acc[TV][TM];
#pragma unroll
    for (int p = 0; p < TV; ++p)
#pragma unroll
        for (int b = 0; b < TM; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[p][b][r] = 0;
    const uint32_t wrow = (uint32_t)(kw * BN + wn * 32 * TV + nn) * kLine, xrow = (uint32_t)(SW * kStW) + (uint32_t)(kw * BM + wm * (BM / kRows) + nn) * kLine, turn = (uint32_t)(nn >> 1 & 7);
    i32x4 wf[2][TV], xf[2][TM];                                       // fragments of two k-steps of 32
    int stw = 0, stx = 0;
    auto read_frags = [&](int ks, int set) {
        const unsigned char* sW = lds + stw * kStW + wrow;
        const unsigned char* sX = lds + stx * kStX + xrow;
        const uint32_t c = ((uint32_t)(2 * ks + half) ^ turn) * 16u;
#pragma unroll
        for (int p = 0; p < TV; ++p) wf[set][p] = *reinterpret_cast<const i32x4*>(sW + p * 32 * kLine + c);
#pragma unroll
        for (int b = 0; b < TM; ++b) xf[set][b] = *reinterpret_cast<const i32x4*>(sX + b * 32 * kLine + c);
    };
    auto products = [&](int ks, int set, auto last) {
        if constexpr (last.value) {                                   // what lies past K counts as zeros
            const bool in = 8 * kw + 2 * ks + half < last_pieces;
#pragma unroll
            for (int b = 0; b < TM; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) xf[set][b][i] = in ? xf[set][b][i] : 0;
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int p = 0; p < TV; ++p)
#pragma unroll
            for (int b = 0; b < TM; ++b) acc[p][b] = __builtin_amdgcn_mfma_i32_32x32x32_i8(wf[set][p], xf[set][b], acc[p][b], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
    };

    static_assert(SW == SH || SW == SH + 1, "the order of requests below");
#pragma unroll
    for (int q = 0; q < SW; ++q) {
        request_w(q, q);
        if (q < SH) request_x(q, q);
    }
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" :: "n"((SW - 1) * WI + (SH - 1) * XI) : "memory");
    read_frags(0, 0);
    auto step = [&](int kb, auto refill, auto left, auto last) {
#pragma unroll
        for (int ks = 0; ks < kLine / 32 - 1; ++ks) {                 // fragments of k-step ks + 1 are read while ks is multiplied
            read_frags(ks + 1, (ks + 1) & 1);
            products(ks, ks & 1, last);
        }
        // The stage's last fragments are in registers: it is free once all waves are here.  k-block kb + 1 is there once no more than what
        // a wave asked for after that (left) is outstanding.
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"(left.value) : "memory");
        if constexpr (refill.value) {
            request_x(kb + SH, stx);
            request_w(kb + SW, stw);
        }
        stw = (stw + 1 == SW) ? 0 : stw + 1;
        stx = (stx + 1 == SH) ? 0 : stx + 1;
        read_frags(0, 0);
        products(kLine / 32 - 1, 1, last);
    };
    int kb = 0;
    for (; kb + SH < KB; ++kb) step(kb, std::true_type{}, std::integral_constant<int, (SW - 2) * WI + (SH - 2) * XI>{}, std::false_type{});
    // The last SH k-blocks.  With fewer than that in all, the first of these steps are left out; requests past the last k-block then
    // re-read it, so that the waits count the same.
    const int skip = max(SH - KB, 0);
    auto tail = [&](auto t) {
        constexpr int pairs = SH - 2 - t.value > 0 ? SH - 2 - t.value : 0;
        if constexpr (t.value < SH)
            if (t.value >= skip)
                step(kb + t.value - skip, std::false_type{}, std::integral_constant<int, pairs * (WI + XI) + (SW - SH) * WI>{}, std::integral_constant<bool, t.value == SH - 1>{});
    };
    static_assert(SH <= 4, "tail");
    tail(std::integral_constant<int, 0>{});
    tail(std::integral_constant<int, 1>{});
    tail(std::integral_constant<int, 2>{});
    tail(std::integral_constant<int, 3>{});

    // ---- scales, then every wave turns its blocks through private patches carved from the stages
    constexpr int kPT = BN / kTileV, kPS = BM * kPT;
    float* const s_sx = reinterpret_cast<float*>(lds + 16 * kPatchBytes);
    float* const s_sw = s_sx + BM;
    float* const s_invt = s_sw + BN;
    float* const s_part = s_invt + BM;                                // [2][BM][kPT]
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");      // nothing is on its way to LDS any more, nothing is read from it
    __syncthreads();
    if (tid < BM) {
        s_sx[tid] = my_sx;
        s_invt[tid] = inv_temperature(my_temp);
    }
    if (tid < BN) s_sw[tid] = my_sw;
    __syncthreads();
    constexpr int kSums = TV * TM * 16 * 64 * 4, kOwn = std::max(2 * kPatchBytes, (KW - 1) * kSums);     // bytes
    static_assert(8 / KW * kOwn <= 16 * kPatchBytes);
    unsigned char* const patch = lds + wave % (8 / KW) * kOwn;
    if constexpr (KW > 1) {                                           // the sums of the waves that share a block go to the first
        i32x4* const sums = reinterpret_cast<i32x4*>(patch) + lane;
        if (kw > 0) {
#pragma unroll
            for (int q = 0; q < TV * TM * 4; ++q) {
                const i32x16& v = acc[q / 4 / TM][q / 4 % TM];
                sums[(kw - 1) * (kSums / 16) + q * 64] = i32x4{v[4 * (q & 3)], v[4 * (q & 3) + 1], v[4 * (q & 3) + 2], v[4 * (q & 3) + 3]};
            }
        }
        __syncthreads();
        if (EPI != kOutHead && kw > 0) return;
#pragma unroll
        for (int u = 0; u < KW - 1; ++u)
#pragma unroll
            for (int q = 0; q < TV * TM * 4; ++q) {
                const i32x4 v = sums[u * (kSums / 16) + q * 64];
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[q / 4 / TM][q / 4 % TM][4 * (q & 3) + i] += v[i];
            }
    }
    const int lr = wm * (BM / kRows), lc = wn * 32 * TV, rows = M - m0 - lr;                  // this wave's block of the tile
    f32x16 y[TV][TM];
#pragma unroll
    for (int b = 0; b < TM; ++b) {
        const float sx = s_sx[lr + b * 32 + nn];
#pragma unroll
        for (int p = 0; p < TV; ++p)
#pragma unroll
            for (int r = 0; r < 16; ++r) y[p][b][r] = (float)acc[p][b][r] * sx;
    }
#pragma unroll
    for (int p = 0; p < TV; ++p)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const float4 sw = *reinterpret_cast<const float4*>(s_sw + lc + p * 32 + 8 * g + 4 * half);
#pragma unroll
            for (int b = 0; b < TM; ++b) {
                y[p][b][4 * g] *= sw.x;
                y[p][b][4 * g + 1] *= sw.y;
                y[p][b][4 * g + 2] *= sw.z;
                y[p][b][4 * g + 3] *= sw.w;
            }
        }
    if constexpr (EPI == kOutHead) {
        float* const L = static_cast<float*>(a.Y);
        constexpr int kW = kPT < 4 ? kPT : 4;                         // partials stored at a time
        typedef float vec __attribute__((ext_vector_type(kW)));
        typedef float vec_e4 __attribute__((ext_vector_type(kW), aligned(4)));
        const int parts = (N + kTileV - 1) / kTileV;
        if (n0 + BN > N) {                                            // uniform: the last column block
            if (kw > 0) return;
#pragma unroll
            for (int p = 0; p < TV; ++p)
#pragma unroll
                for (int b = 0; b < TM; ++b)
                    store_tile_32x32_t<PAST>(y[p][b], m0 + lr + b * 32, n0 + lc + p * 32, M, N, parts, s_invt - m0, L, a.pm, a.ps, patch);
            return;
        }
        if (kw == 0) store_full_tiles<PAST, TV, TM, kPT, kPS>(y, rows, s_invt + lr, s_part + lr * kPT + wn * TV, L + (size_t)(m0 + lr) * N + n0 + lc, N, patch);
        lds_barrier();
#pragma unroll
        for (int t = tid; t < 2 * BM * (kPT / kW); t += kLinearThreads) {
            const int q = t % (kPT / kW), row = t / (kPT / kW) % BM, arr = t / (kPT / kW) / BM;
            const vec x = *reinterpret_cast<const vec*>(s_part + arr * kPS + row * kPT + kW * q);
            if (m0 + row < M) *reinterpret_cast<vec_e4*>((arr == 0 ? a.pm : a.ps) + (size_t)(m0 + row) * parts + n0 / kTileV + kW * q) = vec_e4(x);
        }
    } else if constexpr (EPI == kOutF32) {
        const int q = lane & 7;
#pragma unroll
        for (int p = 0; p < TV; ++p) {
            const int n = n0 + lc + p * 32 + 4 * q;
#pragma unroll
            for (int b = 0; b < TM; ++b) {
                if (b * 32 >= rows) continue;                         // uniform
                unsigned char* const tp = patch + (b & 1) * kPatchBytes;
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    *reinterpret_cast<float4*>(tp + nn * 144 + (8 * g + 4 * half) * 4) =
                        make_float4(y[p][b][4 * g], y[p][b][4 * g + 1], y[p][b][4 * g + 2], y[p][b][4 * g + 3]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int m = b * 32 + 8 * i + (lane >> 3);
                    const float4 v = *reinterpret_cast<const float4*>(tp + (8 * i + (lane >> 3)) * 144 + q * 16);
                    float* const out = static_cast<float*>(a.Y) + (int64_t)(m0 + lr + m) * a.ldy + n;
                    if (m < rows) {
                        if (n + 4 <= N) store_logits<PAST>(out, f32x4u{v.x, v.y, v.z, v.w});
                        else {
                            if (n < N) out[0] = v.x;
                            if (n + 1 < N) out[1] = v.y;
                            if (n + 2 < N) out[2] = v.z;
                        }
                    }
                }
            }
        }
    } else {
        constexpr int LPR = 4 * TV;                                   // lanes of a row: eight columns each
        const int q = lane % LPR, n = n0 + lc + 8 * q;
#pragma unroll
        for (int b = 0; b < TM; ++b) {
            if (b * 32 >= rows) continue;                             // uniform
            unsigned char* const tp = patch + (b & 1) * kPatchBytes;
#pragma unroll
            for (int p = 0; p < TV; ++p)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    *reinterpret_cast<uint2*>(tp + nn * 144 + p * 64 + (8 * g + 4 * half) * 2) =
                        pack_bf16x4(y[p][b][4 * g], y[p][b][4 * g + 1], y[p][b][4 * g + 2], y[p][b][4 * g + 3]);
#pragma unroll
            for (int i = 0; i < 32 * LPR / 64; ++i) {
                const int mr = (64 / LPR) * i + lane / LPR, m = b * 32 + mr;
                const u32x4 v = *reinterpret_cast<const u32x4*>(tp + mr * 144 + q * 16);
                uint16_t* const out = static_cast<uint16_t*>(a.Y) + (int64_t)(m0 + lr + m) * a.ldy + n;
                if (m < rows) {
                    if (n + 8 <= N) *reinterpret_cast<u32x4_e2*>(out) = u32x4_e2(v);
                    else
#pragma unroll
                        for (int e = 0; e < 7; ++e)
                            if (n + e < N) out[e] = (uint16_t)(v[e / 2] >> (16 * (e & 1)));
                }
            }
        }
    }
}

// ---------------------------------------------------------------- host side
// (The limit of a kernel's LDS is raised once for each device.)
template <typename K>
static hipError_t raise_on_device(K kernel, size_t lds, std::once_flag (&once)[kMaxDevices], hipError_t (&rc)[kMaxDevices]) {
    int dev = 0;
    const hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    if (dev < 0 || dev >= kMaxDevices) return hipErrorInvalidDevice;
    return raise_lds_limit(kernel, lds, once[dev], rc[dev]);
}

template <int BM, int BN, int KW, int SW, int SH, int EPI, bool PAST>
static hipError_t launch_tile_q8(const ProfScope* prof, const LinearArgs& a, hipStream_t s) {
    constexpr size_t lds = std::max((size_t)KW * (SW * BN + SH * BM) * kLine, (size_t)16 * kPatchBytes + (2 * BM + BN) * 4 + 2 * BM * (BN / kTileV) * 4);
    static std::once_flag once[kMaxDevices];
    static hipError_t rc[kMaxDevices];
    const hipError_t e = raise_on_device(&k_linear_tile<BM, BN, KW, SW, SH, EPI, PAST>, lds, once, rc);
    if (e != hipSuccess) return e;
    // Column blocks are dealt out one by one, what is left of the last round of them tile by tile.  Where rows of Y do not begin on 64 bytes neighbouring
    // column blocks write parts of the same ones, and many rows' tiles are dealt out in eight runs instead, so that both are in one L2
    // (2000 x 9000, K = 2048: 56.3 us against 61; 1000 x 50000, K = 512: 55.7, 64.4; but 2000 x 20000, K = 512 45.9, 43.8, and 16 x 32000, K = 4096 30.3, 28.6).
    const int mblocks = (a.M + BM - 1) / BM, nblocks = (a.N + BN - 1) / BN;
    const bool runs = a.M > 64 && a.ldy * (EPI == kOutB16 ? 2 : 4) % 64 != 0;
    const int whole = runs ? 0 : nblocks / 8, share = (int)(((int64_t)(nblocks - 8 * whole) * mblocks + 7) / 8);
    launch(prof, k_linear_tile<BM, BN, KW, SW, SH, EPI, PAST>, dim3((whole * mblocks + share) * 8), dim3(kLinearThreads), lds, s, a, mblocks, whole, share);
    return hipGetLastError();
}

// The tile for a product of these sizes, handed to `go`.
template <int BM_, int BN_, int KW_, int SW_, int SH_>
struct Tile { static constexpr int BM = BM_, BN = BN_, KW = KW_, SW = SW_, SH = SH_; };
template <typename Go>
static hipError_t with_tile(int M, int N, int K, bool head, Go&& go) {
    auto tiles = [&](int bm, int bn) { return (long)((M + bm - 1) / bm) * ((N + bn - 1) / bn); };
    // Few tiles: the smaller they are, the more compute units load.  32 x 32 reads X as often as W, so only while all tiles together
    // read little (200 x 1024, K = 2048: 4.7 us against 5.2 in 32 x 64; 16 x 8192, K = 8192: 20.1 against 12.4).  Then the smallest
    // tile that every compute unit has at most one of (64 x 8192, K = 4096: 9.7 us in 32 x 64, 10.1 in 64 x 64, 14.7 in 64 x 128;
    // 128 rows: 13.7, 10.6, 14.8).  With one or two row blocks and more columns than that it is two workgroups a compute unit, or one after the other
    // with deeper stages where K is long enough to fill them (16 x 32000: K = 2048 14.1 us against 15.7, K = 4096 30.4 against 28.7), or one of
    // 64 x 128 where K is short and there are few results or softmax partials, which all eight waves then make (20000 columns, 32 rows, K = 1024 7.9 us
    // against 8.5, LM head of 64 x 32000, K = 768 7.9 against 8.7; but its product alone 8.6 against 8.2, and with K = 4096 35.4 against 31.0).
    if (tiles(32, 32) <= 256 && tiles(32, 32) * K <= 3 << 18) return go(Tile<32, 32, 8, 2, 2>{});
    if (tiles(32, 64) <= 256 || (M <= 32 && K >= 4096)) return go(Tile<32, 64, 4, 3, 3>{});
    if (tiles(64, 64) <= 256) return go(Tile<64, 64, 2, 3, 3>{});
    if (M <= (head ? 64 : 32) && K <= 1024 && tiles(64, 128) <= 256) return go(Tile<64, 128, 1, 3, 3>{});
    if (M <= 64) return go(Tile<64, 64, 2, 2, 2>{});
    // Many tiles: time goes in rounds of as many workgroups as fit the chip, and a round's length with the tile (K = 4096: 57 us in 256 x 256, 36 in
    // 128 x 256, 22 in 128 x 128, 18 in 64 x 128, or 29 where that has two workgroups a compute unit; K = 512: 15.7, 9.6, 5.8, 4.9, 7.9).  Taken is
    // the least product of the two: 160 x 20000, K = 4096 30.5 us in 64 x 128, 32.7 in 128 x 256; 520 x 50000 144 in 128 x 256, 168 in
    // 256 x 256; 1000 x 9000 53 in 256 x 256, 65 in 128 x 256; 520 x 4000 18.8 in 128 x 128, 20.9 in 64 x 128.
    auto cost = [&](int bm, int bn, int length, int at_once) { return (tiles(bm, bn) + at_once - 1) / at_once * length; };
    const long large = cost(256, 256, 16, 256), wide = cost(128, 256, 10, 256), mid = cost(128, 128, 6, 256);
    const long narrow = std::min(cost(64, 128, 5, 256), cost(64, 128, 8, 512));
    if (large <= std::min({wide, mid, narrow})) return go(Tile<256, 256, 1, 3, 2>{});
    if (wide <= std::min(mid, narrow)) return go(Tile<128, 256, 1, 3, 3>{});
    if (mid <= narrow) return go(Tile<128, 128, 1, 4, 4>{});
    return go(Tile<64, 128, 1, 3, 3>{});
}

template <int EPI, bool PAST>
static hipError_t launch_tiles(const ProfScope* prof, const LinearArgs& a, hipStream_t s) {
    return with_tile(a.M, a.N, a.K, EPI == kOutHead, [&](auto t) {
        using T = decltype(t);
        return launch_tile_q8<T::BM, T::BN, T::KW, T::SW, T::SH, EPI, PAST>(prof, a, s);
    });
}

void linear_q8_tile(int M, int N, int K, bool head, int32_t* tile) {
    (void)with_tile(M, N, K, head, [&](auto t) {
        using T = decltype(t);
        tile[0] = T::BM; tile[1] = T::BN; tile[2] = T::KW; tile[3] = T::SW; tile[4] = T::SH;
        return hipSuccess;
    });
}

template <int EPI>
static hipError_t launch_product(const ProfScope* prof, const LinearArgs& a, hipStream_t s) {
    if constexpr (EPI == kOutHead)
        if (a.M > 64 && !past_l2(a.N, a.K / 2, a.M)) return launch_tiles<EPI, false>(prof, a, s);
    return launch_tiles<EPI, EPI == kOutHead>(prof, a, s);
}

hipError_t launch_linear_q8(int M, int N, int K, const int8_t* X, int64_t ldx, const float* sx, const int8_t* W, const float* sw, int y_dtype,
                            void* Y, int64_t ldy, hipStream_t s) {
    const LinearArgs a{M, N, K, X, (uint32_t)ldx, sx, W, sw, Y, ldy, 1, nullptr, nullptr, nullptr};
    ProfScope prof(TABED_K_BODY, s);
    return y_dtype == 1 ? launch_product<kOutB16>(&prof, a, s) : launch_product<kOutF32>(&prof, a, s);
}

hipError_t launch_lmhead_q8(const tabed_cfg& c, const WsLayout& L, char* ws, const int8_t* W, const float* w_scale, const int8_t* H,
                            const float* h_scale, const float* temperature, float* logits, hipStream_t s) {
    const LinearArgs a{L.M, c.V, c.d, H, (uint32_t)c.d, h_scale, W, w_scale, logits, c.V, c.n, temperature,
                       reinterpret_cast<float*>(ws + L.off_pm), reinterpret_cast<float*>(ws + L.off_ps)};
    ProfScope prof(TABED_K_LMHEAD, s);
    return launch_product<kOutHead>(&prof, a, s);
}

}  // namespace tabed
