// Products of int8 rows with int8 weights (tabed_linear_q8): Y[m][n] = (sum_k X[m][k] W[n][k]) * sx[m] * sw[n], and the LM head in
// 8 bits, which is the same with softmax partials.  The sum is in int32 and exact for the K allowed, so the order of its terms is
// free: waves and k-steps share it as suits the memory; one rounding for the integer, one for each scale and one for storage.
// Two kernels: up to 64 rows W is streamed and its bytes bound the product, beyond it is tiled for the matrix cores.
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

typedef uint32_t u32x2_e2 __attribute__((ext_vector_type(2), aligned(2)));

constexpr int kLine = 128;       // bytes of a row that a k-block takes
constexpr int kLinearThreads = 512;

// ---------------------------------------------------------------- up to 64 rows: W is streamed
// Eight waves a workgroup.  KS of them share a tile of 16 NT columns, taking k-steps (128 bytes of 32 rows of W, or 256 of 16) in turn;
// a workgroup owns 8 / KS tiles and walks over the columns.  A wave requests its k-steps as whole lines, kAhead of them ahead of the one being
// multiplied, and turns each through a wave-private LDS patch into operand layout (LDS operations of a wave are in order: no
// barrier).  16 MT rows of X lie in LDS, all of K at once where 64 KB hold them, else in chunks, the next of which is requested while one is
// in use.  The KS integer sums of a tile meet in the patches, 32 rows at a time, from where a row's columns are scaled and stored side by side.
// Loads are never predicated (the number in flight is fixed): what lies past an end re-reads the last of it, and X is zero past K.
constexpr int kAhead = 3;
constexpr int kXPieces = 8;                                       // 16-byte pieces of a chunk of X per thread
constexpr int linear_chunk(int MT) { return kXPieces * kLinearThreads / MT; }        // bytes of K in a chunk, at most

template <int MT, int KS, int NT, int EPI, bool CH /* more than one chunk */>
__global__ __launch_bounds__(kLinearThreads) void k_linear_stream(LinearArgs a, int groups, int kc /* bytes of a chunk */) {
    constexpr int kTiles = 8 / KS, COLS = 16 * NT, VW = kTiles * COLS;
    constexpr int LPR = 16 / NT, RPL = 64 / LPR;                      // lanes of a row in a request; rows of a request
    constexpr int kStep = LPR * 16, kPatchRow = kStep + 16;           // bytes of a k-step; of a row of the patch
    constexpr int SR = (MT == 1) ? 16 : 32, kMeetRow = COLS * 4 + 16;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    __shared__ float s_sx[MT * 16], s_invt[MT * 16];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int ks = wave % KS, tile = wave / KS, r16 = lane & 15, g4 = lane >> 4, lrow = lane / LPR, lpiece = lane % LPR;
    const int M = a.M, N = a.N, K = a.K, xrow = kc + 16;
    unsigned char* const s_x = lds;
    unsigned char* const patches = lds + MT * 16 * xrow;
    unsigned char* const patch = patches + wave * kPatchBytes;
    const float my_sx = a.sx[min(tid, M - 1)];
    float my_temp = 1.f;
    if constexpr (EPI == kOutHead) my_temp = a.temperature[sequence_of(min(tid, M - 1), a.n)];

    // ---- chunks of X
    const int nchunks = CH ? (K + kc - 1) / kc : 1, pieces = MT * kc;
    u32x4 xreg[kXPieces];                                             // (their places are worked out anew for every chunk: not worth the registers)
    auto request_x = [&](int chunk) {
        int per_row = kc / 16;
        asm volatile("" : "+s"(per_row));
#pragma unroll
        for (int q = 0; q < kXPieces; ++q) {
            const int idx = q * kLinearThreads + tid, row = idx / per_row, col = chunk * kc + (idx % per_row) * 16;
            if (q * kLinearThreads < pieces)                          // uniform
                xreg[q] = *reinterpret_cast<const u32x4*>(a.X + (size_t)min(row, M - 1) * a.ldx + min(col, K - 16));
        }
    };
    auto write_x = [&](int chunk) {
        int per_row = kc / 16;
        asm volatile("" : "+s"(per_row));
#pragma unroll
        for (int q = 0; q < kXPieces; ++q) {
            const int idx = q * kLinearThreads + tid, row = idx / per_row, at = (idx % per_row) * 16;
            if (q * kLinearThreads < pieces && idx < pieces) {
                const u32x4 zero = {0u, 0u, 0u, 0u};
                *reinterpret_cast<u32x4*>(s_x + row * xrow + at) = (chunk * kc + at < K) ? xreg[q] : zero;
            }
        }
    };

    // ---- W: step j is bytes (j KS + ks) kStep .. of this wave's tile
    const int steps = (K + kStep * KS - 1) / (kStep * KS), padded = (steps + kAhead - 1) / kAhead * kAhead;
    const int per_chunk = kc / (kStep * KS);
    u32x4 ring[kAhead][4];
    const int8_t* wbase;
    uint32_t woff[4];
    const int q4 = tid % (VW / 4);                                    // the four columns that this thread finishes, of every group
    f32x4 sw;
    auto request_sw = [&](int group) {
#pragma unroll
        for (int u = 0; u < 4; ++u) sw[u] = a.sw[min(group * VW + 4 * q4 + u, N - 1)];
    };
    auto aim = [&](int group) {
        const int first = min(group * VW + tile * COLS, N - 1);
        wbase = a.W + (size_t)first * K;
#pragma unroll
        for (int i = 0; i < 4; ++i) woff[i] = (uint32_t)min(RPL * i + lrow, N - 1 - first) * (uint32_t)K;
    };
    auto request_w = [&](int slot, int j) {
        const uint32_t k = (uint32_t)min((min(j, steps - 1) * KS + ks) * kStep + lpiece * 16, K - 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) ring[slot][i] = *reinterpret_cast<const u32x4*>(wbase + (woff[i] + k));
    };

    request_x(0);
    __builtin_amdgcn_sched_barrier(0);
    aim(blockIdx.x);
#pragma unroll
    for (int q = 0; q < kAhead; ++q) request_w(q, q);
    request_sw(blockIdx.x);
    __builtin_amdgcn_sched_barrier(0);
    write_x(0);
    if (tid < MT * 16) {
        s_sx[tid] = my_sx;
        if constexpr (EPI == kOutHead) s_invt[tid] = inv_temperature(my_temp);
    }
    lds_barrier();

    for (int group = blockIdx.x;; group += gridDim.x) {
        const bool more = group + (int)gridDim.x < groups;
        i32x4 acc[NT][MT];
#pragma unroll
        for (int nb = 0; nb < NT; ++nb)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) acc[nb][mt] = i32x4{0, 0, 0, 0};
        if (group != (int)blockIdx.x) request_sw(group);
        int chunk = 0, in_chunk = 0;                                  // of the step being multiplied
        if constexpr (CH) request_x(1);
        // one round of the ring; ahead 0: the freed slots take steps of this group, 1: the first of the next group, 2: nothing is left
        auto round = [&](int j0, auto ahead) {
#pragma unroll
            for (int q = 0; q < kAhead; ++q) {
                const int j = j0 + q;
                if constexpr (CH)
                    if (in_chunk == per_chunk && j < steps) {         // uniform over the workgroup
                        lds_barrier();                                // every wave is done with the chunk
                        ++chunk;
                        in_chunk = 0;
                        write_x(chunk);
                        lds_barrier();
                        if (chunk + 1 < nchunks) request_x(chunk + 1);
                    }
                if (j < steps) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) *reinterpret_cast<u32x4*>(patch + (RPL * i + lrow) * kPatchRow + lpiece * 16) = ring[q][i];
                }
                __builtin_amdgcn_sched_barrier(0);
                if constexpr (ahead.value == 0) request_w(q, j + kAhead);
                if constexpr (ahead.value == 1) request_w(q, q);
                __builtin_amdgcn_sched_barrier(0);
                if (j < steps) {
                    const unsigned char* const xp = s_x + r16 * xrow + (in_chunk * KS + ks) * kStep + g4 * 16;
                    constexpr int P = kStep / 64;
                    i32x4 w[P][NT];
#pragma unroll
                    for (int p = 0; p < P; ++p)
#pragma unroll
                        for (int nb = 0; nb < NT; ++nb)
                            w[p][nb] = *reinterpret_cast<const i32x4*>(patch + (nb * 16 + r16) * kPatchRow + p * 64 + g4 * 16);
#pragma unroll
                    for (int p = 0; p < P; ++p)
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) {
                            const i32x4 x = *reinterpret_cast<const i32x4*>(xp + mt * 16 * xrow + p * 64);
#pragma unroll
                            for (int nb = 0; nb < NT; ++nb) acc[nb][mt] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[p][nb], x, acc[nb][mt], 0, 0, 0);
                        }
                    ++in_chunk;
                }
            }
        };
        for (int j0 = 0; j0 + kAhead < padded; j0 += kAhead) round(j0, std::integral_constant<int, 0>{});
        if (more) {
            aim(group + gridDim.x);
            round(padded - kAhead, std::integral_constant<int, 1>{});
        } else {
            round(padded - kAhead, std::integral_constant<int, 2>{});
        }
        if constexpr (CH)
            if (more) {
                request_x(0);
                lds_barrier();
                write_x(0);                                           // (seen after the barriers below)
            }

        // ---- the KS sums meet, SR rows at a time
#pragma unroll
        for (int r0 = 0; r0 < MT * 16; r0 += SR) {
            if (r0 < M) {                                             // uniform
#pragma unroll
                for (int i = 0; i < SR / 16; ++i)
#pragma unroll
                    for (int nb = 0; nb < NT; ++nb)
                        *reinterpret_cast<i32x4*>(patch + (i * 16 + r16) * kMeetRow + nb * 64 + g4 * 16) = acc[nb][r0 / 16 + i];
                lds_barrier();
#pragma unroll
                for (int e = 0; e < SR * VW / 4; e += kLinearThreads) {
                    const int idx = e + tid, row = idx / (VW / 4);
                    if (SR * VW / 4 >= kLinearThreads || idx < SR * VW / 4) {
                        const unsigned char* part = patches + (q4 / (COLS / 4)) * KS * kPatchBytes + row * kMeetRow + (q4 % (COLS / 4)) * 16;
                        i32x4 sum = *reinterpret_cast<const i32x4*>(part);
#pragma unroll
                        for (int w = 1; w < KS; ++w) sum += *reinterpret_cast<const i32x4*>(part + w * kPatchBytes);
                        const int m = r0 + row, n0 = group * VW + 4 * q4;
                        const bool live = m < M && n0 < N;
                        float y[4];
#pragma unroll
                        for (int u = 0; u < 4; ++u) y[u] = (float)sum[u] * s_sx[m] * sw[u];
                        if constexpr (EPI == kOutHead) {
                            const float it = s_invt[m];
                            float sc[4], mx = -INFINITY;
#pragma unroll
                            for (int u = 0; u < 4; ++u) {
                                sc[u] = (n0 + u < N) ? y[u] * it : -INFINITY;
                                mx = fmaxf(mx, sc[u]);
                            }
                            mx = fmaxf(mx, dpp_f32<kDppXor1>(mx));
                            mx = fmaxf(mx, dpp_f32<kDppXor2>(mx));
                            mx = fmaxf(mx, dpp_f32<kDppHalfMirror>(mx));
                            float s = 0.f;
#pragma unroll
                            for (int u = 0; u < 4; ++u) s += (sc[u] > -INFINITY) ? __expf(fmaf(y[u], it, -mx)) : 0.f;
                            s += dpp_f32<kDppXor1>(s);
                            s += dpp_f32<kDppXor2>(s);
                            s += dpp_f32<kDppHalfMirror>(s);
                            if (live && (q4 & 7) == 0) {
                                const int parts = (N + kTileV - 1) / kTileV;
                                a.pm[(size_t)m * parts + n0 / kTileV] = mx;
                                a.ps[(size_t)m * parts + n0 / kTileV] = s;
                            }
                        }
                        if (live) {
                            if constexpr (EPI == kOutB16) {
                                uint16_t* out = static_cast<uint16_t*>(a.Y) + m * a.ldy + n0;
                                if (n0 + 4 <= N) {
                                    const uint2 v = pack_bf16x4(y[0], y[1], y[2], y[3]);
                                    *reinterpret_cast<u32x2_e2*>(out) = u32x2_e2{v.x, v.y};
                                } else {
                                    for (int u = 0; n0 + u < N; ++u) out[u] = f32_to_bf16_bits(y[u]);
                                }
                            } else {
                                float* out = static_cast<float*>(a.Y) + m * a.ldy + n0;
                                if (n0 + 4 <= N) {
                                    store_logits<true>(out, f32x4u{y[0], y[1], y[2], y[3]});
                                } else {
                                    for (int u = 0; n0 + u < N; ++u) out[u] = y[u];
                                }
                            }
                        }
                    }
                }
                lds_barrier();                                        // the patches may be written again
            }
        }
        if (!more) break;
    }
}

// ---------------------------------------------------------------- more than 64 rows: tiled
// Workgroup tile BM rows x BN columns x 128 bytes of K, eight waves, each a BM/2 x BN/4 block of 32x32 MFMA tiles with W as the row operand.
// Operands go from memory straight to LDS in SW stages of W and SH of X; a stage has rows of 128 bytes, row r with its
// 16-byte pieces in the order piece ^ (r % 8), which the lanes bring about by the address they load from.  One barrier per k-block, before the
// products of its last k-step: the next k-block's first fragments are read while those run.  Workgroups are numbered so that the row
// blocks that share a column block run back to back on one XCD (workgroup w goes to XCD w % 8): W comes from memory once.
// K past the last whole k-block: loads re-read its last 16 bytes, and X's fragments are zeroed there.
template <int BM, int BN, int SW, int SH, int EPI, bool PAST>
__global__ __launch_bounds__(kLinearThreads, 2) void k_linear_tile(LinearArgs a, int mblocks) {
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    constexpr int kStW = BN * kLine, kStX = BM * kLine;
    constexpr int TV = BN / 128, TM = BM / 64, WI = BN / 64, XI = BM / 64;
    constexpr uint32_t kNext = 8 * 8 * kLine;                         // LDS bytes from one of a wave's loads to its next
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int nn = lane & 31, half = lane >> 5;
    const int w = blockIdx.x, xcd = w & 7, slot = w >> 3;
    const int mb = slot % mblocks, nb = (slot / mblocks) * 8 + xcd;
    const int M = a.M, N = a.N, K = a.K, m0 = mb * BM, n0 = nb * BN;
    if (n0 >= N) return;                                              // uniform: padding workgroups of the last round of XCDs
    const int wm = wave >> 2, wn = wave & 3;
    const float my_sx = a.sx[min(m0 + (tid & (BM - 1)), M - 1)], my_sw = a.sw[min(n0 + (tid & (BN - 1)), N - 1)];      // used after the loop
    float my_temp = 1.f;
    if constexpr (EPI == kOutHead) my_temp = a.temperature[min(m0 + (tid & (BM - 1)), M - 1) / a.n];
    const int KB = (K + kLine - 1) / kLine, last_pieces = (K - (KB - 1) * kLine) / 16;
    const char* const wbase = reinterpret_cast<const char*>(a.W) + (size_t)n0 * K;
    const char* const xbase = reinterpret_cast<const char*>(a.X) + (size_t)m0 * a.ldx;
    uint32_t wo[WI], xo[XI], over;                                    // rows past the end re-read the last one
    {
        const int r = lane >> 3, piece = (lane & 7) ^ r;
#pragma unroll
        for (int i = 0; i < WI; ++i) wo[i] = (uint32_t)min((i * 8 + wave) * 8 + r, N - 1 - n0) * (uint32_t)K + piece * 16;
#pragma unroll
        for (int i = 0; i < XI; ++i) xo[i] = (uint32_t)min((i * 8 + wave) * 8 + r, M - 1 - m0) * a.ldx + piece * 16;
        over = (uint32_t)max(piece - (last_pieces - 1), 0) * 16u;
    }
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds + (uint32_t)wave * 8u * kLine;
    auto request = [&](const char* base, const auto& off, int kb, uint32_t to) {
        kb = min(kb, KB - 1);
        if (kb == KB - 1 && last_pieces < 8) {                        // uniform
            std::remove_cv_t<std::remove_reference_t<decltype(off)>> o;
#pragma unroll
            for (size_t i = 0; i < sizeof(o) / 4; ++i) o[i] = off[i] - over;
            dma_lines(base + (size_t)kb * kLine, o, to, kNext);
        } else {
            dma_lines(base + (size_t)kb * kLine, off, to, kNext);
        }
    };
    auto request_w = [&](int kb, int stage) { request(wbase, wo, kb, lds0 + (uint32_t)(stage * kStW)); };
    auto request_x = [&](int kb, int stage) { request(xbase, xo, kb, lds0 + (uint32_t)(SW * kStW + stage * kStX)); };

    i32x16 acc[TV][TM];
#pragma unroll
    for (int p = 0; p < TV; ++p)
#pragma unroll
        for (int b = 0; b < TM; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[p][b][r] = 0;
    const uint32_t wrow = (uint32_t)(wn * 32 * TV + nn) * kLine, xrow = (uint32_t)(SW * kStW) + (uint32_t)(wm * (BM / 2) + nn) * kLine, turn = (uint32_t)(nn & 7);
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
            const bool in = 2 * ks + half < last_pieces;
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
    unsigned char* const patch = lds + wave * 2 * kPatchBytes;
    const int lr = wm * (BM / 2), lc = wn * 32 * TV, rows = M - m0 - lr;                  // this wave's block of the tile
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
        const int parts = (N + kTileV - 1) / kTileV;
        if (n0 + BN > N) {                                            // uniform: the last column block
#pragma unroll
            for (int p = 0; p < TV; ++p)
#pragma unroll
                for (int b = 0; b < TM; ++b)
                    store_tile_32x32_t<PAST>(y[p][b], m0 + lr + b * 32, n0 + lc + p * 32, M, N, parts, s_invt - m0, L, a.pm, a.ps, patch);
            return;
        }
        store_full_tiles<PAST, TV, TM, kPT, kPS>(y, rows, s_invt + lr, s_part + lr * kPT + wn * TV, L + (size_t)(m0 + lr) * N + n0 + lc, N, patch);
        lds_barrier();
#pragma unroll
        for (int t = tid; t < 2 * BM * (kPT / 4); t += kLinearThreads) {
            const int q = t % (kPT / 4), row = t / (kPT / 4) % BM, arr = t / (kPT / 4) / BM;
            const f32x4 x = *reinterpret_cast<const f32x4*>(s_part + arr * kPS + row * kPT + 4 * q);
            if (m0 + row < M) *reinterpret_cast<f32x4u*>((arr == 0 ? a.pm : a.ps) + (size_t)(m0 + row) * parts + n0 / kTileV + 4 * q) = f32x4u(x);
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

template <int MT, int KS, int NT, int EPI, bool CH>
static hipError_t launch_stream_t(const ProfScope* prof, const LinearArgs& a, int kc, int most, hipStream_t s) {
    constexpr int VW = 8 / KS * 16 * NT;
    auto lds = [](int bytes) { return (size_t)MT * 16 * (bytes + 16) + 8 * (size_t)kPatchBytes; };
    static std::once_flag once[kMaxDevices];
    static hipError_t rc[kMaxDevices];
    const hipError_t e = raise_on_device(&k_linear_stream<MT, KS, NT, EPI, CH>, lds(most), once, rc);
    if (e != hipSuccess) return e;
    const int groups = (a.N + VW - 1) / VW;
    launch(prof, k_linear_stream<MT, KS, NT, EPI, CH>, dim3(std::min(groups, lds(kc) <= 80 * 1024 ? 512 : 256)), dim3(kLinearThreads), lds(kc), s, a, groups, kc);
    return hipGetLastError();
}

template <int MT, int KS, int NT, int EPI>
static hipError_t launch_stream_q8(const ProfScope* prof, const LinearArgs& a, hipStream_t s) {
    constexpr int granule = KS * 256 / NT, most = linear_chunk(MT) / granule * granule;
    static_assert(most > 0, "a chunk holds a step of every wave");
    const int kc = std::min(most, (a.K + granule - 1) / granule * granule);
    return a.K > kc ? launch_stream_t<MT, KS, NT, EPI, true>(prof, a, kc, most, s) : launch_stream_t<MT, KS, NT, EPI, false>(prof, a, kc, most, s);
}

// Waves that share a tile, and its width: as few and as wide as give most compute units a workgroup.
template <int MT, int EPI>
static hipError_t launch_stream_rows(const ProfScope* prof, const LinearArgs& a, hipStream_t s) {
    if (a.N > 192 * 128) return launch_stream_q8<MT, 2, 2, EPI>(prof, a, s);
    if (EPI == kOutHead || a.N > 192 * 64) return launch_stream_q8<MT, 4, 2, EPI>(prof, a, s);
    if constexpr (EPI != kOutHead) return launch_stream_q8<MT, 4, 1, EPI>(prof, a, s);
}

template <int BM, int BN, int SW, int SH, int EPI, bool PAST>
static hipError_t launch_tile_q8(const ProfScope* prof, const LinearArgs& a, hipStream_t s) {
    constexpr size_t lds = std::max((size_t)(SW * BN + SH * BM) * kLine, (size_t)16 * kPatchBytes + (2 * BM + BN) * 4 + 2 * BM * (BN / kTileV) * 4);
    static std::once_flag once[kMaxDevices];
    static hipError_t rc[kMaxDevices];
    const hipError_t e = raise_on_device(&k_linear_tile<BM, BN, SW, SH, EPI, PAST>, lds, once, rc);
    if (e != hipSuccess) return e;
    const int mblocks = (a.M + BM - 1) / BM, nblocks = (a.N + BN - 1) / BN, nrounds = (nblocks + 7) / 8;
    launch(prof, k_linear_tile<BM, BN, SW, SH, EPI, PAST>, dim3(nrounds * mblocks * 8), dim3(kLinearThreads), lds, s, a, mblocks);
    return hipGetLastError();
}

template <int EPI, bool PAST>
static hipError_t launch_tiles(const ProfScope* prof, const LinearArgs& a, hipStream_t s) {
    auto tiles = [&](int bm, int bn) { return (long)((a.M + bm - 1) / bm) * ((a.N + bn - 1) / bn); };
    if (a.M > 128 && (tiles(256, 256) >= 192 || tiles(128, 256) > 256)) return launch_tile_q8<256, 256, 3, 2, EPI, PAST>(prof, a, s);
    if (tiles(128, 256) >= 192) return launch_tile_q8<128, 256, 3, 3, EPI, PAST>(prof, a, s);
    if (tiles(128, 128) > 256) return launch_tile_q8<128, 128, 2, 2, EPI, PAST>(prof, a, s);
    return launch_tile_q8<128, 128, 4, 4, EPI, PAST>(prof, a, s);
}

template <int EPI>
static hipError_t launch_product(const ProfScope* prof, const LinearArgs& a, hipStream_t s) {
    if (a.M <= 16) return launch_stream_rows<1, EPI>(prof, a, s);
    if (a.M <= 32) return launch_stream_rows<2, EPI>(prof, a, s);
    if (a.M <= 64) return launch_stream_rows<4, EPI>(prof, a, s);
    if constexpr (EPI == kOutHead)
        if (!past_l2(a.N, a.K / 2, a.M)) return launch_tiles<EPI, false>(prof, a, s);
    return launch_tiles<EPI, EPI == kOutHead>(prof, a, s);
}

hipError_t launch_linear_q8(int M, int N, int K, const int8_t* X, int64_t ldx, const float* sx, const int8_t* W, const float* sw, int y_dtype,
                            void* Y, int64_t ldy, hipStream_t s) {
    const LinearArgs a{M, N, K, X, (uint32_t)ldx, sx, W, sw, Y, ldy, 1, nullptr, nullptr, nullptr};
    ProfScope prof(TABED_K_LMHEAD, s);
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
