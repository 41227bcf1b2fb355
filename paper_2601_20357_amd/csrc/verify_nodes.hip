// Verification of a tree of drafted tokens: multi-round rejection sampling from the root down, one launch.
//
// The walk is sequential: which node comes next follows from the rows of the one before it, and only the rows of the nodes on the way are
// read.  So that each of these steps has the chip's bandwidth all the same, a sequence's vocabulary is cut into pieces of 1024 or 2048, a workgroup
// each, which walk together: at a step every workgroup reduces its piece, stores what it found, reads what the others found, and comes to
// the same decision as they do from the same numbers in the same order.  A piece stays in registers: the target's row is read once at a node, the
// drafts' once for the distances and once more, out of a cache, where a child is rejected; f is kept from level to level.  The masses of the
// pieces, needed for the sum, are also the prefix in which the last draw is found.
//
// Decisions are in fp64: a draw among 10^5 tokens is decided by sums whose rounding in fp32 exceeds many tokens' probability.
//
// What crosses workgroups is stored past the caches in words of 32 bits of payload and 32 bits of the launch's number, so that a word says by
// itself whether it is this launch's: one trip, no order among stores needed.  Every step has a place of its own (at most N steps: each visits a node
// or rejects one).
//
// Why nothing waits for ever: workgroups are numbered as they start, sequence by sequence, so that a sequence's workgroups wait for ones that run already
// or start as soon as any other sequence, or another kernel, ends; launches on the four queues of a process each hold back less than one sequence's
// workgroups, at most 127 of the 768 that run at a time.  (More launches at a time, as of several processes, can fill the device with workgroups that wait: seven do for rows of
// 262144.  Nothing here can know of them; the caller keeps to a limit.)  A workspace that was never prepared, or for less, is known by a mark.  A wait has a bound of some seconds all
// the same, and what comes of a row is then settled by one word: whoever has all of the walk's records and whoever gives up set it, the first of them for all.  A row that was
// given up is left without a token, flagged, by its first workgroup; where it was not, who would have given up finds the records that it waited for.
//
// What bounds it: the steps, one after the other.  One is 4 to 5 us: 1 for the row's maximum and exponentials, 1.5 until all pieces' are known, 1 for their
// sum, the rest for the distances, the test and the next node's rows; a launch with one node and nothing to test takes 8 to 12, and settling what comes of the row half a us of any.  16
// sequences of 22 nodes, V = 32000, 4 drafts: 40 us (the longest path of 16 visits five nodes); 1 of 6, a path of four: 23 us.  64 sequences, V = 128256, 8 drafts, half of them
// greedy: 208 us for 480 MB and some 10^8 exponentials in 64 bits; 12 sequences run at a time, and while one waits for its pieces its workgroups request the first child's row only.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "nodes.h"
#include "nodes_launch.h"

namespace tabed {

constexpr int kVerThreads = 256, kVerWaves = kVerThreads / 64, kVerMaxPieces = 128;      // pieces are of 4 or 8 elements a thread
constexpr int kVerDraftsAtOnce = 4;
constexpr size_t kVerControl = 256;                                      // uint64: the launch's number and the next workgroup's; in the next line: mark, and what was prepared
constexpr uint32_t kVerMark = 0x7ab3d0deu;
constexpr int kVerSpins = 1 << 24;

struct VerifyArgs {
    int V, n, B, N, G, gamma, tvd;
    uint32_t units;                                                      // of 256 bytes of workspace
    int spins, late;                                                     // polls of a wait; for tests: a workgroup of every sequence that comes 3 ms late, -1: none
    uint64_t seed, round;
    const float* target;
    const float* drafts;
    const double* dlse;
    const int32_t* tokens;
    const float* node_q;
    const int32_t* parents;
    const int32_t* n_nodes;
    const float* weights;
    const float* temperature;
    const float* u_acc;
    const float* u_res;
    int32_t* path;
    int32_t* n_path;
    int32_t* out_tokens;
    uint8_t* flags;
    float* dev;
    int32_t* n_valid;
    uint64_t* ctl;
    uint64_t* rec;
    uint64_t* devrec;
    uint64_t* state;                                                     // [B] the launch's number, and what has come of the row
};
enum : uint32_t { kVerDone = 1, kVerGone = 2 };

__device__ __forceinline__ void say(uint64_t* p, uint32_t v, uint32_t launch) {
    __hip_atomic_store(p, (uint64_t)launch << 32 | v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint32_t lo32(double v) { return (uint32_t)__builtin_bit_cast(uint64_t, v); }
__device__ __forceinline__ uint32_t hi32(double v) { return (uint32_t)(__builtin_bit_cast(uint64_t, v) >> 32); }
__device__ __forceinline__ double from32(uint32_t lo, uint32_t hi) { return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo); }
__device__ __forceinline__ float as_float(uint32_t v) { return __builtin_bit_cast(float, v); }
// What comes of the row: `mine`, unless somebody settled it before.  The word holds the launch before this one, as a rule, or anything else that is not of this launch: a first try
// goes by that, and what it found is looked at when it is back.
__device__ __forceinline__ bool try_settle(uint64_t* state, uint64_t& seen, uint32_t mine, uint32_t launch) {
    return __hip_atomic_compare_exchange_strong(state, &seen, (uint64_t)launch << 32 | mine, __ATOMIC_RELAXED, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
struct Settling {
    uint64_t seen;
    bool won;
    __device__ __forceinline__ void begin(uint64_t* state, uint32_t mine, uint32_t launch) {
        seen = launch == 1 ? 0ull : (uint64_t)(launch - 1) << 32 | kVerDone;
        won = try_settle(state, seen, mine, launch);
    }
    __device__ __forceinline__ uint32_t end(uint64_t* state, uint32_t mine, uint32_t launch) {
        if (!won && (uint32_t)(seen >> 32) != launch) won = try_settle(state, seen, mine, launch);
        return won ? mine : (uint32_t)seen;
    }
};

// The word at p once it is this launch's; ok turns false where it does not come.
__device__ __forceinline__ uint32_t hear(const uint64_t* p, uint32_t launch, int spins, bool& ok) {
    for (int i = 0; i < spins; ++i) {
        const uint64_t w = __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if ((uint32_t)(w >> 32) == launch) return (uint32_t)w;
        if (i > 64) __builtin_amdgcn_s_sleep(1);
    }
    ok = false;
    return 0;
}
// A thread whose words did not come: the row is given up, unless somebody has all records of the walk; then they are there.  (A call, so that what never happens takes no
// registers from what does: within the loops above it cost 5 % of a large batch's time.)
__device__ __attribute__((noinline)) bool hear_or_give_up(const uint64_t* from, int words, uint32_t* to, uint32_t launch, uint64_t* state) {
    Settling settling;
    settling.begin(state, kVerGone, launch);
    if (settling.end(state, kVerGone, launch) != kVerDone) return false;
    bool ok = true;
    for (int w = threadIdx.x; w < words; w += kVerThreads) to[w] = hear(from + w, launch, kVerSpins, ok);
    return ok;
}

// e^x in 64 bits: x = n ln 2 + r, |r| <= ln 2 / 2, the series of e^r up to r^11 / 11! (what is left out is below 7e-15 of the result, ln 2's rounding
// takes n 2.4e-17), times 2^n.  A fifth of the instructions of the library's, which a rejection needs for every element of every draft.
__device__ __forceinline__ double exp64(double x) {
    x = x < -800.0 ? -800.0 : x;                                         // (-inf: 0; a NaN stays one)
    const double n = rint(x * 1.4426950408889634074), r = fma(n, -0.69314718055994530942, x);
    double p = 1.0 / 39916800.0;
    p = fma(p, r, 1.0 / 3628800.0);
    p = fma(p, r, 1.0 / 362880.0);
    p = fma(p, r, 1.0 / 40320.0);
    p = fma(p, r, 1.0 / 5040.0);
    p = fma(p, r, 1.0 / 720.0);
    p = fma(p, r, 1.0 / 120.0);
    p = fma(p, r, 1.0 / 24.0);
    p = fma(p, r, 1.0 / 6.0);
    p = fma(p, r, 0.5);
    p = fma(p, r, 1.0);
    p = fma(p, r, 1.0);
    return __builtin_amdgcn_ldexp(p, (int)n);
}

struct VerifyShared {
    int parent[TABED_MAX_NODES], token[TABED_MAX_NODES];
    float q[TABED_MAX_NODES], u[TABED_MAX_NODES];
    uint32_t rec[kVerMaxPieces][4];                                      // the step's records
    double p_mass[kVerMaxPieces], mass[kVerMaxPieces];                   // of the pieces: p at the node, f of the last level
    double red[kVerWaves][kVerDraftsAtOnce];
    float redf[kVerWaves];
    int redi[kVerWaves], redk[kVerWaves];
    int ticket, bad, done;
    uint32_t launch;
    float weight[TABED_MAX_N], dist[TABED_MAX_N];
    uint8_t flag[TABED_MAX_NODES];
    int path[TABED_MAX_NODES];
    int16_t at_step[TABED_MAX_NODES];                                    // of the path's nodes
};

// Sum over the workgroup, the same in all threads.
__device__ __forceinline__ double group_sum(double v, VerifyShared& s) {
    v = wave_sum(v);
    if ((threadIdx.x & 63) == 0) s.red[threadIdx.x >> 6][0] = v;
    lds_barrier();
    const double t = (s.red[0][0] + s.red[1][0]) + (s.red[2][0] + s.red[3][0]);
    lds_barrier();
    return t;
}

// The first child of `node` behind `after`, -1: none.  Uniform.
__device__ __forceinline__ int next_child(const VerifyShared& s, int node, int after, int count) {
    for (int j0 = after + 1; j0 < count; j0 += 64) {
        const int j = j0 + (threadIdx.x & 63);
        const uint64_t who = __ballot(j < count && s.parent[min(j, count - 1)] == node);
        if (who) return __builtin_amdgcn_readfirstlane(j0 + __ffsll((long long)who) - 1);
    }
    return -1;
}

// A workgroup's part of a row, in groups of four elements a thread.
template <int NG>
struct Piece {
    int v0[NG], at[NG];
};
template <bool SHORT, int NG>                                            // SHORT: rows of fewer than four elements
__device__ __forceinline__ void load_piece(const float* row, int V, const Piece<NG>& p, float4 (&x)[NG]) {
#pragma unroll
    for (int i = 0; i < NG; ++i) {
        if constexpr (SHORT) x[i] = load_short_row(row, p.at[i], V);
        else x[i] = load_group(row, p.at[i]);
    }
#pragma unroll
    for (int i = 0; i < NG; ++i) mask_group(x[i], p.at[i], p.v0[i]);     // (what belongs to other threads, or lies past the row: -inf)
}

template <bool SHORT, int NG>
__global__ __launch_bounds__(kVerThreads, 3) void k_verify_nodes(VerifyArgs a) {
    constexpr int kVerE = 4 * NG, kVerPiece = kVerThreads * kVerE;
    __shared__ VerifyShared s;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, V = a.V, n = a.n;
    if (tid == 0) {
        // One trip: the launch's number and this workgroup's.  The last one to come makes both ready for the next launch.
        const uint64_t known = __hip_atomic_load(a.ctl + 16, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const uint32_t mark = (uint32_t)known;
        const uint64_t got = __hip_atomic_fetch_add(a.ctl, 1ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const uint32_t launch = (uint32_t)(got >> 32), at = (uint32_t)got, count = (uint32_t)(a.B * a.G);
        if (mark == kVerMark && at == count - 1)
            __hip_atomic_store(a.ctl, (uint64_t)(launch == 0xffffffffu ? 1u : launch + 1) << 32, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        s.launch = launch;
        s.bad = 0;
        s.ticket = mark == kVerMark && (uint32_t)(known >> 32) >= a.units && at < count ? (int)at : -1;
    }
    lds_barrier();
    const uint32_t launch = __builtin_amdgcn_readfirstlane(s.launch);
    int ticket = __builtin_amdgcn_readfirstlane(s.ticket);
    const bool prepared = ticket >= 0;
    if (!prepared) ticket = blockIdx.x;
    const int b = ticket / a.G, c = ticket % a.G;
    if (c == a.late) {                                                   // (tests)
        const uint64_t began = __builtin_amdgcn_s_memrealtime();
        while (__builtin_amdgcn_s_memrealtime() - began < 300000) __builtin_amdgcn_s_sleep(8);
    }
    Piece<NG> piece;
#pragma unroll
    for (int i = 0; i < NG; ++i) {
        piece.v0[i] = c * kVerPiece + i * kVerThreads * 4 + tid * 4;
        piece.at[i] = group_at(min(piece.v0[i], V - 1), V);
    }
    float4 x[NG], ahead[NG];                                             // the node's row, and that of its first child
    load_piece<SHORT, NG>(a.target + (size_t)b * a.N * V, V, piece, ahead);
    const int count = nodes_of(a.n_nodes, b, a.N);
    const float T = a.temperature[b], u_res = a.u_res != nullptr ? a.u_res[b] : tabed_uniform(a.seed, a.round, (uint32_t)b, (uint32_t)(a.N - 1), 0);
    if (tid < n) s.weight[tid] = a.weights[(size_t)b * n + tid];
    if (tid < a.N) {
        const size_t j = (size_t)b * a.N + tid;
        s.parent[tid] = tid == 0 ? -1 : parent_of(a.parents, b, tid, a.N);
        s.token[tid] = a.tokens[j];
        s.q[tid] = a.node_q[j];
        s.u[tid] = a.u_acc != nullptr ? a.u_acc[j] : tabed_uniform(a.seed, a.round, (uint32_t)b, (uint32_t)(tid - 1), 1);
        s.flag[tid] = 0;
    }
    lds_barrier();
    const bool greedy = !(T > 0.f);
    const double inv_t = greedy ? 1.0 : 1.0 / (double)T;
    uint64_t* const state = a.state + b;
    uint64_t* const rec_b = a.rec + (size_t)b * a.N * a.G * 4;
    uint64_t* const dev_b = a.devrec + (size_t)b * a.gamma * a.G * n * 2;

    // A step's records, read by all into s.rec; false, for all, where one does not come and the row is given up.
    auto collect = [&](int step) {
        bool ok = true;
        const uint64_t* from = rec_b + (size_t)step * a.G * 4;
        for (int w = tid; w < a.G * 4; w += kVerThreads) s.rec[w / 4][w % 4] = hear(from + w, launch, a.spins, ok);
        if (__builtin_expect(!ok, 0)) ok = hear_or_give_up(from, a.G * 4, &s.rec[0][0], launch, state);
        if (!ok) s.bad = 1;                                              // (never taken back: who reads it behind the barrier reads it before the next)
        lds_barrier();
        return s.bad == 0;
    };
    auto publish = [&](int step, uint32_t w0, uint32_t w1, double z) {   // by one thread
        uint64_t* to = rec_b + ((size_t)step * a.G + c) * 4;
        say(to + 0, w0, launch);
        say(to + 1, w1, launch);
        say(to + 2, lo32(z), launch);
        say(to + 3, hi32(z), launch);
    };

    int cur = 0, depth = 0, step = 0, valid = 0, best = 0, level = 0;
    bool fine = prepared;
    double f[kVerE], q[kVerE], total = 0.0, scale = 0.0;                 // f times scale is p, at level 0
    float4 d[kVerDraftsAtOnce][NG];                                      // the rows of the node's first drafts
    double dl[kVerDraftsAtOnce];                                         // and their log-sum-exp
    auto load_drafts = [&](const float* drafts, const double* dlse, int j0) {
#pragma unroll
        for (int j = 0; j < kVerDraftsAtOnce; ++j) {
            load_piece<SHORT, NG>(drafts + (size_t)min(j0 + j, n - 1) * V, V, piece, d[j]);
            dl[j] = dlse[min(j0 + j, n - 1)];
        }
    };
    while (count > 0 && fine) {
        if (tid == 0) {
            s.path[depth] = cur;
            s.at_step[depth] = (int16_t)step;
        }
        int child = next_child(s, cur, cur, count);
        const int first = child;
        const bool want_dev = child >= 0 && a.dev != nullptr && depth < a.gamma;
        const float* const row = a.target + ((size_t)b * a.N + cur) * V;
        const float* const drafts = a.drafts + ((size_t)cur * a.B + b) * n * V;
        const double* const dlse = a.dlse + ((size_t)cur * a.B + b) * n;
#pragma unroll
        for (int i = 0; i < NG; ++i) x[i] = ahead[i];
        if (want_dev) load_drafts(drafts, dlse, 0);
        int y = child >= 0 ? s.token[child] : -1;
        const float ly = row[(unsigned)y < (unsigned)V ? y : 0];

        // ---- the piece's maximum, and the sum of exp
        ArgMax top{-INFINITY, 0x7fffffff};
#pragma unroll
        for (int i = 0; i < NG; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float v = f4get(x[i], e);
                if (v > top.v) top = ArgMax{v, piece.at[i] + e};         // (ascending within a thread)
            }
        top = wave_argmax(top);
        if (lane == 0) { s.redf[wave] = top.v; s.redi[wave] = top.i; }
        lds_barrier();
        top = argmax_merge(argmax_merge(ArgMax{s.redf[0], s.redi[0]}, ArgMax{s.redf[1], s.redi[1]}),
                           argmax_merge(ArgMax{s.redf[2], s.redi[2]}, ArgMax{s.redf[3], s.redi[3]}));
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < NG; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float v = f4get(x[i], e);
                f[i * 4 + e] = v == -INFINITY ? 0.0 : exp64(((double)v - (double)top.v) * inv_t);
                sum += f[i * 4 + e];
            }
        sum = group_sum(sum, s);
        if (tid == 0) publish(step, __builtin_bit_cast(uint32_t, top.v), (uint32_t)top.i, sum);
        if (first >= 0) load_piece<SHORT, NG>(a.target + ((size_t)b * a.N + first) * V, V, piece, ahead);      // (on its way while the others are waited for)

        if (want_dev) {
            // KL: the piece's sum of exp * ((l - max) / T - log q_j); TVD: of |p - q_j|.  Added up when the walk is over.
            if (!a.tvd) {
                for (int j0 = 0; j0 < n; j0 += kVerDraftsAtOnce) {
                    if (j0 > 0) load_drafts(drafts, dlse, j0);
#pragma unroll
                    for (int j = 0; j < kVerDraftsAtOnce; ++j) {
                        double kl = 0.0;
#pragma unroll
                        for (int i = 0; i < NG; ++i)
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const double w = f[i * 4 + e];
                                const double t = ((double)f4get(x[i], e) - (double)top.v - (double)f4get(d[j][i], e)) * inv_t + dl[j];
                                kl += w == 0.0 ? 0.0 : w * t;
                            }
                        kl = wave_sum(kl);
                        if (lane == 0) s.red[wave][j] = kl;
                    }
                    lds_barrier();
                    if (tid < kVerDraftsAtOnce && j0 + tid < n) {
                        const double kl = (s.red[0][tid] + s.red[1][tid]) + (s.red[2][tid] + s.red[3][tid]);
                        uint64_t* to = dev_b + (((size_t)depth * a.G + c) * n + j0 + tid) * 2;
                        say(to, lo32(kl), launch);
                        say(to + 1, hi32(kl), launch);
                    }
                    lds_barrier();
                }
            }
        }
        // ---- all pieces: maximum, arg-max, sum
        fine = collect(step);
        if (!fine) break;
        ++step;
        ArgMax all{-INFINITY, 0x7fffffff};
        for (int g = lane; g < a.G; g += 64) all = argmax_merge(all, ArgMax{as_float(s.rec[g][0]), (int)s.rec[g][1]});
        all = wave_argmax(all);
        double z = 0.0;
        for (int g = lane; g < a.G; g += 64) {
            const float mg = as_float(s.rec[g][0]);
            const double w = (mg == -INFINITY ? 0.0 : exp64(((double)mg - (double)all.v) * inv_t)) * from32(s.rec[g][2], s.rec[g][3]);      // (a NaN among -inf stays one)
            z += w;
            if (wave == 0) s.p_mass[g] = w;                              // (times 1 / z below)
        }
        const double inv_z = 1.0 / wave_sum(z);
        if (wave == 0)
            for (int g = lane; g < a.G; g += 64) s.p_mass[g] *= inv_z;
        best = all.i < V ? all.i : 0;                                    // (a row of -inf and NaN: 0)
        scale = top.v == -INFINITY ? 0.0 : exp64(((double)top.v - (double)all.v) * inv_t) * inv_z;

        if (want_dev) {
            valid = depth + 1;
            if (a.tvd) {
                for (int j = 0; j < n; ++j) {
                    float4 dj[NG];
                    load_piece<SHORT, NG>(drafts + (size_t)j * V, V, piece, dj);
                    const double lse = dlse[j];
                    double tv = 0.0;
#pragma unroll
                    for (int i = 0; i < NG; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) tv += fabs(f[i * 4 + e] * scale - exp64((double)f4get(dj[i], e) * inv_t - lse));
                    tv = group_sum(tv, s);
                    if (tid == 0) {
                        uint64_t* to = dev_b + (((size_t)depth * a.G + c) * n + j) * 2;
                        say(to, lo32(tv), launch);
                        say(to + 1, hi32(tv), launch);
                    }
                }
            }
        }
        lds_barrier();                                                 // p_mass is whole, s.rec has been read

        // ---- the children, in order
        level = 0;
        total = 1.0;
        double fy = (unsigned)y < (unsigned)V ? exp64(((double)ly - (double)all.v) * inv_t) * inv_z : 0.0;
        int hit = -1;
        while (child >= 0) {
            const bool there = (unsigned)y < (unsigned)V;
            uint8_t flag = there ? 0 : TABED_FLAG_DEGENERATE;
            bool yes = there && y == best;
            if (!greedy) {
                const double want = (double)s.u[child] * (double)s.q[child] * total;
                yes = there && want < fy;
                if (there && fabs(want - fy) < (double)kMargin * fmax(want, fy)) flag |= TABED_FLAG_ACCEPT_MARGIN;
            }
            if (c == 0 && tid == 0) s.flag[child] = flag;
            if (yes) {
                hit = child;
                break;
            }
            child = next_child(s, cur, child, count);
            y = child >= 0 ? s.token[child] : -1;
            if (greedy) continue;
            if (level == 0) {
#pragma unroll
                for (int e = 0; e < kVerE; ++e) {
                    f[e] *= scale;
                    q[e] = 0.0;
                }
                for (int j0 = 0; j0 < n; j0 += kVerDraftsAtOnce) {
                    if (!want_dev || n > kVerDraftsAtOnce) load_drafts(drafts, dlse, j0);
#pragma unroll
                    for (int j = 0; j < kVerDraftsAtOnce; ++j) {
                        if (j0 + j >= n) break;
                        const double w = (double)s.weight[j0 + j];
#pragma unroll
                        for (int i = 0; i < NG; ++i)
#pragma unroll
                            for (int e = 0; e < 4; ++e) q[i * 4 + e] += w * exp64((double)f4get(d[j][i], e) * inv_t - dl[j]);
                    }
                }
            }
            const double inv = total > 0.0 ? 1.0 / total : 0.0;
            double zsum = 0.0, fn = 0.0;
#pragma unroll
            for (int i = 0; i < NG; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    double& fe = f[i * 4 + e];
                    fe = fmax(0.0, fe * inv - q[i * 4 + e]);
                    zsum += fe;
                    if (piece.at[i] + e == y) fn += fe;                  // (an element that is another thread's is 0 here)
                }
            zsum = wave_sum(zsum);
            fn = wave_sum(fn);
            if (lane == 0) { s.red[wave][0] = zsum; s.red[wave][1] = fn; }
            lds_barrier();
            if (tid == 0) {
                const double ft = (s.red[0][1] + s.red[1][1]) + (s.red[2][1] + s.red[3][1]);
                publish(step, lo32(ft), hi32(ft), (s.red[0][0] + s.red[1][0]) + (s.red[2][0] + s.red[3][0]));
            }
            fine = collect(step);
            if (!fine) break;
            ++step;
            ++level;
            double zt = 0.0;
            for (int g = lane; g < a.G; g += 64) {
                const double zg = from32(s.rec[g][2], s.rec[g][3]);
                zt += zg;
                if (wave == 0) s.mass[g] = zg;
            }
            total = wave_sum(zt);
            fy = 0.0;
            if ((unsigned)y < (unsigned)V) fy = from32(s.rec[y / kVerPiece][0], s.rec[y / kVerPiece][1]);
            lds_barrier();                                             // mass is whole, s.rec has been read
        }
        if (!fine || hit < 0) break;
        if (hit != first) load_piece<SHORT, NG>(a.target + ((size_t)b * a.N + hit) * V, V, piece, ahead);
        cur = hit;
        ++depth;
    }

    // ---- the last draw: the piece that it falls into by the masses, in it the token
    bool settles = c == 0 || c < valid;                                  // those that write anything
    Settling settling{};                                                 // (thread 0; on its way while the token is looked for)
    int token = -1;                                                      // the thread that found it, and what is flagged
    uint8_t token_flag = 0;
    if (count > 0 && fine && !greedy) {
        const bool gone = level > 0 && !(total > 0.0);                   // nothing is left of f: p again
        if (gone) {
            float m = -INFINITY;
#pragma unroll
            for (int i = 0; i < NG; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) m = fmaxf(m, f4get(x[i], e));
            m = block_max(m, s.redf);
#pragma unroll
            for (int i = 0; i < NG; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float v = f4get(x[i], e);
                    f[i * 4 + e] = v == -INFINITY ? 0.0 : exp64(((double)v - (double)m) * inv_t) * scale;
                }
        } else if (level == 0) {
#pragma unroll
            for (int e = 0; e < kVerE; ++e) f[e] *= scale;
        }
        const double* const mass = level == 0 || gone ? s.p_mass : s.mass;
        // Every wave of every workgroup the same: the first piece in which the prefix exceeds u Z, else the last with any mass, else the first.
        double whole = 0.0;
        for (int g0 = 0; g0 < a.G; g0 += 64) whole += wave_sum(g0 + lane < a.G ? mass[g0 + lane] : 0.0);
        const double goal = (double)u_res * whole;
        double run = 0.0, before = 0.0;
        int owner = 0;
        bool crossed = false;
        for (int g0 = 0; g0 < a.G && !crossed; g0 += 64) {
            const double mg = g0 + lane < a.G ? mass[g0 + lane] : 0.0;
            const double incl = run + wave_inclusive_scan(mg);
            const uint64_t over = __ballot(mg > 0.0 && incl > goal), some = __ballot(mg > 0.0);
            const int at = over ? __ffsll((long long)over) - 1 : some ? 63 - __clzll((long long)some) : -1;
            if (at >= 0) {
                owner = g0 + at;
                before = lane_f64(incl, at) - lane_f64(mg, at);
            }
            crossed = over != 0;
            run = lane_f64(incl, 63);
        }
        settles = settles || c == owner;
        if (settles && tid == 0) settling.begin(state, kVerDone, launch);
        if (c == owner) {
            int first = 0x7fffffff, last = -1;
            double lo[kVerE];
            for (int i = 0; i < NG; ++i) {                                // (the groups one after the other: the order of the row)
                double part, at = 0.0;
#pragma unroll
                for (int e = 0; e < 4; ++e) at += f[i * 4 + e];
                at = before + block_exclusive_scan(at, &s.red[0][0], &part);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const double fe = f[i * 4 + e];
                    lo[i * 4 + e] = at;
                    at += fe;
                    if (fe > 0.0) {
                        last = piece.at[i] + e;
                        if (at > goal) first = min(first, last);
                    }
                }
                before += part;
            }
            const int pick = block_pick_key(first, last, s.redi, s.redk);
            uint8_t flag = (crossed ? 0 : TABED_FLAG_DEGENERATE) | (gone ? TABED_FLAG_DEGENERATE : 0);
#pragma unroll
            for (int i = 0; i < NG; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (f[i * 4 + e] > 0.0 && piece.at[i] + e == pick) {
                        const double l = lo[i * 4 + e], h = l + f[i * 4 + e];
                        if (fmin(fabs(h - goal), fabs(goal - l)) < (double)kMargin * whole) flag |= TABED_FLAG_SAMPLE_MARGIN;
                        token = pick;
                        token_flag = flag;
                    }
            if (pick < 0 && tid == 0) {                                  // no element has any mass (NaN)
                token = 0;
                token_flag = TABED_FLAG_DEGENERATE;
            }
        }
    } else if (count > 0 && fine && settles && tid == 0) {
        settling.begin(state, kVerDone, launch);
    }

    // ---- the verdict, once it is back
    bool open = settles && count > 0 && fine;
    auto verdict = [&] {
        if (tid == 0) s.done = settling.end(state, kVerDone, launch) == kVerDone;
        lds_barrier();
        fine = s.done != 0;
        open = false;
    };
    if (open && (a.tvd || c >= valid)) verdict();

    // ---- the distances: the positions are dealt to the workgroups, a wave adds up a draft's.  (KL: what is added up is said by all that have come to the position, also by those that
    // give up there, so that the first position need not wait for the verdict.)
    for (int i = c; i < valid && fine; i += a.G) {
        const uint64_t* const from = rec_b + (size_t)s.at_step[i] * a.G * 4;
        for (int j = wave; j < n; j += kVerWaves) {
            bool ok = true;
            float m[2] = {-INFINITY, -INFINITY};
            double sum[2] = {0.0, 0.0}, part[2] = {0.0, 0.0};
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int g = h * 64 + lane;
                if (g >= a.G) continue;
                const uint64_t* const dev = dev_b + (((size_t)i * a.G + g) * n + j) * 2;
                m[h] = as_float(hear(from + g * 4, launch, kVerSpins, ok));
                sum[h] = from32(hear(from + g * 4 + 2, launch, kVerSpins, ok), hear(from + g * 4 + 3, launch, kVerSpins, ok));
                part[h] = from32(hear(dev, launch, kVerSpins, ok), hear(dev + 1, launch, kVerSpins, ok));
            }
            const float top = wave_max(fmaxf(m[0], m[1]));
            double z = 0.0, t = 0.0;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const double up = ((double)m[h] - (double)top) * inv_t;
                if (a.tvd) t += part[h];
                else if (m[h] == -INFINITY) {
                    z += 0.0 * sum[h];
                } else {
                    const double w = exp64(up);
                    z += w * sum[h];
                    t += w * (part[h] + up * sum[h]);
                }
            }
            z = wave_sum(z);
            t = wave_sum(t);
            const bool all = __all(ok);
            if (lane == 0) s.dist[j] = all ? (float)(a.tvd ? 0.5 * t : t / z - log(z)) : __builtin_nanf("");
        }
        if (open) verdict();
        lds_barrier();
        if (tid < n && fine) a.dev[((size_t)b * a.gamma + i) * n + tid] = s.dist[tid];
        lds_barrier();
    }
    if (token >= 0 && fine) {
        a.out_tokens[(size_t)b * a.N + depth] = token;
        a.flags[(size_t)b * a.N] = token_flag;
    }

    // ---- the first workgroup tells the way
    if (c == 0) {
        lds_barrier();
        const int said = count > 0 && fine ? depth + 1 : 0;              // nodes of the path
        if (tid < a.N) {
            const size_t at = (size_t)b * a.N + tid;
            a.path[at] = tid < said ? s.path[tid] : -1;
            if (tid + 1 != said) a.out_tokens[at] = tid + 1 < said ? s.token[s.path[tid + 1]] : -1;
            else if (greedy) a.out_tokens[at] = best;
            if (tid > 0) a.flags[at] = said > 0 ? s.flag[tid] : 0;
            else if (said == 0 || greedy) a.flags[at] = fine ? 0 : TABED_FLAG_DEGENERATE;
        }
        if (tid == 0) {
            a.n_path[b] = said;
            if (a.n_valid != nullptr) a.n_valid[b] = said > 0 ? valid : 0;
        }
    }
}

// Elements of a workgroup's piece: 4 or 8 a thread.  Small pieces end each step sooner as long as a lane polls one workgroup's record and the chip
// has room (rows of 32000: 1 sequence 23.2 us against 25.9, 8 sequences 36.7 against 38.1), and then cost more than they give (16 sequences 42.8
// against 40.6; 1 sequence of 128256 19.4 against 18.5; 4 of them 46.6 against 38.9).
constexpr int kVerSmallGroups = 256;                                     // workgroups of a launch
static int piece_of(const tabed_cfg& c) {
    constexpr int small = kVerThreads * 4;
    const int pieces = (c.V + small - 1) / small;
    return pieces <= 64 && (int64_t)c.B * pieces <= kVerSmallGroups ? small : kVerThreads * 8;
}
NodesVerifyLayout nodes_verify_layout(const tabed_cfg& c, int N) {
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    NodesVerifyLayout L;
    L.G = (c.V + piece_of(c) - 1) / piece_of(c);
    const size_t groups = std::max<size_t>((size_t)c.B * ((c.V + kVerThreads * 8 - 1) / (kVerThreads * 8)), kVerSmallGroups);
    L.off_rec = kVerControl;                                             // (never less for more sequences or longer rows, whatever their pieces)
    L.off_dev = L.off_rec + up(groups * N * 4 * 8);
    L.off_state = L.off_dev + up(groups * c.gamma * c.n * 2 * 8);
    L.total = L.off_state + up((size_t)c.B * 8);
    return L;
}

__global__ void k_verify_nodes_init(uint32_t* ws, size_t words) {
    for (size_t i = blockIdx.x * (size_t)blockDim.x + threadIdx.x; i < words; i += (size_t)gridDim.x * blockDim.x)
        ws[i] = i == 1 ? 1u : i == 32 ? kVerMark : i == 33 ? (uint32_t)(words / 64) : 0u;      // (launch 1, workgroup 0)
}
hipError_t launch_nodes_verify_init(const tabed_cfg& c, int N, char* ws, hipStream_t s) {
    const size_t words = nodes_verify_layout(c, N).total / 4;
    hipLaunchKernelGGL(k_verify_nodes_init, dim3((unsigned)std::min<size_t>((words + 255) / 256, 2048)), dim3(256), 0, s, reinterpret_cast<uint32_t*>(ws), words);
    return hipGetLastError();
}

hipError_t launch_verify_nodes(const tabed_cfg& c, char* ws, uint64_t round, int N, const float* target_logits, const float* draft_logits,
                               const double* draft_lse, const int32_t* tokens, const float* node_q, const int32_t* parents, const int32_t* n_nodes,
                               const float* weights, const float* temperature, const float* u_acc, const float* u_res, int32_t* path, int32_t* n_path,
                               int32_t* out_tokens, uint8_t* flags, float* dev, int32_t* n_valid, hipStream_t s, int spins, int late) {
    ProfScope prof(TABED_K_TREE, s);
    const NodesVerifyLayout L = nodes_verify_layout(c, N);
    const VerifyArgs a{c.V, c.n, c.B, N, L.G, c.gamma, c.distance == 1, (uint32_t)(L.total / 256), spins > 0 ? spins : kVerSpins, late, c.seed, round, target_logits, draft_logits, draft_lse, tokens, node_q, parents,
                       n_nodes, weights, temperature, u_acc, u_res, path, n_path, out_tokens, flags, dev, n_valid, reinterpret_cast<uint64_t*>(ws),
                       reinterpret_cast<uint64_t*>(ws + L.off_rec), reinterpret_cast<uint64_t*>(ws + L.off_dev), reinterpret_cast<uint64_t*>(ws + L.off_state)};
    const dim3 grid((unsigned)(c.B * L.G)), block(kVerThreads);
    if (c.V < 4) launch(&prof, k_verify_nodes<true, 1>, grid, block, 0, s, a);
    else if (piece_of(c) == kVerThreads * 4) launch(&prof, k_verify_nodes<false, 1>, grid, block, 0, s, a);
    else launch(&prof, k_verify_nodes<false, 2>, grid, block, 0, s, a);
    return hipGetLastError();
}

}  // namespace tabed
