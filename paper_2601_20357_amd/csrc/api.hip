// C ABI of the TABED hot path (see include/tabed.h): argument validation on the host, workspace
// layout, launch sequencing, optional per-kernel event timing.  No allocation, no synchronisation,
// except inside the tabed_prof_* calls.
#include <atomic>
#include <cmath>
#include <mutex>
#include <vector>

#include "internal.h"
#include "nodes_launch.h"

namespace tabed {

static thread_local int g_last_hip_error = 0;

static size_t align_up(size_t x, size_t a = 256) { return (x + a - 1) / a * a; }

int validate_cfg(const tabed_cfg* c) {
    if (c == nullptr) return TABED_ENULL;
    if (c->V < 1 || c->d < 1 || c->B < 1 || c->h < 0 || c->n < 1 || c->gamma < 1) return TABED_EINVAL;
    if (c->n > TABED_MAX_N || c->gamma > TABED_MAX_GAMMA) return TABED_ERANGE;
    if (c->w_dtype != 0 && c->w_dtype != 1) return TABED_EINVAL;
    if (c->w_dtype == 1 && (c->d % 8) != 0) return TABED_EINVAL;
    if (c->distance < 0 || c->distance > 2) return TABED_EINVAL;
    if (c->policy < 0 || c->policy > 3) return TABED_EINVAL;
    if (c->policy == 2 && c->n != 2) return TABED_EINVAL;
    if (!(c->tau_w > 0.f) || !(c->eps > 0.f)) return TABED_EINVAL;
    if (c->B > 65535 || (long long)c->B * c->n > (1ll << 24)) return TABED_ERANGE;   // B is a grid dimension
    if (c->V > kTileV * kBlock * 32) return TABED_ERANGE;      // 262144: largest vocabulary the sampler tiles
    return TABED_OK;
}

static WsLayout layout_with(const tabed_cfg& c, int ticket_stride) {
    WsLayout L;
    L.TS = ticket_stride;
    L.M = c.n * c.B;
    L.NT = (c.V + kTileV - 1) / kTileV;
    L.C2 = (c.V + kChunkV - 1) / kChunkV;
    if (L.C2 > kMaxGreedyChunks) L.C2 = kMaxGreedyChunks;
    L.C3max = (c.V + kBlock * 4 - 1) / (kBlock * 4);
    L.NSEG = (c.V + kSegV - 1) / kSegV;
    L.C5 = (c.V + kResidChunkV - 1) / kResidChunkV;
    L.RS = kStatHdr + ((c.policy == 2 && TABED_GRID_CANDIDATES > c.n) ? TABED_GRID_CANDIDATES : c.n);   // A sums: per draft, or per mixture
    L.DW = (c.policy == 2) ? TABED_GRID_CANDIDATES : c.n;
    L.Cd = (c.V + kChunkV - 1) / kChunkV;
    size_t off = 0;
    L.off_tickets = off; off = align_up(off + sizeof(uint32_t) * 5 * (size_t)c.B * L.TS);
    L.off_pm = off;      off = align_up(off + sizeof(float) * (size_t)L.M * L.NT);
    L.off_ps = off;      off = align_up(off + sizeof(float) * (size_t)L.M * L.NT);
    L.off_cand = off;    off = align_up(off + sizeof(Top2Rec) * (size_t)c.B * L.C2);
    L.off_stats = off;   off = align_up(off + sizeof(double) * (size_t)c.B * (c.gamma + 1) * L.C3max * L.RS);
    L.off_seg = off;     off = align_up(off + sizeof(double) * 2 * (size_t)c.B * L.NSEG);
    L.off_wstage = off;  off = align_up(off + sizeof(float) * (size_t)c.B * c.n);
    L.off_dist = off;    off = align_up(off + sizeof(double) * 2 * (size_t)c.B * c.gamma * L.DW * L.Cd);
    L.off_tstate = off;  off = align_up(off + sizeof(double) * kTsSlots * (size_t)c.B);
    L.off_tseg = off;    off = align_up(off + sizeof(double) * 2 * (size_t)c.B * L.NSEG);
    L.total = off;
    return L;
}

// Every sequence's counters have a 128-byte line of their own: atomics on one line are carried out one after the other at
// the memory side, and 600 workgroups of 8 sequences took 4 us to arrive on one.  Where only that would lift a
// configuration over what the built-in scratch holds, the counters stay packed.
WsLayout ws_layout(const tabed_cfg& c) {
    const WsLayout L = layout_with(c, 32);
    if (L.total <= (size_t)TABED_STATIC_SCRATCH_BYTES) return L;
    const WsLayout packed = layout_with(c, 1);
    return packed.total <= (size_t)TABED_STATIC_SCRATCH_BYTES ? packed : L;
}

size_t ws_bytes_unpacked(const tabed_cfg& c) { return layout_with(c, 32).total; }

// ---------------------------------------------------------------- event timing
struct ProfRec {
    int id, also;
    hipEvent_t start, stop;
};
static std::mutex g_prof_mu;
static std::atomic<bool> g_prof_on{false};
static std::vector<ProfRec> g_prof_pending;
static double g_prof_ms[TABED_K_COUNT];
static int64_t g_prof_n[TABED_K_COUNT];

bool prof_on() { return g_prof_on.load(std::memory_order_relaxed); }
void prof_push(int id, int also, hipEvent_t start, hipEvent_t stop) {
    std::lock_guard<std::mutex> lk(g_prof_mu);
    g_prof_pending.push_back(ProfRec{id, also, start, stop});
}
static void prof_drain() {
    for (ProfRec& r : g_prof_pending) {
        float ms = 0.f;
        if (hipEventSynchronize(r.stop) == hipSuccess && hipEventElapsedTime(&ms, r.start, r.stop) == hipSuccess) {
            for (int id : {r.id, r.also})
                if (id >= 0) {
                    g_prof_ms[id] += (double)ms;
                    g_prof_n[id] += 1;
                }
        }
        (void)hipEventDestroy(r.start);
        (void)hipEventDestroy(r.stop);
    }
    g_prof_pending.clear();
}

static int fail_hip(hipError_t e) {
    g_last_hip_error = (int)e;
    return TABED_EHIP;
}
static bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }
static bool storage_type(int32_t t) { return t == 0 || t == 1; }
static bool element_misaligned(const void* p, int32_t type) { return (reinterpret_cast<uintptr_t>(p) & (type == 1 ? 1u : 3u)) != 0; }
constexpr int64_t kMaxWorkgroups = (1 << 23) - 1;      // of the 8-bit cache's launches, up to 2^9 threads each: a grid has fewer than 2^32

static int validate_cache(const tabed_cache_q8* c, bool pointers) {
    if (c == nullptr) return TABED_ENULL;
    if (c->kv_heads < 1 || c->kv_heads > 1024 || c->blocks < 1 || c->max_blocks < 1 || c->max_blocks > (1 << 24)) return TABED_ERANGE;
    if (c->head_dim != 32 && c->head_dim != 64 && c->head_dim != 96 && c->head_dim != 128 && c->head_dim != 256) return TABED_EINVAL;
    if (!pointers) return TABED_OK;
    if (!c->k || !c->v || !c->kscale || !c->vscale || !c->table) return TABED_ENULL;
    if (misaligned(c->k) || misaligned(c->v) || element_misaligned(c->kscale, 0) || element_misaligned(c->vscale, 0) || element_misaligned(c->table, 0))
        return TABED_EALIGN;
    return TABED_OK;
}

static int validate_paged(const tabed_cache_paged* c, bool pointers) {
    if (c == nullptr) return TABED_ENULL;
    if (c->layers < 1 || c->layers > 1024 || c->kv_heads < 1 || c->kv_heads > 1024 || c->blocks < 1 || c->max_blocks < 1 || c->max_blocks > (1 << 24))
        return TABED_ERANGE;
    if (c->head_dim != 32 && c->head_dim != 64 && c->head_dim != 96 && c->head_dim != 128 && c->head_dim != 256) return TABED_EINVAL;
    if (c->type != 1 && c->type != 2) return TABED_EINVAL;
    const int64_t piece = c->type == 2 ? 16 : 8;
    for (int64_t stride : {c->layer_stride, c->block_stride, c->head_stride, c->tok_stride})
        if (stride < c->head_dim || stride % piece != 0 || stride > (1ll << 44)) return TABED_EINVAL;
    if (c->tok_stride > (1 << 24)) return TABED_EINVAL;
    if (!pointers) return TABED_OK;
    if (!c->k || !c->v || !c->table || (c->type == 2 && (!c->kscale || !c->vscale))) return TABED_ENULL;
    if (misaligned(c->k) || misaligned(c->v) || element_misaligned(c->table, 0)) return TABED_EALIGN;
    if (c->type == 2 && (element_misaligned(c->kscale, 0) || element_misaligned(c->vscale, 0))) return TABED_EALIGN;
    return TABED_OK;
}

// ---------------------------------------------------------------- built-in scratch of tabed_draft_step_static
// One array per GPU, part of the loaded code object, so no call ever allocates it.  `scratch` is only a
// host-side handle: the array's device address on the current GPU comes from hipGetSymbolAddress, looked up once
// per device, and that pointer is what kernels and launchers receive.
static __device__ __attribute__((used)) __align__(256) unsigned char scratch[TABED_STATIC_SCRATCH_BYTES];
static std::mutex g_scratch_mu;
static void* g_scratch_ptr[kMaxDevices];

static int static_scratch(char** out) {
    int dev = -1;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return fail_hip(e);
    if (dev < 0 || dev >= kMaxDevices) return TABED_ERANGE;
    std::lock_guard<std::mutex> lk(g_scratch_mu);
    if (g_scratch_ptr[dev] == nullptr) {
        void* p = nullptr;
        e = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch));
        if (e != hipSuccess) return fail_hip(e);
        if (p == nullptr) return fail_hip(hipErrorInvalidSymbol);
        g_scratch_ptr[dev] = p;
    }
    *out = static_cast<char*>(g_scratch_ptr[dev]);
    return TABED_OK;
}

}  // namespace tabed

using namespace tabed;

extern "C" {

int32_t tabed_dev_width(const tabed_cfg* cfg) {
    if (validate_cfg(cfg) != TABED_OK) return 0;
    return ws_layout(*cfg).DW;
}

size_t tabed_workspace_bytes(const tabed_cfg* cfg) {
    if (validate_cfg(cfg) != TABED_OK) return 0;
    return ws_layout(*cfg).total;
}

int tabed_workspace_init(const tabed_cfg* cfg, void* ws, void* stream) {
    const int rc = validate_cfg(cfg);
    if (rc != TABED_OK) return rc;
    if (ws == nullptr) return TABED_ENULL;
    if (misaligned(ws)) return TABED_EALIGN;
    const hipError_t e = launch_ws_init(*cfg, ws_layout(*cfg), static_cast<char*>(ws), static_cast<hipStream_t>(stream));
    return e == hipSuccess ? TABED_OK : fail_hip(e);
}

const char* tabed_strerror(int code) {
    switch (code) {
        case TABED_OK: return "ok";
        case TABED_ENULL: return "a required pointer is NULL";
        case TABED_EINVAL: return "a configuration field is out of range";
        case TABED_ERANGE: return "an index or count exceeds the supported range";
        case TABED_EALIGN: return "a base pointer is not 16-byte aligned";
        case TABED_EUNSUPPORTED: return "valid request that this build does not implement";
        case TABED_EHIP: return "a kernel launch failed";
        case TABED_ETOOBIG: return "the configuration needs more scratch than the built-in buffer holds";
        default: return "unknown error code";
    }
}

int tabed_last_hip_error(void) { return g_last_hip_error; }

int tabed_draft_step(const tabed_cfg* cfg, void* ws, uint64_t round, int32_t pos, const void* W, const void* H,
                     const float* weights, const float* temperature, const float* u_draft, float* draft_logits,
                     double* draft_lse, int32_t* draft_tokens, float* draft_q, uint8_t* flags, void* stream) {
    const int rc = validate_cfg(cfg);
    if (rc != TABED_OK) return rc;
    if (!ws || !W || !H || !weights || !temperature || !draft_logits || !draft_lse || !draft_tokens || !draft_q || !flags)
        return TABED_ENULL;
    if (pos < 0 || pos >= cfg->gamma) return TABED_ERANGE;
    if (misaligned(ws) || misaligned(W) || misaligned(H) || misaligned(draft_logits) || misaligned(draft_lse))
        return TABED_EALIGN;
    const WsLayout L = ws_layout(*cfg);
    hipStream_t s = static_cast<hipStream_t>(stream);
    float* slot = draft_logits + (size_t)pos * L.M * cfg->V;
    hipError_t e = launch_lmhead(*cfg, L, static_cast<char*>(ws), W, H, temperature, slot, s);
    if (e != hipSuccess) return fail_hip(e);
    e = launch_sample(*cfg, L, static_cast<char*>(ws), round, pos, slot, weights, temperature, u_draft, draft_lse,
                      draft_tokens, draft_q, flags, s);
    return e == hipSuccess ? TABED_OK : fail_hip(e);
}

int tabed_draft_step_static(const tabed_cfg* cfg, uint64_t round, int32_t pos, const void* W, const void* H,
                            const float* weights, const float* temperature, const float* u_draft,
                            float* draft_logits, double* draft_lse, int32_t* draft_tokens, float* draft_q,
                            uint8_t* flags, void* stream) {
    const int rc = validate_cfg(cfg);
    if (rc != TABED_OK) return rc;
    if (!W || !H || !weights || !temperature || !draft_logits || !draft_lse || !draft_tokens || !draft_q || !flags)
        return TABED_ENULL;
    if (pos < 0 || pos >= cfg->gamma) return TABED_ERANGE;
    if (misaligned(W) || misaligned(H) || misaligned(draft_logits) || misaligned(draft_lse)) return TABED_EALIGN;
    const WsLayout L = ws_layout(*cfg);
    if (L.total > (size_t)TABED_STATIC_SCRATCH_BYTES) return TABED_ETOOBIG;
    char* ws = nullptr;
    const int rs = static_scratch(&ws);
    if (rs != TABED_OK) return rs;
    hipStream_t s = static_cast<hipStream_t>(stream);
    // the array keeps whatever the last call (of any configuration) left: the arrival counters start at zero
    hipError_t e = launch_ws_init(*cfg, L, ws, s);
    if (e != hipSuccess) return fail_hip(e);
    float* slot = draft_logits + (size_t)pos * L.M * cfg->V;
    e = launch_lmhead(*cfg, L, ws, W, H, temperature, slot, s);
    if (e != hipSuccess) return fail_hip(e);
    e = launch_sample(*cfg, L, ws, round, pos, slot, weights, temperature, u_draft, draft_lse, draft_tokens, draft_q,
                      flags, s);
    return e == hipSuccess ? TABED_OK : fail_hip(e);
}

int tabed_verify(const tabed_cfg* cfg, void* ws, uint64_t round, const float* target_logits,
                 const float* draft_logits, const double* draft_lse, const int32_t* draft_tokens,
                 const float* draft_q, const float* weights, const float* temperature, const float* u_acc,
                 const float* u_res, int32_t* accept_len, int32_t* out_tokens, float* dev, int32_t* n_valid,
                 uint8_t* flags, float* ring, int32_t* ring_head, int32_t* ring_count, float* next_weights,
                 void* stream) {
    const int rc = validate_cfg(cfg);
    if (rc != TABED_OK) return rc;
    if (!ws || !target_logits || !draft_logits || !draft_lse || !draft_tokens || !draft_q || !weights ||
        !temperature || !accept_len || !out_tokens || !dev || !n_valid || !flags)
        return TABED_ENULL;
    if (misaligned(ws) || misaligned(target_logits) || misaligned(draft_logits) || misaligned(draft_lse))
        return TABED_EALIGN;
    const int nwin = (ring != nullptr) + (ring_head != nullptr) + (ring_count != nullptr) + (next_weights != nullptr);
    if (nwin != 0 && nwin != 4) return TABED_ENULL;        // the fused window update takes all four or none
    const WsLayout L = ws_layout(*cfg);
    hipStream_t s = static_cast<hipStream_t>(stream);
    const hipError_t e = launch_verify(*cfg, L, static_cast<char*>(ws), round, target_logits, draft_logits, draft_lse,
                                       draft_tokens, draft_q, weights, temperature, u_acc, u_res, accept_len,
                                       out_tokens, dev, n_valid, flags, ring, ring_head, ring_count, next_weights,
                                       /*tree=*/false, s);
    return e == hipSuccess ? TABED_OK : fail_hip(e);
}

int tabed_draft_siblings(const tabed_cfg* cfg, void* ws, uint64_t round, int32_t pos, int32_t tree_width,
                         const float* draft_logits, const int32_t* draft_tokens, const float* weights,
                         const float* temperature, const float* u_sib, int32_t* sib_tokens, float* sib_q,
                         uint8_t* sib_flags, void* stream) {
    const int rc = validate_cfg(cfg);
    if (rc != TABED_OK) return rc;
    if (tree_width < 1 || tree_width > TABED_MAX_TREE_WIDTH) return TABED_ERANGE;
    if (pos < 0 || pos >= cfg->gamma) return TABED_ERANGE;
    if (tree_width == 1) return TABED_OK;                   // a chain has no siblings
    if (!ws || !draft_logits || !draft_tokens || !weights || !temperature || !sib_tokens || !sib_q || !sib_flags)
        return TABED_ENULL;
    if (misaligned(ws) || misaligned(draft_logits)) return TABED_EALIGN;
    const WsLayout L = ws_layout(*cfg);
    const float* slot = draft_logits + (size_t)pos * L.M * cfg->V;
    const hipError_t e = launch_siblings(*cfg, L, static_cast<char*>(ws), round, pos, tree_width, slot, draft_tokens, weights,
                                         temperature, u_sib, sib_tokens, sib_q, sib_flags, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? TABED_OK : fail_hip(e);
}

int tabed_verify_tree(const tabed_cfg* cfg, void* ws, uint64_t round, int32_t tree_width, const float* target_logits,
                      const float* leaf_logits, const float* draft_logits, const double* draft_lse,
                      const int32_t* draft_tokens, const float* draft_q, const int32_t* sib_tokens, const float* sib_q,
                      const float* weights, const float* temperature, const float* u_acc, const float* u_res,
                      const float* u_acc_sib, int32_t* accept_len, int32_t* out_tokens, float* dev, int32_t* n_valid,
                      uint8_t* flags, int32_t* leaf, int32_t* n_out, float* ring, int32_t* ring_head,
                      int32_t* ring_count, float* next_weights, void* stream) {
    const int rc = validate_cfg(cfg);
    if (rc != TABED_OK) return rc;
    if (tree_width < 1 || tree_width > TABED_MAX_TREE_WIDTH) return TABED_ERANGE;
    if (cfg->distance == 2) return TABED_EUNSUPPORTED;      // hard labels are defined for the chain only
    if (!ws || !target_logits || !draft_logits || !draft_lse || !draft_tokens || !draft_q || !weights ||
        !temperature || !accept_len || !out_tokens || !dev || !n_valid || !flags || !leaf || !n_out)
        return TABED_ENULL;
    if (tree_width > 1 && (!leaf_logits || !sib_tokens || !sib_q)) return TABED_ENULL;
    if (misaligned(ws) || misaligned(target_logits) || misaligned(draft_logits) || misaligned(draft_lse) ||
        (tree_width > 1 && misaligned(leaf_logits)))
        return TABED_EALIGN;
    const int nwin = (ring != nullptr) + (ring_head != nullptr) + (ring_count != nullptr) + (next_weights != nullptr);
    if (nwin != 0 && nwin != 4) return TABED_ENULL;
    if (next_weights == weights) return TABED_EINVAL;       // the tree passes still read this block's weights
    const WsLayout L = ws_layout(*cfg);
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t e = launch_verify(*cfg, L, static_cast<char*>(ws), round, target_logits, draft_logits, draft_lse,
                                 draft_tokens, draft_q, weights, temperature, u_acc, u_res, accept_len, out_tokens, dev,
                                 n_valid, flags, ring, ring_head, ring_count, next_weights, /*tree=*/true, s);
    if (e != hipSuccess) return fail_hip(e);
    e = launch_verify_tree(*cfg, L, static_cast<char*>(ws), round, tree_width, target_logits, leaf_logits, draft_logits,
                           draft_lse, sib_tokens, sib_q, weights, temperature, u_res, u_acc_sib, out_tokens, flags, leaf,
                           n_out, s);
    return e == hipSuccess ? TABED_OK : fail_hip(e);
}

// For the tests, not declared in the header: the grid in which tabed_verify launches the statistics together with hard labels.
int tabed_testing_labels_grid(const tabed_cfg* cfg, uint32_t* grid /* [3] */) {
    const int rc = validate_cfg(cfg);
    if (rc != TABED_OK) return rc;
    const dim3 g = stats_labels_grid(*cfg, ws_layout(*cfg));
    grid[0] = g.x; grid[1] = g.y; grid[2] = g.z;
    return TABED_OK;
}

int tabed_update_weights(const tabed_cfg* cfg, void* ws, uint64_t round, const float* dev, const int32_t* n_valid, float* ring,
                         int32_t* ring_head, int32_t* ring_count, float* weights, void* stream) {
    (void)ws;
    const int rc = validate_cfg(cfg);
    if (rc != TABED_OK) return rc;
    if (!ring || !ring_head || !ring_count || !weights) return TABED_ENULL;
    if ((dev == nullptr) != (n_valid == nullptr)) return TABED_ENULL;
    const hipError_t e = launch_weights(*cfg, round, dev, n_valid, ring, ring_head, ring_count, weights,
                                        static_cast<hipStream_t>(stream));
    return e == hipSuccess ? TABED_OK : fail_hip(e);
}

size_t tabed_body_workspace_bytes(const tabed_body_cfg* cfg, int32_t rows) {
    if (validate_body_cfg(cfg, rows) != TABED_OK) return 0;
    return body_workspace_bytes(*cfg, rows);
}

// For the tests, not declared in the header: how a body step runs.  0: one launch; s > 0: a launch per phase, keys in s ranges.
int tabed_testing_body_route(const tabed_body_cfg* cfg, int32_t rows) {
    const int rc = validate_body_cfg(cfg, rows);
    return rc == TABED_OK ? body_route(*cfg, rows) : rc;
}

int tabed_body_workspace_init(const tabed_body_cfg* cfg, int32_t rows, void* ws, void* stream) {
    const int rc = validate_body_cfg(cfg, rows);
    if (rc != TABED_OK) return rc;
    if (ws == nullptr) return TABED_ENULL;
    if (misaligned(ws)) return TABED_EALIGN;
    const hipError_t e = launch_body_init(*cfg, rows, static_cast<char*>(ws), static_cast<hipStream_t>(stream));
    return e == hipSuccess ? TABED_OK : fail_hip(e);
}

static int check_body_weights(const tabed_body_cfg& cfg, const tabed_body_weights& w) {
    if (!w.embed || !w.g_final) return TABED_ENULL;
    for (int l = 0; l < cfg.layers; ++l) {
        if (!w.g_attn[l] || !w.wqkv[l] || !w.wo[l] || !w.g_mlp[l] || !w.wgu[l] || !w.wdown[l]) return TABED_ENULL;
        if (misaligned(w.wqkv[l]) || misaligned(w.wo[l]) || misaligned(w.wgu[l]) || misaligned(w.wdown[l]) || misaligned(w.g_attn[l]) ||
            misaligned(w.g_mlp[l]))
            return TABED_EALIGN;
    }
    return misaligned(w.embed) || misaligned(w.g_final) ? TABED_EALIGN : TABED_OK;
}

// tabed_draft_body_step, for the tests with workgroups of the one-launch step from number late_from on that come after the others
// have stopped waiting for them, and with one that takes part and does nothing, so that waits for it end unanswered, after
// milliseconds (0: as in earnest).
int tabed_testing_body_step(const tabed_body_cfg* cfg, const tabed_body_weights* weights, void* ws, int32_t rows,
                            const int32_t* token_src, int32_t token_stride, int32_t rows_per_token, int32_t* ctx_len,
                            void* kcache, void* vcache, void* H, void* stream, int32_t late_from, int32_t absent) {
    const int rc = validate_body_cfg(cfg, rows);
    if (rc != TABED_OK) return rc;
    if (!weights || !ws || !token_src || !ctx_len || !kcache || !vcache || !H) return TABED_ENULL;
    if (rows_per_token < 1 || token_stride < 0) return TABED_ERANGE;
    const int rw = check_body_weights(*cfg, *weights);
    if (rw != TABED_OK) return rw;
    if (misaligned(ws) || misaligned(kcache) || misaligned(vcache) || misaligned(H)) return TABED_EALIGN;
    const hipError_t e = launch_body_step(*cfg, *weights, static_cast<char*>(ws), rows, token_src, token_stride, rows_per_token,
                                          ctx_len, static_cast<uint16_t*>(kcache), static_cast<uint16_t*>(vcache),
                                          static_cast<uint16_t*>(H), static_cast<hipStream_t>(stream), late_from, absent);
    return e == hipSuccess ? TABED_OK : fail_hip(e);
}

int tabed_draft_body_step(const tabed_body_cfg* cfg, const tabed_body_weights* weights, void* ws, int32_t rows,
                          const int32_t* token_src, int32_t token_stride, int32_t rows_per_token, int32_t* ctx_len,
                          void* kcache, void* vcache, void* H, void* stream) {
    return tabed_testing_body_step(cfg, weights, ws, rows, token_src, token_stride, rows_per_token, ctx_len, kcache, vcache, H, stream, 0, 0);
}

int tabed_draft_body_rollback(int32_t rows, int32_t rows_per_seq, int32_t gamma, const int32_t* ctx_base,
                              const int32_t* accept_len, int32_t* ctx_len, void* stream) {
    if (!ctx_base || !accept_len || !ctx_len) return TABED_ENULL;
    if (rows < 1 || rows_per_seq < 1 || gamma < 1) return TABED_ERANGE;
    const hipError_t e = launch_body_rollback(rows, rows_per_seq, gamma, ctx_base, accept_len, ctx_len,
                                              static_cast<hipStream_t>(stream));
    return e == hipSuccess ? TABED_OK : fail_hip(e);
}

// ---------------------------------------------------------------- 8-bit operators
int tabed_norm_q8(int32_t rows, int32_t d, int32_t x_dtype, const void* x, int64_t ldx, int32_t delta_dtype, const void* delta, int64_t ldd,
                  void* sum, int64_t lds, const float* gain, float eps, void* q, int64_t ldq, float* scale, void* stream) {
    if (!x || !q || !scale) return TABED_ENULL;
    if (rows < 1 || rows > (1 << 20) || d < 1 || d > 32768) return TABED_ERANGE;
    if (!storage_type(x_dtype) || (delta != nullptr && !storage_type(delta_dtype))) return TABED_EINVAL;
    if (sum != nullptr && delta == nullptr) return TABED_EINVAL;
    if (sum == x && rows > 1 && lds != ldx) return TABED_EINVAL;       // a row's sum would go to where another's values are
    if (ldx < d || ldq < d || (delta != nullptr && ldd < d) || (sum != nullptr && lds < d)) return TABED_EINVAL;
    if (gain != nullptr && !(eps > 0.f)) return TABED_EINVAL;
    if (element_misaligned(x, x_dtype) || element_misaligned(sum, x_dtype) || element_misaligned(delta, delta_dtype) ||
        element_misaligned(gain, 0) || element_misaligned(scale, 0))
        return TABED_EALIGN;
    const hipError_t e = launch_norm_q8(rows, d, x_dtype, x, ldx, delta_dtype, delta, ldd, sum, lds, gain, eps, static_cast<int8_t*>(q), ldq, scale,
                                        nullptr, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? TABED_OK : fail_hip(e);
}

int tabed_linear_q8(int32_t M, int32_t N, int32_t K, const void* X, int64_t ldx, const float* x_scale, const void* W, const float* w_scale,
                    int32_t y_dtype, void* Y, int64_t ldy, void* stream) {
    if (!X || !x_scale || !W || !w_scale || !Y) return TABED_ENULL;
    if (M < 1 || M > (1 << 20) || N < 1 || N > (1 << 24) || K < 16 || K > 131056 || ldx > (1 << 22)) return TABED_ERANGE;
    if ((int64_t)M * N > (1ll << 36)) return TABED_ERANGE;
    if (K % 16 != 0 || ldx % 16 != 0 || ldx < K || ldy < N || !storage_type(y_dtype)) return TABED_EINVAL;
    if (misaligned(X) || misaligned(W) || element_misaligned(Y, y_dtype) || element_misaligned(x_scale, 0) || element_misaligned(w_scale, 0))
        return TABED_EALIGN;
    const hipError_t e = launch_linear_q8(M, N, K, static_cast<const int8_t*>(X), ldx, x_scale, static_cast<const int8_t*>(W), w_scale, y_dtype, Y, ldy,
                                          static_cast<hipStream_t>(stream));
    return e == hipSuccess ? TABED_OK : fail_hip(e);
}

// For the tests, not declared in the header: the tile that a product (head: the LM head) of these sizes runs in: rows, columns, waves that share K, stages
// of W and of X.
int tabed_testing_linear_tile(int32_t M, int32_t N, int32_t K, int32_t head, int32_t* tile /* [5] */) {
    if (M < 1 || N < 1 || K < 16) return TABED_ERANGE;
    linear_q8_tile(M, N, K, head != 0, tile);
    return TABED_OK;
}

int tabed_cache_append_q8(const tabed_cache_q8* cache, int32_t rows, int32_t T, int32_t kv_dtype, const void* k, const void* v,
                          int64_t row_stride, int64_t tok_stride, const int32_t* ctx_len, const int32_t* n_new, void* stream) {
    const int rc = validate_cache(cache, true);
    if (rc != TABED_OK) return rc;
    if (!k || !v || !ctx_len) return TABED_ENULL;
    if (rows < 1 || rows > 65535 || T < 1 || T > (1 << 20)) return TABED_ERANGE;
    if (append_workgroups(*cache, rows, T) > kMaxWorkgroups) return TABED_ERANGE;
    const int64_t heads = (int64_t)cache->kv_heads * cache->head_dim;
    if (!storage_type(kv_dtype) || tok_stride < heads || row_stride < heads) return TABED_EINVAL;
    if (element_misaligned(k, kv_dtype) || element_misaligned(v, kv_dtype) || element_misaligned(ctx_len, 0) || element_misaligned(n_new, 0))
        return TABED_EALIGN;
    const hipError_t e = launch_cache_append(*cache, rows, T, kv_dtype, k, v, row_stride, tok_stride, ctx_len, n_new, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? TABED_OK : fail_hip(e);
}

static int validate_attention(const tabed_cache_q8* cache, int32_t rows, int32_t T, int32_t q_heads, bool pointers) {
    const int rc = validate_cache(cache, pointers);
    if (rc != TABED_OK) return rc;
    if (rows < 1 || rows > 65535 || T < 1 || q_heads < 1) return TABED_ERANGE;
    if ((int64_t)T * q_heads > (1 << 20)) return TABED_ERANGE;
    if (q_heads % cache->kv_heads != 0) return TABED_EINVAL;
    if (attn_workgroups(*cache, rows, T, q_heads) > kMaxWorkgroups) return TABED_ERANGE;
    return TABED_OK;
}

size_t tabed_attention_q8_workspace_bytes(const tabed_cache_q8* cache, int32_t rows, int32_t T, int32_t q_heads) {
    if (validate_attention(cache, rows, T, q_heads, false) != TABED_OK) return 0;
    return attn_layout(*cache, rows, T, q_heads).total;
}

int tabed_attention_q8_workspace_init(const tabed_cache_q8* cache, int32_t rows, int32_t T, int32_t q_heads, void* ws, void* stream) {
    const int rc = validate_attention(cache, rows, T, q_heads, false);
    if (rc != TABED_OK) return rc;
    if (ws == nullptr) return TABED_ENULL;
    if (misaligned(ws)) return TABED_EALIGN;
    const hipError_t e = launch_attn_init(static_cast<char*>(ws), static_cast<hipStream_t>(stream));
    return e == hipSuccess ? TABED_OK : fail_hip(e);
}

int tabed_attention_q8(const tabed_cache_q8* cache, void* ws, int32_t rows, int32_t T, int32_t q_heads, int32_t q_dtype, const void* q,
                       int64_t q_row_stride, int64_t q_tok_stride, const int32_t* ctx_len, const int32_t* n_new, float scale,
                       int32_t out_dtype, void* out, int64_t out_row_stride, int64_t out_tok_stride, float* lse, void* stream) {
    const int rc = validate_attention(cache, rows, T, q_heads, true);
    if (rc != TABED_OK) return rc;
    if (!ws || !q || !ctx_len || !out) return TABED_ENULL;
    const int64_t heads = (int64_t)q_heads * cache->head_dim;
    if (!storage_type(q_dtype) || !storage_type(out_dtype) || !(scale > 0.f) || !(scale < INFINITY)) return TABED_EINVAL;
    if (q_row_stride < heads || q_tok_stride < heads || out_row_stride < heads || out_tok_stride < heads) return TABED_EINVAL;
    if (misaligned(ws) || element_misaligned(q, q_dtype) || element_misaligned(out, out_dtype) || element_misaligned(ctx_len, 0) ||
        element_misaligned(n_new, 0) || element_misaligned(lse, 0))
        return TABED_EALIGN;
    const hipError_t e = launch_attention_q8(*cache, static_cast<char*>(ws), rows, T, q_heads, q_dtype, q, q_row_stride, q_tok_stride, ctx_len, n_new,
                                             scale, out_dtype, out, out_row_stride, out_tok_stride, lse, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? TABED_OK : fail_hip(e);
}

int tabed_draft_step_q8(const tabed_cfg* cfg, void* ws, uint64_t round, int32_t pos, const void* W, const float* w_scale, const void* H,
                        const float* h_scale, const float* weights, const float* temperature, const float* u_draft,
                        float* draft_logits, double* draft_lse, int32_t* draft_tokens, float* draft_q, uint8_t* flags, void* stream) {
    const int rc = validate_cfg(cfg);
    if (rc != TABED_OK) return rc;
    if (!ws || !W || !w_scale || !H || !h_scale || !weights || !temperature || !draft_logits || !draft_lse || !draft_tokens || !draft_q || !flags)
        return TABED_ENULL;
    if (pos < 0 || pos >= cfg->gamma) return TABED_ERANGE;
    if (cfg->d % 16 != 0) return TABED_EINVAL;
    if (cfg->d > 131056 || (int64_t)cfg->B * cfg->n * cfg->V > (1ll << 36)) return TABED_ERANGE;
    if (misaligned(ws) || misaligned(W) || misaligned(H) || misaligned(draft_logits) || misaligned(draft_lse) || element_misaligned(w_scale, 0) ||
        element_misaligned(h_scale, 0))
        return TABED_EALIGN;
    const WsLayout L = ws_layout(*cfg);
    hipStream_t s = static_cast<hipStream_t>(stream);
    float* slot = draft_logits + (size_t)pos * L.M * cfg->V;
    hipError_t e = launch_lmhead_q8(*cfg, L, static_cast<char*>(ws), static_cast<const int8_t*>(W), w_scale, static_cast<const int8_t*>(H), h_scale,
                                    temperature, slot, s);
    if (e != hipSuccess) return fail_hip(e);
    e = launch_sample(*cfg, L, static_cast<char*>(ws), round, pos, slot, weights, temperature, u_draft, draft_lse, draft_tokens, draft_q, flags, s);
    return e == hipSuccess ? TABED_OK : fail_hip(e);
}

static int validate_body_q8(const tabed_body_cfg* cfg, const tabed_cache_q8* cache, int32_t rows, bool pointers) {
    int rc = validate_body_cfg(cfg, rows);
    if (rc == TABED_OK) rc = validate_cache(cache, pointers);
    if (rc != TABED_OK) return rc;
    if (cache->kv_heads != cfg->heads || cache->head_dim != cfg->d / cfg->heads) return TABED_EINVAL;
    if ((int64_t)cache->max_blocks * TABED_CACHE_BLOCK < cfg->max_ctx) return TABED_EINVAL;
    return validate_attention(cache, rows, 1, cfg->heads, false);
}

size_t tabed_body_q8_workspace_bytes(const tabed_body_cfg* cfg, const tabed_cache_q8* cache, int32_t rows) {
    if (validate_body_q8(cfg, cache, rows, false) != TABED_OK) return 0;
    return body_q8_layout(*cfg, *cache, rows).total;
}

int tabed_body_q8_workspace_init(const tabed_body_cfg* cfg, const tabed_cache_q8* cache, int32_t rows, void* ws, void* stream) {
    const int rc = validate_body_q8(cfg, cache, rows, false);
    if (rc != TABED_OK) return rc;
    if (ws == nullptr) return TABED_ENULL;
    if (misaligned(ws)) return TABED_EALIGN;
    const hipError_t e = launch_attn_init(static_cast<char*>(ws), static_cast<hipStream_t>(stream));      // (the attention's workspace comes first)
    return e == hipSuccess ? TABED_OK : fail_hip(e);
}

int tabed_draft_body_step_q8(const tabed_body_cfg* cfg, const tabed_body_weights* weights, void* ws, int32_t rows, const int32_t* token_src,
                             int32_t token_stride, int32_t rows_per_token, int32_t* ctx_len, const tabed_cache_q8* cache, void* H, void* H8,
                             float* h_scale, void* stream) {
    int rc = validate_body_q8(cfg, cache, rows, true);
    if (rc != TABED_OK) return rc;
    if (!weights || !ws || !token_src || !ctx_len || (!H && !H8) || (H8 == nullptr) != (h_scale == nullptr)) return TABED_ENULL;
    if (rows_per_token < 1 || token_stride < 0) return TABED_ERANGE;
    rc = check_body_weights(*cfg, *weights);
    if (rc != TABED_OK) return rc;
    if (misaligned(ws) || misaligned(H) || misaligned(H8) || element_misaligned(h_scale, 0)) return TABED_EALIGN;
    const hipError_t e = launch_body_step_q8(*cfg, *weights, static_cast<char*>(ws), rows, token_src, token_stride, rows_per_token, ctx_len, *cache,
                                             static_cast<uint16_t*>(H), static_cast<int8_t*>(H8), h_scale, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? TABED_OK : fail_hip(e);
}

// ---------------------------------------------------------------- trees given by parents
static int validate_nodes(int32_t rows, int32_t N) {
    return rows < 1 || rows > 65535 || N < 1 || N > TABED_MAX_NODES ? TABED_ERANGE : TABED_OK;
}

int tabed_cache_append_nodes(const tabed_cache_paged* cache, int32_t layer, int32_t rows, int32_t N, int32_t dtype, const void* k, const void* v,
                             int64_t kv_row_stride, int64_t kv_tok_stride, int32_t q_heads, const void* q, int64_t q_row_stride, int64_t q_tok_stride,
                             void* q_out, int64_t out_row_stride, int64_t out_tok_stride, const int32_t* ctx_len, const int32_t* parents,
                             const int32_t* n_nodes, float rope_theta, void* stream) {
    int rc = validate_paged(cache, true);
    if (rc == TABED_OK) rc = validate_nodes(rows, N);
    if (rc != TABED_OK) return rc;
    if (layer < 0 || layer >= cache->layers) return TABED_ERANGE;
    if (!k || !v || !ctx_len || (q == nullptr) != (q_out == nullptr)) return TABED_ENULL;
    const int64_t heads = (int64_t)cache->kv_heads * cache->head_dim;
    if (!storage_type(dtype) || kv_row_stride < heads || kv_tok_stride < heads) return TABED_EINVAL;
    if (!(rope_theta == 0.f || (rope_theta > 0.f && rope_theta < INFINITY))) return TABED_EINVAL;
    if (q != nullptr) {
        if (q_heads < 1 || q_heads > 16384) return TABED_ERANGE;
        const int64_t qh = (int64_t)q_heads * cache->head_dim;
        if (q_row_stride < qh || q_tok_stride < qh || out_row_stride < qh || out_tok_stride < qh) return TABED_EINVAL;
        if (q == q_out && (dtype != 1 || q_row_stride != out_row_stride || q_tok_stride != out_tok_stride)) return TABED_EINVAL;
    }
    if (element_misaligned(k, dtype) || element_misaligned(v, dtype) || element_misaligned(q, dtype) || element_misaligned(q_out, 1) ||
        element_misaligned(ctx_len, 0) || element_misaligned(parents, 0) || element_misaligned(n_nodes, 0))
        return TABED_EALIGN;
    const hipError_t e = launch_append_nodes(*cache, layer, rows, N, dtype, k, v, kv_row_stride, kv_tok_stride, q_heads, q, q_row_stride, q_tok_stride, q_out,
                                             out_row_stride, out_tok_stride, ctx_len, parents, n_nodes, rope_theta, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? TABED_OK : fail_hip(e);
}

static int validate_attention_nodes(const tabed_cache_paged* cache, int32_t rows, int32_t N, int32_t q_heads, bool pointers) {
    int rc = validate_paged(cache, pointers);
    if (rc == TABED_OK) rc = validate_nodes(rows, N);
    if (rc != TABED_OK) return rc;
    if (q_heads < 1 || q_heads > 16384) return TABED_ERANGE;
    if (q_heads % cache->kv_heads != 0) return TABED_EINVAL;
    return nodes_attn_workgroups(*cache, rows, N, q_heads) > kMaxWorkgroups ? TABED_ERANGE : TABED_OK;
}

size_t tabed_attention_nodes_workspace_bytes(const tabed_cache_paged* cache, int32_t rows, int32_t N, int32_t q_heads) {
    if (validate_attention_nodes(cache, rows, N, q_heads, false) != TABED_OK) return 0;
    return nodes_attn_bytes(*cache, rows, N, q_heads);
}

int tabed_attention_nodes_workspace_init(const tabed_cache_paged* cache, int32_t rows, int32_t N, int32_t q_heads, void* ws, void* stream) {
    const int rc = validate_attention_nodes(cache, rows, N, q_heads, false);
    if (rc != TABED_OK) return rc;
    if (ws == nullptr) return TABED_ENULL;
    if (misaligned(ws)) return TABED_EALIGN;
    const hipError_t e = launch_nodes_attn_init(static_cast<char*>(ws), static_cast<hipStream_t>(stream));
    return e == hipSuccess ? TABED_OK : fail_hip(e);
}

int tabed_attention_nodes(const tabed_cache_paged* cache, int32_t layer, void* ws, int32_t rows, int32_t N, int32_t q_heads, const void* q,
                          int64_t q_row_stride, int64_t q_tok_stride, const int32_t* ctx_len, const int32_t* parents, const int32_t* n_nodes, float scale,
                          void* out, int64_t out_row_stride, int64_t out_tok_stride, float* lse, void* stream) {
    const int rc = validate_attention_nodes(cache, rows, N, q_heads, true);
    if (rc != TABED_OK) return rc;
    if (layer < 0 || layer >= cache->layers) return TABED_ERANGE;
    if (!ws || !q || !ctx_len || !out) return TABED_ENULL;
    const int64_t heads = (int64_t)q_heads * cache->head_dim;
    if (!(scale > 0.f) || !(scale < INFINITY)) return TABED_EINVAL;
    if (q_row_stride < heads || q_tok_stride < heads || out_row_stride < heads || out_tok_stride < heads) return TABED_EINVAL;
    if (q == out && (q_row_stride != out_row_stride || q_tok_stride != out_tok_stride)) return TABED_EINVAL;
    if (misaligned(ws) || element_misaligned(q, 1) || element_misaligned(out, 1) || element_misaligned(ctx_len, 0) || element_misaligned(parents, 0) ||
        element_misaligned(n_nodes, 0) || element_misaligned(lse, 0))
        return TABED_EALIGN;
    const hipError_t e = launch_attention_nodes(*cache, layer, static_cast<char*>(ws), rows, N, q_heads, static_cast<const uint16_t*>(q), q_row_stride,
                                                q_tok_stride, ctx_len, parents, n_nodes, scale, static_cast<uint16_t*>(out), out_row_stride,
                                                out_tok_stride, lse, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? TABED_OK : fail_hip(e);
}

static int validate_verify_nodes(const tabed_cfg* cfg, int32_t N) {
    int rc = validate_cfg(cfg);
    if (rc == TABED_OK) rc = validate_nodes(cfg->B, N);
    if (rc != TABED_OK) return rc;
    return nodes_verify_layout(*cfg, N).G * (int64_t)cfg->B > kMaxWorkgroups ? TABED_ERANGE : TABED_OK;
}

size_t tabed_verify_nodes_workspace_bytes(const tabed_cfg* cfg, int32_t N) {
    if (validate_verify_nodes(cfg, N) != TABED_OK) return 0;
    return nodes_verify_layout(*cfg, N).total;
}

int tabed_verify_nodes_workspace_init(const tabed_cfg* cfg, int32_t N, void* ws, void* stream) {
    const int rc = validate_verify_nodes(cfg, N);
    if (rc != TABED_OK) return rc;
    if (ws == nullptr) return TABED_ENULL;
    if (misaligned(ws)) return TABED_EALIGN;
    const hipError_t e = launch_nodes_verify_init(*cfg, N, static_cast<char*>(ws), static_cast<hipStream_t>(stream));
    return e == hipSuccess ? TABED_OK : fail_hip(e);
}

// tabed_verify_nodes, for the tests with waits that end after `spins` polls, and with workgroup `late` of every sequence coming 3 ms after the others (0, -1: as in earnest).
int tabed_testing_verify_nodes(const tabed_cfg* cfg, void* ws, uint64_t round, int32_t N, const float* target_logits, const float* draft_logits,
                       const double* draft_lse, const int32_t* tokens, const float* node_q, const int32_t* parents, const int32_t* n_nodes,
                       const float* weights, const float* temperature, const float* u_acc, const float* u_res, int32_t* path, int32_t* n_path,
                       int32_t* out_tokens, uint8_t* flags, float* dev, int32_t* n_valid, void* stream, int32_t spins, int32_t late) {
    const int rc = validate_verify_nodes(cfg, N);
    if (rc != TABED_OK) return rc;
    if (!ws || !target_logits || !draft_logits || !draft_lse || !tokens || !node_q || !weights || !temperature || !path || !n_path || !out_tokens || !flags)
        return TABED_ENULL;
    if ((dev == nullptr) != (n_valid == nullptr)) return TABED_ENULL;
    if (dev != nullptr && (cfg->distance == 2 || cfg->policy == 2)) return TABED_EUNSUPPORTED;
    if (misaligned(ws) || misaligned(target_logits) || misaligned(draft_logits) || misaligned(draft_lse)) return TABED_EALIGN;
    for (const void* p : std::initializer_list<const void*>{tokens, node_q, parents, n_nodes, weights, temperature, u_acc, u_res, path, n_path, out_tokens, dev, n_valid})
        if (element_misaligned(p, 0)) return TABED_EALIGN;
    const hipError_t e = launch_verify_nodes(*cfg, static_cast<char*>(ws), round, N, target_logits, draft_logits, draft_lse, tokens, node_q, parents, n_nodes,
                                             weights, temperature, u_acc, u_res, path, n_path, out_tokens, flags, dev, n_valid,
                                             static_cast<hipStream_t>(stream), spins, late);
    return e == hipSuccess ? TABED_OK : fail_hip(e);
}

int tabed_verify_nodes(const tabed_cfg* cfg, void* ws, uint64_t round, int32_t N, const float* target_logits, const float* draft_logits,
                       const double* draft_lse, const int32_t* tokens, const float* node_q, const int32_t* parents, const int32_t* n_nodes,
                       const float* weights, const float* temperature, const float* u_acc, const float* u_res, int32_t* path, int32_t* n_path,
                       int32_t* out_tokens, uint8_t* flags, float* dev, int32_t* n_valid, void* stream) {
    return tabed_testing_verify_nodes(cfg, ws, round, N, target_logits, draft_logits, draft_lse, tokens, node_q, parents, n_nodes, weights, temperature, u_acc, u_res, path,
                                      n_path, out_tokens, flags, dev, n_valid, stream, 0, -1);
}

int tabed_cache_keep_nodes(const tabed_cache_paged* cache, int32_t rows, int32_t N, const int32_t* ctx_base, const int32_t* path, const int32_t* n_path,
                           int32_t* ctx_len, void* stream) {
    int rc = validate_paged(cache, true);
    if (rc == TABED_OK) rc = validate_nodes(rows, N);
    if (rc != TABED_OK) return rc;
    if (!ctx_base || !path || !n_path || !ctx_len) return TABED_ENULL;
    if (element_misaligned(ctx_base, 0) || element_misaligned(path, 0) || element_misaligned(n_path, 0) || element_misaligned(ctx_len, 0)) return TABED_EALIGN;
    auto overlaps = [&](const int32_t* in, int64_t n) {                  // (ctx_len is written while others still read)
        const uintptr_t a = reinterpret_cast<uintptr_t>(ctx_len), b = reinterpret_cast<uintptr_t>(in);
        return a < b + n * sizeof(int32_t) && b < a + rows * sizeof(int32_t);
    };
    if (overlaps(ctx_base, rows) || overlaps(path, (int64_t)rows * N) || overlaps(n_path, rows)) return TABED_EINVAL;
    const hipError_t e = launch_keep_nodes(*cache, rows, N, ctx_base, path, n_path, ctx_len, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? TABED_OK : fail_hip(e);
}

int tabed_philox_uniforms(const tabed_cfg* cfg, uint64_t round, float* out, void* stream) {
    const int rc = validate_cfg(cfg);
    if (rc != TABED_OK) return rc;
    if (!out) return TABED_ENULL;
    const hipError_t e = launch_philox(*cfg, round, out, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? TABED_OK : fail_hip(e);
}

int tabed_prof_enable(int on) {
    std::lock_guard<std::mutex> lk(g_prof_mu);
    g_prof_on.store(on != 0, std::memory_order_relaxed);
    return TABED_OK;
}

int tabed_prof_read(int id, double* total_ms, int64_t* launches) {
    if (id < 0 || id >= TABED_K_COUNT) return TABED_ERANGE;
    std::lock_guard<std::mutex> lk(g_prof_mu);
    prof_drain();
    if (total_ms) *total_ms = g_prof_ms[id];
    if (launches) *launches = g_prof_n[id];
    return TABED_OK;
}

int tabed_prof_reset(void) {
    std::lock_guard<std::mutex> lk(g_prof_mu);
    prof_drain();
    for (int i = 0; i < TABED_K_COUNT; ++i) { g_prof_ms[i] = 0.0; g_prof_n[i] = 0; }
    return TABED_OK;
}

int tabed_prof_null(void* stream) {
    const hipError_t e = launch_null(static_cast<hipStream_t>(stream));
    return e == hipSuccess ? TABED_OK : fail_hip(e);
}

const char* tabed_kernel_name(int id) {
    switch (id) {
        case TABED_K_LMHEAD: return "lmhead";
        case TABED_K_SAMPLE: return "sample";
        case TABED_K_STATS: return "stats";
        case TABED_K_RESID: return "resid";
        case TABED_K_WEIGHTS: return "weights";
        case TABED_K_DIST: return "dist";
        case TABED_K_TREE: return "tree";
        case TABED_K_BODY: return "body";
        case TABED_K_NULL: return "null";
        default: return "?";
    }
}

}  // extern "C"
