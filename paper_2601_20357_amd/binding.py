"""Thin ctypes binding of libtabed.so: same names as the C ABI in include/tabed.h, argument marshalling only.

Tensors are torch CUDA (ROCm) tensors; torch is used for device memory and streams, nothing else.
Every step of the path runs inside the library's HIP kernels.  There is no fallback: if the library has
not been built, or a call returns an error code, this module raises.
"""
from __future__ import annotations

import ctypes as C
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libtabed.so")

EXPORTS = [
    "tabed_workspace_bytes", "tabed_workspace_init", "tabed_strerror", "tabed_last_hip_error", "tabed_dev_width",
    "tabed_draft_step", "tabed_draft_step_static", "tabed_verify", "tabed_draft_siblings", "tabed_verify_tree", "tabed_update_weights", "tabed_philox_uniforms",
    "tabed_body_workspace_bytes", "tabed_body_workspace_init", "tabed_draft_body_step", "tabed_draft_body_rollback",
    "tabed_norm_q8", "tabed_linear_q8", "tabed_cache_append_q8",
    "tabed_attention_q8", "tabed_attention_q8_workspace_bytes", "tabed_attention_q8_workspace_init",
    "tabed_draft_step_q8", "tabed_body_q8_workspace_bytes", "tabed_body_q8_workspace_init", "tabed_draft_body_step_q8",
    "tabed_cache_append_nodes", "tabed_attention_nodes", "tabed_attention_nodes_workspace_bytes", "tabed_attention_nodes_workspace_init",
    "tabed_verify_nodes", "tabed_verify_nodes_workspace_bytes", "tabed_verify_nodes_workspace_init", "tabed_cache_keep_nodes",
    "tabed_prof_enable", "tabed_prof_read", "tabed_prof_reset", "tabed_kernel_name", "tabed_prof_null",
]

FLAG_ACCEPT_MARGIN, FLAG_SAMPLE_MARGIN, FLAG_DEGENERATE = 1, 2, 4
K_LMHEAD, K_SAMPLE, K_STATS, K_RESID, K_WEIGHTS, K_DIST, K_TREE, K_BODY, K_NULL, K_COUNT = 0, 1, 2, 3, 4, 5, 6, 7, 8, 9
BODY_MAX_LAYERS = 16


class TabedCfg(C.Structure):
    """Mirror of `tabed_cfg`."""
    _fields_ = [("V", C.c_int32), ("d", C.c_int32), ("n", C.c_int32), ("B", C.c_int32),
                ("gamma", C.c_int32), ("h", C.c_int32), ("w_dtype", C.c_int32), ("distance", C.c_int32),
                ("policy", C.c_int32), ("tau_w", C.c_float), ("eps", C.c_float), ("seed", C.c_uint64)]


class TabedBodyCfg(C.Structure):
    """Mirror of `tabed_body_cfg`."""
    _fields_ = [("layers", C.c_int32), ("d", C.c_int32), ("heads", C.c_int32), ("d_ff", C.c_int32), ("V", C.c_int32),
                ("max_ctx", C.c_int32), ("rope_theta", C.c_float), ("rms_eps", C.c_float)]


class TabedBodyWeights(C.Structure):
    """Mirror of `tabed_body_weights` (device pointers)."""
    _fields_ = [("embed", C.c_void_p), ("g_final", C.c_void_p)] + [
        (name, C.c_void_p * BODY_MAX_LAYERS) for name in ("g_attn", "wqkv", "wo", "g_mlp", "wgu", "wdown")]


class TabedCacheQ8(C.Structure):
    """Mirror of `tabed_cache_q8`."""
    _fields_ = [("kv_heads", C.c_int32), ("head_dim", C.c_int32), ("blocks", C.c_int32), ("max_blocks", C.c_int32),
                ("k", C.c_void_p), ("v", C.c_void_p), ("kscale", C.c_void_p), ("vscale", C.c_void_p), ("table", C.c_void_p)]


class TabedCachePaged(C.Structure):
    """Mirror of `tabed_cache_paged`."""
    _fields_ = [(name, C.c_int32) for name in ("layers", "kv_heads", "head_dim", "blocks", "max_blocks", "type")] + [
        (name, C.c_int64) for name in ("layer_stride", "block_stride", "head_stride", "tok_stride")] + [
        (name, C.c_void_p) for name in ("k", "v", "kscale", "vscale", "table")]


class TabedError(RuntimeError):
    pass


_lib = None


def load():
    """Load libtabed.so; raises if it has not been built (python -m paper_2601_20357_amd.build)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise TabedError(f"{LIB_PATH} is missing: build it first (python paper_2601_20357_amd/build.py); "
                         "there is no CPU fallback")
    lib = C.CDLL(LIB_PATH)
    vp, u64, i32 = C.c_void_p, C.c_uint64, C.c_int32
    cfgp = C.POINTER(TabedCfg)
    lib.tabed_workspace_bytes.restype = C.c_size_t
    lib.tabed_workspace_bytes.argtypes = [cfgp]
    lib.tabed_dev_width.restype = C.c_int32
    lib.tabed_dev_width.argtypes = [cfgp]
    lib.tabed_workspace_init.restype = C.c_int
    lib.tabed_workspace_init.argtypes = [cfgp, vp, vp]
    lib.tabed_strerror.restype = C.c_char_p
    lib.tabed_strerror.argtypes = [C.c_int]
    lib.tabed_last_hip_error.restype = C.c_int
    lib.tabed_draft_step.restype = C.c_int
    lib.tabed_draft_step.argtypes = [cfgp, vp, u64, i32] + [vp] * 11
    lib.tabed_draft_step_static.restype = C.c_int
    lib.tabed_draft_step_static.argtypes = [cfgp, u64, i32] + [vp] * 11
    lib.tabed_verify.restype = C.c_int
    lib.tabed_verify.argtypes = [cfgp, vp, u64] + [vp] * 19
    lib.tabed_draft_siblings.restype = C.c_int
    lib.tabed_draft_siblings.argtypes = [cfgp, vp, u64, i32, i32] + [vp] * 9
    lib.tabed_verify_tree.restype = C.c_int
    lib.tabed_verify_tree.argtypes = [cfgp, vp, u64, i32] + [vp] * 25
    lib.tabed_update_weights.restype = C.c_int
    lib.tabed_update_weights.argtypes = [cfgp, vp, u64] + [vp] * 7
    lib.tabed_philox_uniforms.restype = C.c_int
    lib.tabed_philox_uniforms.argtypes = [cfgp, u64, vp, vp]
    bcfgp = C.POINTER(TabedBodyCfg)
    lib.tabed_body_workspace_bytes.restype = C.c_size_t
    lib.tabed_body_workspace_bytes.argtypes = [bcfgp, i32]
    lib.tabed_body_workspace_init.restype = C.c_int
    lib.tabed_body_workspace_init.argtypes = [bcfgp, i32, vp, vp]
    lib.tabed_draft_body_step.restype = C.c_int
    lib.tabed_draft_body_step.argtypes = [bcfgp, C.POINTER(TabedBodyWeights), vp, i32, vp, i32, i32] + [vp] * 5
    lib.tabed_draft_body_rollback.restype = C.c_int
    lib.tabed_draft_body_rollback.argtypes = [i32, i32, i32, vp, vp, vp, vp]
    i64, f32, cachep = C.c_int64, C.c_float, C.POINTER(TabedCacheQ8)
    lib.tabed_norm_q8.restype = C.c_int
    lib.tabed_norm_q8.argtypes = [i32, i32, i32, vp, i64, i32, vp, i64, vp, i64, vp, f32, vp, i64, vp, vp]
    lib.tabed_linear_q8.restype = C.c_int
    lib.tabed_linear_q8.argtypes = [i32, i32, i32, vp, i64, vp, vp, vp, i32, vp, i64, vp]
    lib.tabed_cache_append_q8.restype = C.c_int
    lib.tabed_cache_append_q8.argtypes = [cachep, i32, i32, i32, vp, vp, i64, i64, vp, vp, vp]
    lib.tabed_attention_q8_workspace_bytes.restype = C.c_size_t
    lib.tabed_attention_q8_workspace_bytes.argtypes = [cachep, i32, i32, i32]
    lib.tabed_attention_q8_workspace_init.restype = C.c_int
    lib.tabed_attention_q8_workspace_init.argtypes = [cachep, i32, i32, i32, vp, vp]
    lib.tabed_attention_q8.restype = C.c_int
    lib.tabed_attention_q8.argtypes = [cachep, vp, i32, i32, i32, i32, vp, i64, i64, vp, vp, f32, i32, vp, i64, i64, vp, vp]
    lib.tabed_draft_step_q8.restype = C.c_int
    lib.tabed_draft_step_q8.argtypes = [cfgp, vp, u64, i32] + [vp] * 13
    lib.tabed_body_q8_workspace_bytes.restype = C.c_size_t
    lib.tabed_body_q8_workspace_bytes.argtypes = [bcfgp, cachep, i32]
    lib.tabed_body_q8_workspace_init.restype = C.c_int
    lib.tabed_body_q8_workspace_init.argtypes = [bcfgp, cachep, i32, vp, vp]
    lib.tabed_draft_body_step_q8.restype = C.c_int
    lib.tabed_draft_body_step_q8.argtypes = [bcfgp, C.POINTER(TabedBodyWeights), vp, i32, vp, i32, i32, vp, cachep] + [vp] * 4
    pagedp = C.POINTER(TabedCachePaged)
    lib.tabed_cache_append_nodes.restype = C.c_int
    lib.tabed_cache_append_nodes.argtypes = [pagedp, i32, i32, i32, i32, vp, vp, i64, i64, i32, vp, i64, i64, vp, i64, i64, vp, vp, vp, f32, vp]
    lib.tabed_attention_nodes_workspace_bytes.restype = C.c_size_t
    lib.tabed_attention_nodes_workspace_bytes.argtypes = [pagedp, i32, i32, i32]
    lib.tabed_attention_nodes_workspace_init.restype = C.c_int
    lib.tabed_attention_nodes_workspace_init.argtypes = [pagedp, i32, i32, i32, vp, vp]
    lib.tabed_attention_nodes.restype = C.c_int
    lib.tabed_attention_nodes.argtypes = [pagedp, i32, vp, i32, i32, i32, vp, i64, i64, vp, vp, vp, f32, vp, i64, i64, vp, vp]
    lib.tabed_verify_nodes_workspace_bytes.restype = C.c_size_t
    lib.tabed_verify_nodes_workspace_bytes.argtypes = [cfgp, i32]
    lib.tabed_verify_nodes_workspace_init.restype = C.c_int
    lib.tabed_verify_nodes_workspace_init.argtypes = [cfgp, i32, vp, vp]
    lib.tabed_verify_nodes.restype = C.c_int
    lib.tabed_verify_nodes.argtypes = [cfgp, vp, u64, i32] + [vp] * 18
    lib.tabed_cache_keep_nodes.restype = C.c_int
    lib.tabed_cache_keep_nodes.argtypes = [pagedp, i32, i32] + [vp] * 5
    lib.tabed_prof_enable.restype = C.c_int
    lib.tabed_prof_enable.argtypes = [C.c_int]
    lib.tabed_prof_read.restype = C.c_int
    lib.tabed_prof_read.argtypes = [C.c_int, C.POINTER(C.c_double), C.POINTER(C.c_int64)]
    lib.tabed_prof_reset.restype = C.c_int
    lib.tabed_kernel_name.restype = C.c_char_p
    lib.tabed_kernel_name.argtypes = [C.c_int]
    lib.tabed_prof_null.restype = C.c_int
    lib.tabed_prof_null.argtypes = [vp]
    _lib = lib
    return lib


GRID_CANDIDATES = 11


def make_cfg(*, V, d, n, B, gamma, h, w_dtype, distance=0, policy=0, tau_w=1.0, eps=1e-6, seed=0) -> TabedCfg:
    return TabedCfg(V, d, n, B, gamma, h, w_dtype, distance, policy, tau_w, eps, seed)


def _check(rc: int, what: str):
    if rc != 0:
        lib = load()
        msg = lib.tabed_strerror(rc).decode()
        raise TabedError(f"{what}: {msg} (code {rc}, hip error {lib.tabed_last_hip_error()})")


def _ptr(t, dtype=None, numel=None, name="tensor"):
    """Device pointer of a contiguous CUDA tensor (None -> NULL), with dtype / size checks."""
    if t is None:
        return None
    if not t.is_cuda:
        raise TabedError(f"{name} must live on the GPU")
    if not t.is_contiguous():
        raise TabedError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise TabedError(f"{name} must be {dtype}, got {t.dtype}")
    if numel is not None and t.numel() != numel:
        raise TabedError(f"{name} must hold {numel} elements, got {t.numel()}")
    return t.data_ptr()


def _stream(stream):
    import torch
    s = torch.cuda.current_stream() if stream is None else stream
    return s.cuda_stream


def tabed_dev_width(cfg: TabedCfg) -> int:
    """Last dimension of `dev` and `ring`: n, or 11 for the two-draft grid policy; 0 for an invalid cfg."""
    return int(load().tabed_dev_width(C.byref(cfg)))


def tabed_workspace_bytes(cfg: TabedCfg) -> int:
    return int(load().tabed_workspace_bytes(C.byref(cfg)))


def tabed_workspace_init(cfg: TabedCfg, ws, stream=None):
    _check(load().tabed_workspace_init(C.byref(cfg), _ptr(ws, name="ws"), _stream(stream)), "tabed_workspace_init")


def new_workspace(cfg: TabedCfg, device="cuda:0", stream=None):
    """Allocate (torch) and prepare a workspace for cfg."""
    import torch
    nbytes = tabed_workspace_bytes(cfg)
    if nbytes == 0:
        raise TabedError("invalid or unsupported tabed_cfg")
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    tabed_workspace_init(cfg, ws, stream)
    return ws


def _store_dtype(cfg):
    import torch
    return torch.float32 if cfg.w_dtype == 0 else torch.bfloat16


def tabed_draft_step(cfg, ws, rnd, pos, W, H, weights, temperature, draft_logits, draft_lse, draft_tokens,
                     draft_q, flags, u_draft=None, stream=None):
    import torch
    V, d, n, B, g = cfg.V, cfg.d, cfg.n, cfg.B, cfg.gamma
    sd = _store_dtype(cfg)
    rc = load().tabed_draft_step(
        C.byref(cfg), _ptr(ws, torch.uint8, name="ws"), rnd, pos,
        _ptr(W, sd, V * d, "W"), _ptr(H, sd, B * n * d, "H"),
        _ptr(weights, torch.float32, B * n, "weights"), _ptr(temperature, torch.float32, B, "temperature"),
        _ptr(u_draft, torch.float32, B * g, "u_draft"),
        _ptr(draft_logits, torch.float32, g * B * n * V, "draft_logits"),
        _ptr(draft_lse, torch.float64, g * B * n, "draft_lse"),
        _ptr(draft_tokens, torch.int32, B * g, "draft_tokens"), _ptr(draft_q, torch.float32, B * g, "draft_q"),
        _ptr(flags, torch.uint8, B * g, "flags"), _stream(stream))
    _check(rc, "tabed_draft_step")


STATIC_SCRATCH_BYTES = 8 << 20
ETOOBIG = -7


def tabed_draft_step_static(cfg, rnd, pos, W, H, weights, temperature, draft_logits, draft_lse, draft_tokens,
                            draft_q, flags, u_draft=None, stream=None):
    """tabed_draft_step on the library's built-in scratch buffer (no workspace argument, nothing allocated)."""
    import torch
    V, d, n, B, g = cfg.V, cfg.d, cfg.n, cfg.B, cfg.gamma
    sd = _store_dtype(cfg)
    rc = load().tabed_draft_step_static(
        C.byref(cfg), rnd, pos,
        _ptr(W, sd, V * d, "W"), _ptr(H, sd, B * n * d, "H"),
        _ptr(weights, torch.float32, B * n, "weights"), _ptr(temperature, torch.float32, B, "temperature"),
        _ptr(u_draft, torch.float32, B * g, "u_draft"),
        _ptr(draft_logits, torch.float32, g * B * n * V, "draft_logits"),
        _ptr(draft_lse, torch.float64, g * B * n, "draft_lse"),
        _ptr(draft_tokens, torch.int32, B * g, "draft_tokens"), _ptr(draft_q, torch.float32, B * g, "draft_q"),
        _ptr(flags, torch.uint8, B * g, "flags"), _stream(stream))
    _check(rc, "tabed_draft_step_static")


def tabed_verify(cfg, ws, rnd, target_logits, draft_logits, draft_lse, draft_tokens, draft_q, weights, temperature,
                 accept_len, out_tokens, dev, n_valid, flags, u_acc=None, u_res=None, ring=None, ring_head=None,
                 ring_count=None, next_weights=None, stream=None):
    import torch
    V, n, B, g = cfg.V, cfg.n, cfg.B, cfg.gamma
    rc = load().tabed_verify(
        C.byref(cfg), _ptr(ws, torch.uint8, name="ws"), rnd,
        _ptr(target_logits, torch.float32, B * (g + 1) * V, "target_logits"),
        _ptr(draft_logits, torch.float32, g * B * n * V, "draft_logits"),
        _ptr(draft_lse, torch.float64, g * B * n, "draft_lse"),
        _ptr(draft_tokens, torch.int32, B * g, "draft_tokens"), _ptr(draft_q, torch.float32, B * g, "draft_q"),
        _ptr(weights, torch.float32, B * n, "weights"), _ptr(temperature, torch.float32, B, "temperature"),
        _ptr(u_acc, torch.float32, B * g, "u_acc"), _ptr(u_res, torch.float32, B, "u_res"),
        _ptr(accept_len, torch.int32, B, "accept_len"), _ptr(out_tokens, torch.int32, B * (g + 1), "out_tokens"),
        _ptr(dev, torch.float32, B * g * tabed_dev_width(cfg), "dev"), _ptr(n_valid, torch.int32, B, "n_valid"),
        _ptr(flags, torch.uint8, B * (g + 1), "flags"),
        _ptr(ring, torch.float32, B * max(cfg.h, 1) * tabed_dev_width(cfg), "ring"),
        _ptr(ring_head, torch.int32, B, "ring_head"), _ptr(ring_count, torch.int32, B, "ring_count"),
        _ptr(next_weights, torch.float32, B * n, "next_weights"), _stream(stream))
    _check(rc, "tabed_verify")


MAX_TREE_WIDTH = 3
SIBLING_STRIDE = 65536


def tabed_draft_siblings(cfg, ws, rnd, pos, tree_width, draft_logits, draft_tokens, weights, temperature, sib_tokens,
                         sib_q, sib_flags, u_sib=None, stream=None):
    import torch
    V, n, B, g = cfg.V, cfg.n, cfg.B, cfg.gamma
    S = tree_width - 1
    rc = load().tabed_draft_siblings(
        C.byref(cfg), _ptr(ws, torch.uint8, name="ws"), rnd, pos, tree_width,
        _ptr(draft_logits, torch.float32, g * B * n * V, "draft_logits"),
        _ptr(draft_tokens, torch.int32, B * g, "draft_tokens"),
        _ptr(weights, torch.float32, B * n, "weights"), _ptr(temperature, torch.float32, B, "temperature"),
        _ptr(u_sib, torch.float32, B * g * S, "u_sib"),
        _ptr(sib_tokens, torch.int32, B * g * S, "sib_tokens"), _ptr(sib_q, torch.float32, B * g * S, "sib_q"),
        _ptr(sib_flags, torch.uint8, B * g * S, "sib_flags"), _stream(stream))
    _check(rc, "tabed_draft_siblings")


def tabed_verify_tree(cfg, ws, rnd, tree_width, target_logits, leaf_logits, draft_logits, draft_lse, draft_tokens,
                      draft_q, sib_tokens, sib_q, weights, temperature, accept_len, out_tokens, dev, n_valid, flags,
                      leaf, n_out, u_acc=None, u_res=None, u_acc_sib=None, ring=None, ring_head=None, ring_count=None,
                      next_weights=None, stream=None):
    import torch
    V, n, B, g = cfg.V, cfg.n, cfg.B, cfg.gamma
    S = tree_width - 1
    dw = tabed_dev_width(cfg)
    rc = load().tabed_verify_tree(
        C.byref(cfg), _ptr(ws, torch.uint8, name="ws"), rnd, tree_width,
        _ptr(target_logits, torch.float32, B * (g + 1) * V, "target_logits"),
        _ptr(leaf_logits, torch.float32, B * g * S * V, "leaf_logits") if S else None,
        _ptr(draft_logits, torch.float32, g * B * n * V, "draft_logits"),
        _ptr(draft_lse, torch.float64, g * B * n, "draft_lse"),
        _ptr(draft_tokens, torch.int32, B * g, "draft_tokens"), _ptr(draft_q, torch.float32, B * g, "draft_q"),
        _ptr(sib_tokens, torch.int32, B * g * S, "sib_tokens") if S else None,
        _ptr(sib_q, torch.float32, B * g * S, "sib_q") if S else None,
        _ptr(weights, torch.float32, B * n, "weights"), _ptr(temperature, torch.float32, B, "temperature"),
        _ptr(u_acc, torch.float32, B * g, "u_acc"), _ptr(u_res, torch.float32, B, "u_res"),
        _ptr(u_acc_sib, torch.float32, B * g * S, "u_acc_sib") if S else None,
        _ptr(accept_len, torch.int32, B, "accept_len"), _ptr(out_tokens, torch.int32, B * (g + 1), "out_tokens"),
        _ptr(dev, torch.float32, B * g * dw, "dev"), _ptr(n_valid, torch.int32, B, "n_valid"),
        _ptr(flags, torch.uint8, B * (g + 1), "flags"), _ptr(leaf, torch.int32, B, "leaf"),
        _ptr(n_out, torch.int32, B, "n_out"),
        _ptr(ring, torch.float32, B * max(cfg.h, 1) * dw, "ring"),
        _ptr(ring_head, torch.int32, B, "ring_head"), _ptr(ring_count, torch.int32, B, "ring_count"),
        _ptr(next_weights, torch.float32, B * n, "next_weights"), _stream(stream))
    _check(rc, "tabed_verify_tree")


def tabed_update_weights(cfg, ws, rnd, dev, n_valid, ring, ring_head, ring_count, weights, stream=None):
    import torch
    n, B, g, h = cfg.n, cfg.B, cfg.gamma, cfg.h
    dw = tabed_dev_width(cfg)
    rc = load().tabed_update_weights(
        C.byref(cfg), _ptr(ws, name="ws"), rnd,
        _ptr(dev, torch.float32, B * g * dw, "dev"), _ptr(n_valid, torch.int32, B, "n_valid"),
        _ptr(ring, torch.float32, B * max(h, 1) * dw, "ring"), _ptr(ring_head, torch.int32, B, "ring_head"),
        _ptr(ring_count, torch.int32, B, "ring_count"), _ptr(weights, torch.float32, B * n, "weights"),
        _stream(stream))
    _check(rc, "tabed_update_weights")


def make_body_cfg(*, layers, d, heads, d_ff, V, max_ctx, rope_theta=1e4, rms_eps=1e-5) -> TabedBodyCfg:
    return TabedBodyCfg(layers, d, heads, d_ff, V, max_ctx, rope_theta, rms_eps)


def make_body_weights(bcfg: TabedBodyCfg, tensors: dict) -> TabedBodyWeights:
    """Pointer table over device tensors: embed [V,d] and the per-layer lists wqkv [3d,d], wo [d,d], wgu [2 d_ff,d],
    wdown [d,d_ff] as bf16 (or their bit patterns as int16 / uint16), gains g_attn, g_mlp (lists) and g_final as fp32.
    The caller keeps `tensors` alive while the table is in use."""
    import torch
    two_byte = (torch.bfloat16, torch.int16, torch.uint16)
    d, ff, L = bcfg.d, bcfg.d_ff, bcfg.layers

    def mat(t, numel, name):
        if t.dtype not in two_byte:
            raise TabedError(f"{name} must hold bf16 values, got {t.dtype}")
        return _ptr(t, None, numel, name)

    w = TabedBodyWeights()
    w.embed = mat(tensors["embed"], bcfg.V * d, "embed")
    w.g_final = _ptr(tensors["g_final"], torch.float32, d, "g_final")
    for key, numel in (("wqkv", 3 * d * d), ("wo", d * d), ("wgu", 2 * ff * d), ("wdown", d * ff)):
        if len(tensors[key]) != L:
            raise TabedError(f"{key} must list {L} layers")
        for l in range(L):
            getattr(w, key)[l] = mat(tensors[key][l], numel, f"{key}[{l}]")
    for key in ("g_attn", "g_mlp"):
        if len(tensors[key]) != L:
            raise TabedError(f"{key} must list {L} layers")
        for l in range(L):
            getattr(w, key)[l] = _ptr(tensors[key][l], torch.float32, d, f"{key}[{l}]")
    return w


def tabed_body_workspace_bytes(bcfg: TabedBodyCfg, rows: int) -> int:
    return int(load().tabed_body_workspace_bytes(C.byref(bcfg), rows))


def tabed_body_workspace_init(bcfg, rows, ws, stream=None):
    import torch
    need = tabed_body_workspace_bytes(bcfg, rows)
    if need == 0:
        raise TabedError("tabed_body_workspace_init: invalid configuration")
    if ws.numel() * ws.element_size() < need:
        raise TabedError(f"body workspace holds {ws.numel() * ws.element_size()} bytes, {need} needed")
    _check(load().tabed_body_workspace_init(C.byref(bcfg), rows, _ptr(ws, torch.uint8, name="ws"), _stream(stream)),
           "tabed_body_workspace_init")


def tabed_draft_body_step(bcfg, weights, ws, rows, token_src, token_stride, rows_per_token, ctx_len, kcache, vcache, H,
                          stream=None):
    """token_src: int32 tensor, or a (tensor, element offset) pair for a view into draft_tokens."""
    import torch
    if isinstance(token_src, tuple):
        base, off = token_src
        need = off + ((rows - 1) // rows_per_token) * token_stride + 1
        if base.dtype != torch.int32 or not base.is_cuda or not base.is_contiguous() or base.numel() < need or off < 0:
            raise TabedError("token_src must be a contiguous int32 GPU tensor covering every token read")
        tok_ptr = base.data_ptr() + 4 * off
    else:
        need = ((rows - 1) // rows_per_token) * token_stride + 1
        if token_src.numel() < need:
            raise TabedError(f"token_src must hold {need} elements, got {token_src.numel()}")
        tok_ptr = _ptr(token_src, torch.int32, None, "token_src")
    if ws.numel() * ws.element_size() < tabed_body_workspace_bytes(bcfg, rows):
        raise TabedError("body workspace too small")
    two_byte = (torch.bfloat16, torch.int16, torch.uint16)
    for t, name in ((kcache, "kcache"), (vcache, "vcache"), (H, "H")):
        if t.dtype not in two_byte:
            raise TabedError(f"{name} must hold bf16 values, got {t.dtype}")
    cache_numel = bcfg.layers * rows * bcfg.max_ctx * bcfg.d
    rc = load().tabed_draft_body_step(
        C.byref(bcfg), C.byref(weights), _ptr(ws, torch.uint8, name="ws"), rows, tok_ptr, token_stride, rows_per_token,
        _ptr(ctx_len, torch.int32, rows, "ctx_len"), _ptr(kcache, None, cache_numel, "kcache"),
        _ptr(vcache, None, cache_numel, "vcache"), _ptr(H, None, rows * bcfg.d, "H"), _stream(stream))
    _check(rc, "tabed_draft_body_step")


def tabed_draft_body_rollback(rows, rows_per_seq, gamma, ctx_base, accept_len, ctx_len, stream=None):
    import torch
    nseq = (rows + rows_per_seq - 1) // rows_per_seq
    rc = load().tabed_draft_body_rollback(
        rows, rows_per_seq, gamma, _ptr(ctx_base, torch.int32, rows, "ctx_base"),
        _ptr(accept_len, torch.int32, nseq, "accept_len"), _ptr(ctx_len, torch.int32, rows, "ctx_len"), _stream(stream))
    _check(rc, "tabed_draft_body_rollback")


def tabed_philox_uniforms(cfg, rnd, out, stream=None):
    import torch
    rc = load().tabed_philox_uniforms(C.byref(cfg), rnd, _ptr(out, torch.float32, cfg.B * (cfg.gamma + 1) * 2, "out"),
                                      _stream(stream))
    _check(rc, "tabed_philox_uniforms")


def tabed_prof_enable(on: bool):
    _check(load().tabed_prof_enable(1 if on else 0), "tabed_prof_enable")


def tabed_prof_reset():
    _check(load().tabed_prof_reset(), "tabed_prof_reset")


def tabed_prof_read(kernel_id: int):
    """(total milliseconds, launches) of one kernel since the last reset; waits for its events."""
    ms, cnt = C.c_double(0), C.c_int64(0)
    _check(load().tabed_prof_read(kernel_id, C.byref(ms), C.byref(cnt)), "tabed_prof_read")
    return ms.value, cnt.value


def tabed_prof_null(stream=None):
    _check(load().tabed_prof_null(_stream(stream)), "tabed_prof_null")


def tabed_kernel_name(kernel_id: int) -> str:
    return load().tabed_kernel_name(kernel_id).decode()


class PreparedCall:
    """A C-ABI call with its arguments already converted to ctypes, for launch loops where the per-call
    tensor checks would cost more than the launch.  Built by RoundBuffers.prepare_*; checks happen once."""

    __slots__ = ("fn", "args", "what", "round_arg")

    def __init__(self, fn, args, what, round_arg=None):
        self.fn, self.args, self.what, self.round_arg = fn, args, what, round_arg

    def set_round(self, rnd: int):
        """Change the SD round number (the Philox counter) the next call passes."""
        if self.round_arg is not None:
            self.round_arg.value = rnd

    def __call__(self):
        rc = self.fn(*self.args)
        if rc != 0:
            _check(rc, self.what)


# ------------------------------------------------------------------ the draft side in 8 bits
CACHE_BLOCK = 64


class DeviceCall(PreparedCall):
    """A PreparedCall that makes its tensors' device current and keeps the tensors (and its HOST structs) alive."""

    __slots__ = ("device", "keep", "current")

    def __init__(self, fn, args, what, device, keep):
        import torch
        for t, a in zip(fn.argtypes, args):
            if t is C.c_int32 and isinstance(a, int) and not -1 << 31 <= a < 1 << 31:
                raise TabedError(f"{what}: a size of {a} does not fit 32 bits")
        simple = (int, float, type(None))                  # converted now, not at every call
        super().__init__(fn, [t(a) if isinstance(a, simple) else a for t, a in zip(fn.argtypes, args)], what)
        self.device, self.keep, self.current = device, keep, torch.cuda.current_device

    def __call__(self):
        if self.current() == self.device:
            rc = self.fn(*self.args)
        else:
            import torch
            with torch.cuda.device(self.device):
                rc = self.fn(*self.args)
        if rc != 0:
            _check(rc, self.what)


def _device_of(named: dict):
    """The one device of the tensors given (None entries are left out)."""
    device = None
    for name, t in named.items():
        if t is None:
            continue
        if not t.is_cuda:
            raise TabedError(f"{name} must live on the GPU")
        if device is not None and t.device != device:
            raise TabedError(f"{name} is on {t.device}, other operands on {device}")
        device = t.device
    return device.index


def _stream_on(device, stream):
    import torch
    if stream is None:
        return torch.cuda.current_stream(device).cuda_stream
    if stream.device.index != device:
        raise TabedError(f"the stream belongs to {stream.device}, the tensors to cuda:{device}")
    return stream.cuda_stream


def _storage_type(t, name):
    import torch
    if t.dtype == torch.float32:
        return 0
    if t.dtype == torch.bfloat16:
        return 1
    raise TabedError(f"{name} must be float32 or bfloat16, got {t.dtype}")


def _matrix(t, rows, cols, name, dtype=None):
    """(pointer, row stride) of a [rows, cols] view whose columns lie side by side (either size may be None: any)."""
    if t is None:
        return None, 0
    if t.dim() != 2 or (rows is not None and t.shape[0] != rows) or (cols is not None and t.shape[1] != cols):
        raise TabedError(f"{name} must be [{'rows' if rows is None else rows}, {'columns' if cols is None else cols}], got {tuple(t.shape)}")
    if dtype is not None and t.dtype != dtype:
        raise TabedError(f"{name} must be {dtype}, got {t.dtype}")
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise TabedError(f"{name}: the values of a row must lie side by side")
    stride = t.stride(0) if t.shape[0] > 1 else t.shape[1]
    if stride < t.shape[1]:
        raise TabedError(f"{name}: rows overlap")
    return t.data_ptr(), stride


def _prepare_norm_q8(x, q, scale, delta, sum_out, gain, eps, stream):
    import torch
    dev = _device_of(dict(x=x, q=q, scale=scale, delta=delta, sum_out=sum_out, gain=gain))
    xp, ldx = _matrix(x, None, None, "x")
    rows, d = x.shape
    xt = _storage_type(x, "x")
    dp, ldd = _matrix(delta, rows, d, "delta")
    sp, lds = _matrix(sum_out, rows, d, "sum_out", x.dtype)
    qp, ldq = _matrix(q, rows, d, "q", torch.int8)
    args = [rows, d, xt, xp, ldx, 0 if delta is None else _storage_type(delta, "delta"), dp, ldd, sp, lds,
            _ptr(gain, torch.float32, d, "gain"), eps, qp, ldq, _ptr(scale, torch.float32, rows, "scale"), _stream_on(dev, stream)]
    return DeviceCall(load().tabed_norm_q8, args, "tabed_norm_q8", dev, (x, q, scale, delta, sum_out, gain))


def tabed_norm_q8(x, q, scale, delta=None, sum_out=None, gain=None, eps=1e-5, stream=None):
    """Residual addition, RMSNorm, int8 rows with a scale each: sum_out = x + delta, q * scale ~ rms_norm(x + delta) * gain; without
    a gain the rows are quantised as they are.  x, delta, sum_out: [rows, d] views with their own row strides; sum_out may be x."""
    _prepare_norm_q8(x, q, scale, delta, sum_out, gain, eps, stream)()


def prepare_norm_q8(x, q, scale, delta=None, sum_out=None, gain=None, eps=1e-5, stream=None) -> PreparedCall:
    return _prepare_norm_q8(x, q, scale, delta, sum_out, gain, eps, stream)


def _prepare_linear_q8(x, x_scale, w, w_scale, y, stream):
    import torch
    dev = _device_of(dict(x=x, x_scale=x_scale, w=w, w_scale=w_scale, y=y))
    xp, ldx = _matrix(x, None, None, "x", torch.int8)
    M, K = x.shape
    if w.dim() != 2 or w.shape[1] != K:
        raise TabedError(f"w must be [N, {K}], got {tuple(w.shape)}")
    N = w.shape[0]
    yp, ldy = _matrix(y, M, N, "y")
    args = [M, N, K, xp, ldx, _ptr(x_scale, torch.float32, M, "x_scale"), _ptr(w, torch.int8, N * K, "w"),
            _ptr(w_scale, torch.float32, N, "w_scale"), _storage_type(y, "y"), yp, ldy, _stream_on(dev, stream)]
    return DeviceCall(load().tabed_linear_q8, args, "tabed_linear_q8", dev, (x, x_scale, w, w_scale, y))


def tabed_linear_q8(x, x_scale, w, w_scale, y, stream=None):
    """y [M, N] = (x [M, K] @ w [N, K].T) * x_scale[:, None] * w_scale, x and w int8, the sum exact."""
    _prepare_linear_q8(x, x_scale, w, w_scale, y, stream)()


def prepare_linear_q8(x, x_scale, w, w_scale, y, stream=None) -> PreparedCall:
    return _prepare_linear_q8(x, x_scale, w, w_scale, y, stream)


class CacheQ8:
    """8-bit key / value cache over tensors of the caller's: k, v [blocks, kv_heads, 64 * head_dim] int8, kscale, vscale
    [blocks, kv_heads] fp32, table [rows, max_blocks] int32 (entries outside [0, blocks): no block); for a body of several layers with
    a leading dimension `layers`, one table for all.  The struct holds the tensors' addresses: the object keeps them alive."""

    def __init__(self, k, v, kscale, vscale, table, head_dim):
        import torch
        self.device = _device_of(dict(k=k, v=v, kscale=kscale, vscale=vscale, table=table))
        if k.dim() not in (3, 4) or k.shape[-1] != CACHE_BLOCK * head_dim:
            raise TabedError(f"k must be [(layers,) blocks, kv_heads, {CACHE_BLOCK * head_dim}], got {tuple(k.shape)}")
        if table.dim() != 2:
            raise TabedError("table must be [rows, max_blocks]")
        blocks, kvh = k.shape[-3:-1]
        if max(blocks, kvh, table.shape[0], table.shape[1]) >= 1 << 31:
            raise TabedError("a cache's sizes must fit 32 bits")
        self.layers = k.shape[0] if k.dim() == 4 else 1
        self.rows, self.head_dim, self.kv_heads = table.shape[0], head_dim, kvh
        self.k, self.v, self.kscale, self.vscale, self.table = k, v, kscale, vscale, table
        self.struct = TabedCacheQ8(kvh, head_dim, blocks, table.shape[1], _ptr(k, torch.int8, None, "k"), _ptr(v, torch.int8, k.numel(), "v"),
                                   _ptr(kscale, torch.float32, self.layers * blocks * kvh, "kscale"),
                                   _ptr(vscale, torch.float32, self.layers * blocks * kvh, "vscale"),
                                   _ptr(table, torch.int32, None, "table"))

    @classmethod
    def allocate(cls, rows, tokens, kv_heads, head_dim, layers=None, device="cuda:0"):
        """An empty cache with room for `tokens` tokens in every row, blocks dealt to the rows in order."""
        import torch
        width = (tokens + CACHE_BLOCK - 1) // CACHE_BLOCK
        lead = () if layers is None else (layers,)
        k = torch.zeros((*lead, rows * width, kv_heads, CACHE_BLOCK * head_dim), dtype=torch.int8, device=device)
        ks = torch.zeros((*lead, rows * width, kv_heads), dtype=torch.float32, device=device)
        table = torch.arange(rows * width, dtype=torch.int32, device=device).view(rows, width)
        return cls(k, torch.zeros_like(k), ks, torch.zeros_like(ks), table, head_dim)


def _heads_view(t, rows, T, heads, hd, name):
    """(pointer, row stride, token stride) of [rows, T, heads, hd] (or [rows, heads * hd] where T is 1), a token's heads side by side."""
    if t.dim() == 2 and T == 1:
        t = t.unsqueeze(1)
    if t.dim() == 4:
        if t.shape[2:] != (heads, hd) or (heads > 1 and t.stride(2) != hd):
            raise TabedError(f"{name}: a token's {heads} heads of {hd} must lie side by side, got {tuple(t.shape)}, strides {t.stride()}")
    elif t.dim() != 3 or t.shape[2] != heads * hd:
        raise TabedError(f"{name} must be [{rows}, {T}, {heads}, {hd}], got {tuple(t.shape)}")
    if t.shape[:2] != (rows, T) or t.stride(-1) != 1:
        raise TabedError(f"{name} must be [{rows}, {T}, {heads}, {hd}] with values side by side, got {tuple(t.shape)}, strides {t.stride()}")
    tok = t.stride(1) if T > 1 else heads * hd               # (a stride that leads nowhere does not count)
    row = t.stride(0) if rows > 1 else T * tok
    if tok < heads * hd or row < heads * hd or (rows > 1 and T > 1 and min(row, tok) * (T if tok < row else rows) > max(row, tok)):
        raise TabedError(f"{name}: tokens overlap")
    return t.data_ptr(), row, tok


def _new_tokens(t, heads, hd):
    return 1 if t.dim() == 2 else t.shape[1]


def _prepare_cache_append_q8(cache, k, v, ctx_len, n_new, stream):
    import torch
    _one_layer(cache, "tabed_cache_append_q8")
    dev = _device_of({"cache": cache.k, "k": k, "v": v, "ctx_len": ctx_len, "n_new": n_new})
    T = _new_tokens(k, cache.kv_heads, cache.head_dim)
    kp, row, tok = _heads_view(k, cache.rows, T, cache.kv_heads, cache.head_dim, "k")
    vp_, vrow, vtok = _heads_view(v, cache.rows, T, cache.kv_heads, cache.head_dim, "v")
    if (row, tok) != (vrow, vtok) or k.dtype != v.dtype:
        raise TabedError("k and v must have the same type and strides")
    args = [C.byref(cache.struct), cache.rows, T, _storage_type(k, "k"), kp, vp_, row, tok, _ptr(ctx_len, torch.int32, cache.rows, "ctx_len"),
            _ptr(n_new, torch.int32, cache.rows, "n_new"), _stream_on(dev, stream)]
    return DeviceCall(load().tabed_cache_append_q8, args, "tabed_cache_append_q8", dev, (cache, k, v, ctx_len, n_new))


def tabed_cache_append_q8(cache: CacheQ8, k, v, ctx_len, n_new=None, stream=None):
    """Quantises k, v [rows, T, kv_heads, head_dim] into the cache at positions ctx_len[r] + t, t < n_new[r] (None: T)."""
    _prepare_cache_append_q8(cache, k, v, ctx_len, n_new, stream)()


def prepare_cache_append_q8(cache: CacheQ8, k, v, ctx_len, n_new=None, stream=None) -> PreparedCall:
    return _prepare_cache_append_q8(cache, k, v, ctx_len, n_new, stream)


def tabed_attention_q8_workspace_bytes(cache: CacheQ8, rows, T, q_heads) -> int:
    return int(load().tabed_attention_q8_workspace_bytes(C.byref(cache.struct), rows, T, q_heads))


def tabed_attention_q8_workspace_init(cache: CacheQ8, rows, T, q_heads, ws, stream=None):
    import torch
    dev = _device_of(dict(cache=cache.k, ws=ws))
    need = tabed_attention_q8_workspace_bytes(cache, rows, T, q_heads)
    if need == 0 or ws.numel() * ws.element_size() < need:
        raise TabedError(f"attention workspace holds {ws.numel() * ws.element_size()} bytes, {need} needed (0: invalid sizes)")
    with torch.cuda.device(dev):
        _check(load().tabed_attention_q8_workspace_init(C.byref(cache.struct), rows, T, q_heads, _ptr(ws, torch.uint8, None, "ws"),
                                                        _stream_on(dev, stream)), "tabed_attention_q8_workspace_init")


def new_attention_workspace(cache: CacheQ8, rows, T, q_heads, stream=None):
    """Allocate (torch) and prepare the workspace of tabed_attention_q8 for these sizes, or others that need no more bytes."""
    import torch
    nbytes = tabed_attention_q8_workspace_bytes(cache, rows, T, q_heads)
    if nbytes == 0:
        raise TabedError("invalid or unsupported attention sizes")
    ws = torch.empty(nbytes, dtype=torch.uint8, device=cache.k.device)
    tabed_attention_q8_workspace_init(cache, rows, T, q_heads, ws, stream)
    return ws


def _prepare_attention_q8(cache, ws, q, ctx_len, out, n_new, scale, lse, stream):
    import torch
    _one_layer(cache, "tabed_attention_q8")
    dev = _device_of(dict(cache=cache.k, ws=ws, q=q, ctx_len=ctx_len, out=out, n_new=n_new, lse=lse))
    hd = cache.head_dim
    T = _new_tokens(q, None, hd)
    heads = q.shape[2] if q.dim() == 4 else q.shape[-1] // hd
    qp, qrow, qtok = _heads_view(q, cache.rows, T, heads, hd, "q")
    op, orow, otok = _heads_view(out, cache.rows, T, heads, hd, "out")
    need = tabed_attention_q8_workspace_bytes(cache, cache.rows, T, heads)
    if ws.numel() * ws.element_size() < need:
        raise TabedError(f"attention workspace holds {ws.numel() * ws.element_size()} bytes, {need} needed")
    args = [C.byref(cache.struct), _ptr(ws, torch.uint8, None, "ws"), cache.rows, T, heads, _storage_type(q, "q"), qp, qrow, qtok,
            _ptr(ctx_len, torch.int32, cache.rows, "ctx_len"), _ptr(n_new, torch.int32, cache.rows, "n_new"),
            hd ** -0.5 if scale is None else scale, _storage_type(out, "out"), op, orow, otok,
            _ptr(lse, torch.float32, cache.rows * T * heads, "lse"), _stream_on(dev, stream)]
    return DeviceCall(load().tabed_attention_q8, args, "tabed_attention_q8", dev, (cache, ws, q, ctx_len, out, n_new, lse))


def tabed_attention_q8(cache: CacheQ8, ws, q, ctx_len, out, n_new=None, scale=None, lse=None, stream=None):
    """out [rows, T, q_heads, head_dim]: causal attention of q over the cache; token t sees positions up to ctx_len[r] + t, which
    tabed_cache_append_q8 has filled.  scale: 1 / sqrt(head_dim) unless given; lse [rows, T, q_heads]: optional."""
    _prepare_attention_q8(cache, ws, q, ctx_len, out, n_new, scale, lse, stream)()


def prepare_attention_q8(cache: CacheQ8, ws, q, ctx_len, out, n_new=None, scale=None, lse=None, stream=None) -> PreparedCall:
    return _prepare_attention_q8(cache, ws, q, ctx_len, out, n_new, scale, lse, stream)


def _one_layer(cache, what):
    if cache.layers != 1:
        raise TabedError(f"{what} takes the cache of one layer, this one has {cache.layers}")


def _prepare_draft_step_q8(cfg, ws, rnd, pos, W, w_scale, H, h_scale, weights, temperature, draft_logits, draft_lse, draft_tokens,
                           draft_q, flags, u_draft, stream):
    import torch
    V, d, n, B, g = cfg.V, cfg.d, cfg.n, cfg.B, cfg.gamma
    dev = _device_of(dict(ws=ws, W=W, w_scale=w_scale, H=H, h_scale=h_scale, weights=weights, temperature=temperature, draft_logits=draft_logits,
                          draft_lse=draft_lse, draft_tokens=draft_tokens, draft_q=draft_q, flags=flags, u_draft=u_draft))
    vp = C.c_void_p
    args = [C.byref(cfg), vp(_ptr(ws, torch.uint8, name="ws")), C.c_uint64(rnd), C.c_int32(pos), vp(_ptr(W, torch.int8, V * d, "W")),
            vp(_ptr(w_scale, torch.float32, V, "w_scale")), vp(_ptr(H, torch.int8, B * n * d, "H")),
            vp(_ptr(h_scale, torch.float32, B * n, "h_scale")), vp(_ptr(weights, torch.float32, B * n, "weights")),
            vp(_ptr(temperature, torch.float32, B, "temperature")), vp(_ptr(u_draft, torch.float32, B * g, "u_draft")),
            vp(_ptr(draft_logits, torch.float32, g * B * n * V, "draft_logits")), vp(_ptr(draft_lse, torch.float64, g * B * n, "draft_lse")),
            vp(_ptr(draft_tokens, torch.int32, B * g, "draft_tokens")), vp(_ptr(draft_q, torch.float32, B * g, "draft_q")),
            vp(_ptr(flags, torch.uint8, B * g, "flags")), vp(_stream_on(dev, stream))]
    call = DeviceCall(load().tabed_draft_step_q8, args, "tabed_draft_step_q8", dev,
                      (cfg, ws, W, w_scale, H, h_scale, weights, temperature, u_draft, draft_logits, draft_lse, draft_tokens, draft_q, flags))
    call.round_arg = args[2]
    return call


def tabed_draft_step_q8(cfg, ws, rnd, pos, W, w_scale, H, h_scale, weights, temperature, draft_logits, draft_lse, draft_tokens,
                        draft_q, flags, u_draft=None, stream=None):
    """tabed_draft_step with int8 W and H and their scales (see tabed_norm_q8)."""
    _prepare_draft_step_q8(cfg, ws, rnd, pos, W, w_scale, H, h_scale, weights, temperature, draft_logits, draft_lse, draft_tokens, draft_q,
                           flags, u_draft, stream)()


def quantize_rows(x, stream=None):
    """(int8 rows, scales) of a [rows, d] bf16 or fp32 matrix: how an LM head or other weights are laid out, once, for the 8-bit products."""
    import torch
    q = torch.empty(x.shape, dtype=torch.int8, device=x.device)
    scale = torch.empty(x.shape[0], dtype=torch.float32, device=x.device)
    tabed_norm_q8(x, q, scale, stream=stream)
    return q, scale


def tabed_body_q8_workspace_bytes(bcfg, cache, rows) -> int:
    return int(load().tabed_body_q8_workspace_bytes(C.byref(bcfg), C.byref(cache.struct), rows))


def tabed_body_q8_workspace_init(bcfg, cache, rows, ws, stream=None):
    import torch
    dev = _device_of(dict(cache=cache.k, ws=ws))
    need = tabed_body_q8_workspace_bytes(bcfg, cache, rows)
    if need == 0 or ws.numel() * ws.element_size() < need:
        raise TabedError(f"body workspace holds {ws.numel() * ws.element_size()} bytes, {need} needed (0: invalid sizes)")
    with torch.cuda.device(dev):
        _check(load().tabed_body_q8_workspace_init(C.byref(bcfg), C.byref(cache.struct), rows, _ptr(ws, torch.uint8, None, "ws"), _stream_on(dev, stream)),
               "tabed_body_q8_workspace_init")


def _prepare_draft_body_step_q8(bcfg, weights, ws, rows, token_src, token_stride, rows_per_token, ctx_len, cache, H, H8, h_scale, stream):
    import torch
    base, off = token_src if isinstance(token_src, tuple) else (token_src, 0)
    need = off + ((rows - 1) // rows_per_token) * token_stride + 1
    if base.dtype != torch.int32 or not base.is_cuda or not base.is_contiguous() or base.numel() < need or off < 0:
        raise TabedError("token_src must be a contiguous int32 GPU tensor covering every token read")
    dev = _device_of(dict(cache=cache.k, ws=ws, token_src=base, ctx_len=ctx_len, H=H, H8=H8, h_scale=h_scale))
    if cache.rows != rows or cache.layers != bcfg.layers:
        raise TabedError(f"the cache is of {cache.rows} rows and {cache.layers} layers, the step of {rows} and {bcfg.layers}")
    if ws.numel() * ws.element_size() < tabed_body_q8_workspace_bytes(bcfg, cache, rows):
        raise TabedError("body workspace too small")
    if H is not None and H.dtype not in (torch.bfloat16, torch.int16, torch.uint16):
        raise TabedError(f"H must hold bf16 values, got {H.dtype}")
    vp = C.c_void_p
    args = [C.byref(bcfg), C.byref(weights), vp(_ptr(ws, torch.uint8, name="ws")), C.c_int32(rows), vp(base.data_ptr() + 4 * off),
            C.c_int32(token_stride), C.c_int32(rows_per_token), vp(_ptr(ctx_len, torch.int32, rows, "ctx_len")), C.byref(cache.struct),
            vp(_ptr(H, None, rows * bcfg.d, "H")), vp(_ptr(H8, torch.int8, rows * bcfg.d, "H8")), vp(_ptr(h_scale, torch.float32, rows, "h_scale")),
            vp(_stream_on(dev, stream))]
    return DeviceCall(load().tabed_draft_body_step_q8, args, "tabed_draft_body_step_q8", dev, (bcfg, weights, ws, base, ctx_len, cache, H, H8, h_scale))


def tabed_draft_body_step_q8(bcfg, weights, ws, rows, token_src, token_stride, rows_per_token, ctx_len, cache, H=None, H8=None, h_scale=None,
                             stream=None):
    """tabed_draft_body_step over an 8-bit cache (CacheQ8 with `layers`), writing H (bf16), H8 and h_scale (int8), or all three.  Faster from about
    32 rows on; with fewer it saves memory, not time."""
    _prepare_draft_body_step_q8(bcfg, weights, ws, rows, token_src, token_stride, rows_per_token, ctx_len, cache, H, H8, h_scale, stream)()


# ------------------------------------------------------------------ trees given by parents
MAX_NODES = 256


class CachePaged:
    """Paged key / value cache over tensors of the caller's: k, v [(layers,) blocks, kv_heads, 64, head_dim] bfloat16 or float8_e4m3fn, of the same
    strides, with the values of a token in a head side by side; for e4m3 kscale, vscale [(layers,) blocks, kv_heads, 64] fp32; table
    [rows, max_blocks] int32, one for all layers (entries outside [0, blocks): no block).  The struct holds the tensors' addresses: the object keeps them alive."""

    def __init__(self, k, v, table, kscale=None, vscale=None):
        import torch
        self.device = _device_of(dict(k=k, v=v, kscale=kscale, vscale=vscale, table=table))
        if k.dim() not in (4, 5) or k.shape[-2] != CACHE_BLOCK:
            raise TabedError(f"k must be [(layers,) blocks, kv_heads, {CACHE_BLOCK}, head_dim], got {tuple(k.shape)}")
        types = {torch.bfloat16: 1, torch.float8_e4m3fn: 2}
        if k.dtype not in types:
            raise TabedError(f"k must be bfloat16 or float8_e4m3fn, got {k.dtype}")
        if v.dtype != k.dtype or v.shape != k.shape or table.dim() != 2:
            raise TabedError("v must have the type and shape of k, table must be [rows, max_blocks]")
        if any(n > 1 and x != y for n, x, y in zip(k.shape, k.stride(), v.stride())):
            raise TabedError("k and v must have the same strides")
        kind, k5 = types[k.dtype], k if k.dim() == 5 else k[None]
        if 0 in k5.shape or 0 in table.shape or max(*k5.shape, *table.shape) >= 1 << 31:
            raise TabedError("a cache's sizes must not be 0, and fit 32 bits")
        layers, blocks, kvh, _, hd = k5.shape
        if hd > 1 and k5.stride(4) != 1:
            raise TabedError("k and v: the values of a token in a head must lie side by side")
        # Strides that lead nowhere do not count; the others must keep entries apart.
        strides, reach = [0] * 4, hd
        for i in sorted((i for i in range(4) if k5.shape[i] > 1), key=lambda i: k5.stride(i)):
            if k5.stride(i) < reach:
                raise TabedError("k and v: entries overlap")
            strides[i], reach = k5.stride(i), k5.stride(i) * k5.shape[i]
        piece = 16 // k.element_size()
        strides = [x if x else (hd + piece - 1) // piece * piece for x in strides]
        if (kscale is None) != (vscale is None) or (kscale is None) != (kind == 1):
            raise TabedError("kscale and vscale go with e4m3, and with it alone")
        self.layers, self.rows, self.kv_heads, self.head_dim = layers, table.shape[0], kvh, hd
        self.k, self.v, self.kscale, self.vscale, self.table = k, v, kscale, vscale, table
        count = layers * blocks * kvh * CACHE_BLOCK
        self.struct = TabedCachePaged(layers, kvh, hd, blocks, table.shape[1], kind, *strides, k.data_ptr(), v.data_ptr(),
                                      _ptr(kscale, torch.float32, count, "kscale"), _ptr(vscale, torch.float32, count, "vscale"),
                                      _ptr(table, torch.int32, None, "table"))

    @classmethod
    def allocate(cls, rows, tokens, kv_heads, head_dim, layers=1, dtype=None, device="cuda:0"):
        """An empty cache with room for `tokens` tokens in every row, blocks dealt to the rows in order; dtype: bfloat16 (None) or float8_e4m3fn."""
        import torch
        dtype = torch.bfloat16 if dtype is None else dtype
        width = (tokens + CACHE_BLOCK - 1) // CACHE_BLOCK
        k = torch.zeros((layers, rows * width, kv_heads, CACHE_BLOCK, head_dim), dtype=dtype, device=device)
        ks = torch.zeros(k.shape[:-1], dtype=torch.float32, device=device) if dtype != torch.bfloat16 else None
        table = torch.arange(rows * width, dtype=torch.int32, device=device).view(rows, width)
        return cls(k, torch.zeros_like(k), table, ks, None if ks is None else torch.zeros_like(ks))

    @classmethod
    def of_body(cls, kcache, vcache, heads):
        """The caches of tabed_draft_body_step, [layers, rows, max_ctx, d] with max_ctx a multiple of 64, seen as a paged one."""
        import torch
        if kcache.dim() != 4 or kcache.shape[2] % CACHE_BLOCK or kcache.shape[3] % heads or not kcache.is_contiguous() or not vcache.is_contiguous():
            raise TabedError(f"kcache and vcache must be contiguous [layers, rows, max_ctx, d], max_ctx a multiple of {CACHE_BLOCK}, got {tuple(kcache.shape)}")
        layers, rows, ctx, d = kcache.shape
        k, v = (x.view(layers, rows * ctx // CACHE_BLOCK, CACHE_BLOCK, heads, d // heads).transpose(2, 3) for x in (kcache, vcache))
        table = torch.arange(rows * ctx // CACHE_BLOCK, dtype=torch.int32, device=kcache.device).view(rows, ctx // CACHE_BLOCK)
        return cls(k, v, table)


def _tree_args(rows, N, parents, n_nodes):
    import torch
    if parents is not None and tuple(parents.shape) != (rows, N):
        raise TabedError(f"parents must be [{rows}, {N}], got {tuple(parents.shape)}")
    return _ptr(parents, torch.int32, rows * N, "parents"), _ptr(n_nodes, torch.int32, rows, "n_nodes")


def _prepare_cache_append_nodes(cache, k, v, ctx_len, parents, n_nodes, q, q_out, rope_theta, layer, stream):
    import torch
    dev = _device_of({"cache": cache.k, "k": k, "v": v, "ctx_len": ctx_len, "parents": parents, "n_nodes": n_nodes, "q": q, "q_out": q_out})
    hd = cache.head_dim
    N = _new_tokens(k, cache.kv_heads, hd)
    kp, row, tok = _heads_view(k, cache.rows, N, cache.kv_heads, hd, "k")
    vp_, vrow, vtok = _heads_view(v, cache.rows, N, cache.kv_heads, hd, "v")
    if (row, tok) != (vrow, vtok) or k.dtype != v.dtype:
        raise TabedError("k and v must have the same type and strides")
    heads, qp, qrow, qtok, op, orow, otok = 0, None, 0, 0, None, 0, 0
    if (q is None) != (q_out is None):
        raise TabedError("q and q_out go together")
    if q is not None:
        heads = q.shape[2] if q.dim() == 4 else q.shape[-1] // hd
        if q.dtype != k.dtype or q_out.dtype != torch.bfloat16:
            raise TabedError("q must have the type of k, q_out must be bfloat16")
        qp, qrow, qtok = _heads_view(q, cache.rows, N, heads, hd, "q")
        op, orow, otok = _heads_view(q_out, cache.rows, N, heads, hd, "q_out")
    pp, np_ = _tree_args(cache.rows, N, parents, n_nodes)
    args = [C.byref(cache.struct), layer, cache.rows, N, _storage_type(k, "k"), kp, vp_, row, tok, heads, qp, qrow, qtok, op, orow, otok,
            _ptr(ctx_len, torch.int32, cache.rows, "ctx_len"), pp, np_, rope_theta, _stream_on(dev, stream)]
    return DeviceCall(load().tabed_cache_append_nodes, args, "tabed_cache_append_nodes", dev, (cache, k, v, ctx_len, parents, n_nodes, q, q_out))


def tabed_cache_append_nodes(cache: CachePaged, k, v, ctx_len, parents=None, n_nodes=None, q=None, q_out=None, rope_theta=0.0, layer=0, stream=None):
    """Writes k, v [rows, N, kv_heads, head_dim] of a tree's nodes into the cache at positions ctx_len[r] + j, turned (with rope_theta > 0) by
    ctx_len[r] + the node's depth, and q [rows, N, q_heads, head_dim], turned likewise, to q_out (bfloat16).  parents [rows, N] (None: chains), n_nodes [rows]."""
    _prepare_cache_append_nodes(cache, k, v, ctx_len, parents, n_nodes, q, q_out, rope_theta, layer, stream)()


def prepare_cache_append_nodes(cache: CachePaged, k, v, ctx_len, parents=None, n_nodes=None, q=None, q_out=None, rope_theta=0.0, layer=0,
                               stream=None) -> PreparedCall:
    return _prepare_cache_append_nodes(cache, k, v, ctx_len, parents, n_nodes, q, q_out, rope_theta, layer, stream)


def tabed_attention_nodes_workspace_bytes(cache: CachePaged, rows, N, q_heads) -> int:
    return int(load().tabed_attention_nodes_workspace_bytes(C.byref(cache.struct), rows, N, q_heads))


def tabed_attention_nodes_workspace_init(cache: CachePaged, rows, N, q_heads, ws, stream=None):
    import torch
    dev = _device_of(dict(cache=cache.k, ws=ws))
    need = tabed_attention_nodes_workspace_bytes(cache, rows, N, q_heads)
    if need == 0 or ws.numel() * ws.element_size() < need:
        raise TabedError(f"attention workspace holds {ws.numel() * ws.element_size()} bytes, {need} needed (0: invalid sizes)")
    with torch.cuda.device(dev):
        _check(load().tabed_attention_nodes_workspace_init(C.byref(cache.struct), rows, N, q_heads, _ptr(ws, torch.uint8, None, "ws"),
                                                           _stream_on(dev, stream)), "tabed_attention_nodes_workspace_init")


def new_attention_nodes_workspace(cache: CachePaged, rows, N, q_heads, stream=None):
    """Allocate (torch) and prepare the workspace of tabed_attention_nodes for these sizes, or others that need no more bytes."""
    import torch
    nbytes = tabed_attention_nodes_workspace_bytes(cache, rows, N, q_heads)
    if nbytes == 0:
        raise TabedError("invalid or unsupported attention sizes")
    ws = torch.empty(nbytes, dtype=torch.uint8, device=cache.k.device)
    tabed_attention_nodes_workspace_init(cache, rows, N, q_heads, ws, stream)
    return ws


def _prepare_attention_nodes(cache, ws, q, ctx_len, out, parents, n_nodes, scale, lse, layer, stream):
    import torch
    dev = _device_of(dict(cache=cache.k, ws=ws, q=q, ctx_len=ctx_len, out=out, parents=parents, n_nodes=n_nodes, lse=lse))
    hd = cache.head_dim
    N = _new_tokens(q, None, hd)
    heads = q.shape[2] if q.dim() == 4 else q.shape[-1] // hd
    if q.dtype != torch.bfloat16 or out.dtype != torch.bfloat16:
        raise TabedError(f"q and out must be bfloat16, got {q.dtype}, {out.dtype}")
    qp, qrow, qtok = _heads_view(q, cache.rows, N, heads, hd, "q")
    op, orow, otok = _heads_view(out, cache.rows, N, heads, hd, "out")
    need = tabed_attention_nodes_workspace_bytes(cache, cache.rows, N, heads)
    if ws.numel() * ws.element_size() < need:
        raise TabedError(f"attention workspace holds {ws.numel() * ws.element_size()} bytes, {need} needed")
    pp, np_ = _tree_args(cache.rows, N, parents, n_nodes)
    args = [C.byref(cache.struct), layer, _ptr(ws, torch.uint8, None, "ws"), cache.rows, N, heads, qp, qrow, qtok,
            _ptr(ctx_len, torch.int32, cache.rows, "ctx_len"), pp, np_, hd ** -0.5 if scale is None else scale, op, orow, otok,
            _ptr(lse, torch.float32, cache.rows * N * heads, "lse"), _stream_on(dev, stream)]
    return DeviceCall(load().tabed_attention_nodes, args, "tabed_attention_nodes", dev, (cache, ws, q, ctx_len, out, parents, n_nodes, lse))


def tabed_attention_nodes(cache: CachePaged, ws, q, ctx_len, out, parents=None, n_nodes=None, scale=None, lse=None, layer=0, stream=None):
    """out [rows, N, q_heads, head_dim]: attention of a tree's nodes over the cache: node j sees the positions before ctx_len[r], the nodes above it and
    itself, which tabed_cache_append_nodes has written.  scale: 1 / sqrt(head_dim) unless given; lse [rows, N, q_heads]: optional."""
    _prepare_attention_nodes(cache, ws, q, ctx_len, out, parents, n_nodes, scale, lse, layer, stream)()


def prepare_attention_nodes(cache: CachePaged, ws, q, ctx_len, out, parents=None, n_nodes=None, scale=None, lse=None, layer=0, stream=None) -> PreparedCall:
    return _prepare_attention_nodes(cache, ws, q, ctx_len, out, parents, n_nodes, scale, lse, layer, stream)


def tabed_verify_nodes_workspace_bytes(cfg: TabedCfg, N) -> int:
    return int(load().tabed_verify_nodes_workspace_bytes(C.byref(cfg), N))


def tabed_verify_nodes_workspace_init(cfg: TabedCfg, N, ws, stream=None):
    import torch
    dev = _device_of(dict(ws=ws))
    need = tabed_verify_nodes_workspace_bytes(cfg, N)
    if need == 0 or ws.numel() * ws.element_size() < need:
        raise TabedError(f"verification workspace holds {ws.numel() * ws.element_size()} bytes, {need} needed (0: invalid sizes)")
    with torch.cuda.device(dev):
        _check(load().tabed_verify_nodes_workspace_init(C.byref(cfg), N, _ptr(ws, torch.uint8, None, "ws"), _stream_on(dev, stream)),
               "tabed_verify_nodes_workspace_init")


def new_verify_nodes_workspace(cfg: TabedCfg, N, device="cuda:0", stream=None):
    """Allocate (torch) and prepare the workspace of tabed_verify_nodes for these sizes, or others that need no more bytes."""
    import torch
    nbytes = tabed_verify_nodes_workspace_bytes(cfg, N)
    if nbytes == 0:
        raise TabedError("invalid or unsupported verification sizes")
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    tabed_verify_nodes_workspace_init(cfg, N, ws, stream)
    return ws


def _prepare_verify_nodes(cfg, ws, rnd, target_logits, draft_logits, draft_lse, tokens, node_q, weights, temperature, path, n_path, out_tokens, flags,
                          parents, n_nodes, u_acc, u_res, dev, n_valid, stream):
    import torch
    index = _device_of(dict(ws=ws, target_logits=target_logits, draft_logits=draft_logits, draft_lse=draft_lse, tokens=tokens, node_q=node_q, weights=weights,
                            temperature=temperature, path=path, n_path=n_path, out_tokens=out_tokens, flags=flags, parents=parents, n_nodes=n_nodes,
                            u_acc=u_acc, u_res=u_res, dev=dev, n_valid=n_valid))
    if tokens.dim() != 2 or tokens.shape[0] != cfg.B:
        raise TabedError(f"tokens must be [{cfg.B}, N], got {tuple(tokens.shape)}")
    B, N, V, n = cfg.B, tokens.shape[1], cfg.V, cfg.n
    slots = draft_logits.shape[0]                        # (slots behind the last node with children may be missing)
    if tuple(draft_logits.shape) != (slots, B, n, V) or tuple(draft_lse.shape) != (slots, B, n) or not (slots >= N or (parents is None and slots == N - 1)):
        raise TabedError(f"draft_logits and draft_lse must be [{N}, {B}, {n}, {V}] and [{N}, {B}, {n}], got {tuple(draft_logits.shape)}, {tuple(draft_lse.shape)}")
    need = tabed_verify_nodes_workspace_bytes(cfg, N)
    if ws.numel() * ws.element_size() < need:
        raise TabedError(f"verification workspace holds {ws.numel() * ws.element_size()} bytes, {need} needed")
    f, i = torch.float32, torch.int32
    pp, np_ = _tree_args(B, N, parents, n_nodes)
    vp = C.c_void_p
    args = [C.byref(cfg), vp(_ptr(ws, torch.uint8, None, "ws")), C.c_uint64(rnd), C.c_int32(N), vp(_ptr(target_logits, f, B * N * V, "target_logits")),
            vp(_ptr(draft_logits, f, None, "draft_logits")), vp(_ptr(draft_lse, torch.float64, None, "draft_lse")), vp(_ptr(tokens, i, B * N, "tokens")),
            vp(_ptr(node_q, f, B * N, "node_q")), vp(pp), vp(np_), vp(_ptr(weights, f, B * n, "weights")), vp(_ptr(temperature, f, B, "temperature")),
            vp(_ptr(u_acc, f, B * N, "u_acc")), vp(_ptr(u_res, f, B, "u_res")), vp(_ptr(path, i, B * N, "path")), vp(_ptr(n_path, i, B, "n_path")),
            vp(_ptr(out_tokens, i, B * N, "out_tokens")), vp(_ptr(flags, torch.uint8, B * N, "flags")), vp(_ptr(dev, f, B * cfg.gamma * n, "dev")),
            vp(_ptr(n_valid, i, B, "n_valid")), vp(_stream_on(index, stream))]
    call = DeviceCall(load().tabed_verify_nodes, args, "tabed_verify_nodes", index,
                      (cfg, ws, target_logits, draft_logits, draft_lse, tokens, node_q, weights, temperature, path, n_path, out_tokens, flags, parents,
                       n_nodes, u_acc, u_res, dev, n_valid))
    call.round_arg = args[2]
    return call


def tabed_verify_nodes(cfg, ws, rnd, target_logits, draft_logits, draft_lse, tokens, node_q, weights, temperature, path, n_path, out_tokens, flags,
                       parents=None, n_nodes=None, u_acc=None, u_res=None, dev=None, n_valid=None, stream=None):
    """Verification of a tree of drafted tokens by multi-round rejection sampling: target_logits [B, N, V], draft_logits [N, B, n, V] and draft_lse [N, B, n]
    as the draft steps write them, tokens and node_q [B, N].  path, out_tokens, flags [B, N], n_path [B]; dev [B, gamma, n] and n_valid [B] for tabed_update_weights."""
    _prepare_verify_nodes(cfg, ws, rnd, target_logits, draft_logits, draft_lse, tokens, node_q, weights, temperature, path, n_path, out_tokens, flags,
                          parents, n_nodes, u_acc, u_res, dev, n_valid, stream)()


def prepare_verify_nodes(cfg, ws, rnd, target_logits, draft_logits, draft_lse, tokens, node_q, weights, temperature, path, n_path, out_tokens, flags,
                         parents=None, n_nodes=None, u_acc=None, u_res=None, dev=None, n_valid=None, stream=None) -> PreparedCall:
    return _prepare_verify_nodes(cfg, ws, rnd, target_logits, draft_logits, draft_lse, tokens, node_q, weights, temperature, path, n_path, out_tokens, flags,
                                 parents, n_nodes, u_acc, u_res, dev, n_valid, stream)


def _prepare_cache_keep_nodes(cache, ctx_base, path, n_path, ctx_len, stream):
    import torch
    dev = _device_of(dict(cache=cache.k, ctx_base=ctx_base, path=path, n_path=n_path, ctx_len=ctx_len))
    if path.dim() != 2 or path.shape[0] != cache.rows:
        raise TabedError(f"path must be [{cache.rows}, N], got {tuple(path.shape)}")
    N = path.shape[1]
    args = [C.byref(cache.struct), cache.rows, N, _ptr(ctx_base, torch.int32, cache.rows, "ctx_base"), _ptr(path, torch.int32, cache.rows * N, "path"),
            _ptr(n_path, torch.int32, cache.rows, "n_path"), _ptr(ctx_len, torch.int32, cache.rows, "ctx_len"), _stream_on(dev, stream)]
    return DeviceCall(load().tabed_cache_keep_nodes, args, "tabed_cache_keep_nodes", dev, (cache, ctx_base, path, n_path, ctx_len))


def tabed_cache_keep_nodes(cache: CachePaged, ctx_base, path, n_path, ctx_len, stream=None):
    """After verification: in all layers the entries of positions ctx_base[r] + path[r][i] move to ctx_base[r] + i, i < n_path[r]; ctx_len[r] becomes
    ctx_base[r] + their number."""
    _prepare_cache_keep_nodes(cache, ctx_base, path, n_path, ctx_len, stream)()


def prepare_cache_keep_nodes(cache: CachePaged, ctx_base, path, n_path, ctx_len, stream=None) -> PreparedCall:
    return _prepare_cache_keep_nodes(cache, ctx_base, path, n_path, ctx_len, stream)


class BodyBuffers:
    """Device buffers of the draft-model body for `rows` rows (allocation only; no arithmetic here): weight table,
    scratch, key / value caches, positions and the hidden states H the LM head reads."""

    def __init__(self, bcfg: TabedBodyCfg, rows: int, tensors: dict, device="cuda:0"):
        import torch
        self.cfg, self.rows, self.tensors = bcfg, rows, tensors
        self.table = make_body_weights(bcfg, tensors)
        need = tabed_body_workspace_bytes(bcfg, rows)
        if need == 0:
            raise TabedError("invalid body configuration")
        self.ws = torch.empty(need, dtype=torch.uint8, device=device)
        tabed_body_workspace_init(bcfg, rows, self.ws)
        self.kcache = torch.zeros((bcfg.layers, rows, bcfg.max_ctx, bcfg.d), dtype=torch.bfloat16, device=device)
        self.vcache = torch.zeros_like(self.kcache)
        self.ctx_len = torch.zeros(rows, dtype=torch.int32, device=device)
        self.ctx_base = torch.zeros(rows, dtype=torch.int32, device=device)
        self.H = torch.zeros((rows, bcfg.d), dtype=torch.bfloat16, device=device)

    def prepare_step(self, token_src, token_offset, token_stride, rows_per_token, stream=None) -> PreparedCall:
        import torch
        need = token_offset + ((self.rows - 1) // rows_per_token) * token_stride + 1
        if token_src.dtype != torch.int32 or not token_src.is_cuda or not token_src.is_contiguous() or token_src.numel() < need:
            raise TabedError("token_src must be a contiguous int32 GPU tensor covering every token read")
        vp = C.c_void_p
        args = [C.byref(self.cfg), C.byref(self.table), vp(self.ws.data_ptr()), C.c_int32(self.rows),
                vp(token_src.data_ptr() + 4 * token_offset), C.c_int32(token_stride), C.c_int32(rows_per_token),
                vp(self.ctx_len.data_ptr()), vp(self.kcache.data_ptr()), vp(self.vcache.data_ptr()), vp(self.H.data_ptr()),
                vp(_stream(stream))]
        return PreparedCall(load().tabed_draft_body_step, args, "tabed_draft_body_step")

    def prepare_rollback(self, rows_per_seq, gamma, accept_len, stream=None) -> PreparedCall:
        import torch
        vp = C.c_void_p
        nseq = (self.rows + rows_per_seq - 1) // rows_per_seq
        args = [C.c_int32(self.rows), C.c_int32(rows_per_seq), C.c_int32(gamma), vp(self.ctx_base.data_ptr()),
                vp(_ptr(accept_len, torch.int32, nseq, "accept_len")), vp(self.ctx_len.data_ptr()), vp(_stream(stream))]
        return PreparedCall(load().tabed_draft_body_rollback, args, "tabed_draft_body_rollback")


class BodyBuffersQ8:
    """BodyBuffers over an 8-bit cache: weight table, scratch, cache of max_ctx tokens a row, positions, hidden states in int8."""

    def __init__(self, bcfg: TabedBodyCfg, rows: int, tensors: dict, device="cuda:0"):
        import torch
        self.cfg, self.rows, self.tensors = bcfg, rows, tensors
        self.table = make_body_weights(bcfg, tensors)
        self.cache = CacheQ8.allocate(rows, bcfg.max_ctx, bcfg.heads, bcfg.d // bcfg.heads, bcfg.layers, device)
        need = tabed_body_q8_workspace_bytes(bcfg, self.cache, rows)
        if need == 0:
            raise TabedError("invalid body configuration")
        self.ws = torch.empty(need, dtype=torch.uint8, device=device)
        tabed_body_q8_workspace_init(bcfg, self.cache, rows, self.ws)
        self.ctx_len = torch.zeros(rows, dtype=torch.int32, device=device)
        self.ctx_base = torch.zeros(rows, dtype=torch.int32, device=device)
        self.H8 = torch.zeros((rows, bcfg.d), dtype=torch.int8, device=device)
        self.h_scale = torch.zeros(rows, dtype=torch.float32, device=device)

    def prepare_step(self, token_src, token_offset, token_stride, rows_per_token, stream=None) -> PreparedCall:
        return _prepare_draft_body_step_q8(self.cfg, self.table, self.ws, self.rows, (token_src, token_offset), token_stride, rows_per_token,
                                           self.ctx_len, self.cache, None, self.H8, self.h_scale, stream)

    prepare_rollback = BodyBuffers.prepare_rollback


class RoundBuffers:
    """Device buffers one sequence batch needs across rounds (allocation only; no arithmetic here)."""

    def __init__(self, cfg: TabedCfg, device="cuda:0"):
        import torch
        V, n, B, g, h = cfg.V, cfg.n, cfg.B, cfg.gamma, cfg.h
        z = lambda shape, dt: torch.zeros(shape, dtype=dt, device=device)
        self.cfg = cfg
        self.ws = new_workspace(cfg, device)
        dw = tabed_dev_width(cfg)
        self.weights = z((B, n), torch.float32)
        self.ring = z((B, max(h, 1), dw), torch.float32)      # h = 0: window ALL keeps one running sum
        self.ring_head = z((B,), torch.int32)
        self.ring_count = z((B,), torch.int32)
        self.draft_logits = z((g, B, n, V), torch.float32)
        self.draft_lse = z((g, B, n), torch.float64)
        self.draft_tokens = z((B, g), torch.int32)
        self.draft_q = z((B, g), torch.float32)
        self.draft_flags = z((B, g), torch.uint8)
        self.accept_len = z((B,), torch.int32)
        self.out_tokens = z((B, g + 1), torch.int32)
        self.dev = z((B, g, dw), torch.float32)
        self.n_valid = z((B,), torch.int32)
        self.verify_flags = z((B, g + 1), torch.uint8)

    # ---- token tree: sibling candidates and the walk's extra outputs
    def enable_tree(self, width: int):
        import torch
        c = self.cfg
        S = width - 1
        dev = self.weights.device
        self.tree_width = width
        self.sib_tokens = torch.zeros((c.B, c.gamma, S), dtype=torch.int32, device=dev)
        self.sib_q = torch.zeros((c.B, c.gamma, S), dtype=torch.float32, device=dev)
        self.sib_flags = torch.zeros((c.B, c.gamma, S), dtype=torch.uint8, device=dev)
        self.leaf = torch.zeros((c.B,), dtype=torch.int32, device=dev)
        self.n_out = torch.zeros((c.B,), dtype=torch.int32, device=dev)

    def prepare_draft_siblings(self, rnd, pos, temperature, stream=None) -> "PreparedCall":
        import torch
        c = self.cfg
        vp = C.c_void_p
        args = [C.byref(c), vp(self.ws.data_ptr()), C.c_uint64(rnd), C.c_int32(pos), C.c_int32(self.tree_width),
                vp(self.draft_logits.data_ptr()), vp(self.draft_tokens.data_ptr()), vp(self.weights.data_ptr()),
                vp(_ptr(temperature, torch.float32, c.B, "temperature")), vp(None),
                vp(self.sib_tokens.data_ptr()), vp(self.sib_q.data_ptr()), vp(self.sib_flags.data_ptr()),
                vp(_stream(stream))]
        return PreparedCall(load().tabed_draft_siblings, args, "tabed_draft_siblings", args[2])

    def prepare_verify_tree(self, rnd, target_logits, leaf_logits, temperature, stream=None) -> "PreparedCall":
        """The window update stays a separate call here (next_weights may not alias weights in tabed_verify_tree)."""
        import torch
        c = self.cfg
        vp = C.c_void_p
        S = self.tree_width - 1
        args = [C.byref(c), vp(self.ws.data_ptr()), C.c_uint64(rnd), C.c_int32(self.tree_width),
                vp(_ptr(target_logits, torch.float32, c.B * (c.gamma + 1) * c.V, "target_logits")),
                vp(_ptr(leaf_logits, torch.float32, c.B * c.gamma * S * c.V, "leaf_logits")),
                vp(self.draft_logits.data_ptr()), vp(self.draft_lse.data_ptr()), vp(self.draft_tokens.data_ptr()),
                vp(self.draft_q.data_ptr()), vp(self.sib_tokens.data_ptr()), vp(self.sib_q.data_ptr()),
                vp(self.weights.data_ptr()), vp(_ptr(temperature, torch.float32, c.B, "temperature")),
                vp(None), vp(None), vp(None),
                vp(self.accept_len.data_ptr()), vp(self.out_tokens.data_ptr()), vp(self.dev.data_ptr()),
                vp(self.n_valid.data_ptr()), vp(self.verify_flags.data_ptr()), vp(self.leaf.data_ptr()),
                vp(self.n_out.data_ptr()), vp(None), vp(None), vp(None), vp(None), vp(_stream(stream))]
        return PreparedCall(load().tabed_verify_tree, args, "tabed_verify_tree", args[2])

    # ---- the same three calls with arguments converted once (hot loops)
    def prepare_update_weights(self, first: bool, rnd=0, stream=None) -> PreparedCall:
        import torch
        c = self.cfg
        vp = C.c_void_p
        args = [C.byref(c), vp(self.ws.data_ptr()), C.c_uint64(rnd),
                vp(None if first else self.dev.data_ptr()), vp(None if first else self.n_valid.data_ptr()),
                vp(self.ring.data_ptr()), vp(self.ring_head.data_ptr()), vp(self.ring_count.data_ptr()),
                vp(self.weights.data_ptr()), vp(_stream(stream))]
        return PreparedCall(load().tabed_update_weights, args, "tabed_update_weights", args[2])

    def prepare_draft_step(self, rnd, pos, W, H, temperature, u_draft=None, stream=None) -> PreparedCall:
        import torch
        c = self.cfg
        sd = _store_dtype(c)
        vp = C.c_void_p
        args = [C.byref(c), vp(self.ws.data_ptr()), C.c_uint64(rnd), C.c_int32(pos),
                vp(_ptr(W, sd, c.V * c.d, "W")), vp(_ptr(H, sd, c.B * c.n * c.d, "H")),
                vp(self.weights.data_ptr()), vp(_ptr(temperature, torch.float32, c.B, "temperature")),
                vp(_ptr(u_draft, torch.float32, c.B * c.gamma, "u_draft")),
                vp(self.draft_logits.data_ptr()), vp(self.draft_lse.data_ptr()), vp(self.draft_tokens.data_ptr()),
                vp(self.draft_q.data_ptr()), vp(self.draft_flags.data_ptr()), vp(_stream(stream))]
        return PreparedCall(load().tabed_draft_step, args, "tabed_draft_step", args[2])

    def prepare_draft_step_q8(self, rnd, pos, W, w_scale, H, h_scale, temperature, u_draft=None, stream=None) -> PreparedCall:
        return _prepare_draft_step_q8(self.cfg, self.ws, rnd, pos, W, w_scale, H, h_scale, self.weights, temperature, self.draft_logits,
                                      self.draft_lse, self.draft_tokens, self.draft_q, self.draft_flags, u_draft, stream)

    def prepare_verify(self, rnd, target_logits, temperature, u_acc=None, u_res=None, stream=None,
                       fused_update=False) -> PreparedCall:
        import torch
        c = self.cfg
        vp = C.c_void_p
        args = [C.byref(c), vp(self.ws.data_ptr()), C.c_uint64(rnd),
                vp(_ptr(target_logits, torch.float32, c.B * (c.gamma + 1) * c.V, "target_logits")),
                vp(self.draft_logits.data_ptr()), vp(self.draft_lse.data_ptr()), vp(self.draft_tokens.data_ptr()),
                vp(self.draft_q.data_ptr()), vp(self.weights.data_ptr()),
                vp(_ptr(temperature, torch.float32, c.B, "temperature")),
                vp(_ptr(u_acc, torch.float32, c.B * c.gamma, "u_acc")), vp(_ptr(u_res, torch.float32, c.B, "u_res")),
                vp(self.accept_len.data_ptr()), vp(self.out_tokens.data_ptr()), vp(self.dev.data_ptr()),
                vp(self.n_valid.data_ptr()), vp(self.verify_flags.data_ptr()),
                vp(self.ring.data_ptr() if fused_update else None), vp(self.ring_head.data_ptr() if fused_update else None),
                vp(self.ring_count.data_ptr() if fused_update else None),
                vp(self.weights.data_ptr() if fused_update else None), vp(_stream(stream))]
        return PreparedCall(load().tabed_verify, args, "tabed_verify", args[2])

    def update_weights(self, first: bool, rnd=0, stream=None):
        tabed_update_weights(self.cfg, self.ws, rnd, None if first else self.dev, None if first else self.n_valid,
                             self.ring, self.ring_head, self.ring_count, self.weights, stream)

    def draft_step(self, rnd, pos, W, H, temperature, u_draft=None, stream=None):
        tabed_draft_step(self.cfg, self.ws, rnd, pos, W, H, self.weights, temperature, self.draft_logits,
                         self.draft_lse, self.draft_tokens, self.draft_q, self.draft_flags, u_draft, stream)

    def verify(self, rnd, target_logits, temperature, u_acc=None, u_res=None, stream=None, fused_update=False):
        """fused_update: the call also opens the next round (window push + next weights, in place)."""
        w = dict(ring=self.ring, ring_head=self.ring_head, ring_count=self.ring_count,
                 next_weights=self.weights) if fused_update else {}
        tabed_verify(self.cfg, self.ws, rnd, target_logits, self.draft_logits, self.draft_lse, self.draft_tokens,
                     self.draft_q, self.weights, temperature, self.accept_len, self.out_tokens, self.dev,
                     self.n_valid, self.verify_flags, u_acc, u_res, stream=stream, **w)
