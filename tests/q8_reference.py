"""Plain definitions of the 8-bit operators for the tests, on the CPU: numpy / torch in 64 bits, or, where the definition fixes every
rounding (appending to the cache), in fp32 step by step."""
import math

import numpy as np
import torch

BLOCK = 64
TINY = np.float32(2.0 ** -100)


def half_step(dtype):
    """Largest relative error of one rounding to the type."""
    return torch.finfo(dtype).eps / 2


# ------------------------------------------------------------------ norm
def norm(x, delta, gain, eps):
    """(r, y, scale) in 64 bits."""
    r = x.double() + (0 if delta is None else delta.double())
    y = r
    if gain is not None:
        y = r / torch.sqrt(r.pow(2).mean(1, keepdim=True) + eps) * gain.double()
    most = y.abs().amax(1)
    return r, y, torch.where(most >= float(TINY), most / 127, torch.zeros_like(most))


# ------------------------------------------------------------------ the cache's layout, element by element
def key_at(tok, dim, hd):
    return (((tok // 4 % 4) * (hd // 16) + dim // 16) * 16 + tok // 16 * 4 + tok % 4) * 16 + dim % 16


def value_at(tok, dim, hd):
    return ((dim // 16 * 4 + tok // 16) * 16 + dim % 16) * 16 + tok % 16


def layout(which, hd):
    """Index [64, hd] into a block's bytes."""
    tok, dim = np.arange(BLOCK)[:, None], np.arange(hd)[None, :]
    return key_at(tok, dim, hd) if which == "k" else value_at(tok, dim, hd)


def fp32_scale(most):
    return np.float32(np.nan) if not np.isfinite(most) else (np.float32(most) / np.float32(127) if most >= TINY else np.float32(0))


def steps(x, s):
    if not s > 0:
        return np.zeros(x.shape, np.int8)
    return np.clip(np.rint(x.astype(np.float32) / np.float32(s)), -127, 127).astype(np.int8)


def append(pool, scales, table, which, new, ctx, n_new, hd):
    """pool [blocks, kv_heads, 64 hd] int8 and scales [blocks, kv_heads] fp32, changed in place; new [rows, T, kv_heads, hd] fp32."""
    where = layout(which, hd)
    blocks, kvh = scales.shape
    rows, T = new.shape[:2]
    for r in range(rows):
        n = T if n_new is None else min(max(int(n_new[r]), 0), T)
        at, end = max(int(ctx[r]), 0), max(int(ctx[r]), 0) + n
        first = at
        while at < end:
            slot, off = divmod(at, BLOCK)
            count = min(BLOCK - off, end - at)
            if slot >= table.shape[1]:
                break
            page = int(table[r, slot])
            if 0 <= page < blocks:
                for h in range(kvh):
                    x = new[r, at - first:at - first + count, h].astype(np.float32)
                    with np.errstate(invalid="ignore"):
                        most = np.float32(np.nan) if not np.isfinite(x).all() else np.abs(x).max()
                    fresh, before = fp32_scale(most), scales[page, h] if off else np.float32(0)
                    s = np.float32(np.nan) if np.isnan(fresh) or np.isnan(before) else max(fresh, before)
                    block = pool[page, h][where]
                    if off and s != before:
                        kept = block[:off].astype(np.float32) * before if s > 0 else np.zeros((off, hd), np.float32)
                        block[:off] = steps(kept, s)
                    block[off:off + count] = steps(x, s)
                    pool[page, h][where] = block
                    scales[page, h] = s
            at += count


# ------------------------------------------------------------------ attention
def attention(pools, scales, table, q, ctx, n_new, scale, hd):
    """(out, lse, bound) in 64 bits; tokens from n_new on hold NaN.  pools, scales: {"k", "v"}; q [rows, T, q_heads, hd].

    bound [rows, T, q_heads]: how far the kernel may be from `out`, by counting its roundings in half steps of fp32 (2^-24).  A score is at most
    four integers, exact, that are rounded to fp32, scaled by a product of four roundings, and added: at most 10 half steps of A = sum_d (|q_d| +
    max|q| 2^-7) |k_d| * scale (a digit's share can exceed its value by the balanced digits' carry, 1/128 of the next one).  The integers
    themselves stand for q to half a unit of max|q| / 0x7f7f78: one half step of B = max|q| sum_d |k_d| * scale.  The exponent is
    rounded once for the maximum (|m| + 14) and once for the result (|s - m| + 14, which matters only while exp2 of it does: |s - m| 2^-|s - m| < 1);
    exp2 is good to 2.  A probability is kept to 2^-22 (two halves of 11 bits; 4) and to 2^-31 of the largest one, so
    it is off by e = ln 2 * (10 A + B + |m| + 29) + 6, A, B, m in base 2.
    Sums of p and of p v run over at most the row's blocks, 64 terms and a chain each, plus joins (waves, ranges): blocks + 220 half steps
    of sum p |v|.  Scale of the value, division: 3 more."""
    rows, T, qh, _ = q.shape
    kvh = scales["k"].shape[1]
    group, u = qh // kvh, 2.0 ** -24
    out, lse = np.full((rows, T, qh, hd), np.nan), np.full((rows, T, qh), np.nan)
    bound = np.zeros((rows, T, qh))
    for r in range(rows):
        n = T if n_new is None else min(max(int(n_new[r]), 0), T)
        cap = table.shape[1] * BLOCK
        c = min(max(int(ctx[r]), 0), cap)
        held = [b for b in range(min(table.shape[1], (c + n + BLOCK - 1) // BLOCK)) if 0 <= table[r, b] < scales["k"].shape[0]]
        pos = np.array([b * BLOCK + i for b in held for i in range(BLOCK)], np.int64)
        for h in range(kvh):
            k, v = (np.concatenate([pools[n_][table[r, b], h][layout(n_, hd)].astype(np.float64) * float(scales[n_][table[r, b], h]) for b in held])
                    if held else np.zeros((0, hd)) for n_ in ("k", "v"))
            for t in range(n):
                seen = pos <= c + t
                for j in range(group):
                    i = h * group + j
                    if not seen.any():
                        out[r, t, i], lse[r, t, i] = 0, -math.inf
                        continue
                    qq = q[r, t, i].astype(np.float64)
                    s = k[seen] @ qq * scale
                    m = s.max()
                    p = np.exp(s - m)
                    out[r, t, i], lse[r, t, i] = p @ v[seen] / p.sum(), m + math.log(p.sum())
                    A = ((np.abs(qq) + np.abs(qq).max() / 128) @ np.abs(k[seen]).T).max() * scale / math.log(2)
                    B = np.abs(qq).max() * np.abs(k[seen]).sum(1).max() * scale / math.log(2)
                    e = math.log(2) * (10 * A + B + abs(m) / math.log(2) + 29) + 6
                    w = p @ np.abs(v[seen]) / p.sum()
                    lost = seen.sum() * 2.0 ** -31 / p.sum() * np.abs(v[seen]).max(0)
                    bound[r, t, i] = ((2 * e + 2 * (len(held) + 220) + 3) * u * w + lost).max()
    return out, lse, bound


# ------------------------------------------------------------------ the draft body over the 8-bit cache
def bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16).double().numpy()


def body_step(bc, w, caches, table, ctx, tokens):
    """One step for all rows in 64 bits with the kernels' storage points: bf16 for weights and whatever feeds a projection or the cache, int8
    for the cache (caches[l] = ({"k", "v"} bytes, {"k", "v"} scales), changed in place).  Returns the final norm's rows, not rounded."""
    rows, d, hd = len(ctx), bc.d, bc.d // bc.heads
    f = lambda bits: (bits.astype(np.uint32) << 16).view(np.float32).astype(np.float64)
    norm = lambda x, g: x / np.sqrt((x * x).mean(1, keepdims=True) + bc.rms_eps) * g
    x = f(w["embed"])[np.asarray(tokens)]
    freq = bc.rope_theta ** (-2.0 * np.arange(hd // 2) / hd)
    cos, sin = (fn(np.asarray(ctx)[:, None] * freq)[:, None, :] for fn in (np.cos, np.sin))

    def rotate(y):
        a, b = y[..., :hd // 2], y[..., hd // 2:]
        return np.concatenate([a * cos - b * sin, b * cos + a * sin], -1)

    for l in range(bc.layers):
        qkv = (bf16(norm(x, w["g_attn"][l])) @ f(w["wqkv"][l]).T).reshape(rows, 3, bc.heads, hd)
        q, k, v = rotate(qkv[:, 0]), bf16(rotate(qkv[:, 1])), bf16(qkv[:, 2])
        pools, scales = caches[l]
        for n, new in (("k", k), ("v", v)):
            append(pools[n], scales[n], table, n, new[:, None].astype(np.float32), ctx, None, hd)
        att, _, _ = attention(pools, scales, table, q[:, None], ctx, None, hd ** -0.5, hd)
        x = x + bf16(att[:, 0].reshape(rows, d)) @ f(w["wo"][l]).T
        gu = bf16(norm(x, w["g_mlp"][l])) @ f(w["wgu"][l]).T
        gate, up = gu[:, :bc.d_ff], gu[:, bc.d_ff:]
        x = x + bf16(gate / (1 + np.exp(-gate)) * up) @ f(w["wdown"][l]).T
    return norm(x, w["g_final"])
