"""Performance cases of the 8-bit operators of the draft model: what one decode step, or one prompt, asks of them.

Four kinds of case:

  norm     residual addition, RMSNorm and int8 rows with a scale each                     (binding.tabed_norm_q8)
  linear   int8 rows times int8 weights, scales for each row and each column              (binding.tabed_linear_q8)
  append   keys and values of new tokens into an int8 cache, a scale for each block of 64
           tokens and head; tokens kept in a begun block are rounded again when its scale
           grows                                                                          (binding.tabed_cache_append_q8)
  attn     causal attention of new tokens over such a cache                               (binding.tabed_attention_q8)

With `own` false `run` computes them in plain torch operations in 32 bits, else by the library's kernels.  What is held
in 8 bits is returned as the values it stands for.
"""
import math

import torch

own = False

DEV = "cuda:0"
BLOCK = 64                     # tokens of a cache block
EPS = 1e-5
TINY = 2.0 ** -100             # rows and blocks with no larger magnitude count as zeros
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


# ------------------------------------------------------------------ the cases
def _norm(name, rows, d, x="fp32", delta="none"):
    return {"name": name, "kind": "norm", "rows": rows, "d": d, "x": x, "delta": delta}


def _linear(name, M, N, K, y="fp32"):
    return {"name": name, "kind": "linear", "M": M, "N": N, "K": K, "y": y}


def _append(name, rows, T, kv_heads, hd, ctx_lo, ctx_hi, kv="bf16", ragged=False):
    return {"name": name, "kind": "append", "rows": rows, "T": T, "kv_heads": kv_heads, "hd": hd, "ctx_lo": ctx_lo, "ctx_hi": ctx_hi,
            "kv": kv, "ragged": ragged}


def _attn(name, rows, T, q_heads, kv_heads, hd, ctx_lo, ctx_hi, q="bf16", out="bf16", ragged=False, holes=False):
    return {"name": name, "kind": "attn", "rows": rows, "T": T, "q_heads": q_heads, "kv_heads": kv_heads, "hd": hd, "ctx_lo": ctx_lo,
            "ctx_hi": ctx_hi, "q": q, "out": out, "ragged": ragged, "holes": holes}


def listed():
    return [
        # final norm of one sequence's four drafting methods, on the way to the LM head: latency alone counts
        _norm("norm_single", 4, 768),
        # a layer's norm over the tokens of several prompts
        _norm("norm_prompt", 8192, 4096, x="bf16", delta="bf16"),
        # sizes nobody rounded: a hidden size that is no multiple of 8, rows of a few requests
        _norm("norm_ragged", 333, 2051, x="bf16", delta="fp32"),
        # LM head of one sequence's four drafting methods
        _linear("linear_single", 4, 32000, 768),
        # LM head of the batched-serving configuration
        _linear("linear_serving", 64, 32000, 768),
        # LM head of the largest batch: eight methods, 64 sequences
        _linear("linear_large", 512, 128256, 2048),
        # a projection over the tokens of several prompts, odd numbers of them and of columns
        _linear("linear_prompt", 3967, 8190, 4096, y="bf16"),
        # a decode step's key and value of every row of the serving configuration
        _append("append_step", 64, 1, 12, 64, 256, 768),
        # prompts of several lengths, behind a shared beginning that ends inside a block
        _append("append_prompt", 16, 1500, 8, 128, 0, 200, ragged=True),
        # decode step of the serving configuration: a few hundred tokens of context a row
        _attn("attn_serving", 64, 1, 12, 12, 64, 256, 768, q="fp32"),
        # one request with a long context, grouped heads
        _attn("attn_long", 1, 1, 32, 8, 128, 120_011, 120_011),
        # verification of a drafted block: up to six tokens a row at once, some rows with fewer, grouped heads
        _attn("attn_verify", 16, 6, 32, 8, 128, 300, 5000, out="fp32", ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "linear", "linear", "append", "attn", "attn", "attn"])
    if kind == "norm":
        while True:
            rows, d = _log_int(rng, 1, 16384), _log_int(rng, 64, 8192)
            d = max(1, d // rng.choice([1, 8, 64])) * rng.choice([1, 8, 64])
            if 64 <= d <= 8192 and rows * d <= 2 ** 24:
                return {"kind": kind, "rows": rows, "d": d, "x": rng.choice(["fp32", "bf16"]), "delta": rng.choice(["none", "fp32", "bf16"])}
    if kind == "linear":
        while True:
            M, N = _log_int(rng, 1, 8192), _log_int(rng, 64, 152064)
            K = 16 * _log_int(rng, 4, 512) if rng.random() < 0.4 else rng.choice([512, 768, 896, 1024, 2048, 4096])
            if M * N * K <= 512 * 128256 * 2048 and M * N <= 512 * 128256:
                return {"kind": kind, "M": M, "N": N, "K": K, "y": rng.choice(["fp32", "bf16"])}
    hd = rng.choice([32, 64, 64, 96, 128, 128, 256])
    kv_heads = _log_int(rng, 1, 16)
    if kind == "append":
        while True:
            rows, T, ctx = _log_int(rng, 1, 256), rng.choice([1, 1, rng.randint(2, 8), _log_int(rng, 9, 2000)]), _log_int(rng, 1, 3000)
            if rows * (T + 2 * BLOCK) * kv_heads * hd <= 16 * 1700 * 8 * 128 and rows * (T + ctx) * kv_heads * hd <= 2 ** 26:
                return {"kind": kind, "rows": rows, "T": T, "kv_heads": kv_heads, "hd": hd, "ctx_lo": 0, "ctx_hi": ctx,
                        "kv": rng.choice(["fp32", "bf16"]), "ragged": T > 1 and rng.random() < 0.7}
    while True:
        rows, group = _log_int(rng, 1, 128), rng.choice([1, 1, 2, 3, 4, 7, 8])
        T, hi = rng.choice([1, 1, rng.randint(2, 8), rng.randint(9, 33)]), _log_int(rng, 1, 120_000)
        lo = rng.choice([0, hi // 3, hi])
        if rows * (hi + T) * kv_heads * hd <= 120_011 * 8 * 128 // 2 and rows * (hi + T) * T * group * kv_heads <= 2 ** 28:
            return {"kind": kind, "rows": rows, "T": T, "q_heads": group * kv_heads, "kv_heads": kv_heads, "hd": hd, "ctx_lo": lo,
                    "ctx_hi": hi, "q": rng.choice(["fp32", "bf16"]), "out": rng.choice(["fp32", "bf16"]),
                    "ragged": T > 1 and rng.random() < 0.5, "holes": rng.random() < 0.15}


# ------------------------------------------------------------------ the cache's blocks
# A block of one head holds 64 tokens.  Keys: [token / 4 % 4][dim / 16][token / 16][token % 4][dim % 16]; values:
# [dim / 16][token / 16][dim % 16][token % 16]; a byte each.
def _keys_in(x):               # [..., 64, hd] -> [..., 64 * hd]
    hd = x.shape[-1]
    return x.unflatten(-2, (4, 4, 4)).unflatten(-1, (hd // 16, 16)).movedim((-4, -2, -5, -3), (-5, -4, -3, -2)).flatten(-5)


def _keys_out(x, hd):          # the way back
    return x.unflatten(-1, (4, hd // 16, 4, 4, 16)).movedim((-3, -5, -2, -4), (-5, -4, -3, -2)).flatten(-5, -3).flatten(-2)


def _values_in(x):
    hd = x.shape[-1]
    return x.unflatten(-2, (4, 16)).unflatten(-1, (hd // 16, 16)).movedim((-2, -4, -1, -3), (-4, -3, -2, -1)).flatten(-4)


def _values_out(x, hd):
    return x.unflatten(-1, (hd // 16, 4, 16, 16)).movedim((-3, -1, -4, -2), (-4, -3, -2, -1)).flatten(-4, -3).flatten(-2)


def _steps(x, s):
    """x in steps of s, rounded to whole ones of at most 127; where s is 0 there are none."""
    return torch.where(s > 0, torch.round(x / torch.where(s > 0, s, torch.ones_like(s))).clamp(-127, 127), torch.zeros_like(x))


def _scale(most):
    return torch.where(most >= TINY, most / 127, torch.zeros_like(most))


# ------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(1_000_003 * seed + 29)


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


def _lengths(g, lo, hi, n):
    return torch.randint(lo, hi + 1, (n,), generator=g, device=DEV, dtype=torch.int32)


def _int8(g, rows, cols):
    """Rows quantised to their largest magnitude, as weights and activations are; made in parts."""
    q, s = torch.empty((rows, cols), dtype=torch.int8, device=DEV), torch.empty(rows, device=DEV)
    part = max(1, 2 ** 26 // cols)
    for at in range(0, rows, part):
        x = _randn(g, min(part, rows - at), cols)
        most = x.abs().amax(1)
        q[at:at + part] = torch.round(x * (127 / most)[:, None]).to(torch.int8)
        s[at:at + part] = most * (0.02 / 127)
    return q, s


def _new_tokens(c, g):
    if not c["ragged"]:
        return torch.full((c["rows"],), c["T"], dtype=torch.int32, device=DEV)
    return _lengths(g, 0, c["T"], c["rows"])


def _pool(c, g):
    """Blocks for the rows' contexts and new tokens, in no order, and the rows' tables."""
    rows, kvh, hd = c["rows"], c["kv_heads"], c["hd"]
    width = (c["ctx_hi"] + c["T"] + BLOCK - 1) // BLOCK
    need = rows * width
    order = torch.randperm(need, generator=g, device=DEV, dtype=torch.int32)
    table = order.view(rows, width).clone()
    st = {"table": table}
    for name, turn in (("k", _keys_in), ("v", _values_in)):
        q, s = torch.empty((need, kvh, BLOCK * hd), dtype=torch.int8, device=DEV), torch.empty((need, kvh), device=DEV)
        part = max(1, 2 ** 25 // (kvh * BLOCK * hd))
        spread = torch.exp(0.5 * _randn(g, kvh, 1, hd))              # some dimensions are larger than others
        for at in range(0, need, part):
            x = _randn(g, min(part, need - at), kvh, BLOCK, hd) * spread
            s[at:at + part] = x.abs().amax((-1, -2)) / 127
            q[at:at + part] = turn(torch.round(x / s[at:at + part, :, None, None]).to(torch.int8))
        st[name], st[name + "scale"] = q, s
    return st


def _inputs(c, seed):
    g = _gen(seed)
    if c["kind"] == "norm":
        st = {"x": (_randn(g, c["rows"], c["d"]) * torch.exp(0.5 * _randn(g, c["d"]))).to(TYPES[c["x"]]), "gain": 1 + 0.1 * _randn(g, c["d"])}
        st["delta"] = None if c["delta"] == "none" else (0.3 * _randn(g, c["rows"], c["d"])).to(TYPES[c["delta"]])
        return st
    if c["kind"] == "linear":
        (x, sx), (w, sw) = _int8(g, c["M"], c["K"]), _int8(g, c["N"], c["K"])
        return {"x": x, "sx": sx, "w": w, "sw": sw}
    ctx = _lengths(g, c["ctx_lo"], c["ctx_hi"], c["rows"])
    st = {"ctx": ctx, "new": _new_tokens(c, g), **_pool(c, g)}
    if c["kind"] == "append":
        for name in ("nk", "nv"):
            st[name] = (1.3 * _randn(g, c["rows"], c["T"], c["kv_heads"], c["hd"])).to(TYPES[c["kv"]])
        return st
    st["q"] = (1.5 * _randn(g, c["rows"], c["T"], c["q_heads"], c["hd"])).to(TYPES[c["q"]])
    full = (ctx // BLOCK)
    if c["rows"] > 1:                                                # row 2 i + 1 begins with a third of the full blocks of row 2 i
        shared = torch.minimum(full[0::2][:len(full[1::2])], full[1::2]) // 3
        at = torch.arange(st["table"].shape[1], device=DEV)[None, :]
        st["table"][1::2] = torch.where(at < shared[:, None], st["table"][0::2][:len(shared)], st["table"][1::2])
    if c["holes"]:                                                   # blocks given up: no table entry
        gone = torch.rand(st["table"].shape, generator=g, device=DEV) < 0.2
        gone[-1] = True
        st["table"] = torch.where(gone, -1, st["table"])
    return st


def prepare(c, seed):
    st = {"case": dict(c), **_inputs(c, seed)}
    if c["kind"] == "attn":
        st["out"] = torch.zeros((c["rows"], c["T"], c["q_heads"], c["hd"]), dtype=TYPES[c["out"]], device=DEV)
        st["lse"] = torch.zeros((c["rows"], c["T"], c["q_heads"]), device=DEV)
    if own:
        _plan(c, st)
    return st


def _plan(c, st):
    """Output buffers, workspace and the call with its arguments converted once, as a serving loop keeps them."""
    from paper_2601_20357_amd import binding as B
    if c["kind"] == "norm":
        st["sum"] = torch.empty_like(st["x"]) if st["delta"] is not None else None
        st["q"] = torch.empty((c["rows"], c["d"]), dtype=torch.int8, device=DEV)
        st["scale"] = torch.empty(c["rows"], device=DEV)
        st["values"] = torch.empty((c["rows"], c["d"]), dtype=torch.bfloat16, device=DEV)
        st["call"] = B.prepare_norm_q8(st["x"], st["q"], st["scale"], delta=st["delta"], sum_out=st["sum"], gain=st["gain"], eps=EPS)
    elif c["kind"] == "linear":
        st["y"] = torch.empty((c["M"], c["N"]), dtype=TYPES[c["y"]], device=DEV)
        st["call"] = B.prepare_linear_q8(st["x"], st["sx"], st["w"], st["sw"], st["y"])
    else:
        st["cache"] = B.CacheQ8(st["k"], st["v"], st["kscale"], st["vscale"], st["table"], head_dim=c["hd"])
        if c["kind"] == "append":
            st["kvalues"], st["vvalues"] = (torch.empty(st["k"].shape, dtype=torch.bfloat16, device=DEV) for _ in range(2))
            st["call"] = B.prepare_cache_append_q8(st["cache"], st["nk"], st["nv"], st["ctx"], n_new=st["new"])
        else:
            st["ws"] = B.new_attention_workspace(st["cache"], c["rows"], c["T"], c["q_heads"])
            st["call"] = B.prepare_attention_q8(st["cache"], st["ws"], st["q"], st["ctx"], st["out"], n_new=st["new"], lse=st["lse"])


# ------------------------------------------------------------------ one pass
def run(st):
    kind = st["case"]["kind"]
    if not own:
        return {"norm": _plain_norm, "linear": _plain_linear, "append": _plain_append, "attn": _plain_attn}[kind](st)
    st["call"]()
    if kind == "norm":
        torch.mul(st["q"], st["scale"][:, None], out=st["values"])
        out = {"values": st["values"], "scale": st["scale"]}
        return out if st["sum"] is None else {"sum": st["sum"], **out}
    if kind == "linear":
        return st["y"]
    if kind == "append":
        torch.mul(st["k"], st["kscale"][..., None], out=st["kvalues"])
        torch.mul(st["v"], st["vscale"][..., None], out=st["vvalues"])
        return {"k": st["kvalues"], "v": st["vvalues"], "kscale": st["kscale"], "vscale": st["vscale"]}
    return {"out": st["out"], "lse": st["lse"]}


def _plain_norm(st):
    r = st["x"].float()
    if st["delta"] is not None:
        r = r + st["delta"].float()
    y = r * torch.rsqrt((r * r).mean(1, keepdim=True) + EPS) * st["gain"]
    s = _scale(y.abs().amax(1, keepdim=True))
    out = {"values": (_steps(y, s) * s).to(torch.bfloat16), "scale": s[:, 0]}
    return out if st["delta"] is None else {"sum": r.to(st["x"].dtype), **out}


def _plain_linear(st):
    y = torch.mm(st["x"].float(), st["w"].float().t())
    return (y * st["sx"][:, None] * st["sw"][None, :]).to(TYPES[st["case"]["y"]])


def _plain_append(st):
    c, table, ctx = st["case"], st["table"].long(), st["ctx"].long()
    rows, hd, blocks, width = c["rows"], c["hd"], st["k"].shape[0], table.shape[1]
    nb = (c["T"] + BLOCK - 2) // BLOCK + 1                            # blocks that T tokens can touch
    slot = (ctx // BLOCK)[:, None] + torch.arange(nb, device=DEV)     # [rows, nb] of the table
    pos = slot[..., None] * BLOCK + torch.arange(BLOCK, device=DEV)   # [rows, nb, 64]
    t = pos - ctx[:, None, None]
    fresh = (t >= 0) & (t < st["new"][:, None, None])
    page = torch.where(fresh.any(2) & (slot < width), table.gather(1, slot.clamp(max=width - 1)), blocks)   # `blocks`: a block of no one
    page = torch.where(page < 0, blocks, page)
    at = (torch.arange(rows, device=DEV)[:, None, None], t.clamp(0, c["T"] - 1))
    kept = (t < 0)[:, :, None, :, None]
    out = {}
    for name, turn_in, turn_out in (("k", _keys_in, _keys_out), ("v", _values_in, _values_out)):
        pool, scales = (torch.cat([x, torch.zeros_like(x[:1])]) for x in (st[name], st[name + "scale"]))
        x = st["n" + name].float()[at].transpose(2, 3)                # [rows, nb, kv_heads, 64, hd]
        now = fresh[:, :, None, :, None]
        most = torch.where(now, x.abs(), torch.zeros_like(x)).amax((-1, -2))
        before = torch.where((t[:, :, 0] < 0)[..., None], scales[page], torch.zeros_like(most))
        s = torch.maximum(before, _scale(most))
        old = turn_out(pool[page], hd).float()
        wide = s[..., None, None]
        q = torch.where(now, _steps(x, wide), torch.where(kept, _steps(old * before[..., None, None], wide), old))
        pool[page], scales[page] = turn_in(q).to(torch.int8), s
        pool, scales = pool[:-1], scales[:-1].clone()
        out[name], out[name + "scale"] = (pool.float() * scales[..., None]).to(torch.bfloat16), scales
    return {n: out[n] for n in ("k", "v", "kscale", "vscale")}


def _plain_attn(st):
    c = st["case"]
    rows, T, kvh, hd, group = c["rows"], c["T"], c["kv_heads"], c["hd"], c["q_heads"] // c["kv_heads"]
    table = st["table"].long()
    page = table.clamp(min=0)
    k, v = (turn(st[n][page], hd).float() * st[n + "scale"][page][..., None, None] for n, turn in (("k", _keys_out), ("v", _values_out)))
    k, v = (x.transpose(1, 2).flatten(2, 3) for x in (k, v))          # [rows, kv_heads, tokens, hd]
    q = st["q"].float().view(rows, T, kvh, group, hd).permute(0, 2, 1, 3, 4).reshape(rows, kvh, T * group, hd)
    s = torch.matmul(q, k.transpose(2, 3).contiguous()) * (1 / math.sqrt(hd))
    pos = torch.arange(k.shape[2], device=DEV)
    seen = (pos <= (st["ctx"][:, None] + torch.arange(T, device=DEV))[..., None]) & (table >= 0).repeat_interleave(BLOCK, 1)[:, None, :]
    s = s.view(rows, kvh, T, group, -1).masked_fill(~seen[:, None, :, None, :], -math.inf)
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(m > -math.inf, m, torch.zeros_like(m)))
    z = p.sum(-1, keepdim=True)
    o = torch.matmul(p.flatten(2, 3), v.contiguous()).view(rows, kvh, T, group, hd) / torch.where(z > 0, z, torch.ones_like(z))
    lse = (m + torch.log(z))[..., 0]
    live = (torch.arange(T, device=DEV) < st["new"][:, None])[:, :, None]
    o = o.permute(0, 2, 1, 3, 4).reshape(rows, T, c["q_heads"], hd)
    lse = lse.permute(0, 2, 1, 3).reshape(rows, T, c["q_heads"])
    return {"out": torch.where(live[..., None], o.to(st["out"].dtype), st["out"]), "lse": torch.where(live, lse, st["lse"])}


# ------------------------------------------------------------------ what a pass cannot do without
def work(c):
    size = {"fp32": 4, "bf16": 2, "none": 0}
    if c["kind"] == "norm":
        n = c["rows"] * c["d"]
        kept = 0 if c["delta"] == "none" else size[c["x"]]
        return {"bytes": n * (size[c["x"]] + size[c["delta"]] + kept + 1) + 4 * (c["d"] + c["rows"]), "flops": 8 * n}
    if c["kind"] == "linear":
        M, N, K = c["M"], c["N"], c["K"]
        return {"bytes": M * K + N * K + M * N * size[c["y"]] + 4 * (M + N), "flops": 2 * M * N * K}
    part = 0.5 if c["ragged"] else 1.0
    head = c["rows"] * c["kv_heads"] * c["hd"]
    if c["kind"] == "append":
        new = part * head * c["T"]
        return {"bytes": int(2 * new * (size[c["kv"]] + 1)), "flops": int(6 * new)}
    ctx = (c["ctx_lo"] + c["ctx_hi"]) / 2
    queries = part * c["rows"] * c["T"] * c["q_heads"] * c["hd"]
    held = (0.8 if c["holes"] else 1.0) * head * (ctx + part * c["T"])
    return {"bytes": int(2 * held * (1 + 4 / (BLOCK * c["hd"])) + queries * (size[c["q"]] + size[c["out"]])),
            "flops": int(4 * queries * (ctx + part * c["T"] / 2))}


# ------------------------------------------------------------------ in 64 bits, from the definitions
def exact(c, seed):
    st = _inputs(c, seed)
    if c["kind"] == "norm":
        r = st["x"].double() + (0 if st["delta"] is None else st["delta"].double())
        y = r / (r.pow(2).sum(1, keepdim=True) / c["d"] + EPS).sqrt() * st["gain"].double()
        s = y.abs().max(1, keepdim=True).values / 127
        out = {"values": (y / s).round() * s, "scale": s.squeeze(1)}
        return out if st["delta"] is None else {"sum": r, **out}
    if c["kind"] == "linear":
        wt = (st["w"].double() * st["sw"].double().unsqueeze(1)).t().contiguous()
        return (st["x"].double() * st["sx"].double().unsqueeze(1)) @ wt
    ctx, new, table = st["ctx"].tolist(), st["new"].tolist(), st["table"].tolist()
    hd = c["hd"]
    tok, dim = torch.arange(BLOCK, device=DEV)[:, None], torch.arange(hd, device=DEV)[None, :]
    where = {"k": (((tok // 4 % 4) * (hd // 16) + dim // 16) * 16 + tok // 16 * 4 + tok % 4) * 16 + dim % 16,
             "v": ((dim // 16 * 4 + tok // 16) * 16 + dim % 16) * 16 + tok % 16}
    if c["kind"] == "append":
        if c["rows"] * c["T"] > 40_000 or c["rows"] * (c["T"] // BLOCK + 1) > 2000:
            return None
        out = {}
        for n in ("k", "v"):
            q, s = st[n].double(), st[n + "scale"].double()
            for r in range(c["rows"]):
                at = ctx[r]
                while at < ctx[r] + new[r]:
                    b, off = divmod(at, BLOCK)
                    count = min(BLOCK - off, ctx[r] + new[r] - at)
                    x = st["n" + n][r, at - ctx[r]:at - ctx[r] + count].double().transpose(0, 1)         # [kv_heads, count, hd]
                    page = table[r][b]
                    most = x.abs().amax((1, 2)) / 127
                    s_new = torch.maximum(most, s[page]) if off else most
                    block = q[page][:, where[n].flatten()].view(-1, BLOCK, hd).clone()
                    if off:
                        block[:, :off] = (block[:, :off] * s[page][:, None, None] / s_new[:, None, None]).round()
                    block[:, off:off + count] = (x / s_new[:, None, None]).round()
                    q[page][:, where[n].flatten()] = block.flatten(1)
                    s[page] = s_new
                    at += count
            out[n], out[n + "scale"] = q * s[..., None], s
        return {n: out[n] for n in ("k", "v", "kscale", "vscale")}
    group = c["q_heads"] // c["kv_heads"]
    out = torch.zeros((c["rows"], c["T"], c["q_heads"], hd), dtype=torch.float64, device=DEV)
    lse = torch.zeros(out.shape[:3], dtype=torch.float64, device=DEV)
    for r in range(c["rows"]):
        count = min(len(table[r]), (ctx[r] + new[r] + BLOCK - 1) // BLOCK)
        held = [b for b in range(count) if table[r][b] >= 0]
        pages = torch.tensor([table[r][b] for b in held], dtype=torch.long, device=DEV)
        pos = (torch.tensor(held, dtype=torch.long, device=DEV)[:, None] * BLOCK + torch.arange(BLOCK, device=DEV)).flatten()
        for h in range(c["kv_heads"]):
            k, v = ((st[n][pages, h].double() * st[n + "scale"][pages, h].double()[:, None])[:, where[n]].flatten(0, 1) for n in ("k", "v"))
            for t in range(new[r]):
                if not held:
                    lse[r, t, h * group:(h + 1) * group] = -math.inf
                    continue
                s = st["q"][r, t, h * group:(h + 1) * group].double() @ k.t() / math.sqrt(hd)
                s[:, pos > ctx[r] + t] = -math.inf
                lse[r, t, h * group:(h + 1) * group] = z = torch.logsumexp(s, 1)
                some = torch.isfinite(z)
                out[r, t, h * group:(h + 1) * group][some] = torch.exp(s[some] - z[some, None]) @ v
    return {"out": out, "lse": lse}
