"""Performance cases of the operators for a tree of drafted tokens: what one forward pass over the tree, and its verification, ask for.

A tree is given by its nodes' parents (node 0: the last token emitted, which the cache does not hold yet).  Four kinds of case:

  append   queries and keys rotated by their nodes' depths, keys and values into a paged cache, in bfloat16 or
           in e4m3 with a scale for each token and head                                       (binding.tabed_cache_append_nodes)
  attn     attention of the nodes over such a cache: the context, the node's ancestors, itself (binding.tabed_attention_nodes)
  verify   multi-round rejection sampling down the tree, the token that follows, the distances of
           the positions on the way                                                           (binding.tabed_verify_nodes)
  keep     the cache's entries of the accepted path moved to where the context ends, all layers (binding.tabed_cache_keep_nodes)

With `own` false `run` computes them in plain torch operations, in 32 bits, the verification's decisions in 64; else by the
library's kernels.  What is held in 8 bits is returned as the values it stands for.
"""
import math

import torch

own = False

DEV = "cuda:0"
BLOCK = 64                     # tokens of a cache block
TINY = 2.0 ** -100             # tokens with no larger magnitude in a head count as zeros
MARGIN = 1e-6                  # decisions closer than this are flagged
THETA = 10000.0


# ------------------------------------------------------------------ the cases
def _append(name, rows, N, q_heads, kv_heads, hd, ctx_hi, src="bf16", cache="bf16", ragged=False, chain=False, rotate=True):
    return {"name": name, "kind": "append", "rows": rows, "N": N, "q_heads": q_heads, "kv_heads": kv_heads, "hd": hd, "ctx_lo": 0, "ctx_hi": ctx_hi,
            "src": src, "cache": cache, "ragged": ragged, "chain": chain, "rotate": rotate, "by_token": False, "layers": 1}


def _attn(name, rows, N, q_heads, kv_heads, hd, ctx_lo, ctx_hi, cache="bf16", ragged=False, chain=False, holes=False, by_token=False):
    return {"name": name, "kind": "attn", "rows": rows, "N": N, "q_heads": q_heads, "kv_heads": kv_heads, "hd": hd, "ctx_lo": ctx_lo, "ctx_hi": ctx_hi,
            "cache": cache, "ragged": ragged, "chain": chain, "holes": holes, "by_token": by_token, "layers": 1}


def _verify(name, B, N, n, V, greedy=0.0, temp=1.0, ragged=False, chain=False, noise=1.0):
    return {"name": name, "kind": "verify", "B": B, "N": N, "n": n, "V": V, "greedy": greedy, "temp": temp, "ragged": ragged, "chain": chain, "noise": noise}


def _keep(name, rows, N, layers, kv_heads, hd, ctx_hi, most, cache="bf16", by_token=False):
    return {"name": name, "kind": "keep", "rows": rows, "N": N, "layers": layers, "kv_heads": kv_heads, "hd": hd, "ctx_lo": 0, "ctx_hi": ctx_hi, "most": most,
            "cache": cache, "by_token": by_token}


def listed():
    return [
        # one sequence's drafted block of five and the token before it: latency alone counts
        _append("append_single", 1, 6, 12, 12, 64, 600, chain=True),
        # trees of many sequences into an 8-bit cache, grouped heads, some trees smaller
        _append("append_trees", 64, 24, 32, 8, 128, 40, cache="e4m3", ragged=True),
        # the same drafted block, scored over a few hundred tokens of context
        _attn("attn_single", 1, 6, 12, 12, 64, 600, 600, chain=True),
        # batched serving: small trees of every row, in the layout of a body's cache (a token's heads side by side)
        _attn("attn_serving", 64, 16, 12, 12, 64, 256, 768, by_token=True),
        # one request with a long context, grouped heads
        _attn("attn_long", 1, 16, 32, 8, 128, 120_011, 120_011),
        # trees over an 8-bit cache, contexts of all lengths, some trees smaller
        _attn("attn_trees", 16, 33, 32, 8, 128, 300, 5000, cache="e4m3", ragged=True),
        # the widest trees: the matrix products weigh as much as the cache
        _attn("attn_wide", 8, 256, 32, 8, 128, 4000, 16000),
        # one sequence's drafted block
        _verify("verify_single", 1, 6, 4, 32000, chain=True),
        # batched serving: a tree for each sequence
        _verify("verify_serving", 16, 22, 4, 32000),
        # the largest batch: eight drafting methods, greedy rows among the sampling ones
        _verify("verify_large", 64, 10, 8, 128256, greedy=0.5, temp=0.7, ragged=True),
        # after the verification of one sequence, a small model's cache
        _keep("keep_single", 1, 6, 2, 12, 64, 600, 4),
        # after the verification of many sequences, all layers at once
        _keep("keep_trees", 32, 24, 12, 8, 128, 40, 7),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "attn", "attn", "attn", "verify", "verify", "keep"])
    if kind == "verify":
        while True:
            B, N, n = _log_int(rng, 1, 64), _log_int(rng, 1, 40), rng.choice([1, 2, 3, 4, 8])
            V = _log_int(rng, 200, 152064) if rng.random() < 0.5 else rng.choice([1000, 32000, 128256, 152064])
            if B * N * (n + 1) * V <= 2 ** 29:
                return {"kind": kind, "B": B, "N": N, "n": n, "V": V, "greedy": rng.choice([0.0, 0.0, 0.3, 1.0]), "temp": rng.choice([0.3, 0.7, 1.0, 1.5]),
                        "ragged": N > 1 and rng.random() < 0.5, "chain": rng.random() < 0.25, "noise": rng.choice([0.1, 0.5, 1.0, 2.0])}
    hd, cache, by_token = rng.choice([32, 64, 64, 96, 128, 128, 256]), rng.choice(["bf16", "bf16", "e4m3"]), rng.random() < 0.4
    kv_heads, group = _log_int(rng, 1, 16), rng.choice([1, 1, 2, 3, 4, 7, 8])
    N = rng.choice([1, rng.randint(2, 8), _log_int(rng, 9, 64), _log_int(rng, 9, 256)])
    both = {"N": N, "kv_heads": kv_heads, "hd": hd, "cache": cache, "by_token": by_token, "ctx_lo": 0}
    if kind == "append":
        while True:
            rows, ctx = _log_int(rng, 1, 256), rng.randint(0, 300)
            if rows * N * kv_heads * (group + 2) * hd <= 2 ** 25 and rows * (N + ctx) * kv_heads * hd <= 2 ** 25:
                return {"kind": kind, "rows": rows, **both, "q_heads": group * kv_heads, "ctx_hi": ctx, "src": rng.choice(["fp32", "bf16"]), "layers": 1,
                        "ragged": N > 1 and rng.random() < 0.5, "chain": rng.random() < 0.3, "rotate": rng.random() < 0.8}
    if kind == "keep":
        while True:
            rows, layers, ctx = _log_int(rng, 1, 128), _log_int(rng, 1, 32), rng.randint(0, 300)
            if rows * layers * (N + ctx + BLOCK) * kv_heads * hd <= 2 ** 25:
                return {"kind": kind, "rows": rows, "layers": layers, **both, "ctx_hi": ctx, "most": rng.randint(1, min(N, 12))}
    while True:
        rows, hi = _log_int(rng, 1, 128), _log_int(rng, 1, 120_000)
        lo = rng.choice([0, hi // 3, hi])
        if rows * (hi + N) * kv_heads * hd <= 120_011 * 8 * 128 and rows * (hi + N) * N * group * kv_heads * hd <= 8 * 10_000 * 256 * 32 * 128:
            return {"kind": kind, "rows": rows, **both, "q_heads": group * kv_heads, "ctx_lo": lo, "ctx_hi": hi, "layers": 1,
                    "ragged": N > 1 and rng.random() < 0.5, "chain": rng.random() < 0.3, "holes": rng.random() < 0.15}


# ------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(1_000_003 * seed + 41)


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


def _rand(g, *shape):
    return torch.rand(shape, generator=g, device=DEV)


def _lengths(g, lo, hi, n):
    return torch.randint(lo, hi + 1, (n,), generator=g, device=DEV, dtype=torch.int32)


def _parents(c, g, rows):
    """Trees that grow by levels: a node's parent is one of the nodes not far before it.  None: chains."""
    N = c["N"]
    if c["chain"]:
        return None
    at = torch.arange(N, device=DEV)
    reach = torch.minimum(at, torch.full_like(at, max(4, N // 6)))
    back = (_rand(g, rows, N) * reach).long().clamp(max=N)
    return torch.where(at > 0, (at - 1 - back).clamp(min=0), -1).to(torch.int32).contiguous()


def _nodes(c, g, rows):
    return _lengths(g, 1, c["N"], rows) if c["ragged"] else torch.full((rows,), c["N"], dtype=torch.int32, device=DEV)


def _e4m3(x, scale):
    """x in steps of e4m3 times scale; where scale is 0 there are none."""
    return torch.where(scale > 0, x / torch.where(scale > 0, scale, 1.0), 0.0).clamp(-448, 448).to(torch.float8_e4m3fn)


def _pool(c, g):
    """Blocks for the rows' contexts and nodes, in no order, and the rows' tables."""
    rows, kvh, hd, layers = c["rows"], c["kv_heads"], c["hd"], c["layers"]
    width = (c["ctx_hi"] + c["N"] + BLOCK - 1) // BLOCK
    need = rows * width
    st = {"table": torch.randperm(need, generator=g, device=DEV, dtype=torch.int32).view(rows, width).clone()}
    shape = (layers, need, BLOCK, kvh, hd) if c["by_token"] else (layers, need, kvh, BLOCK, hd)
    for name in ("k", "v"):
        x = torch.empty(shape, dtype=torch.bfloat16 if c["cache"] == "bf16" else torch.float8_e4m3fn, device=DEV)
        s = torch.empty(shape[:-1], device=DEV) if c["cache"] == "e4m3" else None
        spread = torch.exp(0.5 * _randn(g, hd))                          # some dimensions are larger than others
        part = max(1, 2 ** 25 // (kvh * BLOCK * hd))
        for layer in range(layers):
            for at in range(0, need, part):
                y = _randn(g, min(part, need - at), *shape[2:]) * spread
                if s is None:
                    x[layer, at:at + part] = y.to(torch.bfloat16)
                else:
                    s[layer, at:at + part] = y.abs().amax(-1) / 448
                    x[layer, at:at + part] = _e4m3(y, s[layer, at:at + part, ..., None])
        if c["by_token"]:                                                # seen as [layers, blocks, kv_heads, 64, hd] either way
            x, s = x.transpose(2, 3), None if s is None else s.transpose(2, 3).contiguous()
        st[name], st[name + "scale"] = x, s
    return st


def _verify_inputs(c, g):
    B, N, n, V = c["B"], c["N"], c["n"], c["V"]
    parents = _parents(c, g, B)
    st = {"parents": parents, "nodes": _nodes(c, g, B)}
    temp = torch.full((B,), c["temp"], device=DEV)
    st["temp"] = torch.where(_rand(g, B) < c["greedy"], torch.zeros_like(temp), temp)
    eff = torch.where(st["temp"] > 0, st["temp"], 1.0)
    w = torch.exp(0.7 * _randn(g, B, n))
    st["weights"] = w / w.sum(1, keepdim=True)
    st["target"] = torch.empty((B, N, V), device=DEV)
    st["drafts"] = torch.empty((N, B, n, V), device=DEV)
    st["lse"] = torch.empty((N, B, n), dtype=torch.float64, device=DEV)
    mix = torch.empty((N, B, V), device=DEV)
    for j in range(N):                                                   # the drafts and the target agree in part, token by token
        base = 2.5 * _randn(g, B, 1, V)
        st["target"][:, j] = base[:, 0] + c["noise"] * _randn(g, B, V)
        st["drafts"][j] = base + _randn(g, B, n, V)
        x = st["drafts"][j].double() / eff[:, None, None]
        st["lse"][j] = torch.logsumexp(x, -1)
        mix[j] = (torch.exp(x - st["lse"][j][..., None]) * st["weights"][..., None]).sum(1).float()
    pa = torch.arange(-1, N - 1, device=DEV).expand(B, N) if parents is None else parents.long()
    st["tokens"] = torch.zeros((B, N), dtype=torch.int32, device=DEV)
    st["q"] = torch.ones((B, N), device=DEV)
    rows = torch.arange(B, device=DEV)
    for j in range(1, N):                                                # a node's token is drawn from its parent's mixture
        q = mix[pa[:, j], rows]
        e = q / -torch.log(_rand(g, B, V).clamp(min=1e-30))
        y = torch.where(st["temp"] > 0, e.argmax(1), q.argmax(1) if j % 3 else e.argmax(1))
        st["tokens"][:, j], st["q"][:, j] = y.to(torch.int32), q[rows, y]
    st["u_acc"], st["u_res"] = _rand(g, B, N), _rand(g, B)
    return st


def _inputs(c, seed):
    g = _gen(seed)
    if c["kind"] == "verify":
        return _verify_inputs(c, g)
    rows, N, hd = c["rows"], c["N"], c["hd"]
    st = {"ctx": _lengths(g, c["ctx_lo"], c["ctx_hi"], rows), **_pool(c, g)}
    if c["kind"] == "keep":
        # accepted paths; a node either stays where it is or comes from behind the path's end, so that a pass can be repeated
        count = _lengths(g, 1, c["most"], rows)
        i = torch.arange(N, device=DEV)
        stay = _lengths(g, 1, c["most"], rows)[:, None]
        later = torch.where(torch.arange(N, device=DEV) < count[:, None], 2.0, _rand(g, rows, N)).sort(1).indices.to(torch.int32)
        room = N - count[:, None]
        moved = torch.minimum(stay, count[:, None])
        moved = torch.maximum(moved, count[:, None] - room)              # as many come from behind as there are nodes there
        picked = torch.where(i < (count[:, None] - moved), later, N).sort(1).values
        path = torch.where(i < moved, i, picked.gather(1, (i - moved).clamp(min=0)))
        st["path"] = torch.where(i < count[:, None], path, -1).to(torch.int32).contiguous()
        st["count"] = count
        return st
    st["parents"], st["nodes"] = _parents(c, g, rows), _nodes(c, g, rows)
    if c["kind"] == "append":
        for name, heads in (("nq", c["q_heads"]), ("nk", c["kv_heads"]), ("nv", c["kv_heads"])):
            x = 1.3 * _randn(g, rows, N, heads, hd)
            st[name] = x if c["src"] == "fp32" else x.to(torch.bfloat16)
        return st
    st["q"] = (1.5 * _randn(g, rows, N, c["q_heads"], hd)).to(torch.bfloat16)
    if c["holes"]:                                                       # blocks given up: no table entry
        gone = _rand(g, *st["table"].shape) < 0.2
        gone[-1] = True
        st["table"] = torch.where(gone, -1, st["table"])
    return st


def prepare(c, seed):
    st = {"case": dict(c), **_inputs(c, seed)}
    if c["kind"] == "append":
        st["q_out"] = torch.zeros((c["rows"], c["N"], c["q_heads"], c["hd"]), dtype=torch.bfloat16, device=DEV)
    elif c["kind"] == "attn":
        st["out"] = torch.zeros_like(st["q"])
        st["out_lse"] = torch.zeros(st["q"].shape[:3], device=DEV)
    elif c["kind"] == "verify":
        B, N, gamma = c["B"], c["N"], _gamma(c)
        for name, shape, kind in (("path", (B, N), torch.int32), ("n_path", (B,), torch.int32), ("out_tokens", (B, N), torch.int32),
                                  ("dev", (B, gamma, c["n"]), torch.float32), ("n_valid", (B,), torch.int32), ("flags", (B, N), torch.uint8)):
            st[name] = torch.zeros(shape, dtype=kind, device=DEV)
    else:
        st["ctx_out"] = torch.zeros_like(st["ctx"])
    if own:
        _plan(c, st)
    return st


def _gamma(c):
    return min(32, c["N"])                                               # positions whose distances are wanted


def _plan(c, st):
    """Workspace and the call with its arguments converted once, as a serving loop keeps them."""
    from paper_2601_20357_amd import binding as B
    if c["kind"] == "verify":
        st["cfg"] = B.make_cfg(V=c["V"], d=64, n=c["n"], B=c["B"], gamma=_gamma(c), h=8, w_dtype=1)
        st["ws"] = B.new_verify_nodes_workspace(st["cfg"], c["N"])
        st["call"] = B.prepare_verify_nodes(st["cfg"], st["ws"], 0, st["target"], st["drafts"], st["lse"], st["tokens"], st["q"], st["weights"], st["temp"],
                                            st["path"], st["n_path"], st["out_tokens"], st["flags"], parents=st["parents"], n_nodes=st["nodes"],
                                            u_acc=st["u_acc"], u_res=st["u_res"], dev=st["dev"], n_valid=st["n_valid"])
        return
    st["pool"] = B.CachePaged(st["k"], st["v"], st["table"], kscale=st["kscale"], vscale=st["vscale"])
    if c["kind"] == "append":
        st["call"] = B.prepare_cache_append_nodes(st["pool"], st["nk"], st["nv"], st["ctx"], parents=st["parents"], n_nodes=st["nodes"], q=st["nq"],
                                                  q_out=st["q_out"], rope_theta=THETA if c["rotate"] else 0.0)
    elif c["kind"] == "attn":
        st["ws"] = B.new_attention_nodes_workspace(st["pool"], c["rows"], c["N"], c["q_heads"])
        st["call"] = B.prepare_attention_nodes(st["pool"], st["ws"], st["q"], st["ctx"], st["out"], parents=st["parents"], n_nodes=st["nodes"],
                                               lse=st["out_lse"])
    else:
        st["call"] = B.prepare_cache_keep_nodes(st["pool"], st["ctx"], st["path"], st["count"], st["ctx_out"])


# ------------------------------------------------------------------ one pass
def run(st):
    kind = st["case"]["kind"]
    if not own:
        return {"append": _plain_append, "attn": _plain_attn, "verify": _plain_verify, "keep": _plain_keep}[kind](st)
    st["call"]()
    if kind == "append":
        return {"q": st["q_out"], **_held(st)}
    if kind == "attn":
        return {"out": st["out"], "lse": st["out_lse"]}
    if kind == "verify":
        return {n: st[n] for n in ("path", "n_path", "out_tokens", "dev", "n_valid", "flags")}
    return {"ctx": st["ctx_out"], **_held(st)}


def _held(st):
    """The cache's values."""
    if st["case"]["cache"] == "bf16":
        return {"k": st["k"], "v": st["v"]}
    values = {n: (st[n].float() * st[n + "scale"][..., None]).to(torch.bfloat16) for n in ("k", "v")}
    return {**values, "kscale": st["kscale"], "vscale": st["vscale"]}


def _ancestors(parents, rows, N):
    """[rows, N, N] truth values: does node i see node j (itself and the nodes above it)?"""
    at = torch.arange(N, device=DEV)
    if parents is None:
        return (at[:, None] >= at).expand(rows, N, N)
    seen = (at[:, None] == at) | (parents[..., None] == at)
    for _ in range(max(1, (N - 1).bit_length())):
        seen = torch.matmul(seen.float(), seen.float()) > 0
    return seen


def _rotated(x, pos):
    """x [rows, N, heads, hd] turned by pos [rows, N]; the angles in 64 bits."""
    half = x.shape[-1] // 2
    angle = pos.double()[..., None] * THETA ** (-torch.arange(half, device=DEV, dtype=torch.float64) / half)
    cos, sin = torch.cos(angle).float()[:, :, None], torch.sin(angle).float()[:, :, None]
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * cos - b * sin, a * sin + b * cos], -1)


def _plain_append(st):
    c = st["case"]
    rows, N = c["rows"], c["N"]
    live = torch.arange(N, device=DEV) < st["nodes"][:, None]
    q, k = st["nq"].float(), st["nk"].float()
    if c["rotate"]:
        pos = st["ctx"][:, None] + _ancestors(st["parents"], rows, N).sum(-1) - 1
        q, k = _rotated(q, pos), _rotated(k, pos)
    at = st["ctx"][:, None].long() + torch.arange(N, device=DEV)
    page, slot = st["table"].long().gather(1, at // BLOCK), at % BLOCK
    for name, x in (("k", k), ("v", st["nv"].float())):
        pool = st[name][0]
        old = pool[page, :, slot]                                        # [rows, N, kv_heads, hd]
        if c["cache"] == "bf16":
            pool[page, :, slot] = torch.where(live[..., None, None], x.to(torch.bfloat16), old)
            continue
        most = x.abs().amax(-1)
        s = torch.where(most >= TINY, most / 448, 0.0)
        scales = st[name + "scale"][0]
        scales[page, :, slot] = torch.where(live[..., None], s, scales[page, :, slot])
        pool.view(torch.uint8)[page, :, slot] = torch.where(live[..., None, None], _e4m3(x, s[..., None]).view(torch.uint8), old.view(torch.uint8))
    return {"q": torch.where(live[..., None, None], q.to(torch.bfloat16), st["q_out"]), **_held(st)}


def _plain_attn(st):
    c = st["case"]
    rows, N, kvh, hd, group = c["rows"], c["N"], c["kv_heads"], c["hd"], c["q_heads"] // c["kv_heads"]
    table = st["table"].long()
    page = table.clamp(min=0)
    k, v = ((st[n][0].view(torch.uint8)[page].view(torch.float8_e4m3fn) if c["cache"] == "e4m3" else st[n][0][page]).float() for n in ("k", "v"))
    if c["cache"] == "e4m3":
        k, v = k * st["kscale"][0][page][..., None], v * st["vscale"][0][page][..., None]
    k, v = (x.transpose(1, 2).flatten(2, 3) for x in (k, v))             # [rows, kv_heads, tokens, hd]
    q = st["q"].float().view(rows, N, kvh, group, hd).permute(0, 2, 1, 3, 4).reshape(rows, kvh, N * group, hd)
    s = torch.matmul(q, k.transpose(2, 3).contiguous()) * (1 / math.sqrt(hd))
    node = torch.arange(k.shape[2], device=DEV) - st["ctx"][:, None].long()              # [rows, tokens]: the node that a position holds
    above = _ancestors(st["parents"], rows, N).gather(2, node.clamp(0, N - 1)[:, None, :].expand(rows, N, -1))
    seen = (node < 0)[:, None] | (above & (node < N)[:, None])
    seen = seen & (table >= 0).repeat_interleave(BLOCK, 1)[:, None, :]
    s = s.view(rows, kvh, N, group, -1).masked_fill_(~seen[:, None, :, None, :], -math.inf)
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(m > -math.inf, m, 0.0))
    z = p.sum(-1, keepdim=True)
    o = torch.matmul(p.flatten(2, 3), v.contiguous()).view(rows, kvh, N, group, hd) / torch.where(z > 0, z, 1.0)
    lse = (m + torch.log(z))[..., 0]
    live = (torch.arange(N, device=DEV) < st["nodes"][:, None])[:, :, None]
    o = o.permute(0, 2, 1, 3, 4).reshape(rows, N, c["q_heads"], hd)
    lse = lse.permute(0, 2, 1, 3).reshape(rows, N, c["q_heads"])
    return {"out": torch.where(live[..., None], o.to(torch.bfloat16), st["out"]), "lse": torch.where(live, lse, st["out_lse"])}


def _softmax64(x):
    e = torch.exp(x - x.amax(-1, keepdim=True))
    return e / e.sum(-1, keepdim=True)


def _plain_verify(st):
    c = st["case"]
    B, N, n, V, gamma = c["B"], c["N"], c["n"], c["V"], _gamma(c)
    b = torch.arange(B, device=DEV)
    at = torch.arange(N, device=DEV)
    pa = at.expand(B, N) - 1 if st["parents"] is None else st["parents"].long()
    there = (pa >= 0) & (pa < at) & (at < st["nodes"][:, None])                           # nodes that are somebody's children
    inner = ((pa[:, None, :] == at[:, None]) & there[:, None, :]).any(2)                   # [B, N]: has children
    eff = torch.where(st["temp"] > 0, st["temp"], 1.0).double()
    greedy = st["temp"] <= 0
    p = _softmax64(st["target"].double() / eff[:, None, None])
    best = torch.where(st["target"] == st["target"].amax(-1, keepdim=True), torch.arange(V, device=DEV), V).amin(-1)
    logp = torch.where(p > 0, torch.log(p), 0.0)
    own_term = (p * logp).sum(-1)
    q, dist = torch.zeros_like(p), torch.zeros((B, N, n), dtype=torch.float64, device=DEV)
    for j in range(n):
        logq = (st["drafts"][:, :, j].double() / eff[:, None] - st["lse"][:, :, j, None]).transpose(0, 1)
        dist[..., j] = own_term - (p * logq).sum(-1)
        q += st["weights"][:, j, None, None] * torch.exp(logq)
    f, z = p.clone(), torch.ones((B, N), dtype=torch.float64, device=DEV)
    taken = torch.full((B, N), -1, device=DEV)
    test_flag = torch.zeros((B, N), dtype=torch.uint8, device=DEV)
    for j in range(1, N):
        at_pa = pa[:, j].clamp(min=0)
        up, y = f[b, at_pa], st["tokens"][:, j].long()
        left, right = st["u_acc"][:, j].double() * st["q"][:, j].double() * z[b, at_pa], up[b, y]
        open_ = there[:, j] & (taken[b, at_pa] < 0)
        yes = torch.where(greedy, y == best[b, at_pa], left < right)
        near = (left - right).abs() < MARGIN * torch.maximum(left, right)
        test_flag[:, j] = (open_ & near & ~greedy).to(torch.uint8)
        taken[b, at_pa] = torch.where(open_ & yes, j, taken[b, at_pa])
        no = open_ & ~yes & ~greedy
        was = z[b, at_pa][:, None]
        rest = (torch.where(was > 0, up / torch.where(was > 0, was, 1.0), 0.0) - q[b, at_pa]).clamp(min=0)
        f[b, at_pa] = torch.where(no[:, None], rest, up)
        z[b, at_pa] = torch.where(no, rest.sum(1), z[b, at_pa])
    path = torch.full((B, N), -1, dtype=torch.int32, device=DEV)
    cur, end = torch.zeros(B, dtype=torch.long, device=DEV), torch.zeros(B, dtype=torch.long, device=DEV)
    dev, count = st["dev"].clone(), torch.zeros(B, dtype=torch.int32, device=DEV)
    going = st["nodes"] > 0
    for i in range(N):
        path[:, i] = torch.where(going, cur, -1)
        count += going
        if i < gamma:
            dev[:, i] = torch.where((going & inner[b, cur])[:, None], dist[b, cur].float(), dev[:, i])
        end = torch.where(going, cur, end)
        step = taken[b, cur]
        going = going & (step >= 0)
        cur = torch.where(going, step, cur)
    out = torch.where(path >= 0, st["tokens"].gather(1, path.long().clamp(min=0)), -1)
    out = torch.cat([out[:, 1:], torch.full((B, 1), -1, dtype=torch.int32, device=DEV)], 1)
    row = f[b, end]
    row = torch.where((row.sum(1) > 0)[:, None], row, p[b, end])
    total = row.sum(1, keepdim=True)
    cdf, mark = row.cumsum(1), st["u_res"].double()[:, None] * total
    over = (cdf > mark) & (row > 0)
    first = torch.where(over, torch.arange(V, device=DEV), V).amin(1)
    last = torch.where(row > 0, torch.arange(V, device=DEV), -1).amax(1)
    pick = torch.where(first < V, first, last)
    hi = cdf[b, pick]
    near = torch.minimum((hi - mark[:, 0]).abs(), (mark[:, 0] - (hi - row[b, pick])).abs()) < MARGIN * total[:, 0]
    pick = torch.where(greedy, best[b, end], pick)
    flags = torch.where(greedy[:, None], 0, test_flag)
    walked = (pa[:, None, :] == path[:, :, None].long()).any(1) & there                    # tested: children of the path's nodes, up to the one accepted
    before = taken.gather(1, pa.clamp(min=0))
    flags = torch.where(walked & ((before < 0) | (at <= before)), flags, 0)
    flags[:, 0] = torch.where(greedy, 0, (near * 2 + (first >= V) * 4 + (f[b, end].sum(1) <= 0) * 4)).to(torch.uint8)
    some = count > 0
    out[b, (count.long() - 1).clamp(min=0)] = torch.where(some, pick, out[b, 0]).to(torch.int32)
    flags = torch.where(some[:, None], flags, 0)
    valid = torch.where(some, torch.clamp(count - (~inner[b, end]).int(), max=gamma), 0).to(torch.int32)
    return {"path": path, "n_path": count, "out_tokens": out, "dev": dev, "n_valid": valid, "flags": flags}


def _plain_keep(st):
    c = st["case"]
    i = torch.arange(c["N"], device=DEV)
    base = st["ctx"][:, None].long()
    keep = i < st["count"][:, None]
    src, dst = base + torch.where(keep, st["path"], i), base + i
    table = st["table"].long()
    from_page, from_slot, to_page, to_slot = table.gather(1, src // BLOCK), src % BLOCK, table.gather(1, dst // BLOCK), dst % BLOCK
    for name in ("k", "v"):
        x = st[name] if c["cache"] == "bf16" else st[name].view(torch.uint8)
        for y in (x, st[name + "scale"]):
            if y is not None:
                y = y.transpose(2, 3)                                    # [layers, blocks, 64, kv_heads, ...]
                y[:, to_page, to_slot] = y[:, from_page, from_slot]
    return {"ctx": st["ctx"] + st["count"], **_held(st)}


# ------------------------------------------------------------------ what a pass cannot do without
def work(c):
    size = {"fp32": 4, "bf16": 2}
    if c["kind"] == "verify":
        # the target's and the drafts' rows of the nodes on an accepted path, half of a tree's depth at a guess
        way = 1 + (c["N"] - 1) / 2 if c["chain"] else 1 + math.log2(c["N"]) / 2
        way = way / 2 + 0.5 if c["ragged"] else way
        rows = c["B"] * (way * (c["n"] + 1) - (c["n"] if c["N"] == 1 else 0))
        return {"bytes": int(rows * c["V"] * 4), "flops": int(rows * c["V"] * 20)}
    head = c["hd"] * (2 if c["cache"] == "bf16" else 1) + (0 if c["cache"] == "bf16" else 4)        # bytes of a token's key or value in a head
    if c["kind"] == "keep":
        moved = c["rows"] * c["layers"] * c["kv_heads"] * (c["most"] - 1) / 4
        return {"bytes": int(4 * moved * head + 8 * c["rows"] + 1), "flops": 0}
    part = 0.5 if c["ragged"] else 1.0
    nodes = part * c["rows"] * c["N"]
    if c["kind"] == "append":
        values = nodes * c["hd"] * (c["q_heads"] + 2 * c["kv_heads"])
        return {"bytes": int(values * size[c["src"]] + 2 * nodes * c["q_heads"] * c["hd"] + 2 * nodes * c["kv_heads"] * head), "flops": int(3 * values)}
    ctx = (c["ctx_lo"] + c["ctx_hi"]) / 2
    held = (0.8 if c["holes"] else 1.0) * c["rows"] * c["kv_heads"] * (ctx + part * c["N"])
    queries = nodes * c["q_heads"] * c["hd"]
    return {"bytes": int(2 * held * head + queries * 4), "flops": int(4 * queries * (ctx + part * c["N"] / 2))}


# ------------------------------------------------------------------ in 64 bits, from the definitions
def _above(st, r, j):
    """The nodes that node j of row r sees, itself first."""
    found = [j]
    while True:
        up = found[-1] - 1 if st["parents"] is None else st["up"][r][found[-1]]
        if up < 0:
            return found
        found.append(up)


def _nearest_e4m3(y):
    """The nearest e4m3 value, ties to even: 3 bits behind the leading one, exponents from -6 on."""
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step


def exact(c, seed):
    st = _inputs(c, seed)
    if c["kind"] != "keep" and st["parents"] is not None:
        st["up"] = st["parents"].tolist()
    if c["kind"] == "verify":
        return _exact_verify(c, st)
    ctx, table = st["ctx"].tolist(), st["table"].tolist()
    values = {n: st[n].double() * (1 if st[n + "scale"] is None else st[n + "scale"].double()[..., None]) for n in ("k", "v")} if c["kind"] != "attn" else {}
    scales = {n + "scale": st[n + "scale"].double() for n in ("k", "v")} if c["cache"] == "e4m3" else {}
    if c["kind"] == "keep":
        if c["rows"] * c["most"] > 4000:
            return None
        for r, (count, path) in enumerate(zip(st["count"].tolist(), st["path"].tolist())):
            for i in range(count):
                (to, ts), (fr, fs) = divmod(ctx[r] + i, BLOCK), divmod(ctx[r] + path[i], BLOCK)
                for x in (*values.values(), *scales.values()):
                    x[:, table[r][to], :, ts] = x[:, table[r][fr], :, fs]
        return {"ctx": st["ctx"] + st["count"], **values, **scales}
    new, hd = st["nodes"].tolist(), c["hd"]
    if c["kind"] == "append":
        if sum(new) > 4000:
            return None
        q = torch.zeros((c["rows"], c["N"], c["q_heads"], hd), dtype=torch.float64, device=DEV)
        turn = torch.exp(torch.arange(hd // 2, device=DEV, dtype=torch.float64) * (-2 * math.log(THETA) / hd))
        for r in range(c["rows"]):
            for j in range(new[r]):
                phase = torch.polar(torch.ones_like(turn), turn * (ctx[r] + len(_above(st, r, j)) - 1))
                got = {"v": st["nv"][r, j].double()}
                for name in ("q", "k"):
                    x = st["n" + name][r, j].double()
                    if c["rotate"]:
                        x = torch.complex(x[:, :hd // 2], x[:, hd // 2:]) * phase
                        x = torch.cat([x.real, x.imag], 1)
                    got[name] = x
                q[r, j] = got["q"]
                to, slot = divmod(ctx[r] + j, BLOCK)
                for name in ("k", "v"):
                    x = got[name]
                    if scales:
                        s = x.abs().max(1).values / 448
                        scales[name + "scale"][0, table[r][to], :, slot] = s
                        x = _nearest_e4m3(x / s[:, None]) * s[:, None]
                    values[name][0, table[r][to], :, slot] = x
        return {"q": q, **values, **scales}
    group = c["q_heads"] // c["kv_heads"]
    out = torch.zeros((c["rows"], c["N"], c["q_heads"], hd), dtype=torch.float64, device=DEV)
    lse = torch.zeros(out.shape[:3], dtype=torch.float64, device=DEV)
    for r in range(c["rows"]):
        count = min(len(table[r]), (ctx[r] + c["N"] + BLOCK - 1) // BLOCK)
        pages = [t for t in range(count) if table[r][t] >= 0]
        held = [x * BLOCK + s for x in pages for s in range(BLOCK)]
        seen = torch.zeros((new[r], max(ctx[r] + c["N"], len(table[r]) * BLOCK)), dtype=torch.bool)
        seen[:, :ctx[r]] = True
        for j in range(new[r]):
            seen[j, [ctx[r] + a for a in _above(st, r, j)]] = True
        seen = seen[:, held].to(DEV)
        at = torch.tensor([table[r][x] for x in pages], dtype=torch.long, device=DEV)
        for h in range(c["kv_heads"]):
            part = slice(h * group, (h + 1) * group)
            k, v = (((st[n][0].view(torch.uint8)[at, h].view(torch.float8_e4m3fn) if scales else st[n][0][at, h]).double()
                     * (scales[n + "scale"][0, at, h].unsqueeze(-1) if scales else 1)).flatten(0, 1) for n in ("k", "v"))
            s = torch.einsum("jgd,td->gjt", st["q"][r, :new[r], part].double(), k) / math.sqrt(hd)
            s[:, ~seen] = -math.inf
            z = torch.logsumexp(s, 2)
            lse[r, :new[r], part] = z.t()
            p = torch.where(torch.isfinite(z)[..., None], torch.exp(s - z[..., None]), 0.0)
            out[r, :new[r], part] = torch.einsum("gjt,td->jgd", p, v)
    return {"out": out, "lse": lse}


def _exact_verify(c, st):
    B, N, n, gamma = c["B"], c["N"], c["n"], _gamma(c)
    path, out = [[-1] * N for _ in range(B)], [[-1] * N for _ in range(B)]
    flags, dev = [[0] * N for _ in range(B)], torch.zeros((B, gamma, n), dtype=torch.float64, device=DEV)
    count, valid = [0] * B, [0] * B
    tokens, qs, us, temps, ns = (st[x].tolist() for x in ("tokens", "q", "u_acc", "temp", "nodes"))
    last_u = st["u_res"].tolist()
    for b in range(B):
        node, T = 0, temps[b] or 1.0
        T = float(torch.tensor(T, dtype=torch.float32))
        for i in range(N if ns[b] > 0 else 0):
            path[b][i], count[b] = node, i + 1
            logp = torch.log_softmax(st["target"][b, node].double() / T, 0)
            children = [j for j in range(node + 1, ns[b]) if (j - 1 if st["parents"] is None else st["up"][b][j]) == node]
            if children:
                valid[b] = min(i + 1, gamma)
                logq = st["drafts"][node, b].double() / T - st["lse"][node, b][:, None]
                if i < gamma:
                    dev[b, i] = (logp.exp() * (logp - logq)).sum(1)
            top, mass, level, hit = int(logp.argmax()), 1.0, logp.exp(), None
            if children and temps[b] > 0:
                mixture = (st["weights"][b].double()[:, None] * logq.exp()).sum(0)
            for j in children:
                if temps[b] == 0:
                    if tokens[b][j] == top:
                        hit = j
                        break
                    continue
                want, have = us[b][j] * qs[b][j] * mass, float(level[tokens[b][j]])
                flags[b][j] = int(abs(want - have) < MARGIN * max(want, have))
                if want < have:
                    hit = j
                    break
                level = torch.relu(level / mass - mixture) if mass > 0 else level * 0
                mass = float(level.sum())
            if hit is not None:
                out[b][i], node = tokens[b][hit], hit
                continue
            if temps[b] == 0:
                out[b][i] = top
                break
            if mass <= 0:
                level, flags[b][0] = logp.exp(), 4
            sums = torch.cumsum(level, 0)
            goal = last_u[b] * float(level.sum())
            crossed = torch.nonzero((sums > goal) & (level > 0))
            pick = int(crossed[0]) if len(crossed) else int(torch.nonzero(level > 0)[-1])
            flags[b][0] |= 0 if len(crossed) else 4
            edge = min(abs(float(sums[pick]) - goal), abs(goal - float(sums[pick] - level[pick])))
            flags[b][0] |= 2 if edge < MARGIN * float(level.sum()) else 0
            out[b][i] = pick
            break
    whole = lambda x, t=torch.int32: torch.tensor(x, dtype=t, device=DEV)  # noqa: E731
    return {"path": whole(path), "n_path": whole(count), "out_tokens": whole(out), "dev": dev, "n_valid": whole(valid), "flags": whole(flags, torch.uint8)}
