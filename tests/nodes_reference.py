"""The operators on trees of drafted tokens in 64 bits, from their definitions, on the CPU and in plain loops.  Used by the tests only."""
import math

import torch

BLOCK = 64
MARGIN = 1e-6


def tree(N, kind, seed=0):
    """Parents of a tree of N nodes: 'chain' (None), 'star', 'random', 'deep', 'forest' (several roots and entries that name no node before them)."""
    g = torch.Generator().manual_seed(seed * 7919 + N)
    if kind == "chain":
        return None
    if kind == "star":
        return torch.tensor([-1] + [0] * (N - 1), dtype=torch.int32)
    if kind == "deep":
        return torch.tensor([j - 1 if j % 5 else max(j - 3, -1) for j in range(N)], dtype=torch.int32)
    p = [-1] + [int(torch.randint(max(0, j - max(4, N // 6)), j, (1,), generator=g)) for j in range(1, N)]
    if kind == "forest":
        for j in range(1, N):
            if j % 3 == 0:
                p[j] = (-1, -7, j, N + 3, 2 ** 31 - 1, -2 ** 31)[j // 3 % 6]
    return torch.tensor(p, dtype=torch.int32)


def parent(parents, r, j):
    p = j - 1 if parents is None else int(parents[r, j])
    return p if 0 <= p < j else -1


def above(parents, r, j):
    """Node j of row r and the nodes above it."""
    found = []
    while j >= 0:
        found.append(j)
        j = parent(parents, r, j)
    return found


def place(table, blocks, r, pos):
    """(block, slot) of a position, None where it is in none."""
    if pos // BLOCK >= table.shape[1]:
        return None
    b = int(table[r, pos // BLOCK])
    return (b, pos % BLOCK) if 0 <= b < blocks else None


def rotated(x, pos, theta):
    """x [heads, hd] in 64 bits turned by pos: a complex product."""
    hd = x.shape[-1]
    if theta == 0:
        return x
    angle = pos * torch.exp(torch.arange(hd // 2, dtype=torch.float64) * (-2 * math.log(theta) / hd))
    z = torch.complex(x[:, :hd // 2], x[:, hd // 2:]) * torch.polar(torch.ones_like(angle), angle)
    return torch.cat([z.real, z.imag], 1)


def attention(q, k, v, table, blocks, ctx, parents, nodes, scale):
    """q [rows, N, q_heads, hd], k, v [blocks, kv_heads, 64, hd] in 64 bits: (out, lse, mass) with mass = sum p |v|, NaN rows where a node is absent."""
    rows, N, qh, hd = q.shape
    group = qh // k.shape[1]
    out = torch.full(q.shape, math.nan, dtype=torch.float64)
    lse, mass = torch.full(q.shape[:3], math.nan, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
    for r in range(rows):
        for j in range(nodes[r]):
            see = [place(table, blocks, r, p) for p in [*range(ctx[r]), *(ctx[r] + a for a in sorted(above(parents, r, j)))]]
            see = [w for w in see if w is not None]
            if not see:
                out[r, j], lse[r, j] = 0.0, -math.inf
                continue
            b, s = (torch.tensor(x) for x in zip(*see))
            kk, vv = (x[b, :, s].repeat_interleave(group, 1).transpose(0, 1) for x in (k, v))        # [q_heads, seen, hd]
            score = (kk @ q[r, j].unsqueeze(-1)).squeeze(-1) * scale
            lse[r, j] = torch.logsumexp(score, 1)
            p = torch.softmax(score, 1).unsqueeze(1)
            out[r, j], mass[r, j] = (p @ vv).squeeze(1), (p @ vv.abs()).squeeze(1)
    return out, lse, mass


def verify(target, drafts, dlse, tokens, q, parents, nodes, weights, temp, u_acc, u_res, gamma, tvd=False):
    """One list of outputs a row: (path, out_tokens, {node: flag}, last flag, distances [valid][n], closest margin of any decision)."""
    B, N, V = target.shape
    rows = []
    for b in range(B):
        T = float(temp[b]) or 1.0
        cur, path, out, flags, dist, close = 0, [], [], {}, [], 1.0
        last = 0
        while nodes[b] > 0:
            path.append(cur)
            p = torch.softmax(target[b, cur].double() / T, 0)
            kids = [j for j in range(cur + 1, int(nodes[b])) if parent(parents, b, j) == cur]
            if kids:
                logq = drafts[cur, b].double() / T - dlse[cur, b].double()[:, None]
                if len(path) <= gamma:
                    if tvd:
                        dist.append([0.5 * float((p - x.exp()).abs().sum()) for x in logq])
                    else:
                        logp = torch.log_softmax(target[b, cur].double() / T, 0)
                        dist.append([float(torch.where(p > 0, p * (logp - x), 0.0).sum()) for x in logq])
                mix = (weights[b].double()[:, None] * logq.exp()).sum(0)
            best = int((target[b, cur] == target[b, cur].max()).nonzero()[0])
            f, Z, hit = p, 1.0, None
            for j in kids:
                y = int(tokens[b, j])
                inside = 0 <= y < V
                flags[j] = 0 if inside else 4
                if temp[b] == 0:
                    if y == best:
                        hit = j
                        break
                    continue
                want, have = float(u_acc[b, j]) * float(q[b, j]) * Z, float(f[y]) if inside else 0.0
                if inside:
                    flags[j] |= int(abs(want - have) < MARGIN * max(want, have))
                    close = min(close, abs(want - have) / max(want, have, 1e-300))
                if inside and want < have:
                    hit = j
                    break
                f = torch.clamp(f / Z - mix, min=0) if Z > 0 else torch.zeros_like(f)
                Z = float(f.sum())
            if hit is not None:
                out.append(int(tokens[b, hit]))
                cur = hit
                continue
            if temp[b] == 0:
                out.append(best)
                break
            if not Z > 0:
                f, last = p, 4
            whole = float(f.sum())
            cdf, goal = torch.cumsum(f, 0), float(u_res[b]) * whole
            over = ((cdf > goal) & (f > 0)).nonzero()
            pick = int(over[0]) if len(over) else int((f > 0).nonzero()[-1])
            last |= 0 if len(over) else 4
            edge = min(abs(float(cdf[pick]) - goal), abs(goal - float(cdf[pick] - f[pick])))
            last |= 2 if edge < MARGIN * whole else 0
            close = min(close, edge / whole)
            out.append(pick)
            break
        rows.append((path, out, flags, last, dist, close))
    return rows
