"""Verification of trees is lossless behind an accepted node too."""
import pytest
import torch

import test_gpu_nodes_verify as tv

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("temp", [1.0, 0.6])
def test_token_behind_an_accepted_node_follows_its_target(temp):
    """Over 60000 rows of one tree with Philox's uniforms, children drawn from their parent's mixture: given the node accepted, the next token is distributed as the target's there
    (chi-square, 1 in 10^6), behind a node with children and behind one without."""
    from paper_2601_20357_amd import binding
    Bn, N, V, n = 60_000, 5, 6, 2
    g = torch.Generator().manual_seed(9)
    c = tv.make(1, N, n, V, kind="star", seed=14, temp=[temp], noise=1.0, spread=1.0)
    parents = torch.tensor([[-1, 0, 0, 1, 1]], dtype=torch.int32)
    drafts, lse = c["drafts"][:, 0].double() / temp, c["lse"][:, 0]
    mix = (torch.exp(drafts - lse[..., None]) * c["weights"][0][:, None]).sum(1)
    tokens, q = torch.zeros(Bn, N, dtype=torch.int32), torch.ones(Bn, N)
    for j in range(1, N):
        row = mix[parents[0, j]].float()
        y = torch.multinomial(row, Bn, replacement=True, generator=g)
        tokens[:, j], q[:, j] = y.to(torch.int32), row[y]
    big = {"parents": parents.expand(Bn, N).contiguous(), "nodes": torch.full((Bn,), N), "temp": torch.full((Bn,), temp), "target": c["target"].expand(Bn, N, V).contiguous(),
           "drafts": c["drafts"].expand(N, Bn, n, V).contiguous(), "lse": c["lse"].expand(N, Bn, n).contiguous(), "weights": c["weights"].expand(Bn, n).contiguous(),
           "u_acc": None, "u_res": None, "tokens": tokens, "q": q}
    o, _, _ = tv.run(binding, big, uniforms=False, rnd=6)
    path, out = o["path"].cpu(), o["out"].cpu()
    for node in (1, 2, 3, 4):
        depth = 2 if node > 2 else 1
        at = path[:, depth] == node
        count = int(at.sum())
        assert count > 1000, node
        p = torch.softmax(c["target"][0, node].double() / temp, 0)
        seen = torch.bincount(out[at, depth].long(), minlength=V).double()
        chi = float(((seen - count * p) ** 2 / (count * p)).sum())
        assert chi < 36.2, (node, seen / count, p)                       # 5 degrees of freedom: 10^-6 above 36.2
