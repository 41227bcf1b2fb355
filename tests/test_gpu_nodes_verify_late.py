"""Verification of trees where a workgroup comes so late that others have stopped waiting for it: a row has a verdict that is whole, or none, flagged."""
import ctypes
import math

import pytest
import torch

import test_gpu_nodes_verify as tv

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def call_late(binding, c, ws, cfg, spins, late, gamma):
    """tabed_verify_nodes with waits of `spins` polls, and workgroup `late` of every sequence coming after the others have stopped waiting."""
    B, N, V = c["target"].shape
    n = c["drafts"].shape[2]
    keep = {k: c[k].to(DEV) for k in ("target", "drafts", "lse", "q", "weights", "temp", "u_acc", "u_res")}
    for k in ("tokens", "parents", "nodes"):
        keep[k] = None if c[k] is None else c[k].to(torch.int32).to(DEV)
    o = {"path": torch.full((B, N), 99, dtype=torch.int32, device=DEV), "n_path": torch.full((B,), 99, dtype=torch.int32, device=DEV),
         "out": torch.full((B, N), 99, dtype=torch.int32, device=DEV), "flags": torch.full((B, N), 99, dtype=torch.uint8, device=DEV),
         "dev": torch.full((B, gamma, n), 7.0, device=DEV), "n_valid": torch.full((B,), 99, dtype=torch.int32, device=DEV)}
    p = lambda t: ctypes.c_void_p(None if t is None else t.data_ptr())  # noqa: E731
    rc = binding.load().tabed_testing_verify_nodes(
        ctypes.byref(cfg), p(ws), ctypes.c_uint64(0), ctypes.c_int32(N), *(p(keep[k]) for k in ("target", "drafts", "lse", "tokens", "q", "parents", "nodes", "weights", "temp",
                                                                                             "u_acc", "u_res")),
        *(p(o[k]) for k in ("path", "n_path", "out", "flags", "dev", "n_valid")), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream),
        ctypes.c_int32(spins), ctypes.c_int32(late))
    assert rc == 0
    torch.cuda.synchronize()
    return {k: v.cpu() for k, v in o.items()}


@pytest.mark.parametrize("tvd", [False, True])
@pytest.mark.parametrize("N,kind", [(1, "star"), (2, "chain"), (7, "random")])
def test_a_row_has_a_whole_verdict_or_none(N, kind, tvd):
    """Every workgroup late in turn; the next call in earnest, on the same workspace, as ever.  (Rows of 5000 tokens: five workgroups a sequence.)"""
    from paper_2601_20357_amd import binding
    Bn, V, n, gamma = 6, 5000, 2, 5
    c = tv.make(Bn, N, n, V, kind=kind, seed=N, temp=[1.0, 0.7, 0.0])
    c["u_res"] = torch.tensor([0.001, 0.3, 0.5, 0.6, 0.8, 0.999])        # (last draws in all pieces)
    cfg = binding.make_cfg(V=V, d=64, n=n, B=Bn, gamma=gamma, h=8, w_dtype=1, seed=77, distance=int(tvd))
    want, _, ws = tv.run(binding, c, gamma=gamma, cfg=cfg)
    want = {k: v.cpu() for k, v in want.items()}
    ended = 0
    for late in range(5):
        for spins in (40, 1 << 24):
            o = call_late(binding, c, ws, cfg, spins, late, gamma)
            for b in range(Bn):
                if int(o["n_path"][b]) == 0:
                    ended += 1
                    assert spins == 40
                    assert (o["path"][b] == -1).all() and (o["out"][b] == -1).all() and o["flags"][b].tolist() == [4] + [0] * (N - 1) and o["n_valid"][b] == 0
                    assert (o["dev"][b] == 7).all()
                else:
                    for k in o:
                        assert torch.equal(o[k][b], want[k][b]), (late, spins, b, k)
        again, _, _ = tv.run(binding, c, gamma=gamma, cfg=cfg, ws=ws)
        for k in want:
            assert torch.equal(again[k].cpu(), want[k]), (late, k)
    assert ended > 0                                                     # (waits of 40 polls end before 3 ms)


def test_a_workspace_prepared_for_less_ends_flagged():
    """A buffer that is large enough, prepared for a smaller call: what lies behind that may look like anything, here like words of the next launches."""
    from paper_2601_20357_amd import binding
    large, small = tv.make(8, 9, 3, 7000, seed=1), tv.make(2, 3, 1, 500, seed=2)
    make = lambda c: binding.make_cfg(V=c["target"].shape[2], d=64, n=c["drafts"].shape[2], B=len(c["target"]), gamma=c["target"].shape[1], h=8, w_dtype=1, seed=77)  # noqa: E731
    cfg, less = make(large), make(small)
    need = binding.tabed_verify_nodes_workspace_bytes(cfg, 9)
    assert binding.tabed_verify_nodes_workspace_bytes(less, 3) < need
    want, want_small = tv.run(binding, large, cfg=cfg)[0], tv.run(binding, small, cfg=less)[0]
    for launch in (1, 2):
        ws = torch.full((need // 8,), launch << 32 | 1, dtype=torch.int64, device=DEV).view(torch.uint8)
        binding.tabed_verify_nodes_workspace_init(less, 3, ws)
        for _ in range(2):
            o = tv.run(binding, large, ws=ws, cfg=cfg)[0]
            assert o["n_path"].tolist() == [0] * 8 and (o["path"] == -1).all() and (o["out"] == -1).all() and (o["flags"][:, 0] == 4).all() and (o["n_valid"] == 0).all()
            again = tv.run(binding, small, ws=ws, cfg=less)[0]
            for k in want_small:
                assert torch.equal(again[k], want_small[k]), k
        binding.tabed_verify_nodes_workspace_init(cfg, 9, ws)
        again = tv.run(binding, large, ws=ws, cfg=cfg)[0]
        for k in want:
            assert torch.equal(again[k], want[k]), k


@pytest.mark.parametrize("at", [0, 1024, 4096])
def test_nan_among_masked_logits_ends_flagged(at):
    """A NaN is one also where all others of its workgroup's 1024 logits are -inf."""
    from paper_2601_20357_amd import binding
    c = tv.make(3, 4, 2, 5000, seed=8, temp=[1.0])
    c["target"][1, 0, at:at + 1024] = -math.inf
    want = tv.run(binding, c)[0]
    c["target"][1, 0, at + 500] = math.nan
    o = tv.run(binding, c)[0]
    assert o["n_path"][1] == 1 and o["path"][1].tolist() == [0, -1, -1, -1] and o["flags"][1, 0] == 4 and 0 <= int(o["out"][1, 0]) < 5000
    assert int(o["n_valid"][1]) == 0 or bool(o["dev"][1, 0].isnan().all())
    for k in o:
        assert torch.equal(o[k][[0, 2]], want[k][[0, 2]]), k
