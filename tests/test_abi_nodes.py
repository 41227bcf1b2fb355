"""Refusals of the operators on trees of drafted tokens, on the host: nothing is enqueued, no GPU is touched."""
import ctypes as C
import os
import re

import pytest
import torch

from paper_2601_20357_amd import binding

ENULL, EINVAL, ERANGE, EALIGN, EUNSUPPORTED = -1, -2, -3, -4, -5
P, ODD = C.c_void_p(0x1000), C.c_void_p(0x1001)          # never dereferenced
HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "tabed.h")


@pytest.fixture(scope="module")
def lib():
    return binding.load()


def call(fn, names, good, **changed):
    args = dict(good, **changed)
    assert set(args) == set(names), set(args) ^ set(names)
    return fn(*[args[n] for n in names])


def cache(**kw):
    f = dict(layers=2, kv_heads=2, head_dim=64, blocks=10, max_blocks=5, type=1, layer_stride=81920, block_stride=8192, head_stride=4096, tok_stride=64,
             k=0x1000, v=0x1000, kscale=None, vscale=None, table=0x1000)
    f.update(kw)
    return C.byref(binding.TabedCachePaged(*[f[n] for n, _ in binding.TabedCachePaged._fields_]))


def test_struct_matches_header():
    body = re.search(r"typedef struct tabed_cache_paged \{(.*?)\} tabed_cache_paged;", open(HEADER).read(), flags=re.S).group(1)
    fields = re.findall(r"\b(?:int32_t|int64_t|void\*|float\*|const int32_t\*)\s+([a-z_]+);", re.sub(r"/\*.*?\*/", "", body, flags=re.S))
    assert fields == [f[0] for f in binding.TabedCachePaged._fields_]
    assert C.sizeof(binding.TabedCachePaged) == 6 * 4 + 4 * 8 + 5 * 8
    assert int(re.search(r"#define TABED_MAX_NODES (\d+)", open(HEADER).read()).group(1)) == binding.MAX_NODES


BAD_CACHES = [(dict(layers=0), ERANGE), (dict(layers=1025), ERANGE), (dict(kv_heads=0), ERANGE), (dict(kv_heads=1025), ERANGE), (dict(blocks=0), ERANGE),
              (dict(max_blocks=0), ERANGE), (dict(max_blocks=2 ** 24 + 1), ERANGE), (dict(head_dim=48), EINVAL), (dict(head_dim=0), EINVAL), (dict(type=0), EINVAL),
              (dict(type=3), EINVAL), (dict(tok_stride=63), EINVAL), (dict(tok_stride=68), EINVAL), (dict(head_stride=-4096), EINVAL), (dict(block_stride=0), EINVAL),
              (dict(layer_stride=2 ** 45), EINVAL), (dict(tok_stride=2 ** 24 + 16), EINVAL), (dict(type=2, tok_stride=72, kscale=0x1000, vscale=0x1000), EINVAL), (dict(k=None), ENULL), (dict(v=None), ENULL),
              (dict(table=None), ENULL), (dict(type=2), ENULL), (dict(type=2, kscale=0x1000), ENULL), (dict(k=0x1008), EALIGN), (dict(v=0x1002), EALIGN),
              (dict(table=0x1002), EALIGN), (dict(type=2, kscale=0x1002, vscale=0x1000), EALIGN)]
APPEND = "cache layer rows N dt k v row tok qh q qrow qtok out orow otok ctx parents nodes theta stream".split()
APPEND_OK = dict(cache=cache(), layer=1, rows=3, N=8, dt=1, k=P, v=P, row=1024, tok=128, qh=4, q=P, qrow=2048, qtok=256, out=C.c_void_p(0x9000), orow=2048, otok=256,
                 ctx=P, parents=None, nodes=None, theta=1e4, stream=None)


@pytest.mark.parametrize("changed,code", [(dict(cache=cache(**c)), e) for c, e in BAD_CACHES] + [
    (dict(cache=None), ENULL), (dict(layer=-1), ERANGE), (dict(layer=2), ERANGE), (dict(rows=0), ERANGE), (dict(rows=65536), ERANGE), (dict(N=0), ERANGE),
    (dict(N=257), ERANGE), (dict(dt=2), EINVAL), (dict(k=None), ENULL), (dict(v=None), ENULL), (dict(ctx=None), ENULL), (dict(q=None), ENULL), (dict(out=None), ENULL),
    (dict(row=127), EINVAL), (dict(tok=127), EINVAL), (dict(qh=0), ERANGE), (dict(qh=16385), ERANGE), (dict(qrow=255), EINVAL), (dict(qtok=255), EINVAL),
    (dict(orow=255), EINVAL), (dict(otok=-256), EINVAL), (dict(theta=-1.0), EINVAL), (dict(theta=float("nan")), EINVAL), (dict(theta=float("inf")), EINVAL),
    (dict(out=P, dt=0), EINVAL), (dict(out=P, orow=4096), EINVAL), (dict(k=ODD), EALIGN), (dict(k=C.c_void_p(0x1002), dt=0), EALIGN), (dict(out=ODD), EALIGN),
    (dict(q=ODD), EALIGN), (dict(ctx=ODD), EALIGN), (dict(parents=ODD), EALIGN), (dict(nodes=C.c_void_p(0x1002)), EALIGN)])
def test_append_refuses(lib, changed, code):
    assert call(lib.tabed_cache_append_nodes, APPEND, APPEND_OK, **changed) == code


ATTN = "cache layer ws rows N qh q qrow qtok ctx parents nodes scale out orow otok lse stream".split()
ATTN_OK = dict(cache=cache(), layer=0, ws=P, rows=3, N=8, qh=4, q=P, qrow=2048, qtok=256, ctx=P, parents=None, nodes=None, scale=0.125, out=P, orow=2048, otok=256,
               lse=None, stream=None)


@pytest.mark.parametrize("changed,code", [(dict(cache=cache(**c)), e) for c, e in BAD_CACHES] + [
    (dict(cache=None), ENULL), (dict(layer=-1), ERANGE), (dict(layer=2), ERANGE), (dict(ws=None), ENULL), (dict(rows=0), ERANGE), (dict(rows=65536), ERANGE),
    (dict(N=0), ERANGE), (dict(N=257), ERANGE), (dict(cache=cache(kv_heads=1024), rows=65535, qh=1024, qrow=65536, qtok=65536, orow=65536, otok=65536), ERANGE), (dict(qh=0), ERANGE), (dict(qh=3), EINVAL), (dict(qh=16386), ERANGE), (dict(q=None), ENULL), (dict(ctx=None), ENULL),
    (dict(out=None), ENULL), (dict(qrow=255), EINVAL), (dict(qtok=0), EINVAL), (dict(orow=255), EINVAL), (dict(otok=255), EINVAL), (dict(scale=0.0), EINVAL),
    (dict(scale=float("nan")), EINVAL), (dict(scale=float("inf")), EINVAL), (dict(ws=C.c_void_p(0x1008)), EALIGN), (dict(q=ODD), EALIGN), (dict(out=ODD), EALIGN),
    (dict(ctx=ODD), EALIGN), (dict(parents=ODD), EALIGN), (dict(nodes=ODD), EALIGN), (dict(lse=ODD), EALIGN)])
def test_attention_refuses(lib, changed, code):
    assert call(lib.tabed_attention_nodes, ATTN, ATTN_OK, **changed) == code


def test_attention_workspace(lib):
    need = lib.tabed_attention_nodes_workspace_bytes
    assert need(cache(), 3, 8, 4) > 0 and need(cache(k=None, v=None, table=None), 3, 8, 4) > 0
    for bad in ((cache(type=0), 3, 8, 4), (cache(), 0, 8, 4), (cache(), 3, 257, 4), (cache(), 3, 8, 3), (None, 3, 8, 4)):
        assert need(*bad) == 0
    init = lib.tabed_attention_nodes_workspace_init
    assert init(cache(), 3, 8, 4, None, None) == ENULL and init(cache(), 3, 8, 4, C.c_void_p(0x1008), None) == EALIGN and init(cache(), 3, 0, 4, P, None) == ERANGE


VERIFY = "cfg ws rnd N target drafts lse tokens q parents nodes weights temp ua ur path count out flags dev valid stream".split()


def cfg(**kw):
    return C.byref(binding.make_cfg(**dict(dict(V=32000, d=768, n=4, B=16, gamma=5, h=8, w_dtype=1), **kw)))


VERIFY_OK = dict(cfg=cfg(), ws=P, rnd=0, N=8, target=P, drafts=P, lse=P, tokens=P, q=P, parents=None, nodes=None, weights=P, temp=P, ua=None, ur=None, path=P, count=P,
                 out=P, flags=P, dev=P, valid=P, stream=None)


@pytest.mark.parametrize("changed,code", [(dict([(name, None)]), ENULL) for name in
                                          ("cfg", "ws", "target", "drafts", "lse", "tokens", "q", "weights", "temp", "path", "count", "out", "flags", "dev", "valid")] + [
    (dict([(name, ODD)]), EALIGN) for name in ("ws", "target", "drafts", "lse", "tokens", "q", "parents", "nodes", "weights", "temp", "ua", "ur", "path", "count", "out",
                                               "dev", "valid")] + [
    (dict(cfg=cfg(V=0)), EINVAL), (dict(cfg=cfg(n=17)), ERANGE), (dict(cfg=cfg(B=65536)), ERANGE), (dict(N=0), ERANGE), (dict(N=257), ERANGE),
    (dict(cfg=cfg(distance=2)), EUNSUPPORTED), (dict(cfg=cfg(policy=2, n=2)), EUNSUPPORTED)])
def test_verify_refuses(lib, changed, code):
    assert call(lib.tabed_verify_nodes, VERIFY, VERIFY_OK, **changed) == code


def test_verify_workspace(lib):
    need, init = lib.tabed_verify_nodes_workspace_bytes, lib.tabed_verify_nodes_workspace_init
    assert need(cfg(), 8) > 0 and need(cfg(), 0) == 0 and need(cfg(), 257) == 0 and need(cfg(V=0), 8) == 0
    assert init(cfg(), 8, None, None) == ENULL and init(cfg(), 8, C.c_void_p(0x1008), None) == EALIGN and init(cfg(), 0, P, None) == ERANGE


KEEP = "cache rows N base path count ctx stream".split()
KEEP_OK = dict(cache=cache(), rows=3, N=8, base=P, path=P, count=P, ctx=C.c_void_p(0x2000), stream=None)


@pytest.mark.parametrize("changed,code", [(dict(cache=cache(**c)), e) for c, e in BAD_CACHES] + [
    (dict(cache=None), ENULL), (dict(rows=0), ERANGE), (dict(rows=65536), ERANGE), (dict(N=0), ERANGE), (dict(N=257), ERANGE), (dict(base=None), ENULL),
    (dict(path=None), ENULL), (dict(count=None), ENULL), (dict(ctx=None), ENULL), (dict(ctx=P), EINVAL), (dict(base=ODD), EALIGN), (dict(path=ODD), EALIGN),
    (dict(count=ODD), EALIGN), (dict(ctx=ODD), EALIGN)])
def test_keep_refuses(lib, changed, code):
    assert call(lib.tabed_cache_keep_nodes, KEEP, KEEP_OK, **changed) == code


# ------------------------------------------------------------------ the binding's own checks (no call is made: tensors that claim to be on a GPU are not needed)
def views(monkeypatch):
    monkeypatch.setattr(binding, "_device_of", lambda named: 0)
    monkeypatch.setattr(binding, "_ptr", lambda t, dtype=None, numel=None, name="": None if t is None else t.data_ptr())


def test_cache_views(monkeypatch):
    views(monkeypatch)
    table = torch.zeros(2, 3, dtype=torch.int32)
    k = torch.zeros(6, 2, 64, 32, dtype=torch.bfloat16)
    c = binding.CachePaged(k, k.clone(), table)
    assert (c.layers, c.struct.block_stride, c.struct.head_stride, c.struct.tok_stride) == (1, 4096, 2048, 32) and c.struct.layer_stride >= 32
    body = torch.zeros(4, 2, 192, 96, dtype=torch.bfloat16)
    c = binding.CachePaged.of_body(body, body.clone(), 3)
    assert (c.layers, c.rows, c.kv_heads, c.head_dim, c.struct.blocks) == (4, 2, 3, 32, 6)
    assert (c.struct.layer_stride, c.struct.block_stride, c.struct.head_stride, c.struct.tok_stride) == (2 * 192 * 96, 64 * 96, 32, 96)
    one = torch.zeros(1, 1, 64, 32, dtype=torch.bfloat16)
    c = binding.CachePaged(one.as_strided((1, 1, 64, 32), (7, 3, 32, 1)), one.clone(), table)            # strides that lead nowhere
    assert c.struct.block_stride % 8 == 0 and c.struct.head_stride >= 32
    wrong = [(k, k.clone()[:5], table), (k, k.float(), table), (k.float(), k.float(), table), (k[..., :63, :], k[..., :63, :], table), (k, k.clone(), table[0]),
             (k.transpose(0, 1), k, table), (k.expand(6, 2, 64, 32)[:1].expand(6, 2, 64, 32), k, table), (k[:0], k[:0], table),
             (k.as_strided((6, 2, 64, 32), (4096, 2048, 16, 1)), k.as_strided((6, 2, 64, 32), (4096, 2048, 16, 1)), table)]
    for bad in wrong:
        with pytest.raises(binding.TabedError):
            binding.CachePaged(*bad)
    s = torch.zeros(6, 2, 64)
    with pytest.raises(binding.TabedError):
        binding.CachePaged(k, k.clone(), table, s, s)
    with pytest.raises(binding.TabedError):
        binding.CachePaged(k.to(torch.float8_e4m3fn), k.to(torch.float8_e4m3fn), table)
    for shape, heads in (((4, 2, 100, 96), 3), ((4, 2, 128, 96), 5), ((4, 128, 96), 3)):
        with pytest.raises(binding.TabedError):
            binding.CachePaged.of_body(torch.zeros(shape), torch.zeros(shape), heads)


def test_verify_workspace_of_a_larger_call_serves_smaller_ones():
    def need(B, V, N=22, n=4, gamma=5):
        return binding.tabed_verify_nodes_workspace_bytes(binding.make_cfg(V=V, d=64, n=n, B=B, gamma=gamma, h=8, w_dtype=1), N)
    for V in (300, 32000, 65536, 65537, 262144):
        sizes = [need(B, V) for B in range(1, 300)]
        assert sizes == sorted(sizes)
    for B in (1, 4, 5, 8, 16):
        sizes = [need(B, V) for V in range(1, 262145, 511)]
        assert sizes == sorted(sizes)


def test_attention_workspace_of_a_larger_call_serves_smaller_ones(lib):
    for hd in (32, 64, 96, 128, 256):
        for kv, group in ((8, 4), (12, 1), (1, 8)):
            for mb in (10, 100, 130, 2000):
                def need(rows, N):
                    c = cache(kv_heads=kv, head_dim=hd, max_blocks=mb, tok_stride=hd, head_stride=64 * hd, block_stride=64 * hd * kv, layer_stride=640 * hd * kv)
                    return lib.tabed_attention_nodes_workspace_bytes(c, rows, N, kv * group)
                rows, nodes = (1, 2, 8, 31, 32, 63, 64, 257, 1024, 1025), (1, 2, 4, 5, 8, 9, 16, 17, 32, 33, 64, 65, 128, 129, 255, 256)
                sizes = [[need(r, n) for n in nodes] for r in rows]
                assert sizes[0][0] > 0
                for line in sizes + [list(x) for x in zip(*sizes)]:
                    line = [x for x in line if x]                        # (0: more than a launch holds)
                    assert line == sorted(line), (hd, kv, mb)


@pytest.mark.parametrize("name,at", [("base", 0x1000), ("base", 0x2008), ("base", 0x1ff8), ("path", 0x2008), ("path", 0x1fa4), ("count", 0x2000), ("count", 0x1ff8)])
def test_keep_refuses_lengths_that_overlap_what_is_read(lib, name, at):
    changed = {name: C.c_void_p(at)}
    if at == 0x1000:
        changed["ctx"] = C.c_void_p(0x1000)
    assert call(lib.tabed_cache_keep_nodes, KEEP, KEEP_OK, **changed) == EINVAL


def test_attention_refuses_results_in_place_of_queries_with_other_strides(lib):
    for changed in (dict(orow=4096), dict(otok=512)):
        assert call(lib.tabed_attention_nodes, ATTN, ATTN_OK, **changed) == EINVAL
