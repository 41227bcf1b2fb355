"""Refusals of the 8-bit operators, on the host: nothing is enqueued, no GPU is touched."""
import ctypes as C

import pytest

from paper_2601_20357_amd import binding

ENULL, EINVAL, ERANGE, EALIGN = -1, -2, -3, -4
P, ODD = C.c_void_p(0x1000), C.c_void_p(0x1001)          # never dereferenced


@pytest.fixture(scope="module")
def lib():
    return binding.load()


def call(fn, names, good, **changed):
    args = dict(good, **changed)
    assert set(args) == set(names), set(args) ^ set(names)
    return fn(*[args[n] for n in names])


NORM = "rows d xt x ldx dt delta ldd sum lds gain eps q ldq scale stream".split()
NORM_OK = dict(rows=4, d=768, xt=0, x=P, ldx=768, dt=0, delta=P, ldd=768, sum=P, lds=768, gain=P, eps=1e-5, q=P, ldq=768, scale=P, stream=None)


@pytest.mark.parametrize("changed,code", [
    (dict(x=None), ENULL), (dict(q=None), ENULL), (dict(scale=None), ENULL), (dict(rows=0), ERANGE), (dict(rows=-1), ERANGE),
    (dict(rows=2 ** 20 + 1), ERANGE), (dict(d=0), ERANGE), (dict(d=32769), ERANGE), (dict(xt=2), EINVAL), (dict(dt=-1), EINVAL), (dict(delta=None), EINVAL),
    (dict(ldx=767), EINVAL), (dict(ldd=0), EINVAL), (dict(lds=-768), EINVAL), (dict(ldq=1), EINVAL), (dict(eps=0.0), EINVAL), (dict(eps=float("nan")), EINVAL),
    (dict(x=ODD), EALIGN), (dict(delta=ODD, dt=1), EALIGN), (dict(sum=ODD), EALIGN), (dict(gain=ODD), EALIGN), (dict(scale=ODD), EALIGN),
    (dict(x=C.c_void_p(0x1002)), EALIGN)])
def test_norm_q8_refuses(lib, changed, code):
    assert call(lib.tabed_norm_q8, NORM, NORM_OK, **changed) == code


LINEAR = "M N K x ldx sx w sw yt y ldy stream".split()
LINEAR_OK = dict(M=4, N=100, K=768, x=P, ldx=768, sx=P, w=P, sw=P, yt=0, y=P, ldy=100, stream=None)


@pytest.mark.parametrize("changed,code", [
    (dict(x=None), ENULL), (dict(sx=None), ENULL), (dict(w=None), ENULL), (dict(sw=None), ENULL), (dict(y=None), ENULL), (dict(M=0), ERANGE),
    (dict(M=2 ** 20 + 1), ERANGE), (dict(N=0), ERANGE), (dict(N=2 ** 24 + 1), ERANGE), (dict(K=0), ERANGE), (dict(K=131072, ldx=131072), ERANGE),
    (dict(K=760), EINVAL), (dict(ldx=776), EINVAL), (dict(ldx=752), EINVAL), (dict(ldy=99), EINVAL), (dict(yt=2), EINVAL), (dict(x=C.c_void_p(0x1008)), EALIGN),
    (dict(w=C.c_void_p(0x1008)), EALIGN), (dict(y=C.c_void_p(0x1002)), EALIGN), (dict(sx=ODD), EALIGN), (dict(sw=ODD), EALIGN)])
def test_linear_q8_refuses(lib, changed, code):
    assert call(lib.tabed_linear_q8, LINEAR, LINEAR_OK, **changed) == code


def cache(**kw):
    f = dict(kv_heads=2, head_dim=64, blocks=10, max_blocks=5, k=0x1000, v=0x1000, kscale=0x1000, vscale=0x1000, table=0x1000)
    f.update(kw)
    return C.byref(binding.TabedCacheQ8(*[f[n] for n, _ in binding.TabedCacheQ8._fields_]))


BAD_CACHES = [(dict(kv_heads=0), ERANGE), (dict(kv_heads=1025), ERANGE), (dict(blocks=0), ERANGE), (dict(max_blocks=0), ERANGE), (dict(max_blocks=2 ** 24 + 1), ERANGE),
              (dict(head_dim=48), EINVAL), (dict(head_dim=0), EINVAL), (dict(k=None), ENULL), (dict(vscale=None), ENULL), (dict(table=None), ENULL),
              (dict(v=0x1008), EALIGN), (dict(kscale=0x1002), EALIGN)]
APPEND = "cache rows T kvt k v row tok ctx new stream".split()
APPEND_OK = dict(cache=cache(), rows=3, T=2, kvt=1, k=P, v=P, row=256, tok=128, ctx=P, new=None, stream=None)
ATTN = "cache ws rows T heads qt q qrow qtok ctx new scale ot out orow otok lse stream".split()
ATTN_OK = dict(cache=cache(), ws=P, rows=3, T=2, heads=4, qt=0, q=P, qrow=512, qtok=256, ctx=P, new=None, scale=0.125, ot=1, out=P, orow=512, otok=256,
               lse=None, stream=None)


@pytest.mark.parametrize("changed,code", BAD_CACHES)
def test_cache_calls_refuse_bad_caches(lib, changed, code):
    assert call(lib.tabed_cache_append_q8, APPEND, APPEND_OK, cache=cache(**changed)) == code
    assert call(lib.tabed_attention_q8, ATTN, ATTN_OK, cache=cache(**changed)) == code
    if code in (ERANGE, EINVAL):
        assert lib.tabed_attention_q8_workspace_bytes(cache(**changed), 3, 2, 4) == 0
        assert lib.tabed_attention_q8_workspace_init(cache(**changed), 3, 2, 4, P, None) == code


@pytest.mark.parametrize("changed,code", [
    (dict(cache=None), ENULL), (dict(k=None), ENULL), (dict(v=None), ENULL), (dict(ctx=None), ENULL), (dict(rows=0), ERANGE), (dict(rows=65536), ERANGE),
    (dict(T=0), ERANGE), (dict(T=2 ** 20 + 1), ERANGE), (dict(rows=65535, T=4096), ERANGE), (dict(kvt=2), EINVAL), (dict(tok=127), EINVAL), (dict(row=0), EINVAL),
    (dict(k=ODD), EALIGN), (dict(v=ODD), EALIGN), (dict(k=C.c_void_p(0x1002), kvt=0), EALIGN), (dict(ctx=ODD), EALIGN), (dict(new=ODD), EALIGN)])
def test_cache_append_q8_refuses(lib, changed, code):
    assert call(lib.tabed_cache_append_q8, APPEND, APPEND_OK, **changed) == code


@pytest.mark.parametrize("changed,code", [
    (dict(cache=None), ENULL), (dict(ws=None), ENULL), (dict(q=None), ENULL), (dict(ctx=None), ENULL), (dict(out=None), ENULL), (dict(rows=0), ERANGE),
    (dict(rows=65536), ERANGE), (dict(T=0), ERANGE), (dict(heads=0), ERANGE), (dict(T=2 ** 19, heads=4), ERANGE), (dict(rows=65535, T=2 ** 14, heads=64), ERANGE),
    (dict(heads=5), EINVAL), (dict(qt=3), EINVAL), (dict(ot=-1), EINVAL), (dict(scale=0.0), EINVAL), (dict(scale=float("inf")), EINVAL),
    (dict(scale=float("nan")), EINVAL), (dict(qrow=255), EINVAL), (dict(qtok=255), EINVAL), (dict(orow=0), EINVAL), (dict(otok=-256), EINVAL),
    (dict(ws=C.c_void_p(0x1008)), EALIGN), (dict(q=C.c_void_p(0x1002)), EALIGN), (dict(out=ODD), EALIGN), (dict(lse=ODD), EALIGN), (dict(ctx=ODD), EALIGN)])
def test_attention_q8_refuses(lib, changed, code):
    assert call(lib.tabed_attention_q8, ATTN, ATTN_OK, **changed) == code


def test_attention_workspace_sizes(lib):
    assert lib.tabed_attention_q8_workspace_bytes(cache(), 3, 2, 4) > 0
    assert lib.tabed_attention_q8_workspace_bytes(cache(k=None, table=None), 3, 2, 4) > 0        # sizes alone decide
    assert lib.tabed_attention_q8_workspace_bytes(cache(), 3, 2, 3) == 0
    assert lib.tabed_attention_q8_workspace_bytes(None, 3, 2, 4) == 0
    assert lib.tabed_attention_q8_workspace_init(cache(), 3, 2, 4, None, None) == ENULL
    assert lib.tabed_attention_q8_workspace_init(cache(), 3, 2, 4, C.c_void_p(0x1008), None) == EALIGN


def test_binding_refuses_what_does_not_fit():
    import torch
    x, q, s = torch.zeros(4, 8), torch.zeros((4, 8), dtype=torch.int8), torch.zeros(4)
    with pytest.raises(binding.TabedError, match="GPU"):
        binding.tabed_norm_q8(x, q, s)
    with pytest.raises(binding.TabedError, match="GPU"):
        binding.tabed_linear_q8(q, s, q, s, x)
    with pytest.raises(binding.TabedError, match="GPU"):
        binding.CacheQ8(q, q, s, s, q, 64)
    with pytest.raises(binding.TabedError, match="side by side"):
        binding._matrix(torch.zeros(8, 4).t(), 4, 8, "x")
    with pytest.raises(binding.TabedError, match="overlap"):
        binding._matrix(torch.zeros(8).expand(4, 8), 4, 8, "x")
    with pytest.raises(binding.TabedError, match="must be"):
        binding._matrix(x, 4, 9, "x")
    view = binding._heads_view
    assert view(torch.zeros(3, 2, 4, 64), 3, 2, 4, 64, "q")[1:] == (512, 256)
    assert view(torch.zeros(3, 256), 3, 1, 4, 64, "q")[1:] == (256, 256)
    assert view(torch.zeros(2, 3, 256).transpose(0, 1), 3, 2, 4, 64, "q")[1:] == (256, 768)
    for bad in (torch.zeros(3, 2, 64, 4).transpose(2, 3), torch.zeros(3, 4, 2, 64).transpose(1, 2), torch.zeros(3, 1, 256).expand(3, 2, 256), torch.zeros(3, 2, 255),
                torch.zeros(2, 2, 256)):
        with pytest.raises(binding.TabedError):
            view(bad, 3, 2, 4, 64, "q")


STEP = "cfg ws round pos W wsc H hsc weights temp u logits lse tokens q flags stream".split()


def step_ok(**kw):
    cfg = dict(V=32000, d=768, n=4, B=16, gamma=5, h=8, w_dtype=1)
    cfg.update(kw)
    return dict({n: P for n in STEP}, cfg=C.byref(binding.make_cfg(**cfg)), round=0, pos=0, u=None, stream=None)


def test_draft_step_q8_refuses(lib):
    fn = lib.tabed_draft_step_q8
    for name in STEP:
        if name not in ("cfg", "round", "pos", "u", "stream"):
            assert call(fn, STEP, step_ok(), **{name: None}) == ENULL, name
    assert call(fn, STEP, step_ok(), cfg=None) == ENULL
    assert call(fn, STEP, step_ok(), pos=5) == ERANGE and call(fn, STEP, step_ok(), pos=-1) == ERANGE
    assert call(fn, STEP, step_ok(d=776)) == EINVAL
    assert call(fn, STEP, step_ok(d=131072)) == ERANGE
    assert call(fn, STEP, step_ok(V=262144, B=65535, n=16)) == ERANGE
    assert call(fn, STEP, step_ok(n=17)) == ERANGE
    for name in ("ws", "W", "H", "logits", "lse"):
        assert call(fn, STEP, step_ok(), **{name: C.c_void_p(0x1008)}) == EALIGN, name
    for name in ("wsc", "hsc"):
        assert call(fn, STEP, step_ok(), **{name: ODD}) == EALIGN, name


BODY = "cfg weights ws rows src stride per ctx cache H H8 hs stream".split()


def body_ok(cache_kw=None, **kw):
    cfg = dict(layers=2, d=128, heads=2, d_ff=256, V=1000, max_ctx=320)
    cfg.update(kw)
    w = binding.TabedBodyWeights()
    w.embed = w.g_final = 0x1000
    for l in range(2):
        for key in ("g_attn", "wqkv", "wo", "g_mlp", "wgu", "wdown"):
            getattr(w, key)[l] = 0x1000
    return dict(cfg=C.byref(binding.make_body_cfg(**cfg)), weights=C.byref(w), ws=P, rows=3, src=P, stride=1, per=1, ctx=P, cache=cache(**(cache_kw or {})),
                H=P, H8=P, hs=P, stream=None)


def test_body_step_q8_refuses(lib):
    fn = lib.tabed_draft_body_step_q8
    for name in ("cfg", "weights", "ws", "src", "ctx", "cache"):
        assert call(fn, BODY, body_ok(), **{name: None}) == ENULL, name
    assert call(fn, BODY, body_ok(), H=None, H8=None, hs=None) == ENULL
    assert call(fn, BODY, body_ok(), hs=None) == ENULL and call(fn, BODY, body_ok(), H8=None) == ENULL
    assert call(fn, BODY, body_ok(), rows=0) == ERANGE and call(fn, BODY, body_ok(), per=0) == ERANGE and call(fn, BODY, body_ok(), stride=-1) == ERANGE
    assert call(fn, BODY, body_ok(layers=17)) == ERANGE
    assert call(fn, BODY, body_ok(max_ctx=321)) == EINVAL                     # five blocks hold 320 tokens
    for bad in (dict(kv_heads=1), dict(head_dim=128)):
        assert call(fn, BODY, body_ok(bad)) == EINVAL
        assert lib.tabed_body_q8_workspace_bytes(body_ok()["cfg"], cache(**bad), 3) == 0
    assert call(fn, BODY, body_ok(dict(head_dim=16), heads=8)) == EINVAL       # heads of 16: no such cache
    assert call(fn, BODY, body_ok(dict(kscale=None))) == ENULL
    for name in ("ws", "H", "H8"):
        assert call(fn, BODY, body_ok(), **{name: C.c_void_p(0x1008)}) == EALIGN, name
    assert call(fn, BODY, body_ok(), hs=ODD) == EALIGN
    assert lib.tabed_body_q8_workspace_bytes(body_ok()["cfg"], cache(k=None), 3) > 0
    assert lib.tabed_body_q8_workspace_init(body_ok()["cfg"], cache(), 3, None, None) == ENULL
    assert lib.tabed_body_q8_workspace_init(body_ok()["cfg"], cache(), 3, C.c_void_p(0x1008), None) == EALIGN
    assert lib.tabed_body_q8_workspace_init(body_ok()["cfg"], cache(kv_heads=1), 3, P, None) == EINVAL


def test_sizes_past_32_bits_are_refused_by_the_binding(lib):
    args = [1, 16, 16, 0x1000, 16, 0x1000, 0x1000, 0x1000, 0, 0x1000, 16, None]
    assert binding.DeviceCall(lib.tabed_linear_q8, args, "tabed_linear_q8", 0, ()).device == 0
    for at, size in ((0, 2 ** 32 + 1), (1, 2 ** 31), (2, -2 ** 31 - 1)):
        with pytest.raises(binding.TabedError, match="32 bits"):
            binding.DeviceCall(lib.tabed_linear_q8, args[:at] + [size] + args[at + 1:], "tabed_linear_q8", 0, ())
