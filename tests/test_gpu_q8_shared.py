"""Workspaces of the 8-bit calls that captured graphs, eager calls and 16-bit calls use in turn."""
import pytest
import torch

from paper_2601_20357_amd import binding
from test_gpu_q8 import DEV, Cache, check_attention, gen, randn

pytestmark = pytest.mark.gpu


def test_two_captured_graphs_and_eager_calls_share_an_attention_workspace():
    """Single tokens and blocks of six over rows that are cut into ranges, whose joins count arrivals in the workspace: replayed in any order, with
    eager calls of a third size in between and rows that grow."""
    c = Cache(3, 130, 2, 64, seed=51)
    sizes = [(1, 4), (6, 4), (3, 8)]                                   # the last is the eager one
    need = max(binding.tabed_attention_q8_workspace_bytes(c.gpu, 3, T, heads) for T, heads in sizes)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    ws.fill_(0x5a)
    binding.tabed_attention_q8_workspace_init(c.gpu, 3, 1, 4, ws)
    ctx = torch.tensor([8000, 700, 3100], dtype=torch.int32, device=DEV)
    q = [randn(gen(T), 3, T, heads, 64).to(DEV) for T, heads in sizes]
    out = [torch.zeros_like(x) for x in q]
    call = lambda i, into, w: binding.tabed_attention_q8(c.gpu, w, q[i], ctx, into)
    side, graphs = torch.cuda.Stream(), []
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for i in (0, 1):
            graph = torch.cuda.CUDAGraph()
            graph.capture_begin()
            call(i, out[i], ws)
            graph.capture_end()
            graphs.append(graph)
    torch.cuda.current_stream().wait_stream(side)
    for step, order in enumerate(((0, 1, 2), (1, 0, 2, 0), (2, 2, 1, 1), (0, 0, 1, 2), (1, 2, 0))):
        fresh = [torch.zeros_like(x) for x in q]
        for i in range(3):
            call(i, fresh[i], binding.new_attention_workspace(c.gpu, 3, *sizes[i]))
        for i in order:
            out[i].zero_()
            if i < 2:
                graphs[i].replay()
            else:
                call(i, out[i], ws)
        torch.cuda.synchronize()
        for i in set(order):                                           # (an output that was not asked for is the last step's)
            assert torch.equal(out[i], fresh[i]), (step, i)
        if step == 0:
            check_attention(c, q[1].cpu(), ctx.tolist(), None, out[1].cpu(), None)
        ctx += 61


def test_draft_steps_of_both_widths_share_a_workspace():
    """8-bit and 16-bit steps in turn, eager and replayed, leave what each leaves with a workspace of its own."""
    n, B, V, d = 4, 9, 5003, 256
    g = torch.Generator().manual_seed(4)
    W, H = (torch.randn(V, d, generator=g) * 0.05).bfloat16().to(DEV), torch.randn(B * n, d, generator=g).bfloat16().to(DEV)
    (W8, ws8), (H8, hs8) = binding.quantize_rows(W), binding.quantize_rows(H)
    temp = torch.tensor([0.0, 1.0, 0.7] * 3, device=DEV)
    cfg = binding.make_cfg(V=V, d=d, n=n, B=B, gamma=2, h=4, w_dtype=1, seed=6)

    def buffers():
        b = binding.RoundBuffers(cfg)
        b.weights.copy_(torch.softmax(torch.randn(B, n, generator=torch.Generator().manual_seed(3)), 1).to(DEV))
        return b

    calls = lambda b, pos: (lambda: b.draft_step(1, pos, W, H, temp), b.prepare_draft_step_q8(1, pos, W8, ws8, H8, hs8, temp))
    left = lambda b: [t.clone() for t in (b.draft_logits, b.draft_lse, b.draft_tokens, b.draft_q, b.draft_flags)]

    def alone(which):
        b = buffers()
        b.draft_logits.zero_(), b.draft_lse.zero_(), b.draft_tokens.zero_(), b.draft_q.zero_(), b.draft_flags.zero_()
        calls(b, 0)[which](), calls(b, 1)[1 - which]()
        torch.cuda.synchronize()
        return left(b)

    want = [alone(0), alone(1)]
    assert not torch.equal(want[0][0], want[1][0])
    b = buffers()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        captured = b.prepare_draft_step_q8(1, 0, W8, ws8, H8, hs8, temp)
        graph.capture_begin()
        captured()
        graph.capture_end()
    torch.cuda.current_stream().wait_stream(side)
    for turn in range(4):
        b.draft_logits.zero_(), b.draft_lse.zero_(), b.draft_tokens.zero_(), b.draft_q.zero_(), b.draft_flags.zero_()
        which = turn % 2
        if which == 1 and turn > 1:
            graph.replay()
        else:
            calls(b, 0)[which]()
        calls(b, 1)[1 - which]()
        torch.cuda.synchronize()
        for x, y in zip(left(b), want[which]):
            assert torch.equal(x, y), turn
