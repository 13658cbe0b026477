"""The operators as a decoder layer uses them: a prompt into the cache and attention over it, against the softmax chain on what the cache holds;
then tokens one by one, eagerly and as one captured step; and the gradients of a layer's queries and keys."""
import math

import pytest
import torch

import cache_reference as ref
import paper_2506_22169_amd as mcf

pytestmark = pytest.mark.gpu

HQ, H, D, PAGE = 8, 2, 64, 16


class Layer:
    def __init__(self, gen, dtype, batch, width):
        self.cos, self.sin = (t.cuda() for t in ref.tables(D, width * PAGE))
        self.wq, self.wk = ((1 + 0.1 * torch.randn(D, generator=gen)).to(dtype).cuda() for _ in range(2))
        self.cache = mcf.kv_cache(batch * width + 1, H, PAGE, D)
        self.table = torch.randperm(batch * width + 1, generator=gen)[:batch * width].view(batch, width).int().cuda()
        self.scale = 1 / math.sqrt(D)

    def step(self, qkv, lengths, starts=None, out=None):
        q, k, v = qkv[:, :HQ], qkv[:, HQ:HQ + H], qkv[:, HQ + H:]
        q = mcf.append_cache(self.cache, k, v, self.table, lengths, starts, self.cos, self.sin, self.wk, q, self.wq)
        return q, mcf.cache_attention(q, self.cache, self.table, lengths, self.scale, starts, out=out)

    def held(self):
        return [(t.double() * s.double()[:, :, None, None]).cpu() for t, s in ((self.cache.k, self.cache.k_scale), (self.cache.v, self.cache.v_scale))]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
def test_prompt_then_tokens(dtype):
    gen = torch.Generator().manual_seed(41)
    news = [100, 1, 77]
    layer = Layer(gen, dtype, 3, 8)
    lengths = torch.tensor(news, dtype=torch.int32).cuda()
    starts = torch.tensor([0, 100, 101, 178], dtype=torch.int32).cuda()
    qkv = torch.randn(178, HQ + 2 * H, D, generator=gen).to(dtype).cuda()
    q, out = layer.step(qkv, lengths, starts)
    # norm_rotate does the same to the queries, and the softmax chain the same attention on what the cache holds (exact in 16 bits)
    at = torch.cat([torch.arange(n) for n in news]).cuda()
    assert torch.equal(q, mcf.norm_rotate(qkv[:, :HQ], None, layer.cos, layer.sin, at, layer.wq)[0])
    k, v = layer.held()
    for b, n in enumerate(news):
        ids = layer.table[b].long().cpu()
        kk, vv = (t[ids].transpose(0, 1).reshape(H, -1, D)[:, :n].to(dtype).cuda() for t in (k, v))
        rows = slice(sum(news[:b]), sum(news[:b + 1]))
        qq = q[rows].transpose(0, 1).contiguous()
        chain = mcf.causal_softmax_gemm_chain(qq, kk.repeat_interleave(HQ // H, 0).transpose(1, 2), vv.repeat_interleave(HQ // H, 0), layer.scale)
        # each rounds its weights and its result once; the results are means of values below 5
        most = vv.abs().max().item()
        assert (chain.transpose(0, 1).double() - out[rows].double()).abs().max().item() <= 4 * ref.half_step(dtype) * most
    want, bound = ref.attention(q.cpu(), k, v, layer.table.cpu(), news, news, PAGE, layer.scale, True)
    ref.check(out, want, bound, dtype, "prompt")
    # tokens one by one
    for i in range(1, 20):
        lengths += 1
        q, out = layer.step(torch.randn(3, HQ + 2 * H, D, generator=gen).to(dtype).cuda(), lengths)
        k, v = layer.held()
        want, bound = ref.attention(q.cpu(), k, v, layer.table.cpu(), [1, 1, 1], [n + i for n in news], PAGE, layer.scale, True)
        ref.check(out, want, bound, dtype, f"token {i}")


def test_captured_step():
    """One decoding step as a graph: its replays follow the lengths, and equal the eager steps."""
    gen = torch.Generator().manual_seed(42)
    tokens = [torch.randn(2, HQ + 2 * H, D, generator=gen).bfloat16().cuda() for _ in range(6)]
    first = [30, 500]
    results = []
    for captured in (False, True):
        gen2 = torch.Generator().manual_seed(43)
        layer = Layer(gen2, torch.bfloat16, 2, 40)
        lengths = torch.tensor(first, dtype=torch.int32).cuda()
        starts = torch.tensor([0, 30, 530], dtype=torch.int32).cuda()
        layer.step(torch.randn(530, HQ + 2 * H, D, generator=gen2).bfloat16().cuda(), lengths, starts)
        x, out = torch.zeros_like(tokens[0]), torch.zeros(2, HQ, D, dtype=torch.bfloat16, device="cuda")
        if captured:
            saved = [t.clone() for t in layer.cache]
            lengths += 1
            layer.step(x, lengths, out=out)
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                layer.step(x, lengths, out=out)
            lengths -= 1
            for t, s in zip(layer.cache, saved):
                t.copy_(s)
        outs = []
        for t in tokens:
            x.copy_(t)
            lengths += 1
            if captured:
                g.replay()
            else:
                layer.step(x, lengths, out=out)
            torch.cuda.synchronize()
            outs.append(out.clone())
        results.append(outs + [t.clone() for t in layer.cache])
    for a, b in zip(*results):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_training_layer():
    """Queries and keys normed and rotated into the chain's layout, and their gradients through a linear loss of the scores."""
    gen = torch.Generator().manual_seed(44)
    T = 65
    qkv = torch.randn(T, HQ + 2 * HQ, D, generator=gen).bfloat16().cuda()
    layer = Layer(gen, torch.bfloat16, 1, 5)
    q, k = torch.empty(HQ, T, D, dtype=torch.bfloat16, device="cuda"), torch.empty(HQ, T, D, dtype=torch.bfloat16, device="cuda")
    mcf.norm_rotate(qkv[:, :HQ], qkv[:, HQ:2 * HQ], layer.cos, layer.sin, None, layer.wq, layer.wk, q_out=q.transpose(0, 1), k_out=k.transpose(0, 1))
    out = mcf.softmax_gemm_chain(q, k.transpose(1, 2), qkv[:, 2 * HQ:].transpose(0, 1), layer.scale)
    s = layer.scale * q.double() @ k.double().transpose(1, 2)
    want = torch.softmax(s, -1) @ qkv[:, 2 * HQ:].transpose(0, 1).double()
    assert (out.double() - want).abs().max() <= 2 * ref.half_step(torch.bfloat16) * qkv[:, 2 * HQ:].abs().max().item()
    # d loss / d q for loss = sum of (q k^T) g, through the norm and the rotation, where the weights' sums run over all heads
    g = torch.randn(HQ, T, T, generator=gen).cuda()
    dq, dk = (g @ k.float()).bfloat16(), (g.transpose(1, 2).contiguous() @ q.float()).bfloat16()
    got = mcf.norm_rotate_backward(dq.transpose(0, 1), dk.transpose(0, 1), qkv[:, :HQ], qkv[:, HQ:2 * HQ], layer.cos, layer.sin, None, layer.wq, layer.wk)
    at = torch.arange(T)
    for x, dy, w, dx, dw in ((qkv[:, :HQ], dq, layer.wq, got[0], got[2]), (qkv[:, HQ:2 * HQ], dk, layer.wk, got[1], got[3])):
        want, want_w, bx, bw = ref.norm_rotate_backward(dy.transpose(0, 1).cpu(), x.cpu(), layer.cos.cpu(), layer.sin.cpu(), at, w.cpu(), 1e-6, False)
        ref.check(dx, want, bx, torch.bfloat16)
        ref.check(dw, want_w, bw, torch.float32)


@pytest.mark.parametrize("name", ["norm_rotate", "norm_rotate_backward", "append_cache", "cache_attention"])
def test_memory_of_another_stream(name):
    """A call on another stream while the current one, or that one, is busy: results do not lie in memory that the current stream still writes, and
    what the call reads may be dropped right behind it."""
    gen = torch.Generator().manual_seed(43)
    layer = Layer(gen, torch.float16, 4, 8)
    lengths = torch.full((4,), 100, dtype=torch.int32).cuda()
    starts = torch.arange(5, dtype=torch.int32).cuda() * 100
    qkv = torch.randn(400, HQ + 2 * H, D, generator=gen).half().cuda()
    q, k, v = (t.contiguous() for t in (qkv[:, :HQ], qkv[:, HQ:HQ + H], qkv[:, HQ + H:]))
    layer.step(qkv, lengths, starts)

    def call(q, k, v, stream=None):
        if name == "norm_rotate":
            return mcf.norm_rotate(q, k, layer.cos, layer.sin, None, layer.wq, layer.wk, stream=stream)
        if name == "norm_rotate_backward":
            return mcf.norm_rotate_backward(q, k, q, k, layer.cos, layer.sin, None, layer.wq, layer.wk, stream=stream)
        if name == "append_cache":
            return (mcf.append_cache(layer.cache, k, v, layer.table, lengths, starts, layer.cos, layer.sin, layer.wk, q, layer.wq, stream=stream),)
        return (mcf.cache_attention(q, layer.cache, layer.table, lengths, layer.scale, starts, stream=stream),)

    want = [t.clone() for t in call(q, k, v)]
    held = layer.held()

    def same(got):  # (bytes: positions beyond the tables give NaN)
        for a, b in zip(got, want):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))

    busy, to = torch.randn(4096, 4096, device="cuda"), torch.empty(4096, 4096, device="cuda")
    stream = torch.cuda.Stream()
    torch.mm(busy, busy, out=to)
    with torch.cuda.stream(stream):
        torch.mm(busy, busy, out=to)
    torch.cuda.synchronize()
    # the current stream writes memory that it has given back
    for _ in range(20):
        torch.mm(busy, busy, out=to)
    for t in want:
        torch.empty_like(t).fill_(7)
    got = call(q, k, v, stream)
    torch.cuda.synchronize()
    same(got)
    # the call's stream is behind with what it reads
    drop = [t.clone() for t in (q, k, v)]
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        for _ in range(20):
            torch.mm(busy, busy, out=to)
    got = call(*drop, stream)
    del drop
    over = [torch.full_like(t, float("nan")) for t in (q, k, v)]
    torch.cuda.synchronize()
    same(got)
    assert all(torch.equal(a, b) for a, b in zip(layer.held(), held)) and over[0].isnan().all()
