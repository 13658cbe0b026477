"""Attention over the paged cache of 8 bits, against the definition in 64 bits on what the cache holds."""
import math

import pytest
import torch

import cache_reference as ref
import paper_2506_22169_amd as mcf

pytestmark = pytest.mark.gpu


def _cache(gen, pages, heads, page, size, spread=0, joined=False):
    """Random pages; spread: binary orders that the scales of V range over; joined: K and V of a page in one tensor."""
    dev, host = [], []
    both = torch.zeros(pages, 2, heads, page, size, dtype=ref.E4M3, device="cuda") if joined else None
    for i in range(2):
        q = (torch.randn(pages, heads, page, size, generator=gen) * 100).clamp(-448, 448).to(ref.E4M3)
        s = 0.01 * (0.5 + torch.rand(pages, heads, generator=gen))
        if i and spread:
            s = s * 2.0 ** torch.randint(-spread, spread + 1, (pages, heads), generator=gen)
        d = both[:, i].copy_(q) if joined else q.cuda()
        sd = torch.zeros(pages, heads + joined, device="cuda")[:, :heads].copy_(s)
        dev.append((d, sd))
        host.append(q.double() * s.double()[:, :, None, None])
    return mcf.KVCache(dev[0][0], dev[1][0], dev[0][1], dev[1][1]), host


def _problem(gen, news, lengths, hq, heads, size, page, dtype, spread=0, joined=False, width=None, spare=3):
    width = width or max(1, max(-(-n // page) for n in lengths))
    need = sum(min(width, -(-n // page)) for n in lengths)
    cache, host = _cache(gen, need + spare, heads, page, size, spread, joined)
    table = torch.full((len(news), width), -1)
    ids = torch.randperm(need + spare, generator=gen).tolist()
    for b, n in enumerate(lengths):
        for c in range(min(width, -(-n // page))):
            table[b, c] = ids.pop()
    q = torch.randn(sum(news), hq, size, generator=gen).to(dtype)
    return q, cache, host, table


def _run(q, cache, table, news, lengths, scale, causal, single=None, pad=0, **kw):
    single = all(n == 1 for n in news) if single is None else single
    starts = None if single else (pad + torch.tensor([sum(news[:i]) for i in range(len(news) + 1)])).int().cuda()
    return mcf.cache_attention(q.cuda(), cache, table.int().cuda(), torch.tensor(lengths).int().cuda(), scale, starts, causal=causal, **kw)


def _check(q, cache, host, table, news, lengths, page, scale, causal, what="", **kw):
    got = _run(q, cache, table, news, lengths, scale, causal, **kw)
    want, bound = ref.attention(q, host[0], host[1], table, news, lengths, page, scale, causal)
    ref.check(got, want, bound, q.dtype, what)
    return got


# rows that each sequence brings, tokens that it has, heads of q, heads, size, page
CASES = [
    ([1], [1], 1, 1, 64, 16), ([1, 1, 1], [5, 0, 129], 8, 2, 128, 16), ([1], [2000], 4, 1, 128, 64), ([1, 1], [700, 33], 5, 5, 80, 32),
    ([1, 1], [515, 1030], 16, 1, 96, 128), ([1], [300], 20, 1, 192, 16), ([1, 1, 1], [40, 41, 1200], 6, 3, 256, 64), ([1] * 67, list(range(67)), 2, 1, 64, 16),
    ([3], [100], 4, 2, 64, 16), ([5, 2, 0, 1], [5, 90, 7, 0], 8, 2, 128, 32), ([7, 4], [3, 4], 3, 1, 80, 16), ([16], [1000], 12, 4, 96, 64), ([9, 13], [400, 13], 40, 8, 256, 16),
    ([33], [64], 4, 4, 128, 16), ([100, 1, 57], [100, 300, 257], 4, 2, 128, 64), ([65, 200], [65, 333], 3, 1, 192, 32), ([130], [700], 6, 6, 64, 128), ([77], [77], 2, 2, 80, 16),
    ([300], [301], 7, 1, 96, 16), ([129, 64], [129, 64], 5, 5, 256, 128), ([2] * 70, [2 + i for i in range(70)], 2, 2, 64, 16),
]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "whole"])
@pytest.mark.parametrize("i", range(len(CASES)))
def test_attention(i, causal, dtype):
    news, lengths, hq, heads, size, page = CASES[i]
    gen = torch.Generator().manual_seed(500 + i)
    q, cache, host, table = _problem(gen, news, lengths, hq, heads, size, page, dtype, joined=causal)
    _check(q, cache, host, table, news, lengths, page, 1 / math.sqrt(size), causal, str(CASES[i]))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("scale", [0.0, -0.125, 2.0, 1e-4])
def test_scales_of_the_scores(scale, dtype):
    gen = torch.Generator().manual_seed(31)
    for news, lengths in (([1, 1], [300, 77]), ([70], [150])):
        q, cache, host, table = _problem(gen, news, lengths, 4, 2, 128, 16, dtype)
        _check(q, cache, host, table, news, lengths, 16, scale, True)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("news", [[1, 1], [6, 90]], ids=str)
def test_scales_of_the_values(news, dtype):
    """Scales of V that differ by 2^20 between pages: every weight has all its bits, whatever the scale of its page."""
    gen = torch.Generator().manual_seed(32)
    lengths = [160, 320]
    q, cache, host, table = _problem(gen, news, lengths, 4, 2, 64, 16, dtype, spread=10)
    scale = 0.3
    got = _run(q, cache, table, news, lengths, scale, True).double().cpu()
    want, bound = ref.attention(q, host[0], host[1], table, news, lengths, 16, scale, True)
    if dtype == torch.float16:  # weights times the scale are rounded: 2^-25 of the largest such product in the place of one weight's
        bound = bound * 2 ** 4
    ok = want.abs() < 6e4
    assert ((got - want).abs()[ok] <= (bound + ref.half_step(dtype) * want.abs())[ok] + 2.0 ** -25).all()


@pytest.mark.parametrize("news,lengths", [([1, 1, 1], [300, 20, 0]), ([4, 2, 3], [130, 17, 9]), ([70, 3], [200, 3])], ids=str)
def test_what_a_row_does_not_see(news, lengths):
    """NaN in every place behind a sequence's last token, in pages of others and in pages that are not there, and (causal) NaN tokens that only
    later rows see."""
    gen = torch.Generator().manual_seed(33)
    page = 16
    for dtype in (torch.float16, torch.bfloat16):
        q, cache, host, table = _problem(gen, news, lengths, 4, 2, 128, page, dtype)
        want = _check(q, cache, host, table, news, lengths, page, 0.1, True)
        seen = torch.zeros(cache.k.shape[0], page, dtype=torch.bool)
        for b, n in enumerate(lengths):
            for t in range(n):
                seen[int(table[b, t // page]), t % page] = True
        hidden = ~seen.cuda()
        for t in (cache.k, cache.v):
            t.view(torch.uint8).transpose(1, 2)[hidden] = 0x7f
        unused = ~seen.any(1).cuda()
        for t in (cache.k_scale, cache.v_scale):
            t[unused] = float("nan")
        assert torch.equal(_run(q, cache, table, news, lengths, 0.1, True), want)
        if max(news) == 1:
            continue
        # the last token of the first sequence: NaN in one column of V for the last row alone, in K for all of that row
        last = lengths[0] - 1
        p, place = int(table[0, last // page]), last % page
        cache.v.view(torch.uint8)[p, 1, place, 77] = 0xff
        got = _run(q, cache, table, news, lengths, 0.1, True)
        r = news[0] - 1
        assert torch.isnan(got[r, 2:, 77]).all()
        got[r, 2:, 77] = want[r, 2:, 77]
        assert torch.equal(got, want)
        cache.k.view(torch.uint8)[p, 0, place, 3] = 0x7f
        got = _run(q, cache, table, news, lengths, 0.1, True)
        assert torch.isnan(got[r, :2]).all()
        got[r, :2] = want[r, :2]
        got[r, 2:, 77] = want[r, 2:, 77]
        assert torch.equal(got, want)


def test_nan_and_infinite_queries():
    gen = torch.Generator().manual_seed(34)
    news, lengths = [3, 40], [50, 60]
    q, cache, host, table = _problem(gen, news, lengths, 4, 2, 64, 16, torch.float16)
    want = _run(q, cache, table, news, lengths, 0.1, True)
    q[1, 2, 5], q[20, 0, 0] = float("nan"), float("inf")
    got = _run(q, cache, table, news, lengths, 0.1, True)
    assert torch.isnan(got[1, 2]).all() and torch.isnan(got[20, 0]).all()
    got[1, 2], got[20, 0] = want[1, 2], want[20, 0]
    assert torch.equal(got, want)


@pytest.mark.parametrize("news", [[1, 1, 1, 1, 1], [2, 3, 1, 4, 6], [40, 1, 90, 3, 2]], ids=str)
def test_pages_that_are_not_there(news):
    """Page numbers outside of the cache anywhere in a sequence, tokens beyond the table, sequences without any page: zeros."""
    gen = torch.Generator().manual_seed(35)
    lengths = [100, 90, 130, 64, 500]
    for dtype in (torch.float16, torch.bfloat16):
        q, cache, host, table = _problem(gen, news, lengths, 4, 2, 64, 16, dtype, width=8)
        table[0, 0], table[1, 3], table[2, 2:5], table[3, :] = -1, 10 ** 6, -2 ** 31, 2 ** 31 - 1
        got = _check(q, cache, host, table, news, lengths, 16, 0.2, True)
        row = sum(news[:3])
        assert (got[row:row + news[3]] == 0).all()


def test_rows_outside_and_strides():
    """Padding before the first and behind the last sequence, queries and results as slices of wider tensors, a table that is a slice."""
    gen = torch.Generator().manual_seed(36)
    news, lengths = [3, 1, 80], [60, 33, 100]
    q, cache, host, table = _problem(gen, news, lengths, 4, 2, 96, 16, torch.bfloat16)
    want = _check(q, cache, host, table, news, lengths, 16, 0.1, True)
    wide = torch.full((sum(news) + 7, 9, 96), float("nan"), dtype=torch.bfloat16, device="cuda")
    out = torch.full_like(wide, 5.0)
    wide[2:2 + sum(news), 3:7] = q.cuda()
    tables = torch.full((3, table.shape[1] + 5), -7, dtype=torch.int32, device="cuda")
    tables[:, 2:2 + table.shape[1]] = table.int().cuda()
    starts = 2 + torch.tensor([0, 3, 4, 84], dtype=torch.int32, device="cuda")
    got = mcf.cache_attention(wide[:, 3:7], cache, tables[:, 2:2 + table.shape[1]], torch.tensor(lengths).int().cuda(), 0.1, starts, out=out[:, 1:5])
    assert torch.equal(got[2:2 + sum(news)], want)
    out[2:2 + sum(news), 1:5] = 5.0
    assert (out == 5).all()


def test_starts_of_no_order():
    q = torch.randn(6, 2, 64).half().cuda()
    c = mcf.kv_cache(8, 1, 16, 64)
    table = torch.arange(8, dtype=torch.int32).view(4, 2).cuda()
    lengths = torch.tensor([3, 9, -2, 2 ** 31 - 1], dtype=torch.int32).cuda()
    for starts in ([0, -5, 3, 9, 2], [7, 7, 7, 7, 100], [2 ** 31 - 1, -2 ** 31, 0, 1, 6], [6, 4, 2, 0, -1]):
        mcf.cache_attention(q, c, table, lengths, 0.1, torch.tensor(starts, dtype=torch.int32).cuda())
    torch.cuda.synchronize()


@pytest.mark.parametrize("tokens,heads,width", [(64, 16, 8), (64, 2, 8), (300, 16, 2), (64, 4, 100)])
def test_starts_that_overlap(tokens, heads, width):
    """Every second sequence claims all rows: many times the tiles that rows and sequences allow for."""
    batch = 60
    q = torch.randn(tokens, heads, 64).half().cuda()
    c = mcf.kv_cache(8, 1, 16, 64)
    table = torch.zeros(batch, width, dtype=torch.int32, device="cuda")
    lengths = torch.full((batch,), 16 * width, dtype=torch.int32, device="cuda")
    starts = torch.tensor([0, tokens] * (batch // 2) + [0], dtype=torch.int32, device="cuda")
    out = mcf.cache_attention(q, c, table, lengths, 0.1, starts)
    torch.cuda.synchronize()
    assert out.shape == q.shape


@pytest.mark.parametrize("batch", [64, 66])
def test_starts_that_overlap_beyond_what_is_counted(batch):
    """Sequences of 2^30 tokens that claim all rows each: more than 2^32 pieces of work.  Nothing is computed, and nothing is joined."""
    tokens = 6 * batch
    q = torch.randn(tokens, 8, 64).half().cuda()
    c = mcf.kv_cache(8, 1, 128, 64)
    table = torch.zeros(1, 1 << 23, dtype=torch.int32, device="cuda").expand(batch, -1)
    lengths = torch.full((batch,), 1 << 30, dtype=torch.int32, device="cuda")
    starts = torch.tensor([0, tokens] * (batch // 2) + [0], dtype=torch.int32, device="cuda")
    out = torch.full_like(q, 3.0)
    mcf.cache_attention(q, c, table, lengths, 0.1, starts, out=out)
    assert (out == 3).all()


def test_empty():
    c = mcf.kv_cache(2, 1, 16, 64)
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    q = torch.zeros(0, 4, 64, dtype=torch.float16, device="cuda")
    assert mcf.cache_attention(q, c, torch.zeros(0, 3, dtype=torch.int32, device="cuda"), none, 1.0).shape == (0, 4, 64)
    q = torch.ones(2, 4, 64, dtype=torch.float16, device="cuda")
    length = torch.tensor([9, 0], dtype=torch.int32, device="cuda")
    for cache, table in ((c, torch.zeros(2, 0, dtype=torch.int32, device="cuda")), (mcf.kv_cache(0, 1, 16, 64), torch.zeros(2, 1, dtype=torch.int32, device="cuda"))):
        assert (mcf.cache_attention(q, cache, table, length, 1.0) == 0).all()


def _long(dtype, new, n, pages_before=0, size=128):
    """A long sequence and a 64-bit reference on the device."""
    gen = torch.Generator(device="cuda").manual_seed(37)
    page, heads = 64, 1
    pages = pages_before + -(-n // page)
    c = mcf.kv_cache(pages, heads, page, size)
    used = c.k[pages_before:], c.v[pages_before:]
    for t in used:
        t.copy_((torch.randn(t.shape, generator=gen, device="cuda") * 100).clamp(-448, 448).to(ref.E4M3))
    c.k_scale.fill_(2.0 ** -7)
    c.v_scale.fill_(2.0 ** -6)
    table = pages_before + torch.randperm(pages - pages_before, generator=gen, device="cuda").int()[None]
    q = torch.randn(new, 4, size, generator=gen, device="cuda").to(dtype)
    got = mcf.cache_attention(q, c, table, torch.tensor([n], dtype=torch.int32, device="cuda"), 0.09, torch.tensor([0, new], dtype=torch.int32, device="cuda"))
    at = table[0].long()
    k, v = ((t[at, 0].double() * s).flatten(0, 1)[:n] for t, s in ((c.k, 2.0 ** -7), (c.v, 2.0 ** -6)))
    s = 0.09 * q.double().flatten(0, 1) @ k.T
    limit = (n - new + torch.arange(new, device="cuda") + 1).repeat_interleave(4)
    s.masked_fill_(torch.arange(n, device="cuda")[None] >= limit[:, None], -math.inf)
    p = torch.softmax(s, -1)
    want, mean = p @ v, p @ v.abs()
    big = 0.09 * (q.double().flatten(0, 1).abs() @ k.abs().T).amax(-1, keepdim=True)
    # as in the reference, and sums over the tokens in fp32 of up to n terms in chains of n / 128 and their joining
    bound = mean * (ref.half_step(dtype) + 2 * (size + 32) * 2.0 ** -24 * big + (n / 64 + 64) * 2.0 ** -24)
    if dtype == torch.float16:
        bound = bound + 2.0 ** -25 * p.amax(-1, keepdim=True) * v.abs().sum(0)
    off = (got.double().flatten(0, 1) - want).abs() - bound - ref.half_step(dtype) * want.abs()
    assert off.max() <= 2.0 ** -25, off.max()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("new", [1, 3, 150])
def test_long(new, dtype):
    _long(dtype, new, 50001)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("new", [1, 7, 12, 16, 30, 60])
@pytest.mark.parametrize("size", [64, 80, 96, 128, 192, 256])
def test_parts(size, new, dtype):
    """Tiles whose tokens are split over blocks, of every number of rows and every size."""
    _long(dtype, new, 5003, size=size)


@pytest.mark.parametrize("new,hq,heads", [(70, 2, 2), (1, 40, 2), (9, 4, 1)])
def test_more_sequences_than_lanes(new, hq, heads):
    """67 sequences, of one length that is long enough to be split and many short ones."""
    gen = torch.Generator().manual_seed(39)
    news = [new if i % 9 else 0 for i in range(67)]
    lengths = [new + (3 * i) % 40 for i in range(66)] + [1500]
    q, cache, host, table = _problem(gen, news, lengths, hq, heads, 64, 16, torch.bfloat16)
    _check(q, cache, host, table, news, lengths, 16, 0.1, True)


@pytest.mark.parametrize("new", [1, 3, 60])
def test_captured_by_others(new):
    """A stream that the HIP runtime captures for someone else has no workspace: the call is one kernel, and its replays equal the eager call."""
    import ctypes
    import re
    hip = ctypes.CDLL(re.search(r"\S*/libamdhip64\.so\S*", open("/proc/self/maps").read()).group())
    gen = torch.Generator().manual_seed(40)
    q, cache, host, table = _problem(gen, [new], [2500], 4, 1, 64, 16, torch.float16)
    starts = torch.tensor([0, new], dtype=torch.int32, device="cuda")
    args = [q.cuda(), cache, table.int().cuda(), torch.tensor([2500]).int().cuda(), 0.1, starts]
    out = mcf.cache_attention(*args)
    want, bound = ref.attention(q, host[0], host[1], table, [new], [2500], 16, 0.1, True)
    ref.check(out, want, bound, torch.float16)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    handle, graph, exe, n = ctypes.c_void_p(stream.cuda_stream), ctypes.c_void_p(), ctypes.c_void_p(), ctypes.c_size_t()
    assert hip.hipStreamBeginCapture(handle, 1) == 0
    try:
        mcf.cache_attention(*args, out=out, stream=stream)
        with pytest.raises(mcf.McfError) as refused:
            mcf.norm_rotate_backward(args[0], None, args[0], q_weight=torch.ones(64, dtype=torch.float16, device="cuda"), stream=stream)
    finally:
        assert hip.hipStreamEndCapture(handle, ctypes.byref(graph)) == 0
    assert refused.value.status == 2
    assert hip.hipGraphGetNodes(graph, None, ctypes.byref(n)) == 0 and n.value == 1
    assert hip.hipGraphInstantiate(ctypes.byref(exe), graph, None, None, ctypes.c_size_t(0)) == 0
    for rep in range(3):
        out.fill_(-3.0)
        torch.cuda.synchronize()
        assert hip.hipGraphLaunch(exe, handle) == 0
        torch.cuda.synchronize()
        ref.check(out, want, bound, torch.float16)
    assert hip.hipGraphExecDestroy(exe) == 0 and hip.hipGraphDestroy(graph) == 0


def test_beyond_32_bits():
    """Pages behind 4 GiB of cache."""
    _long(torch.bfloat16, 2, 1000, pages_before=(5 << 30) // (64 * 128))


@pytest.mark.parametrize("new", [1, 3])
def test_streams_graphs_and_workspaces(new):
    """Split calls on two streams at once and captured into two graphs that are replayed one after the other: every result is that of the call
    alone, bit for bit; lengths that change between replays are followed."""
    gen = torch.Generator().manual_seed(38)
    problems = []
    for n in (900, 1300):
        news, lengths = [new], [n]
        q, cache, host, table = _problem(gen, news, lengths, 4, 2, 64, 16, torch.bfloat16)
        starts = torch.tensor([0, new], dtype=torch.int32, device="cuda")
        args = [q.cuda(), cache, table.int().cuda(), torch.tensor(lengths).int().cuda(), 0.1, starts]
        problems.append((args, mcf.cache_attention(*args), (q, host, table, n)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in problems]
    outs = [torch.empty_like(p[1]) for p in problems]
    for _ in range(10):
        for s, (args, _, _), out in zip(streams, problems, outs):
            mcf.cache_attention(*args, out=out, stream=s)
    torch.cuda.synchronize()
    for (_, want, _), out in zip(problems, outs):
        assert torch.equal(out, want)
    graphs = []
    for (args, _, _), out in zip(problems, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            mcf.cache_attention(*args, out=out)
        graphs.append(g)
    for rep in range(4):
        junk = [torch.full((1 << i,), float("nan"), device="cuda") for i in range(10, 20)]
        for out in outs:
            out.fill_(-3.0)
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for (_, want, _), out in zip(problems, outs):
            assert torch.equal(out, want), rep
        del junk
    args, _, (q, host, table, n) = problems[0]
    args[3].fill_(n - 700)
    graphs[0].replay()
    torch.cuda.synchronize()
    want, bound = ref.attention(q, host[0], host[1], table, [new], [n - 700], 16, 0.1, True)
    ref.check(outs[0], want, bound, torch.bfloat16)
