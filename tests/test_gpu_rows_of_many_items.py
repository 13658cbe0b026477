"""The kernels' forms for many rows (four heads an item, lanes that go through several items), which start at some ten thousand rows: against the
definition in 64 bits, against the same rows in calls below that number, and for the weights' gradients in sums that are exact, so that
one row too few or too many shows."""
import pytest
import torch

import cache_reference as ref
import paper_2506_22169_amd as mcf

pytestmark = pytest.mark.gpu


def _lanes(size):
    return 4 if size <= 64 else 8 if size <= 128 else 16 if size <= 256 else 32


def _rows(gen, tokens, heads, size, dtype):
    return torch.randn(tokens, heads, size, generator=gen, device="cuda").to(dtype)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("norm,interleaved", [(True, False), (False, True)])
@pytest.mark.parametrize("size,hq,hk", [(48, 9, 4), (64, 13, 3), (80, 4, 1), (128, 13, 3), (192, 6, 0), (256, 1, 3), (512, 9, 4)])
def test_forward(size, hq, hk, norm, interleaved, dtype):
    gen = torch.Generator(device="cuda").manual_seed(size)
    tokens = -(-8192 * 64 // ((hq + hk) * _lanes(size))) + 5  # a little above where items of four heads begin
    rotary = size if size % 32 else size // 2
    q, k = _rows(gen, tokens, hq, size, dtype), _rows(gen, tokens, hk, size, dtype) if hk else None
    wq, wk = ((1 + 0.2 * torch.randn(size, generator=gen, device="cuda")).to(dtype) for _ in range(2)) if norm else (None, None)
    cos, sin = (t.cuda() for t in ref.tables(rotary, 1000))
    at = torch.randint(0, 1000, (tokens,), generator=gen, device="cuda")
    kw = dict(eps=1e-5, interleaved=interleaved)
    got = mcf.norm_rotate(q, k, cos, sin, at, wq, wk, **kw)
    for x, w, y in ((q, wq, got[0]), (k, wk, got[1])):
        if x is None:
            continue
        want = ref.norm_rotate(x, cos, sin, at, w, 1e-5, interleaved)
        ref.check(y, want.cpu(), ref.norm_rotate_bound(x, want, cos, w, 1e-5, interleaved, dtype).cpu(), dtype)
    half = tokens // 2
    for rows in (slice(0, half), slice(half, tokens)):
        part = mcf.norm_rotate(q[rows], None if k is None else k[rows], cos, sin, at[rows], wq, wk, **kw)
        assert torch.equal(part[0], got[0][rows]) and (k is None or torch.equal(part[1], got[1][rows]))


# blocks of items of two heads (256 / lanes an item each): more than 768 of them and more than 1536, q and k uneven
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("blocks", [700, 1100, 2500])
@pytest.mark.parametrize("size,hq,hk", [(64, 5, 1), (80, 1, 6), (128, 13, 3), (192, 2, 3), (256, 3, 0), (512, 1, 4)])
def test_backward(size, hq, hk, blocks, dtype):
    """x of ones under either sign (its norm is 1), gradients of small whole numbers, angles of quarter turns: every sum is a whole number."""
    gen = torch.Generator(device="cuda").manual_seed(size + blocks)
    tokens = blocks * (256 // _lanes(size)) // ((hq + 1) // 2 + (hk + 1) // 2) + 1
    whole = size & (size - 1) == 0
    cos = torch.tensor([1.0, 0.0, -1.0, 0.0], device="cuda")[:, None].expand(4, size // 2 if size % 32 == 0 else 8).contiguous()
    sin = torch.tensor([0.0, 1.0, 0.0, -1.0], device="cuda")[:, None].expand(4, cos.shape[1]).contiguous()
    at = torch.randint(0, 4, (tokens,), generator=gen, device="cuda")
    w = torch.ones(size, dtype=dtype, device="cuda")

    def signs(h):
        return (torch.randint(0, 2, (tokens, h, size), generator=gen, device="cuda") * 2 - 1).to(dtype)

    def numbers(h):  # of other sizes, whose 1 / size is rounded, a row in 32 has any, and its sums stay within a hundredth
        x = torch.randint(-4, 5, (tokens, h, size), generator=gen, device="cuda")
        return (x if whole else x * (torch.randint(0, 32, (tokens, h, 1), generator=gen, device="cuda") == 0)).to(dtype)

    q, dq, k, dk = signs(hq), numbers(hq), signs(hk) if hk else None, numbers(hk) if hk else None
    got = mcf.norm_rotate_backward(dq, dk, q, k, cos, sin, at, w, w if hk else None, eps=0.0)
    for x, dy, dx, dw in ((q, dq, got[0], got[2]), (k, dk, got[1], got[3])):
        if x is None:
            assert dx is None and dw is None
            continue
        g = ref.turn(dy.double(), cos, sin, at, False, back=True)
        terms = g * x.double()
        want, want_w = g - x.double() * terms.mean(-1, keepdim=True), terms.sum((0, 1))
        if whole:  # nothing is rounded but dx, once
            assert torch.equal(dx, want.to(dtype)) and torch.equal(dw.double(), want_w)
        else:
            # r is 1 within 4 steps of 2^-24; chains of a lane's items, 64 groups, 12 parts and 64 slices at most
            most = terms.abs().sum((0, 1)).max().item()
            bound = (4 + 2 * tokens * (hq + hk) // (blocks * 256 // _lanes(size)) + 64 + 12 + 64 + 40) * 2.0 ** -24 * most
            assert bound < 0.5
            assert ((dw.double() - want_w).abs() <= bound).all()
            ref.check(dx, want.cpu(), torch.full_like(want, 64 * 2.0 ** -24 * 8).cpu(), dtype)
    again = mcf.norm_rotate_backward(dq, dk, q, k, cos, sin, at, w, w if hk else None, eps=0.0)
    assert all(a is b is None or torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("size,page,hq,heads,norm", [(64, 16, 13, 1, True), (80, 32, 9, 2, False), (128, 64, 6, 2, True), (192, 32, 13, 1, False), (256, 128, 9, 2, True)])
def test_append(size, page, hq, heads, norm, dtype):
    """Queries four heads at a time: the bits of norm_rotate, and the cache as by calls of a page or two each."""
    gen = torch.Generator(device="cuda").manual_seed(size)
    total = -(-8192 * 64 // (hq * _lanes(size))) + 7
    news = [total // 2, 0, total // 3, total - total // 2 - total // 3]
    width = -(-max(news) // page)
    q, k, v = (_rows(gen, total, h, size, dtype) for h in (hq, heads, heads))
    wq, wk = ((1 + 0.2 * torch.randn(size, generator=gen, device="cuda")).to(dtype) for _ in range(2)) if norm else (None, None)
    cos, sin = (t.cuda() for t in ref.tables(size, max(news)))
    table = torch.randperm(4 * width, generator=gen, device="cuda").view(4, width).int()
    starts = [sum(news[:i]) for i in range(5)]
    whole = mcf.kv_cache(4 * width, heads, page, size)
    got = mcf.append_cache(whole, k, v, table, torch.tensor(news).int().cuda(), torch.tensor(starts).int().cuda(), cos, sin, wk, q, wq)
    at = torch.cat([torch.arange(n) for n in news]).cuda()
    half = total // 2
    for rows in (slice(0, half), slice(half, total)):
        assert torch.equal(got[rows], mcf.norm_rotate(q[rows], None, cos, sin, at[rows], wq)[0])
    parts = mcf.kv_cache(4 * width, heads, page, size)
    for first in range(0, max(news), 2 * page):
        these = [min(n, first + 2 * page) for n in news]
        rows = torch.cat([torch.arange(s + min(first, n), s + n) for s, n in zip(starts, these)]).cuda()
        cut = [0] + torch.tensor([max(0, n - first) for n in these]).cumsum(0).tolist()
        mcf.append_cache(parts, k[rows], v[rows], table, torch.tensor(these).int().cuda(), torch.tensor(cut).int().cuda(), cos, sin, wk)
    for a, b in zip(whole, parts):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
