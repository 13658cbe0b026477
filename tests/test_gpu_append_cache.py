"""Keys and values into the paged cache of 8 bits, against the definition in 64 bits: scales have to be equal, held values within half a step of
e4m3 of the 64-bit value (so that a value next to a border may be held as either neighbour), everything else untouched."""
import pytest
import torch

import cache_reference as ref
import paper_2506_22169_amd as mcf

pytestmark = pytest.mark.gpu


def half_step_e4m3(x, s):
    """Half a step of e4m3 at x / s, times s (and a hair for the sides of a border)."""
    m = (x / s).abs().clamp_min(2.0 ** -6)
    return torch.exp2(torch.floor(torch.log2(m)) - 4) * s * (1 + 2.0 ** -20)


class Cache:
    """A cache on the device with random contents, and the same in 64 bits."""

    def __init__(self, gen, pages, heads, page, size, wide=False):
        x = torch.randn(pages, heads, page, size, generator=gen)
        self.parts = {}
        dev = []
        for name in ("k", "v"):
            s = 2.0 ** torch.randint(-8, -5, (pages, heads), generator=gen).double()
            q = (torch.randn(pages, heads, page, size, generator=gen) * 100).clamp(-448, 448).to(ref.E4M3)
            self.parts[name] = {"v": q.double(), "s": s}
            if wide:  # both in one tensor, page by page
                both = torch.zeros(pages, 2, heads, page, size, dtype=ref.E4M3, device="cuda")
                t = both[:, 0 if name == "k" else 1]
                t.copy_(q)
                scales = torch.zeros(pages, heads + 3, device="cuda")[:, :heads]
            else:
                t, scales = q.cuda(), torch.zeros(pages, heads, device="cuda")
            scales.copy_(s)
            dev += [t, scales]
        self.dev = mcf.KVCache(dev[0], dev[2], dev[1], dev[3])
        self.before = [t.clone() for t in self.dev]

    def touched(self, table, news, lengths, page):
        """Masks of pages and of places that the new tokens go to, and of places that may be rounded again."""
        pages, heads = self.parts["k"]["s"].shape
        new = torch.zeros(pages, page, dtype=torch.bool)
        again = torch.zeros(pages, page, dtype=torch.bool)
        for b, n in enumerate(news):
            for at in range(max(0, lengths[b] - n), min(lengths[b], table.shape[1] * page)):
                p = int(table[b, at // page])
                if 0 <= p < pages:
                    new[p, at % page] = True
                    if at == max(0, lengths[b] - n):
                        again[p, :at % page] = True
        return new, again

    def check(self, xk, xv, table, news, lengths, page):
        new, again = self.touched(table, news, lengths, page)
        for name, x, held, scale, was, was_scale in (("k", xk, self.dev.k, self.dev.k_scale, self.before[0], self.before[2]),
                                                     ("v", xv, self.dev.v, self.dev.v_scale, self.before[1], self.before[3])):
            want = self.parts[name]
            ref.append(want, x, table, news, lengths, page, name)
            got, s = held.double().cpu(), scale.double().cpu()
            assert torch.equal(s[new.any(1)], want["s"][new.any(1)]), name
            assert torch.equal(s[~new.any(1)], was_scale.double().cpu()[~new.any(1)]), name
            bytes_now, bytes_was = held.cpu().view(torch.uint8), was.cpu().view(torch.uint8)
            same = (bytes_now == bytes_was).all(-1).transpose(1, 2)  # [pages, page, heads]
            assert same[~(new | again)].all(), f"{name}: a place that no token goes to was written"
            # rounded again: exact, from the same values
            where = again[:, None, :, None].expand_as(got)
            assert torch.equal(torch.nan_to_num(got[where], nan=-1e9), torch.nan_to_num(want["v"][where], nan=-1e9)), name
            # new ones: within half a step of the value
            row = 0
            for b, n in enumerate(news):
                for i in range(n):
                    at = lengths[b] - n + i
                    if at < 0 or at // page >= table.shape[1] or not 0 <= int(table[b, at // page]) < got.shape[0]:
                        continue
                    p = int(table[b, at // page])
                    value, sc = x[row + i], s[p][:, None]
                    g = got[p, :, at % page] * sc
                    fine = torch.isfinite(value)
                    assert torch.equal(torch.isnan(g), ~fine), (name, b, i)
                    off = torch.where(fine, (g - value).abs() - half_step_e4m3(torch.nan_to_num(value), sc), -1.0)
                    assert off.max() <= 0, (name, b, i, off.max())
                row += n


def _step(cache, gen, table, news, lengths, page, dtype, hq, heads, size, norm=True, rotary=None, interleaved=False, pad=0, single=False, change=None, positions=None):
    total = sum(news)
    qkv = torch.randn(total + 2 * pad, hq + 2 * heads, size, generator=gen).to(dtype)
    if change:
        change(qkv)
    w = [(1 + 0.2 * torch.randn(size, generator=gen)).to(dtype) for _ in range(2)] if norm else [None, None]
    rotary = size if rotary is None else rotary
    cos, sin = ref.tables(rotary, positions or max(lengths) + 1) if rotary else (None, None)
    at = torch.cat([torch.arange(n - m, n) for m, n in zip(news, lengths)] + [torch.zeros(0, dtype=torch.long)])
    starts = None if single else (pad + torch.tensor([sum(news[:i]) for i in range(len(news) + 1)])).int().cuda()
    d = qkv.cuda()
    dev = lambda t: None if t is None else t.cuda()
    out = torch.full((total + 2 * pad, hq, size), 7.0, dtype=dtype, device="cuda")
    got = mcf.append_cache(cache.dev, d[:, hq:hq + heads], d[:, hq + heads:], table.int().cuda(), torch.tensor(lengths).int().cuda(), starts, dev(cos), dev(sin),
                           dev(w[1]), d[:, :hq] if hq else None, dev(w[0]) if hq else None, eps=1e-5, interleaved=interleaved, q_out=out if hq else None)
    x = qkv[pad:pad + total]
    xk = ref.norm_rotate(x[:, hq:hq + heads], cos, sin, at, w[1], 1e-5, interleaved)
    cache.check(xk, x[:, hq + heads:].double(), table, news, lengths, page)
    if hq:
        want = ref.norm_rotate(x[:, :hq], cos, sin, at, w[0], 1e-5, interleaved)
        ref.check(got[pad:pad + total], want, ref.norm_rotate_bound(x[:, :hq], want, cos, w[0], 1e-5, interleaved, dtype), dtype, "q")
        assert (got[:pad] == 7).all() and (got[pad + total:] == 7).all()


def _table(gen, pages, batch, width):
    t = torch.full((batch, width), -1)
    t.view(-1)[:min(pages, batch * width)] = torch.randperm(pages, generator=gen)[:batch * width]
    return t


# news, lengths (with the new ones), heads of q, heads, size, page
CASES = [
    ([1], [1], 1, 1, 64, 16), ([1, 1, 1], [17, 16, 33], 4, 2, 128, 16), ([5, 0, 40], [5, 9, 47], 3, 3, 80, 32), ([130, 1], [200, 128], 0, 2, 96, 64),
    ([260], [300], 2, 1, 256, 128), ([17, 31, 16], [33, 31, 48], 2, 2, 192, 16), ([0, 0], [0, 5], 2, 1, 64, 16), ([64, 64], [64, 128], 8, 8, 64, 64),
    ([1] * 70, list(range(1, 71)), 2, 1, 64, 16), ([2] * 130, list(range(2, 132)), 1, 1, 64, 16),
]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("norm,interleaved,pad", [(True, False, 0), (False, True, 3)])
@pytest.mark.parametrize("i", range(len(CASES)))
def test_append(i, norm, interleaved, pad, dtype):
    news, lengths, hq, heads, size, page = CASES[i]
    gen = torch.Generator().manual_seed(300 + i)
    width = max(-(-n // page) for n in lengths) + 1
    pages = len(news) * width + 2
    cache = Cache(gen, pages, heads, page, size, wide=norm)
    _step(cache, gen, _table(gen, pages, len(news), width), news, lengths, page, dtype, hq, heads, size, norm=norm, interleaved=interleaved, pad=pad)


@pytest.mark.parametrize("page,size", [(16, 64), (128, 128)])
def test_one_by_one_and_at_once(page, size):
    """A prompt at once, in pieces and token by token: the same scales, and values that differ only where a page's scale grew on the way
    (a value that fell below the smallest exponent in between)."""
    gen = torch.Generator().manual_seed(9)
    n = 2 * page + 5
    k, v = (torch.randn(n, 2, size, generator=gen).bfloat16().cuda() for _ in range(2))
    cos, sin = (t.cuda() for t in ref.tables(size, n))
    w = torch.ones(size, dtype=torch.bfloat16, device="cuda")
    table = torch.tensor([[3, 0, 2]], dtype=torch.int32, device="cuda")
    results = []
    for cut in (n, 7, 1):
        c = mcf.kv_cache(4, 2, page, size)
        for at in range(0, n, cut):
            m = min(cut, n - at)
            mcf.append_cache(c, k[at:at + m], v[at:at + m], table, torch.tensor([at + m], dtype=torch.int32, device="cuda"),
                             torch.tensor([0, m], dtype=torch.int32, device="cuda"), cos, sin, w)
        results.append([t.double().cpu() for t in c])
    for r in results[1:]:
        assert torch.equal(r[2], results[0][2]) and torch.equal(r[3], results[0][3])
        for a, b, s in zip(r[:2], results[0][:2], r[2:]):
            # rounded at a smaller scale first, then again: within half a step of the smallest exponent more
            assert ((a - b).abs() <= 2.0 ** -9).all()
            big = b.abs() >= 2.0 ** -6
            assert torch.equal(a[big], b[big])


@pytest.mark.parametrize("hq", [0, 3, 64])
def test_more_blocks_than_two_rounds(hq):
    # 34 pages of 32 heads in blocks of 512 lanes, of which 512 are resident: they lie among those of the queries
    gen = torch.Generator().manual_seed(hq)
    page, size, heads = 64, 128, 32
    news = [1, 130, 0, 64, 65, 33, 190, 2, 60, 61, 62, 32]
    lengths = [9, 130, 7, 128, 200, 40, 192, 66, 64, 100, 62, 33]
    table = _table(gen, 64, len(news), 4)
    _step(Cache(gen, 64, heads, page, size), gen, table, news, lengths, page, torch.bfloat16, hq, heads, size, pad=1)


def test_scales():
    """Borders of the scale (448 and just above, times powers of two), zeros, the smallest and the largest values, infinities and NaN."""
    gen = torch.Generator().manual_seed(11)
    rows = torch.zeros(12, 2, 64, dtype=torch.bfloat16)
    big = [448.0, 450.0, 1.75, 1.7578125, 0.0, 2.0 ** -126, 3e38, 2.0 ** -95, 1.0, 1.0, 2.0 ** -133, -448.0]
    for t, m in enumerate(big):
        rows[t, 0, 5] = m
        rows[t, 1] = (torch.randn(64, generator=gen).bfloat16() * 0.01).bfloat16()
    rows[8, 0, 9] = float("inf")
    rows[9, 0, 9], rows[9, 1, 3] = float("nan"), -float("inf")
    cache = Cache(gen, 14, 2, 16, 64)
    table = torch.arange(12)[:, None]
    w = dict(starts=None, cos=None)
    lengths = torch.full((12,), 1, dtype=torch.int32).cuda()
    mcf.append_cache(cache.dev, rows.cuda(), rows.flip(0).contiguous().cuda(), table.int().cuda(), lengths, **w)
    cache.check(rows.double(), rows.flip(0).double(), table, [1] * 12, [1] * 12, 16)


def test_places_that_are_not_there():
    """Pages outside of the cache, tokens beyond the table, more rows than tokens, positions beyond the tables: nothing is written for them,
    or NaN where only the rotation has no row."""
    gen = torch.Generator().manual_seed(12)
    table = torch.tensor([[0, -1, 2], [3, 99, 5], [2 ** 31 - 1, 6, 7], [8, 9, 10], [-2 ** 31, 11, 12]])
    news, lengths = [40, 40, 20, 30, 9], [40, 48, 20, 60, 4]
    cache = Cache(gen, 13, 2, 16, 64)
    _step(cache, gen, table, news, lengths, 16, torch.float16, 3, 2, 64)
    cache = Cache(gen, 13, 2, 16, 64)
    _step(cache, gen, table, news, lengths, 16, torch.bfloat16, 3, 2, 64, positions=17)


def test_starts_of_no_order():
    """starts that run backwards or outside of the rows: no row out of bounds is touched."""
    k = torch.randn(6, 1, 64).half().cuda()
    table = torch.arange(8, dtype=torch.int32).view(4, 2).cuda()
    lengths = torch.tensor([3, 9, 2, 30], dtype=torch.int32).cuda()
    c = mcf.kv_cache(8, 1, 16, 64)
    for starts in ([0, -5, 3, 9, 2], [7, 7, 7, 7, 100], [2 ** 31 - 1, -2 ** 31, 0, 1, 6], [6, 4, 2, 0, -1]):
        mcf.append_cache(c, k, k, table, lengths, torch.tensor(starts, dtype=torch.int32).cuda(), q=k)
    torch.cuda.synchronize()


def test_empty():
    c = mcf.kv_cache(2, 1, 16, 64)
    e = torch.zeros(0, 1, 64, dtype=torch.float16, device="cuda")
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    assert mcf.append_cache(c, e, e, torch.zeros(0, 3, dtype=torch.int32, device="cuda"), none, q=e).shape == (0, 1, 64)
    one = torch.ones(1, 1, 64, dtype=torch.float16, device="cuda")
    length = torch.ones(1, dtype=torch.int32, device="cuda")
    mcf.append_cache(c, one, one, torch.zeros(1, 0, dtype=torch.int32, device="cuda"), length)  # no column in the table
    mcf.append_cache(mcf.kv_cache(0, 1, 16, 64), one, one, torch.zeros(1, 1, dtype=torch.int32, device="cuda"), length)  # no pages
    assert (c.k.view(torch.uint8) == 0).all() and (c.v_scale == 0).all()


def test_beyond_32_bits():
    """Pages behind 4 GiB of cache."""
    heads, page, size = 8, 128, 256
    pages = (5 << 30) // (heads * page * size)
    c = mcf.kv_cache(pages, heads, page, size)
    gen = torch.Generator().manual_seed(13)
    k, v = (torch.randn(2, heads, size, generator=gen).half() for _ in range(2))
    table = torch.tensor([[pages - 1], [pages - 2]], dtype=torch.int32)
    mcf.append_cache(c, k.cuda(), v.cuda(), table.cuda(), torch.tensor([1, 1], dtype=torch.int32).cuda())
    for b, p in enumerate((pages - 1, pages - 2)):
        for x, held, s in ((k, c.k, c.k_scale), (v, c.v, c.v_scale)):
            got = held[p, :, 0].double().cpu() * s[p].double().cpu()[:, None]
            value = x[b].double()
            assert ((got - value).abs() <= half_step_e4m3(value, s[p].double().cpu()[:, None])).all()
