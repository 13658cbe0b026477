"""Starts that do not ascend, run outside of the rows or overlap: what the calls write stays within the rows of sequences and within the pages that their table
names, and what they read stays within what belongs to the call.  Every operand lies between guards: of those that are written a pattern that has
to be there afterwards, of those that are read what would show in a result (NaN, numbers of pages of NaN)."""
import ctypes

import pytest
import torch

import cache_reference as ref
import paper_2506_22169_amd as mcf
from paper_2506_22169_amd.binding import load_library

pytestmark = pytest.mark.gpu

TOKENS, HEADS, SIZE, PAGE, PAGES = 6, 2, 64, 16, 12  # pages 0 .. 7 are named by the tables, the others by the guards of the tables alone
GUARD = 5
STARTS = [[0, -5, 3, 9, 2], [7, 7, 7, 7, 100], [2 ** 31 - 1, -2 ** 31, 0, 1, 6], [6, 4, 2, 0, -1], [-3, 2, 2, 5, 2 ** 31 - 1], [0, 6, 0, 6, 0], [0, 1, 3, 4, 6]]
LENGTHS = [[3, 9, 2, 30], [32, 0, -4, 2 ** 31 - 1], [17, 16, 33, 6]]


def guarded(x, value):
    """A copy of x between rows of `value`, and the tensor of all."""
    rows = torch.full((x.shape[0] + 2 * GUARD, *x.shape[1:]), value, dtype=x.dtype, device="cuda")
    rows[GUARD:GUARD + x.shape[0]] = x.cuda()
    return rows[GUARD:GUARD + x.shape[0]], rows


def claims(starts):
    """Of every row the sequences that it belongs to."""
    cut = [min(max(s, 0), TOKENS) for s in starts]
    return [[b for b in range(4) if cut[b] <= t < cut[b + 1]] for t in range(TOKENS)]


def problem(gen, lengths, starts, dtype):
    table, _ = guarded(torch.arange(8, dtype=torch.int32).view(4, 2), 9)
    length, _ = guarded(torch.tensor(lengths, dtype=torch.int32), 12)
    start, _ = guarded(torch.tensor(starts, dtype=torch.int32), 3)
    parts, wholes = [], []
    for _ in range(2):
        pages = (torch.randn(PAGES, HEADS, PAGE, SIZE, generator=gen) * 100).clamp(-448, 448).to(ref.E4M3)
        pages.view(torch.uint8)[8:] = 0x7f
        p, all_pages = guarded(pages.view(torch.uint8), 0x7f)
        s, all_scales = guarded(torch.full((PAGES, HEADS), 2.0 ** -6), float("nan"))
        parts.append((p.view(ref.E4M3), s))
        wholes += [all_pages, all_scales]
    cache = mcf.KVCache(parts[0][0], parts[1][0], parts[0][1], parts[1][1])
    return table, length, start, cache, wholes


def same(a, b):
    return torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("lengths", LENGTHS, ids=str)
@pytest.mark.parametrize("starts", STARTS, ids=str)
@pytest.mark.parametrize("group", [1, 24])  # tiles of 16 rows, and of more
def test_attention(group, starts, lengths, dtype):
    gen = torch.Generator().manual_seed(81)
    table, length, start, cache, _ = problem(gen, lengths, starts, dtype)
    q, _ = guarded(torch.randn(TOKENS, HEADS * group, SIZE, generator=gen).to(dtype), float("nan"))
    out, all_out = guarded(torch.full(q.shape, 7.0, dtype=dtype), 7.0)
    for causal in (True, False):
        all_out.fill_(7.0)
        mcf.cache_attention(q, cache, table, length, 0.01, start, causal=causal, out=out)
        assert (all_out[:GUARD] == 7).all() and (all_out[-GUARD:] == 7).all()
        k, v = ((t.double() * s.double()[:, :, None, None]).cpu() for t, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)))
        owners = claims(starts)
        cut = [min(max(s, 0), TOKENS) for s in starts]
        for t, of in enumerate(owners):
            if not of:
                assert (out[t] == 7).all(), t
            if len(of) != 1 or max(map(len, owners)) > 1:
                continue
            b = of[0]  # the row alone, as the last of those before it in its sequence
            n = max(0, lengths[b])
            i, rows = t - cut[b], cut[b + 1] - cut[b]
            seen = max(0, min(n - rows + i + 1, 2 * PAGE)) if causal else min(n, 2 * PAGE)
            want, bound = ref.attention(q[t:t + 1].cpu(), k, v, table[b:b + 1].cpu(), [1], [seen], PAGE, 0.01, True)
            ref.check(out[t:t + 1], want, bound, dtype, (t, b))
        assert not torch.isnan(out).any()  # nothing was read from pages that no table names, nor between the guards


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("lengths", LENGTHS, ids=str)
@pytest.mark.parametrize("starts", STARTS, ids=str)
@pytest.mark.parametrize("q_heads", [0, 3])
def test_append(q_heads, starts, lengths, dtype):
    gen = torch.Generator().manual_seed(82)
    table, length, start, cache, wholes = problem(gen, lengths, starts, dtype)
    before = [t.clone() for t in wholes]
    k, _ = guarded(torch.randn(TOKENS, HEADS, SIZE, generator=gen).to(dtype), float("nan"))
    v, _ = guarded(torch.randn(TOKENS, HEADS, SIZE, generator=gen).to(dtype), float("nan"))
    q, _ = guarded(torch.randn(TOKENS, max(q_heads, 1), SIZE, generator=gen).to(dtype), float("nan"))
    out, all_out = guarded(torch.full(q.shape, 7.0, dtype=dtype), 7.0)
    mcf.append_cache(cache, k, v, table, length, start, q=q if q_heads else None, q_out=out if q_heads else None)
    assert (all_out[:GUARD] == 7).all() and (all_out[-GUARD:] == 7).all()
    cut = [min(max(s, 0), TOKENS) for s in starts]
    for t, of in enumerate(claims(starts)):  # (without tables and norm a query that is written is itself)
        assert (out[t] == 7).all() or (of and q_heads and same(out[t], q[t])), t
    # places that any sequence's new rows have, and pages that hold any
    places = torch.zeros(PAGES + 2 * GUARD, PAGE, dtype=torch.bool, device="cuda")
    again = places.clone()
    for b in range(4):
        n, rows = max(0, lengths[b]), max(0, cut[b + 1] - cut[b])
        for at in range(max(0, n - rows), min(n, 2 * PAGE)):
            if rows:
                places[GUARD + 2 * b + at // PAGE, at % PAGE] = True
                if at == max(0, n - rows):
                    again[GUARD + 2 * b + at // PAGE, :at % PAGE] = True
    for i, (now, was) in enumerate(zip(wholes, before)):
        if i % 2:  # scales
            kept = ~places.any(1)
            assert same(now[kept], was[kept])
        else:
            kept = ~(places | again)[:, None, :].expand(-1, HEADS, -1)
            assert torch.equal(now[kept], was[kept])
    assert not torch.isnan(cache.k[:8].float()).any() and not torch.isnan(cache.v[:8].float()).any()  # no row of the guards went in
    if all(len(of) == 1 for of in claims(starts)):  # each row of one sequence: its values are where they belong
        for t, (b,) in enumerate(claims(starts)):
            at = max(0, lengths[b]) - (cut[b + 1] - cut[b]) + t - cut[b]
            if 0 <= at < 2 * PAGE:
                p = 2 * b + at // PAGE
                for x, pages, scale in ((k, cache.k, cache.k_scale), (v, cache.v, cache.v_scale)):
                    s = scale[p].double()[:, None]
                    off = (pages[p, :, at % PAGE].double() * s - x[t].double()).abs()
                    assert (off <= x[t].double().abs() * 2.0 ** -4 + 2.0 ** -10 * s).all(), (t, b)


class Rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("stride", ctypes.c_int64 * 3)]


class Cache(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("pages", "heads", "page_size", "size")] + [(n, ctypes.c_void_p) for n in ("k", "v", "k_scale", "v_scale")] + [
        ("k_stride", ctypes.c_int64 * 2), ("v_stride", ctypes.c_int64 * 2), ("k_scale_stride", ctypes.c_int64), ("v_scale_stride", ctypes.c_int64)]


class Sequences(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("batch", "tokens", "table_width", "table_stride")] + [(n, ctypes.c_void_p) for n in ("starts", "lengths", "table")]


class Call(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("causal", ctypes.c_int32), ("q_heads", ctypes.c_int64), ("scale", ctypes.c_float), ("reserved", ctypes.c_int32),
                ("q", Rows), ("out", Rows), ("cache", Cache), ("seq", Sequences)]


@pytest.mark.parametrize("batch,tokens,q_heads,heads,width", [(60, 64, 16, 1, 8), (60, 64, 2, 1, 200), (4, 12, 4, 1, 700), (9, 300, 8, 2, 100), (66, 132, 8, 1, 200), (3, 150, 4, 1, 400)])
def test_workspace(batch, tokens, q_heads, heads, width):
    """Ascending starts and starts that overlap, in a workspace of the bytes that are asked for between guards, through the C ABI."""
    lib = load_library()
    q = torch.randn(tokens, q_heads, SIZE).half().cuda()
    c = mcf.kv_cache(8, heads, PAGE, SIZE)
    table = torch.zeros(batch, width, dtype=torch.int32, device="cuda")
    lengths = torch.full((batch,), PAGE * width, dtype=torch.int32, device="cuda")
    out, all_out = guarded(torch.full(q.shape, 7.0, dtype=torch.float16), 7.0)
    split = 0
    for starts in (torch.linspace(0, tokens, batch + 1).int().tolist(), [0, tokens] * (batch // 2) + [0] * (1 + batch % 2), [tokens - i for i in range(batch + 1)]):
        start = torch.tensor(starts, dtype=torch.int32, device="cuda")
        rows = [Rows(t.data_ptr(), (ctypes.c_int64 * 3)(0, q_heads * SIZE, SIZE)) for t in (q, out)]
        strides = (ctypes.c_int64 * 2)(heads * PAGE * SIZE, PAGE * SIZE)
        call = Call(0, 1, q_heads, 0.1, 0, *rows, Cache(8, heads, PAGE, SIZE, *(t.data_ptr() for t in c), strides, strides, heads, heads),
                    Sequences(batch, tokens, width, width, start.data_ptr(), lengths.data_ptr(), table.data_ptr()))
        size = ctypes.c_int64()
        assert lib.mcf_cache_attention_workspace(ctypes.byref(call), ctypes.byref(size)) == 0
        split += size.value > 0
        guard = 1 << 20
        work = torch.full((size.value + 2 * guard,), 0x5a, dtype=torch.uint8, device="cuda")
        stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
        assert lib.mcf_cache_attention(ctypes.byref(call), ctypes.c_void_p(work.data_ptr() + guard), size, stream) == 0
        assert (work[:guard] == 0x5a).all() and (work[guard + size.value:] == 0x5a).all()
        assert (all_out[:GUARD] == 7).all() and (all_out[-GUARD:] == 7).all()
    assert split  # (the shapes are ones that the host splits)
