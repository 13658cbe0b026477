"""Plain implementations in 64 bits, on the CPU, of the operators around the paged cache, and the error that each may have."""
import math

import torch

E4M3 = torch.float8_e4m3fn


def half_step(dtype):
    """Largest relative error of one rounding to a type."""
    return torch.finfo(dtype).eps / 2


def tables(rotary, positions):
    half = rotary // 2
    angle = torch.arange(positions, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(half, dtype=torch.float64) / max(half, 1))
    return angle.cos().float(), angle.sin().float()


def turn(x, cos, sin, positions, interleaved, back=False):
    """Rotation of the last dimension of x [..., tokens, heads, size] (float64); positions [..., tokens]."""
    rotary = 2 * cos.shape[-1]
    known = (positions >= 0) & (positions < cos.shape[0])
    at = torch.where(known, positions, 0).long()
    nan = torch.where(known, 0.0, math.nan).double()[..., None, None]
    c, s = cos.double()[at][..., None, :] + nan, sin.double()[at][..., None, :] + nan
    if back:
        s = -s
    y = x.clone()
    if interleaved:
        a, b = x[..., 0:rotary:2], x[..., 1:rotary:2]
        y[..., 0:rotary:2], y[..., 1:rotary:2] = a * c - b * s, b * c + a * s
    else:
        a, b = x[..., :rotary // 2], x[..., rotary // 2:rotary]
        y[..., :rotary // 2], y[..., rotary // 2:rotary] = a * c - b * s, b * c + a * s
    return y


def normed(x, weight, eps):
    if weight is None:
        return x
    return x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * weight.double()


def norm_rotate(x, cos, sin, positions, weight, eps, interleaved):
    x = normed(x.double(), weight, eps)
    return x if cos is None else turn(x, cos, sin, positions, interleaved)


def norm_rotate_bound(x, ref, cos, weight, eps, interleaved, dtype):
    """One rounding to the type (an absolute step below its smallest exponent) and fp32 arithmetic before it: the sum of squares
    (a chain of at most 32 additions and 5 exchanges, of positive terms), its root, three products and two of the rotation,
    each 2^-24 of the pair that is rotated: 64 of them are more than enough."""
    y = normed(x.double(), weight, eps).abs()
    pair = y.clone()
    if cos is not None:
        rotary = 2 * cos.shape[-1]
        if interleaved:
            both = y[..., 0:rotary:2] + y[..., 1:rotary:2]
            pair[..., 0:rotary:2] = pair[..., 1:rotary:2] = both
        else:
            both = y[..., :rotary // 2] + y[..., rotary // 2:rotary]
            pair[..., :rotary] = torch.cat((both, both), -1)
    return half_step(dtype) * ref.abs() + 64 * 2.0 ** -24 * pair + torch.finfo(dtype).smallest_normal * half_step(dtype)


def norm_rotate_backward(dy, x, cos, sin, positions, weight, eps, interleaved):
    """(dx, dw, bound of dx before its last rounding, bound of dw)"""
    x, g = x.double(), dy.double()
    if cos is not None:
        g = turn(g, cos, sin, positions, interleaved, back=True)
    if weight is None:
        return g, None, 8 * 2.0 ** -24 * dy.double().abs().amax(-1, keepdim=True) * 2, None
    n = x.shape[-1]
    r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    u = g * weight.double()
    dx = r * (u - x * r * r * (u * x).sum(-1, keepdim=True) / n)
    terms = g * x * r
    rows = tuple(range(x.dim() - 1))
    # dx: sums of at most 32 terms a lane and 5 exchanges, a dozen operations around them; the rotation's operands are
    # at most the row's largest element each.  dw: each term as above, in chains that these tests keep below 2^10
    big = dy.double().abs().amax(-1, keepdim=True) * 2 * weight.double().abs().amax()
    bx = 64 * 2.0 ** -24 * r * (big + x.abs() * r * r * (big * x.abs()).sum(-1, keepdim=True) / n)
    bw = (2.0 ** 10 + 64) * 2.0 ** -24 * ((dy.double().abs().amax(-1, keepdim=True) * 2) * (x * r).abs()).sum(rows)
    return dx, terms.sum(rows), bx, bw


def power_of_two(amax):
    """The least power of two that brings amax to 448 at most, 2^-100 at least."""
    s = 2.0 ** -100
    while amax > 448 * s:
        s *= 2
    return s


def to_e4m3(x):
    """Rounded to the nearest e4m3 (ties to even); what is not finite becomes NaN.  x: float64, at most 448."""
    y = x.clone()
    fine = torch.isfinite(x)
    m = x[fine].abs()
    step = torch.exp2(torch.floor(torch.log2(m.clamp_min(2.0 ** -6))) - 3)
    y[fine] = torch.round(m / step) * step * torch.sign(x[fine])  # (round halves to even)
    y[~fine] = math.nan
    return y


def append(cache, x, table, news, lengths, page, which):
    """Puts the rows x [tokens, heads, size] (float64, normed and rotated) of sequences that bring `news` tokens into the cache's
    dicts cache["v"] [pages, heads, page, size] and cache["s"] [pages, heads], both float64, in place."""
    pages = cache["v"].shape[0]
    row = 0
    for b, n in enumerate(news):
        parts = {}
        for i in range(n):
            at = lengths[b] - n + i
            if at < 0 or at // page >= table.shape[1]:
                continue
            p = int(table[b, at // page])
            if 0 <= p < pages:
                parts.setdefault(p, []).append((at % page, row + i))
        for p, tokens in parts.items():
            first = tokens[0][0]
            for h in range(x.shape[1]):
                new = torch.stack([x[r, h] for _, r in tokens])
                fine = new[torch.isfinite(new)]
                s = power_of_two(float(fine.abs().max()) if fine.numel() else 0.0)
                old = float(cache["s"][p, h])
                if first > 0:
                    s = max(s, old)
                    if s != old:
                        cache["v"][p, h, :first] = to_e4m3(cache["v"][p, h, :first] * (old / s))
                cache["s"][p, h] = s
                for place, r in tokens:
                    cache["v"][p, h, place] = to_e4m3(x[r, h] / s)
        row += n


def attention(q, k, v, table, news, lengths, page, scale, causal):
    """q [tokens, q_heads, size]; k, v float64 [pages, heads, page, size], scales applied.  Returns (out, bound without the last rounding)
    for the rows of the sequences, in fp16 or bf16."""
    pages, heads = k.shape[:2]
    group = q.shape[1] // heads
    out = torch.zeros(q.shape, dtype=torch.float64)
    bound = torch.zeros(q.shape, dtype=torch.float64)
    size, step = q.shape[2], half_step(q.dtype)
    row = 0
    for b, n in enumerate(news):
        seen = min(lengths[b], table.shape[1] * page)
        ids = [int(table[b, t // page]) for t in range(seen)]
        there = torch.tensor([0 <= p < pages for p in ids], dtype=torch.bool)
        where = torch.tensor([p if 0 <= p < pages else 0 for p in ids], dtype=torch.long)
        place = torch.arange(seen) % page
        for i in range(n):
            limit = max(0, min(seen, lengths[b] - n + i + 1)) if causal else seen
            ok = there[:limit]
            if not ok.any():
                continue
            for h in range(heads):
                kk, vv = k[where[:limit][ok], h, place[:limit][ok]], v[where[:limit][ok], h, place[:limit][ok]]
                qq = q[row + i, h * group:(h + 1) * group].double()
                s = scale * qq @ kk.T
                p = torch.softmax(s, -1)
                out[row + i, h * group:(h + 1) * group] = p @ vv
                # the weights' rounding; scores of fp32 sums (size + 32 steps of the sum of magnitudes), as an error of both
                # the weights and their sum; the exponential; fp16 weights below 2^-14 of the largest
                big = abs(scale) * (qq.abs() @ kk.abs().T).amax(-1, keepdim=True)
                mean = p @ vv.abs()
                bound[row + i, h * group:(h + 1) * group] = mean * (step + 2 * (size + 32) * 2.0 ** -24 * big + 2.0 ** -20) + (
                    len(vv) * 2.0 ** -25 * vv.abs().amax(0) if q.dtype == torch.float16 else 0.0)
        row += n
    return out, bound


def check(got, ref, bound, dtype, what=""):
    """got (of a type) against ref (float64) within `bound` and one rounding to the type."""
    got = got.double().cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(ref)), f"{what}: NaN in other places"
    off = (got - ref).abs() - (bound + half_step(dtype) * ref.abs() + torch.finfo(dtype).smallest_normal * half_step(dtype))
    off = torch.where(torch.isnan(ref), -1.0, off)
    worst = off.max().item() if off.numel() else 0.0
    assert worst <= 0, f"{what}: over its bound by {worst:.3g} (largest difference {torch.nan_to_num((got - ref).abs()).max().item():.3g})"
