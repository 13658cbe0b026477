"""Attention over the paged cache where scales of V are far apart, so that a page of tiny weights counts (any finite scale is allowed)."""
import math

import pytest
import torch

import cache_reference as ref
import paper_2506_22169_amd as mcf

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("new", [1, 9, 70])
@pytest.mark.parametrize("large,small", [(70, 75), (100, 102), (119, 118), (-70, 60), (-100, 100), (-126, 90)], ids=str)
def test_wide_scales(large, small, new, dtype):
    """A page of ones under 2^large whose weights are 2^-small of the other's: the definition in 64 bits, within the bound that other cases have."""
    size, page = 64, 16
    c = mcf.kv_cache(3, 1, page, size)
    c.k[2].fill_(1.0)
    c.v[0].fill_(1.0)
    c.v[2, ..., ::2] = 1.0
    c.k_scale.fill_(1.0)
    c.v_scale[:, 0] = torch.tensor([2.0 ** large, 1.0, 1.0])
    table = torch.tensor([[0, 2] + [0, 2] * 4])
    n = page * table.shape[1]
    q = torch.ones(new, 2, size, dtype=dtype)
    scale = small * math.log(2) / size
    starts = torch.tensor([0, new]).int().cuda()
    got = mcf.cache_attention(q.cuda(), c, table.int().cuda(), torch.tensor([n]).int().cuda(), scale, starts, causal=False)
    k, v = ((t.double() * s.double()[:, :, None, None]).cpu() for t, s in ((c.k, c.k_scale), (c.v, c.v_scale)))
    # (bf16's bound: that of fp16 has a term for weights below its smallest exponent beside, which would hide what is looked for)
    want, bound = ref.attention(q.bfloat16(), k, v, table, [new], [n], page, scale, False)
    assert 2.0 ** (large - small) * 0.9 < want[0, 0, 1].item() < 2.0 ** (large - small) * 1.1
    ref.check(got, want, bound, dtype)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("new", [1, 9, 70])
@pytest.mark.parametrize("large,small", [(6, -4), (6, -15), (7, -22), (-3, -24)], ids=str)
@pytest.mark.parametrize("size,factor", [(64, 1.0), (80, 1.37), (128, 1.0)])
def test_small_pages_beside_large_ones(size, factor, large, small, new, dtype):
    """Pages of like weights under scales far apart, where the large ones hold zeros in every second column: what is left there is of the small ones
    alone, and has the bits that it would have without the large ones beside."""
    gen = torch.Generator().manual_seed(61)
    page = 16
    c = mcf.kv_cache(4, 1, page, size)
    for t in c[:2]:
        t.copy_((torch.randn(t.shape, generator=gen) * 100).clamp(-448, 448).to(ref.E4M3))
    c.v[::2, ..., ::2] = 0.0
    c.k_scale.fill_(2.0 ** -10)
    c.v_scale[:, 0] = torch.tensor([2.0 ** large, 2.0 ** small, 2.0 ** large, 2.0 ** (small + 1)]) * factor
    table = torch.tensor([[2, 3, 0, 1, 3, 2]])
    n = page * table.shape[1] - 3
    q = torch.randn(new, 2, size, generator=gen).to(dtype)
    starts = torch.tensor([0, new]).int().cuda()
    got = mcf.cache_attention(q.cuda(), c, table.int().cuda(), torch.tensor([n]).int().cuda(), 0.1, starts, causal=False)
    k, v = ((t.double() * s.double()[:, :, None, None]).cpu() for t, s in ((c.k, c.k_scale), (c.v, c.v_scale)))
    want, bound = ref.attention(q, k, v, table, [new], [n], page, 0.1, False)
    ref.check(got, want, bound, dtype)
