"""What the operators around the paged cache refuse, before anything is launched: shapes, types, strides and alignment.  The check for
device tensors comes last, so that the others are tested without a GPU."""
import pytest
import torch

import paper_2506_22169_amd as mcf

EINVAL, EUNSUPPORTED, EALIGN = 1, 2, 3


def z(*s, dtype=torch.float16):
    return torch.zeros(s, dtype=dtype)


def i32(*v):
    return torch.tensor(v, dtype=torch.int32)


def refused(call, status, text=""):
    with pytest.raises(mcf.McfError) as e:
        call()
    assert e.value.status == status, str(e.value)
    assert text in str(e.value)


def misaligned(*s):
    return z(int(torch.tensor(s).prod()) + 1)[1:].view(s)


NORM = [
    (dict(q=z(4, 64)), EINVAL, "rows are"),
    (dict(q=z(4, 2, 64, dtype=torch.float32)), EUNSUPPORTED, "float16 or bfloat16"),
    (dict(q=z(4, 2, 40)), EUNSUPPORTED, "multiple of 16"),
    (dict(q=z(4, 2, 528)), EUNSUPPORTED, "multiple of 16"),
    (dict(q=z(4, 64, 2).transpose(1, 2)), EUNSUPPORTED, "packed"),
    (dict(q=z(4, 2, 68)[..., :64]), EALIGN, ""),
    (dict(q=misaligned(4, 2, 64)), EALIGN, ""),
    (dict(k=z(4, 2, 64, dtype=torch.bfloat16)), EINVAL, "q and k differ"),
    (dict(k=z(5, 2, 64)), EINVAL, "q and k differ"),
    (dict(k=z(1, 4, 2, 64)), EINVAL, "q and k differ"),
    (dict(cos=z(9, 32, dtype=torch.float32)), EINVAL, "come together"),
    (dict(cos=z(9, 32), sin=z(9, 32)), EINVAL, "float32"),
    (dict(cos=z(9, 33, dtype=torch.float32), sin=z(9, 33, dtype=torch.float32)), EINVAL, ""),
    (dict(cos=z(9, 4, dtype=torch.float32), sin=z(9, 4, dtype=torch.float32)), EINVAL, ""),
    (dict(cos=z(9, 64, dtype=torch.float32)[:, ::2], sin=z(9, 64, dtype=torch.float32)[:, ::2]), EINVAL, "packed"),
    (dict(positions=torch.arange(4).float()), EINVAL, "int32 or int64"),
    (dict(positions=torch.arange(5)), EINVAL, "one for each"),
    (dict(positions=torch.tensor(3)), EINVAL, "one for each"),
    (dict(positions=torch.arange(4)[None]), EINVAL, "one for each"),
    (dict(positions=torch.arange(8)[::2]), EINVAL, "packed"),
    (dict(q_weight=z(32)), EINVAL, "a weight"),
    (dict(q_weight=z(64, dtype=torch.bfloat16)), EINVAL, "type of the rows"),
    (dict(q_weight=z(64), k_weight=z(64, dtype=torch.float32)), EINVAL, "one type"),
    (dict(eps=-1.0), EINVAL, ""),
    (dict(eps=float("nan")), EINVAL, ""),
    (dict(q_out=z(4, 2, 64, dtype=torch.bfloat16)), EINVAL, "q_out"),
    (dict(q_out=z(4, 1, 64).expand(4, 2, 64)), EINVAL, ""),
    (dict(q_out=z(4 * 2 * 64 + 64).as_strided((4, 2, 64), (64, 64, 1))), EINVAL, ""),
    (dict(q=z(1, 1, 64).expand(1 << 16, 1 << 16, 64), k=None, q_out=None), EUNSUPPORTED, "too many rows"),
    (dict(), EINVAL, "device"),
]


@pytest.mark.parametrize("i", range(len(NORM)))
def test_norm_rotate(i):
    change, status, text = NORM[i]
    a = dict(q=z(4, 2, 64), k=z(4, 1, 64), cos=None, sin=None, positions=None, q_weight=None, k_weight=None, eps=1e-6)
    if "q" in change:
        a["k"] = None
    a.update(change)
    refused(lambda: mcf.norm_rotate(**a), status, text)
    q, k = a.pop("q"), a.pop("k")
    refused(lambda: mcf.norm_rotate_backward(q, k, q, k, **a), status, text)


def test_norm_rotate_backward_shapes():
    q, k = z(4, 2, 64), z(4, 1, 64)
    refused(lambda: mcf.norm_rotate_backward(z(4, 3, 64), k, q, k), EINVAL, "dq")
    refused(lambda: mcf.norm_rotate_backward(q, z(4, 2, 64), q, k), EINVAL, "dk")
    refused(lambda: mcf.norm_rotate_backward(q, None, q, k), EINVAL, "come together")
    refused(lambda: mcf.norm_rotate_backward(q, k, q), EINVAL, "come together")
    refused(lambda: mcf.norm_rotate_backward(None, k, q, k), EINVAL, "missing")


def cache(pages=3, heads=2, page=16, size=64):
    return mcf.kv_cache(pages, heads, page, size, device="cpu")


def fp8(*s):
    return torch.zeros(s, dtype=torch.float8_e4m3fn)


def f32(*s):
    return torch.zeros(s, dtype=torch.float32)


CACHES = [
    (cache(page=8), EUNSUPPORTED, "pages hold"),
    (cache(page=48), EUNSUPPORTED, "pages hold"),
    (cache(size=32), EUNSUPPORTED, "the cache holds"),
    (cache(size=112), EUNSUPPORTED, "the cache holds"),
    (tuple(cache())[:3], EINVAL, "a cache is"),
    (list(cache()), EINVAL, "a cache is"),
    (cache()._replace(v=fp8(3, 2, 16, 80)), EINVAL, "the pages are"),
    (cache()._replace(v=z(3, 2, 16, 64)), EINVAL, "the pages are"),
    (cache()._replace(k=fp8(3, 2, 32, 64)[:, :, ::2]), EUNSUPPORTED, "packed"),
    (cache()._replace(k=fp8(3, 16, 2, 64).transpose(1, 2)), EUNSUPPORTED, "packed"),
    (cache()._replace(k_scale=z(3, 2)), EINVAL, "the scales"),
    (cache()._replace(k_scale=f32(3, 3)), EINVAL, "the scales"),
    (cache()._replace(k_scale=f32(2, 3).t()), EUNSUPPORTED, "the scales"),
    (cache()._replace(k_scale=f32(1, 2).expand(3, 2)), EINVAL, ""),
    (cache()._replace(k=fp8(1, 2, 16, 64).expand(3, 2, 16, 64)), EINVAL, ""),
    (cache()._replace(k=fp8(3 * 2 * 16 * 64 + 8)[8:].view(3, 2, 16, 64)), EALIGN, ""),
    (cache()._replace(k=fp8(3 * (2 * 16 * 64 + 8)).as_strided((3, 2, 16, 64), (2 * 16 * 64 + 8, 16 * 64, 64, 1))), EALIGN, ""),
    (cache(), EINVAL, "device"),
]

SEQUENCES = [
    (dict(table=torch.zeros(2, 3, dtype=torch.int64)), EINVAL, "int32"),
    (dict(table=torch.zeros(3, dtype=torch.int32)), EINVAL, "the table is"),
    (dict(table=torch.zeros(3, 3, dtype=torch.int32)), EINVAL, "the table is"),
    (dict(table=torch.zeros(2, 6, dtype=torch.int32)[:, ::2]), EUNSUPPORTED, "packed"),
    (dict(lengths=torch.ones(2)), EINVAL, "int32"),
    (dict(lengths=i32(1, 1, 1, 1)[::2]), EUNSUPPORTED, "packed"),
    (dict(starts=i32(0, 2)), EINVAL, "one entry more"),
    (dict(starts=i32(0, 1, 2, 3)), EINVAL, "one entry more"),
    (dict(starts=None), EINVAL, "one row"),
]


@pytest.mark.parametrize("i", range(len(CACHES)))
def test_caches(i):
    c, status, text = CACHES[i]
    size = c[0].shape[3] if len(c) == 4 else 64
    page = dict(table=torch.zeros(2, 3, dtype=torch.int32), lengths=i32(1, 1))
    refused(lambda: mcf.append_cache(c, z(2, 2, size), z(2, 2, size), **page), status, text)
    refused(lambda: mcf.cache_attention(z(2, 4, size), c, scale=1.0, **page), status, text)


@pytest.mark.parametrize("i", range(len(SEQUENCES)))
def test_sequences(i):
    change, status, text = SEQUENCES[i]
    a = dict(table=torch.zeros(2, 3, dtype=torch.int32), lengths=i32(3, 2), starts=i32(0, 3, 5))
    a.update(change)
    refused(lambda: mcf.append_cache(cache(), z(5, 2, 64), z(5, 2, 64), **a), status, text)
    refused(lambda: mcf.cache_attention(z(5, 4, 64), cache(), scale=1.0, **a), status, text)


def test_append():
    page = dict(table=torch.zeros(2, 3, dtype=torch.int32), lengths=i32(1, 1))
    k = z(2, 2, 64)
    refused(lambda: mcf.append_cache(cache(), k, z(2, 1, 64), **page), EINVAL, "k and v differ")
    refused(lambda: mcf.append_cache(cache(), z(2, 3, 64), z(2, 3, 64), **page), EINVAL, "than the cache")
    refused(lambda: mcf.append_cache(cache(), z(2, 2, 80), z(2, 2, 80), **page), EINVAL, "than the cache")
    refused(lambda: mcf.append_cache(cache(), z(1, 2, 2, 64), z(1, 2, 2, 64), **page), EINVAL, "rows are")
    refused(lambda: mcf.append_cache(cache(), k.float(), k.float(), **page), EUNSUPPORTED, "float16")
    refused(lambda: mcf.append_cache(cache(), k, k, q=z(3, 2, 64), **page), EINVAL, "q and k differ")
    refused(lambda: mcf.append_cache(cache(), k, k, q_out=z(2, 2, 64), **page), EINVAL, "without q")
    refused(lambda: mcf.append_cache(cache(), k, k, q=z(2, 4, 64), q_out=z(2, 3, 64), **page), EINVAL, "q_out")
    refused(lambda: mcf.append_cache(cache(), k, k, k_weight=z(64), q=z(2, 4, 64), q_weight=f32(64), **page), EINVAL, "one type")
    refused(lambda: mcf.append_cache(cache(), k, k, cos=f32(9, 40), sin=f32(9, 40), **page), EINVAL, "")
    refused(lambda: mcf.append_cache(cache(), k, k, eps=-1, **page), EINVAL, "")


def test_attention():
    page = dict(table=torch.zeros(2, 3, dtype=torch.int32), lengths=i32(1, 1))
    q = z(2, 4, 64)
    refused(lambda: mcf.cache_attention(z(2, 3, 64), cache(), scale=1.0, **page), EINVAL, "multiple")
    refused(lambda: mcf.cache_attention(z(2, 4, 80), cache(), scale=1.0, **page), EINVAL, "size")
    refused(lambda: mcf.cache_attention(q.float(), cache(), scale=1.0, **page), EUNSUPPORTED, "float16")
    refused(lambda: mcf.cache_attention(q, cache(), scale=float("nan"), **page), EINVAL, "")
    refused(lambda: mcf.cache_attention(q, cache(), scale=float("inf"), **page), EINVAL, "")
    refused(lambda: mcf.cache_attention(q, cache(), scale=1e300, **page), EINVAL, "")
    refused(lambda: mcf.cache_attention(q, cache(), scale=1.0, out=z(2, 4, 64, dtype=torch.bfloat16), **page), EINVAL, "out has")
    refused(lambda: mcf.cache_attention(q, cache(), scale=1.0, out=z(1, 4, 64).expand(2, 4, 64), **page), EINVAL, "")
    with pytest.raises(TypeError):
        mcf.cache_attention(q, cache(), scale=object(), **page)
