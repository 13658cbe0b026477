"""Attention over the paged cache where scales are not finite: whoever sees their pages gets NaN, nobody else is touched."""
import math

import pytest
import torch

from test_gpu_cache_attention import _problem, _run

pytestmark = pytest.mark.gpu

# rows, tokens, size: single tokens (the second in parts), a few rows, many; later rows of the first sequence alone see its last page
CASES = [([1, 1], [40, 3000], 128), ([4, 2], [130, 17], 64), ([9, 3], [135, 2000], 96), ([40, 3], [200, 3], 80), ([150], [230], 128), ([70], [165], 256),
         ([12], [140], 192), ([30, 30], [100, 90], 256)]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("value", [math.nan, math.inf], ids=["nan", "inf"])
@pytest.mark.parametrize("which", ["k_scale", "v_scale"])
@pytest.mark.parametrize("news,lengths,size", CASES, ids=str)
def test_scales(news, lengths, size, which, value, dtype):
    gen = torch.Generator().manual_seed(51)
    page = 16
    q, cache, _, table = _problem(gen, news, lengths, 4, 2, size, page, dtype)
    scales = getattr(cache, which)
    for causal in (True, False):
        want = _run(q, cache, table, news, lengths, 0.1, causal)
        assert torch.isfinite(want).all()
        for b, n in enumerate(lengths):
            for column in sorted({0, (n - 1) // page // 2, (n - 1) // page}):
                p = int(table[b, column])
                was = scales[p, 1].item()
                scales[p, 1] = value
                got = _run(q, cache, table, news, lengths, 0.1, causal)
                scales[p, 1] = was
                first = sum(news[:b])
                sees = [r for r in range(news[b]) if not causal or n - news[b] + r >= column * page]
                rows = torch.tensor(sees, device="cuda") + first
                assert torch.isnan(got[rows, 2:]).all(), (b, column, causal)
                got[rows, 2:] = want[rows, 2:]
                assert torch.equal(got, want), (b, column, causal)
