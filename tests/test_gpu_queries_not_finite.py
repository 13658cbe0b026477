"""Attention over the paged cache for queries that are not finite: NaN where they see a token, zeros where they see none (as every row that sees none),
and no other row is touched."""
import math

import pytest
import torch

from test_gpu_cache_attention import _problem, _run

pytestmark = pytest.mark.gpu

PAGE = 16
# rows, tokens, size; the second sequence has no page, the last one more rows than tokens; tiles of 16 rows in one part and in several, 32, 48, 128, 256
CASES = [([1, 1, 1], [40, 50, 0], 128), ([1, 1, 1], [3000, 2000, 0], 64), ([4, 3, 2], [130, 40, 1], 96), ([12, 10, 14], [140, 90, 6], 192), ([22, 20, 19], [200, 60, 9], 80),
         ([60, 50, 50], [100, 200, 20], 256), ([150, 70, 100], [230, 70, 40], 128)]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf], ids=str)
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "whole"])
@pytest.mark.parametrize("news,lengths,size", CASES, ids=str)
def test_queries(news, lengths, size, causal, value, dtype):
    gen = torch.Generator().manual_seed(52)
    q, cache, _, table = _problem(gen, news, lengths, 4, 2, size, PAGE, dtype)
    table[1] = torch.tensor([-1, 10 ** 6])[torch.arange(table.shape[1]) % 2]
    want = _run(q, cache, table, news, lengths, 0.1, causal)
    assert torch.isfinite(want).all() and (want[news[0]:news[0] + news[1]] == 0).all()
    total = sum(news)
    sees = [r < news[0] or (r >= news[0] + news[1] and (lengths[2] > 0 if not causal else lengths[2] - (total - r) >= 0)) for r in range(total)]
    bad = torch.zeros(total, 4, dtype=torch.bool)
    for r, h in ((0, 1), (news[0] - 1, 2), (news[0], 0), (news[0] + news[1] - 1, 3), (news[0] + news[1], 0), (total - 1, 1)):
        bad[r, h] = True
    q[bad, size - 3] = value
    got = _run(q, cache, table, news, lengths, 0.1, causal)
    gone = (bad & torch.tensor(sees)[:, None]).cuda()
    assert torch.isnan(got[gone]).all()
    got[gone] = want[gone]
    assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("news", [[1, 1], [5, 60], [90, 40]], ids=str)
def test_scores_of_minus_infinity_alone(news, dtype):
    """Every score of a row is -inf: it sees tokens, and their weights are 0 / 0."""
    gen = torch.Generator().manual_seed(53)
    lengths = [100, 2500]
    q, cache, _, table = _problem(gen, news, lengths, 4, 2, 64, PAGE, dtype)
    cache.k[..., 7] = 2.0
    q[:, 1, 7] = -math.inf
    for scale in (0.1, 0.0):
        got = _run(q, cache, table, news, lengths, scale, True)
        assert torch.isnan(got[:, 1]).all() and torch.isfinite(got[:, [0, 2, 3]]).all()
