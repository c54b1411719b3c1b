"""Queries that are not finite: what bsfa_paged_attention and bsfa_prefix_attention give for their rows, and for the others."""
import math

import pytest
import torch

from paper_2512_07011_amd import binding
from tests import paged

pytestmark = pytest.mark.gpu
DEV = "cuda"

# lens, new tokens, query and KV heads, prefix, columns of the table: few rows written at once and joined, many rows written at
# once and dealt, prefixes of few and of many rows with few and many own rows behind them
FORMS = {"few, whole": ([40, 77], 1, 8, 2, 0, 8), "few, joined": ([3000, 77], 2, 16, 2, 0, 200), "many, whole": ([90, 177], 30, 8, 2, 0, 12),
         "many, dealt": ([2000, 177], 30, 8, 2, 0, 130), "few behind a prefix": ([40, 77], 1, 8, 2, 300, 8),
         "prefix of many rows": ([40, 77, 0, 9, 30], 4, 16, 2, 300, 8), "many behind a prefix": ([40, 77], 30, 8, 2, 300, 8)}


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("d,dtype", [(128, "bf16"), (64, "fp16")])
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_queries_that_are_not_finite(form, d, dtype, value):
    """Result and log-sum-exp of such a row are NaN (a softmax of NaN, or of infinities of both signs), never 0 and -inf, which stand
    for a row that sees nothing; the other rows' are the same, bit for bit."""
    lens, s, hq, hkv, prefix, columns = FORMS[form]
    dt = paged.DTYPES[dtype]
    kc, vc, table, prefix_table = paged.filled(lens, 16, hkv, d, dt, "nhd", 11, columns=columns, prefix=prefix)
    q = torch.randn(len(lens), s, hq, d, generator=torch.Generator().manual_seed(12)).to(dt)
    rows = [(0, s - 1, 0), (1, s // 2, hq - 1)]
    print("case", form, d, dtype, value, flush=True)
    kc, vc, table, prefix_table = (t.to(DEV) for t in (kc, vc, table, prefix_table))
    held = torch.tensor(lens, dtype=torch.int32, device=DEV)

    def call(q):
        lse = torch.full(q.shape[:3], 7.0, device=DEV)
        more = dict(lse=lse, max_cache_len=200 if form.endswith("whole") else 0)
        if prefix:
            out = binding.bsfa_prefix_attention(q.to(DEV), kc, vc, prefix_table, prefix, table, held, **more)
        else:
            out = binding.bsfa_paged_attention(q.to(DEV), kc, vc, table, held, **more)
        return out.cpu(), lse.cpu()

    want = call(q)
    bad = q.clone()
    for b, i, h in rows:
        bad[b, i, h, 3] = value
    got = call(bad)
    for b, i, h in rows:
        assert got[0][b, i, h].isnan().all(), (b, i, h)
        assert got[1][b, i, h].isnan(), (b, i, h, got[1][b, i, h].item())
    for x, y in zip(got, want):
        for row in rows:
            x[row] = y[row]
        assert torch.equal(x, y)
