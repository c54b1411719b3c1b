"""One key that draws most of the weight, and very many that have little each but not little together."""
import math

import pytest
import torch

from paper_2512_07011_amd import binding
from tests import paged

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("b,s,hq,prefix", [(128, 1, 16, 0), (64, 16, 64, 0), (2, 64, 16, 8192)])
@pytest.mark.parametrize("gap", [16.0, 17.5, 19.0])
def test_small_weights_add_up(dtype, d, b, s, hq, prefix, gap):
    """The first key's score lies `gap` above all others', which are equal; its value is 0 and theirs 1, so that the result is the sum of
    the small weights, n e^-gap / (1 + n e^-gap).  In fp16 each of them lies below 2^-22 of the first one's.  The tolerance is the one of
    paged.check_attention.  (Every sequence is in the same pages, and in one range: all keys meet in one accumulator, or four.)"""
    dt, page, hkv = paged.DTYPES[dtype], 128, 8
    n = prefix or 16384
    kc, vc = torch.zeros(n // page, page, hkv, d, dtype=dt), torch.ones(n // page, page, hkv, d, dtype=dt)
    q = torch.zeros(1, 1, hq, d, dtype=dt)
    q[..., 0] = 8.0
    kc[0, 0, :, 0] = gap * math.sqrt(d) / 8.0
    vc[0, 0] = 0.0
    table = torch.arange(n // page, dtype=torch.int32)
    if prefix:
        ref = paged.run_oracle(q, kc, vc, table[None, :1], [0], prefix_table=table, prefix_len=n)
    else:
        ref = paged.run_oracle(q, kc, vc, table[None], [n], causal=False)
    print("case", dtype, d, b, s, hq, prefix, gap, ref[0].amax().item(), flush=True)
    q, kc, vc, table = q.to(DEV).expand(b, s, hq, d).contiguous(), kc.to(DEV), vc.to(DEV), table.to(DEV)
    lse = torch.empty(b, s, hq, device=DEV)
    held = torch.full((b,), 0 if prefix else n, dtype=torch.int32, device=DEV)
    if prefix:
        out = binding.bsfa_prefix_attention(q, kc, vc, table, n, table[None, :1].expand(b, 1), held, lse=lse)
    else:
        out = binding.bsfa_paged_attention(q, kc, vc, table[None].expand(b, -1), held, causal=False, lse=lse)
    paged.check_attention(out.cpu(), lse.cpu(), tuple(t.expand(b, s, *t.shape[2:]) for t in ref), dt, math.nan)
