"""Rows that a call does not have: sequences that rest (q_lens 0, tokens in the cache) and the rows behind q_lens."""
import pytest
import torch

from paper_2512_07011_amd import binding
from tests import paged

pytestmark = pytest.mark.gpu
DEV = "cuda"


def call(lens, q_lens, s, hq, hkv, d, prefix=0, columns=600):
    """Result, log-sum-exp and the scratch memory as the call leaves it (255 where it wrote nothing); the inputs follow from the sizes
    of `lens` of the first call alone."""
    kc, vc, table, prefix_table = paged.filled([columns * 16 - 16] * len(lens), 16, hkv, d, torch.bfloat16, "hnd", 21, columns=columns, prefix=prefix)
    q = torch.randn(len(lens), s, hq, d, generator=torch.Generator().manual_seed(22)).to(torch.bfloat16).to(DEV)
    kc, vc, table, prefix_table = (t.to(DEV) for t in (kc, vc, table, prefix_table))
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    need = binding.paged_workspace_bytes(q, kc, table, prefix_table if prefix else None, prefix)
    ws = torch.full((need,), 255, dtype=torch.uint8, device=DEV)
    out, lse = torch.full(q.shape, 7.0, dtype=q.dtype, device=DEV), torch.full(q.shape[:3], 7.0, device=DEV)
    print("case", lens, q_lens, s, hq, hkv, d, prefix, flush=True)
    kw = dict(q_lens=ints(q_lens), out=out, lse=lse, workspace=ws)
    if prefix:
        binding.bsfa_prefix_attention(q, kc, vc, prefix_table, prefix, table, ints(lens), **kw)
    else:
        binding.bsfa_paged_attention(q, kc, vc, table, ints(lens), **kw)
    torch.cuda.synchronize()
    return out, lse, ws


@pytest.mark.parametrize("s,hq,hkv,d,prefix", [(1, 8, 2, 128, 0), (4, 16, 2, 64, 0), (30, 8, 2, 128, 0), (1, 8, 2, 64, 300), (4, 16, 2, 128, 300),
                                               (30, 8, 2, 64, 300)])
def test_a_resting_sequence_counts_as_one_without_tokens(s, hq, hkv, d, prefix):
    """Neither its keys nor a share of the chip: the others' ranges are cut as if it had none, and nothing is kept for it.  The scratch
    memory shows both, and is the same to the bit."""
    q_lens = [s, 0, 0, max(1, s - 1), 0]
    resting = call([2500, 9000, 4000, 33, 700], q_lens, s, hq, hkv, d, prefix)
    empty = call([2500, 0, 0, 33, 0], q_lens, s, hq, hkv, d, prefix)
    for x, y in zip(resting, empty):
        assert torch.equal(x, y)
    for b in (1, 2, 4):
        assert (resting[0][b] == 7.0).all() and (resting[1][b] == 7.0).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("prefix", [0, 300])
def test_row_groups_behind_q_lens_are_left(d, prefix):
    """64 rows of 256 exist, in the first of two groups of 128: the second group's own ranges are not worked on.  What it would leave
    in the scratch memory is as much as the first group's."""
    def written(q_lens):
        return (call([5000], q_lens, 64, 8, 2, d, prefix)[2] != 255).sum().item()

    none, some, full = written([0]), written([16]), written([64])
    assert full - none > 0.9 * 256 * 2 * d * 4, (none, some, full)        # (both groups' results of one range at least)
    assert some - none < 0.6 * (full - none), (none, some, full)
