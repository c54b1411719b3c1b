"""bsfa_paged_attention and bsfa_prefix_attention against the 64-bit oracle."""
import itertools
import math

import pytest
import torch

from paper_2512_07011_amd import binding
from tests import paged

pytestmark = pytest.mark.gpu
DEV = "cuda"


def run_case(lens, s, hq, hkv, d, page, dtype="bf16", layout="nhd", causal=True, q_lens=None, prefix=0, seed=0, columns=None,
             max_cache_len=0, spread_q=1.0, stream=None):
    dt = paged.DTYPES[dtype]
    kc, vc, table, prefix_table = paged.filled(lens, page, hkv, d, dt, layout, seed, columns=columns, prefix=prefix)
    g = torch.Generator().manual_seed(seed + 1)
    q = (spread_q * torch.randn(len(lens), s, hq, d, generator=g)).to(dt)
    if q_lens is not None:
        for b, m in enumerate(q_lens):
            q[b, m:] = math.nan
    print("case", lens, s, hq, hkv, d, page, dtype, layout, causal, q_lens, prefix, columns, max_cache_len, flush=True)
    kw = dict(causal=causal)
    ref = paged.run_oracle(q, kc, vc, table, lens, q_lens=q_lens, prefix_table=prefix_table if prefix else None, prefix_len=prefix, **kw)
    to = lambda t: None if t is None else t.to(DEV)
    # (a copy to the GPU keeps strides only of dense tensors: the others are built there)
    dkc, dvc = (paged.pool(*kc.shape, dt, layout).to(DEV) if layout != "wide" else torch.full((kc.shape[0], page + 3, hkv + 1, d + 8), math.nan, dtype=dt, device=DEV)[:, 1:page + 1, 1:, 8:] for _ in "kv")
    dkc.copy_(kc)
    dvc.copy_(vc)
    out = torch.full(q.shape, 7.0, dtype=dt, device=DEV)
    lse = torch.full(q.shape[:3], 7.0, device=DEV)
    ints = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device=DEV)
    kw.update(out=out, lse=lse, q_lens=ints(q_lens), max_cache_len=max_cache_len)
    if prefix:
        binding.bsfa_prefix_attention(to(q), dkc, dvc, to(prefix_table), prefix, to(table), ints(lens), **kw)
    else:
        binding.bsfa_paged_attention(to(q), dkc, dvc, to(table), ints(lens), **kw)
    torch.cuda.synchronize()
    paged.check_attention(out.cpu(), lse.cpu(), ref, dt, 7.0)
    # without lse, with scratch memory of the caller's
    again = torch.full(q.shape, 7.0, dtype=dt, device=DEV)
    need = binding.paged_workspace_bytes(to(q), dkc, to(table), to(prefix_table) if prefix else None, prefix, max_cache_len)
    kw.update(out=again, lse=None, workspace=torch.full((need + 512,), 255, dtype=torch.uint8, device=DEV))
    if prefix:
        binding.bsfa_prefix_attention(to(q), dkc, dvc, to(prefix_table), prefix, to(table), ints(lens), **kw)
    else:
        binding.bsfa_paged_attention(to(q), dkc, dvc, to(table), ints(lens), **kw)
    assert torch.equal(again, out)
    assert need == 0 or (kw["workspace"][need:] == 255).all()


LENGTHS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 255, 256]


@pytest.mark.parametrize("d,dtype,page,layout", [(128, "bf16", 16, "nhd"), (128, "fp16", 64, "hnd"), (64, "bf16", 32, "wide"), (64, "fp16", 128, "nhd"),
                                                 (128, "bf16", 256, "wide")])
def test_single_tokens_of_all_short_lengths(d, dtype, page, layout):
    run_case(LENGTHS, 1, 8, 2, d, page, dtype, layout)
    run_case(LENGTHS, 1, 8, 2, d, page, dtype, layout, columns=-(-1100 // page))          # (room for long ones: ranges)


@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 1), (4, 2), (7, 1), (8, 8), (16, 1), (17, 1), (24, 2), (33, 1), (64, 1), (66, 2), (130, 1)])
def test_head_groups(hq, hkv):
    run_case([70, 301, 0, 1], 1, hq, hkv, 128, 32)
    run_case([70, 301, 0, 1], 1, hq, hkv, 64, 16, "fp16", "hnd")


@pytest.mark.parametrize("s,group", [(2, 1), (3, 4), (5, 3), (9, 7), (16, 4), (17, 4), (33, 2), (70, 1), (100, 4), (129, 3)])
@pytest.mark.parametrize("causal", [True, False])
def test_several_tokens(s, group, causal):
    """Among them sequences shorter than their new tokens: the first rows see nothing."""
    lens = [s, s + 1, 300 + s, max(0, s - 3), 1, 0, 513]
    run_case(lens, s, 2 * group, 2, 128, 16, causal=causal)
    run_case(lens, s, 2 * group, 2, 64, 64, "fp16", "wide", causal=causal, q_lens=[s, 1, s // 2, s, 0, s, s - 1])


@pytest.mark.parametrize("lens", [[2000], [5003, 1, 0, 77], [1024, 1024], [4097] + [33] * 70])
def test_ranges_joined(lens):
    run_case(lens, 1, 8, 2, 128, 64, layout="hnd")
    run_case(lens, 2, 4, 4, 64, 16, "fp16", q_lens=[2 - b % 3 % 2 for b in range(len(lens))])


@pytest.mark.parametrize("tiles", [1, 2, 3, 4, 5, 6, 8])
@pytest.mark.parametrize("d", [64, 128])
def test_even_and_odd_numbers_of_tiles(tiles, d):
    """The kernel of many rows looks a tile ahead, at the end at one that does not exist, whose zeros must not come late.  Many
    workgroups at a time, and results that are dense enough to show a lost row anywhere."""
    for page in (16, 128):
        run_case([64 * tiles - 3] * 40, 9, 32, 8, d, page, "bf16", "hnd", max_cache_len=64 * tiles)
        run_case([5] * 95, 1, 32, 8, d, page, "bf16", prefix=64 * tiles - 16, max_cache_len=16)
    run_case([64 * tiles + 589] * 2, 589, 4, 2, d, 128, "fp16", "hnd")


def _dealt(name):
    g = torch.Generator().manual_seed(len(name))
    rnd = lambda n, hi: torch.randint(0, hi, (n,), generator=g).tolist()
    return {"equal": [340] * 5, "one long": rnd(20, 40) + [4000] + rnd(20, 40), "many": rnd(130, 200) + [0] * 3, "odd": [1, 2500, 0, 17, 16, 900, 15, 901],
            "borders": [256, 257, 255, 512, 496, 528, 1024, 1, 1023], "empty": [0] * 70, "last": [0] * 64 + [700]}[name]


@pytest.mark.parametrize("name", ["equal", "one long", "many", "odd", "borders", "empty", "last"])
@pytest.mark.parametrize("s,hq,hkv,d", [(1, 1, 1, 128), (1, 8, 8, 64), (3, 8, 1, 128), (5, 16, 2, 64), (9, 16, 2, 128)])
def test_a_batch_dealt_to_the_chip(name, s, hq, hkv, d):
    """Sequences of different lengths share workgroups, and workgroups share sequences: 3 x 8 and 5 x 8 and 9 x 8 rows to a KV head
    take the streaming kernel's wide form and the kernel of many rows."""
    lens = _dealt(name)
    columns = max(17, -(-max(lens) // 16))
    run_case(lens, s, hq, hkv, d, 16, "bf16" if d == 128 else "fp16", columns=columns)
    run_case(lens, s, hq, hkv, d, 32, q_lens=[(b + s) % (s + 1) for b in range(len(lens))], columns=columns)


def test_many_sequences_one_range_each():
    lens = [(7 * i) % 300 for i in range(600)]
    run_case(lens, 1, 4, 2, 64, 16)
    run_case([n % 100 for n in lens], 1, 4, 2, 64, 16, max_cache_len=100)


def test_bound_cuts_lengths():
    """max_cache_len clamps, as the table's size does."""
    dt = torch.bfloat16
    kc, vc, table, _ = paged.filled([300, 40], 16, 2, 128, dt, "nhd", 3)
    q = torch.randn(2, 1, 4, 128, generator=torch.Generator().manual_seed(5)).to(dt)
    ref = paged.run_oracle(q, kc, vc, table, [200, 40])
    got = binding.bsfa_paged_attention(q.to(DEV), kc.to(DEV), vc.to(DEV), table.to(DEV), torch.tensor([300, 40], dtype=torch.int32, device=DEV), max_cache_len=200)
    paged.check_attention(got.cpu(), None, ref, dt, 0.0)
    full = table[:, :19].contiguous()                       # 304 places
    ref = paged.run_oracle(q, kc, vc, full, [300, 40])
    got = binding.bsfa_paged_attention(q.to(DEV), kc.to(DEV), vc.to(DEV), full.to(DEV), torch.tensor([300, 40], dtype=torch.int32, device=DEV))
    paged.check_attention(got.cpu(), None, ref, dt, 0.0)


@pytest.mark.parametrize("s", [1, 3, 40])
def test_pages_that_the_cache_does_not_have(s):
    """Tokens in them are not seen; a sequence of nothing else is empty."""
    dt = torch.bfloat16
    lens = [100, 350, 64, 16]
    kc, vc, table, _ = paged.filled(lens, 16, 2, 128, dt, "nhd", 9)
    table[0, 2], table[0, 6], table[1, 0], table[1, 20], table[3, 0] = -1, kc.shape[0], -(1 << 31), (1 << 31) - 1, -1
    table[2, :] = -1
    q = torch.randn(4, s, 8, 128, generator=torch.Generator().manual_seed(5)).to(dt)
    ref = paged.run_oracle(q, kc, vc, table, lens)
    out, lse = torch.full(q.shape, 7.0, dtype=dt, device=DEV), torch.full(q.shape[:3], 7.0, device=DEV)
    binding.bsfa_paged_attention(q.to(DEV), kc.to(DEV), vc.to(DEV), table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), out=out, lse=lse)
    paged.check_attention(out.cpu(), lse.cpu(), ref, dt, 7.0)


@pytest.mark.parametrize("b,s", [(2, 1), (6, 1), (20, 1), (3, 12)])
def test_pages_of_the_prefix_that_the_cache_does_not_have(b, s):
    dt = torch.bfloat16
    lens = [(40 * x) % 100 for x in range(b)]
    for prefix, holes in ((600, [0, 7, 37]), (600, range(38)), (16, [0])):
        kc, vc, table, prefix_table = paged.filled(lens, 16, 2, 128, dt, "nhd", 9, prefix=prefix)
        for x in holes:
            prefix_table[x] = -1 if x % 2 else kc.shape[0] + x
        q = torch.randn(b, s, 8, 128, generator=torch.Generator().manual_seed(5)).to(dt)
        ref = paged.run_oracle(q, kc, vc, table, lens, prefix_table=prefix_table, prefix_len=prefix)
        out, lse = torch.full(q.shape, 7.0, dtype=dt, device=DEV), torch.full(q.shape[:3], 7.0, device=DEV)
        binding.bsfa_prefix_attention(q.to(DEV), kc.to(DEV), vc.to(DEV), prefix_table.to(DEV), prefix, table.to(DEV),
                                      torch.tensor(lens, dtype=torch.int32, device=DEV), out=out, lse=lse)
        paged.check_attention(out.cpu(), lse.cpu(), ref, dt, 7.0)


@pytest.mark.parametrize("s", [1, 5, 70])
def test_views(s):
    """Queries out of a fused projection, results heads first, a table that is a slice of a wider one: nothing beside the
    results is written."""
    dt, lens = torch.float16, [300, 9, 77]
    kc, vc, table, _ = paged.filled(lens, 16, 2, 64, dt, "nhd", 2)
    g = torch.Generator().manual_seed(5)
    fused = torch.randn(3, s, 12, 64, generator=g).to(dt)
    ref = paged.run_oracle(fused[:, :, 2:10], kc, vc, table, lens)
    wide = torch.full((3, table.shape[1] + 5), 3, dtype=torch.int32)
    wide[:, 2:-3] = table
    room = torch.full((3, 10, s + 2, 72), 7.0, dtype=dt, device=DEV)
    out = room[:, 1:9, 1:-1, :64].transpose(1, 2)
    binding.bsfa_paged_attention(fused.to(DEV)[:, :, 2:10], kc.to(DEV), vc.to(DEV), wide.to(DEV)[:, 2:-3], torch.tensor(lens, dtype=torch.int32, device=DEV), out=out)
    paged.check_attention(out.cpu().contiguous(), None, ref, dt, 7.0)
    out.fill_(7.0)
    assert (room == 7.0).all()


@pytest.mark.parametrize("b,s,hq,hkv", [(1, 1, 4, 2), (5, 1, 8, 2), (9, 2, 12, 4), (20, 1, 4, 1), (40, 1, 8, 2), (70, 3, 3, 1)])
@pytest.mark.parametrize("prefix", [1, 63, 64, 200, 1000, 2500])
def test_shared_prefix(b, s, hq, hkv, prefix):
    lens = [max(0, (37 * i + s) % 90) for i in range(b)]
    d, page, dtype, layout = [(128, 16, "bf16", "nhd"), (64, 64, "fp16", "hnd"), (128, 32, "fp16", "wide")][(b + prefix) % 3]
    run_case(lens, s, hq, hkv, d, page, dtype, layout, prefix=prefix)


def test_shared_prefix_with_long_own_parts_and_idle_elements():
    run_case([700, 0, 3, 1500, 10], 4, 8, 2, 128, 64, prefix=900, q_lens=[4, 0, 2, 1, 3])
    run_case([700, 0, 3, 1500, 10], 4, 8, 2, 64, 16, "fp16", "hnd", prefix=900, causal=False)


@pytest.mark.parametrize("scale", [1e-3, 30.0])
def test_flat_and_peaked_scores(scale):
    run_case([900, 77], 2, 8, 2, 128, 64, spread_q=scale)


@pytest.mark.parametrize("layout", ["nhd", "hnd"])
def test_offsets_beyond_32_bits(layout):
    """A cache whose last pages lie more than 2^32 bytes behind its first: appended to, and read by every kernel."""
    dt, page, hkv, d = torch.bfloat16, 64, 2, 128
    n = (1 << 32) // (page * hkv * d * 2) + 40
    shape = (n, page, hkv, d) if layout == "nhd" else (n, hkv, page, d)
    kc, vc = (torch.empty(shape, dtype=dt, device=DEV) for _ in "kv")
    if layout == "hnd":
        kc, vc = kc.transpose(1, 2), vc.transpose(1, 2)
    small_k, small_v, table, _ = paged.filled([300, 65], page, hkv, d, dt, "nhd", 4)
    m = small_k.shape[0]
    moved = torch.where((table >= 0) & (table < m), table + (n - m), table).to(DEV)
    for b, lens in enumerate((300, 65)):                     # (through the operator that writes it)
        t = torch.arange(lens)
        ids = table[b].long()[t // page]
        rows = [x[ids, t % page][None].to(DEV) for x in (small_k, small_v)]
        binding.bsfa_cache_append(None, *rows, kc, vc, moved[b:b + 1], torch.zeros(1, dtype=torch.int32, device=DEV))
        for x, y in ((kc, small_k), (vc, small_v)):
            assert torch.equal(x[ids.to(DEV) + (n - m), t.to(DEV) % page].cpu(), y[ids, t % page])
    lens = torch.tensor([300, 65], dtype=torch.int32, device=DEV)
    for s in (2, 50):
        q = torch.randn(2, s, 4, d, generator=torch.Generator().manual_seed(5)).to(dt)
        ref = paged.run_oracle(q, small_k, small_v, table, [300, 65])
        got = binding.bsfa_paged_attention(q.to(DEV), kc, vc, moved, lens)
        paged.check_attention(got.cpu(), None, ref, dt, 0.0)
        none = torch.zeros(2, dtype=torch.int32, device=DEV)
        got = binding.bsfa_prefix_attention(q.to(DEV), kc, vc, moved[0, :5].contiguous(), 300, moved, none)
        ref = paged.run_oracle(q, small_k, small_v, table, [0, 0], prefix_table=table[0, :5], prefix_len=300)
        paged.check_attention(got.cpu(), None, ref, dt, 0.0)
