"""bsfa_cache_append against the 64-bit oracle, and appending, prompts, decoding and shared prefixes in one run."""
import math

import pytest
import torch

from oracle import paged_oracle
from paper_2512_07011_amd import binding
from tests import paged

pytestmark = pytest.mark.gpu
DEV = "cuda"


def bits(t):
    return t.contiguous().view(torch.int16)


def ints(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device=DEV)


def append_case(b, n, hq, hkv, d, page, rot, start, seqlens=None, interleaved=False, dtype="bf16", layout="nhd", q_layout="fused",
                in_place=False, seed=0, holes=(), columns=None, keys_only=False):
    dt = paged.DTYPES[dtype]
    g = torch.Generator().manual_seed(seed)
    ends = [s + (n if seqlens is None else seqlens[i]) for i, s in enumerate(start)]
    columns = columns or max(1, -(-max(ends) // page))
    ids = torch.randperm(b * columns + 3, generator=g)[:b * columns].int().view(b, columns)
    for x, y, to in holes:
        ids[x, y] = to
    kc, vc = (paged.pool(b * columns + 3, page, hkv, d, dt, layout) for _ in "kv")
    fused = torch.randn(b, n, hq + 2 * hkv, d, generator=g).to(dt)
    if seqlens is not None:
        for i, m in enumerate(seqlens):
            fused[i, max(0, m):] = math.nan
    table = binding.rotary_table(columns * page, rot, device="cpu") if rot else None
    q, k, v = fused.split([hq, hkv, hkv], dim=2)
    if keys_only:
        q = None
    ref = paged_oracle.append(k, v, kc, vc, ids, start, table, q, seqlens, interleaved)
    df = fused.to(DEV)
    dq, dk, dv = df.split([hq, hkv, hkv], dim=2)
    if q_layout == "bhnd":
        dq, dk, dv = (t.transpose(1, 2).contiguous().transpose(1, 2) for t in (dq, dk, dv))
    dkc, dvc = (torch.empty(0) for _ in "kv")
    if layout == "wide":
        dkc, dvc = (torch.full((kc.shape[0], page + 3, hkv + 1, d + 8), math.nan, dtype=dt, device=DEV) for _ in "kv")
        whole = (dkc, dvc)
        dkc, dvc = (t[:, 1:page + 1, 1:, 8:] for t in whole)
    else:
        dkc, dvc = kc.to(DEV), vc.to(DEV)
    q_out = None if keys_only else dq if in_place else torch.full((b, n, hq, d), 7.0, dtype=dt, device=DEV)
    k_out = dk if in_place else torch.full((b, n, hkv, d), 7.0, dtype=dt, device=DEV)
    before = df.clone()
    print("case", b, n, hq, hkv, d, page, rot, start, seqlens, interleaved, dtype, layout, q_layout, in_place, flush=True)
    got_q, got_k = binding.bsfa_cache_append(None if keys_only else dq, dk, dv, dkc, dvc, ids.to(DEV), ints(start), None if table is None else table.to(DEV),
                                             seqlens=ints(seqlens), interleaved=interleaved, q_out=q_out, k_out=k_out)
    torch.cuda.synchronize()
    rkc, rvc, rq, rk = ref
    u = paged.half_step(dt)

    def close(got, want, what, size):
        """One rounding, u of the value; two products and a sum in 32 bits before it, 3 * 2^-24 of their sizes at most."""
        there = ~want.isnan()
        tol = u * want.abs() + (3 * 2.0 ** -24 * (1 + u)) * size + torch.finfo(dt).smallest_normal
        bad = there & ~((got.double() - want).abs() <= tol)
        assert not bad.any(), (what, bad.sum().item(), bad.nonzero()[0].tolist())
        return there

    biggest = 2 * fused.double().nan_to_num().abs().amax()
    if not keys_only:
        there = close(got_q.cpu(), rq, "q", biggest)
        if not in_place:
            assert (got_q.cpu()[~there] == 7.0).all()
    there = close(got_k.cpu(), rk, "k", biggest)
    if not in_place:
        assert (got_k.cpu()[~there] == 7.0).all()
        assert torch.equal(bits(df), bits(before))
    there = close(dkc.cpu(), rkc, "k cache", biggest)
    assert dkc.cpu()[~there].isnan().all()
    assert torch.equal(bits(dvc.cpu().nan_to_num(nan=9.0)), bits(rvc.nan_to_num(nan=9.0).to(dt)))       # values are copied
    if layout == "wide":
        for t, view in zip(whole, (dkc, dvc)):
            view.fill_(math.nan)
            assert t.isnan().all()                          # nothing beside the cache's own places was written


@pytest.mark.parametrize("d,rot", [(128, 128), (128, 64), (128, 16), (128, 112), (64, 64), (64, 32), (64, 48)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotations(d, rot, interleaved):
    append_case(2, 5, 4, 2, d, 16, rot, [0, 29], interleaved=interleaved)
    append_case(3, 1, 8, 1, d, 32, rot, [0, 31, 64], interleaved=interleaved, dtype="fp16", layout="hnd", q_layout="bhnd")


@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 1), (12, 4), (28, 4), (32, 8), (64, 8)])
def test_heads(hq, hkv):
    append_case(2, 3, hq, hkv, 128, 64, 128, [62, 5], layout="wide")
    append_case(2, 3, hq, hkv, 64, 16, 32, [62, 5], dtype="fp16")


def test_lengths_and_positions():
    append_case(5, 40, 4, 2, 128, 16, 128, [0, 3, 100, 17, 1], seqlens=[40, 0, 1, 39, 17])
    append_case(1, 300, 4, 2, 64, 64, 64, [1000])
    append_case(7, 1, 4, 2, 128, 16, 128, [0, 15, 16, 17, 31, 32, 200])


def test_in_place_and_without_rotation():
    append_case(2, 9, 4, 2, 128, 16, 128, [0, 7], in_place=True)
    append_case(2, 9, 4, 2, 64, 16, 32, [0, 7], in_place=True, interleaved=True, q_layout="bhnd")
    append_case(2, 9, 4, 2, 64, 16, 0, [0, 7], keys_only=True)
    append_case(2, 9, 4, 2, 128, 16, 64, [0, 7], keys_only=True)


def test_places_that_do_not_exist():
    """Tokens beyond the table are left out; those of a page that is none are rotated, and stored nowhere."""
    append_case(3, 20, 4, 2, 128, 16, 128, [10, -5, 0], columns=1, holes=[(2, 0, -1)])
    append_case(2, 40, 4, 2, 64, 16, 64, [0, 16], columns=3, holes=[(0, 1, 1 << 30), (1, 2, -(1 << 31))])


def test_serving_run():
    """Prompts go through append and bsfa_forward; decoding appends a token at a time to three sequences of which two share a
    prefix, and every step's attention equals dense attention over the whole sequence."""
    dt, hq, hkv, d, page = torch.bfloat16, 8, 2, 128, 32
    g = torch.Generator().manual_seed(3)
    prefix, own, steps = 150, [40, 1, 70], 5
    total = [prefix + n + steps for n in own]
    table = binding.rotary_table(512, d, 10000.0)
    kc, vc = (t.fill_(math.nan) for t in binding.alloc_cache(40, page, hkv, d))
    ids = torch.randperm(40, generator=g).int()
    prefix_table = ids[:5].to(DEV)                                         # 160 places
    own_table = ids[5:5 + 3 * 4].view(3, 4).contiguous().to(DEV)           # 128 places each
    rnd = lambda *s: torch.randn(*s, generator=g).to(dt).to(DEV)
    pq, pk, pv = rnd(1, prefix, hq, d), rnd(1, prefix, hkv, d), rnd(1, prefix, hkv, d)
    rq, rk = binding.bsfa_cache_append(pq, pk, pv, kc, vc, prefix_table[None], ints([0]), table, k_out=True)
    dense = torch.full((hq,), -math.inf, device=DEV)
    prompt = binding.bsfa_forward(rq, rk, pv, dense)
    paged_prompt = binding.bsfa_paged_attention(rq, kc, vc, prefix_table[None], ints([prefix]))
    ref = paged_oracle.attend(rq.cpu(), rk.cpu(), pv.cpu(), torch.zeros(1, 1, dtype=torch.int32), [prefix])   # (one page of 150 places)
    paged.check_attention(paged_prompt.cpu(), None, ref, dt, 0.0)
    assert (prompt.float() - ref[0].to(DEV)).abs().max() <= 2e-2
    # each sequence's own tokens so far, in its own pages, at positions behind the prefix: the table is read from there on
    behind = table[prefix:].contiguous()
    n = max(own)
    oq, ok, ov = rnd(3, n, hq, d), rnd(3, n, hkv, d), rnd(3, n, hkv, d)
    _, rok = binding.bsfa_cache_append(oq, ok, ov, kc, vc, own_table, ints([0, 0, 0]), behind, seqlens=ints(own), k_out=True)
    keys = [torch.cat([rk[0], rok[b, :own[b]]]) for b in range(3)]
    values = [torch.cat([pv[0], ov[b, :own[b]]]) for b in range(3)]
    for step in range(steps):
        q, k, v = rnd(3, 1, hq, d), rnd(3, 1, hkv, d), rnd(3, 1, hkv, d)
        at = [m + step for m in own]
        q, kr = binding.bsfa_cache_append(q, k, v, kc, vc, own_table, ints(at), behind, q_out=q, k_out=True)
        out = binding.bsfa_prefix_attention(q, kc, vc, prefix_table, prefix, own_table, ints([m + 1 for m in at]))
        for b in range(3):
            keys[b], values[b] = torch.cat([keys[b], kr[b]]), torch.cat([values[b], v[b]])
            ref = paged_oracle.attend(q[b:b + 1].cpu(), keys[b][None].cpu(), values[b][None].cpu(), torch.zeros(1, 1, dtype=torch.int32), [len(keys[b])])
            paged.check_attention(out[b:b + 1].cpu(), None, ref, dt, 0.0)
    assert [len(x) for x in keys] == total


def test_graph_replays_follow_the_lengths():
    """One captured step of append and attention, replayed as the sequences grow, with eager work between the replays."""
    dt, hq, hkv, d, page, b = torch.bfloat16, 8, 2, 128, 16, 3
    g = torch.Generator().manual_seed(8)
    kc, vc = (t.zero_() for t in binding.alloc_cache(3 * 40, page, hkv, d))
    table = torch.randperm(120, generator=g).int().view(3, 40).to(DEV)
    prefix_table = torch.tensor([119, 3], dtype=torch.int32, device=DEV)   # (any pages: what lies there is the prefix)
    cos_sin = binding.rotary_table(640, d)
    q, k, v = (torch.zeros(b, 1, h, d, dtype=dt, device=DEV) for h in (hq, hkv, hkv))
    start, held = ints([0, 0, 0]), ints([0, 0, 0])

    def step():
        rq, _ = binding.bsfa_cache_append(q, k, v, kc, vc, table, start, cos_sin)
        return (binding.bsfa_paged_attention(rq, kc, vc, table, held),
                binding.bsfa_prefix_attention(rq, kc, vc, prefix_table, 20, table, held))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    at = [0, 100, 500]
    for turn in range(6):
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, generator=g).to(dt))
        start.copy_(ints(at))
        held.copy_(ints([x + 1 for x in at]))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in captured]
        want = step()
        torch.cuda.synchronize()
        there = [x for x in range(b) if at[x] < 640]          # (the last token of the third has no place: its query is not written)
        for x, y in zip(got, want):
            assert torch.equal(x[there], y[there]), turn
        at = [x + 1 + 20 * turn for x in at]


def test_calls_on_other_streams():
    """A call is ordered by the stream it is given, and its scratch memory is its own."""
    dt = torch.bfloat16
    lens = [3000, 700]
    kc, vc, table, _ = paged.filled(lens, 16, 2, 128, dt, "nhd", 1)
    q = torch.randn(2, 1, 8, 128, generator=torch.Generator().manual_seed(5)).to(dt)
    ref = paged.run_oracle(q, kc, vc, table, lens)
    args = [t.to(DEV) for t in (q, kc, vc, table)] + [ints(lens)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = [binding.bsfa_paged_attention(*args, stream=s) for s in streams for _ in range(2)]
    torch.cuda.synchronize()
    for o in outs:
        paged.check_attention(o.cpu(), None, ref, dt, 0.0)
