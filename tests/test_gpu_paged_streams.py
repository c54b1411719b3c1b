"""Calls on streams that are not the current one: ordered by their own stream, each with scratch memory of its own."""
import pytest
import torch

from oracle import paged_oracle
from paper_2512_07011_amd import binding
from tests import paged

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _busy(x, n):
    """About n * 0.5 ms of work on the current stream."""
    for _ in range(n):
        x = x @ x
        x /= x.norm()
    return x


@pytest.mark.parametrize("prefix", [0, 500])
def test_calls_wait_for_their_stream_and_share_no_scratch_memory(prefix, monkeypatch):
    """Queries, lengths and tables are written on a call's own stream behind long work there, which the host does not wait for, and
    the result is read there: a call on another stream would see what was there before.  The streams' calls differ in their inputs, and
    overlap: calls that shared scratch memory would join each other's ranges."""
    dt, lens = torch.bfloat16, [[3000, 700], [2100, 2900], [64, 3000]]
    kc, vc, table, prefix_table = paged.filled([3000, 3000], 16, 2, 128, dt, "nhd", 1, prefix=prefix)
    g = torch.Generator().manual_seed(5)
    queries = [torch.randn(2, 2, 8, 128, generator=g).to(dt) for _ in lens]
    tables = [table.clone(), table.flip(0), table.clone()]
    refs = [paged.run_oracle(q, kc, vc, t, n, prefix_table=prefix_table if prefix else None, prefix_len=prefix) for q, t, n in zip(queries, tables, lens)]
    kc, vc, prefix_table = (t.to(DEV) for t in (kc, vc, prefix_table))
    ready = [(q.to(DEV), t.to(DEV), torch.tensor(n, dtype=torch.int32, device=DEV)) for q, t, n in zip(queries, tables, lens)]
    late = [(torch.zeros_like(q), torch.full_like(t, -1), torch.zeros_like(n)) for q, t, n in ready]
    work = [torch.randn(4096, 4096, device=DEV) for _ in lens]
    taken, scratch = [], binding._scratch

    def record(nbytes, device, stream):
        t = scratch(nbytes, device, stream)
        taken.append((t.data_ptr(), nbytes, stream.cuda_stream))
        return t

    def call(q, t, n, stream):
        if prefix:
            return binding.bsfa_prefix_attention(q, kc, vc, prefix_table, prefix, t, n, stream=stream)
        return binding.bsfa_paged_attention(q, kc, vc, t, n, stream=stream)

    streams = [torch.cuda.Stream() for _ in lens]
    with torch.cuda.stream(streams[0]):
        _busy(work[0], 1)                                    # (loads the kernels)
    call(*late[0], None)
    torch.cuda.synchronize()
    monkeypatch.setattr(binding, "_scratch", record)
    events, outs = [], []
    for s, w, new, old in zip(streams, work, ready, late):
        with torch.cuda.stream(s):
            _busy(w, 40)
            for x, y in zip(old, new):
                x.copy_(y)
            events.append(s.record_event())
    for turn in range(2):                                    # (a stream's two calls may use one piece of memory after each other)
        outs += [call(*x, s) for s, x in zip(streams, late)]
    assert not any(e.query() for e in events), "the work in front of the calls was too short to tell"
    got = []
    for x, out in enumerate(outs):
        with torch.cuda.stream(streams[x % 3]):
            got.append(out.cpu())
    for x, out in enumerate(got):
        print("call", x, flush=True)
        paged.check_attention(out, None, refs[x % 3], dt, 0.0)
    assert len(taken) == 6 and [t[2] for t in taken] == [s.cuda_stream for s in streams] * 2
    for p, n, s in taken:
        assert all(s == s2 or p + n <= p2 or p2 + n2 <= p for p2, n2, s2 in taken)


def test_appending_waits_for_its_stream():
    """Tokens and positions are written on the call's stream behind long work; what the call stores and returns is theirs."""
    dt, page = torch.bfloat16, 16
    g = torch.Generator().manual_seed(6)
    cos_sin = binding.rotary_table(160, 64, device="cpu")
    table = torch.randperm(20, generator=g).int().view(2, 10)
    q, k, v = (torch.randn(2, 3, h, 64, generator=g).to(dt) for h in (4, 2, 2))
    start = [40, 157]
    kc, vc = (paged.pool(20, page, 2, 64, dt, "nhd", 7.0) for _ in "kv")
    want = paged_oracle.append(k, v, kc, vc, table, start, cos_sin, q)
    kc, vc, table, cos_sin = (t.to(DEV) for t in (kc, vc, table, cos_sin))
    ready = [t.to(DEV) for t in (q, k, v, torch.tensor(start, dtype=torch.int32))]
    late = [torch.zeros_like(t) for t in ready]
    late[3].fill_(-1000)                                     # (no place: a call that came too early would store nothing)
    w = torch.randn(4096, 4096, device=DEV)
    _busy(w, 1)
    binding.bsfa_cache_append(*late[:3], kc, vc, table, late[3], cos_sin)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        _busy(w, 40)
        for x, y in zip(late, ready):
            x.copy_(y)
        event = stream.record_event()
    rq, rk = binding.bsfa_cache_append(*late[:3], kc, vc, table, late[3], cos_sin, k_out=True, stream=stream)
    assert not event.query(), "the work in front of the call was too short to tell"
    with torch.cuda.stream(stream):
        got = [t.cpu().double() for t in (kc, vc, rq, rk)]
    u = paged.half_step(dt)
    for x, y in zip(got, want):
        # one rounding of the result; two products and a sum in 32 bits of values below 8 before it
        assert ((x - y).abs() <= u * y.abs() + 3 * 2.0 ** -24 * 16).all()
