"""The scratch memory of the attention over a paged cache, as the host is told of it (no GPU)."""
import pytest
import torch

from paper_2512_07011_amd import binding


@pytest.fixture(autouse=True)
def on_the_host(monkeypatch):
    monkeypatch.setattr(binding, "_same_device", lambda *a: None)
    monkeypatch.setattr(binding, "_on_device", lambda *a: pytest.fail("launched"))


def need(q, d=128, pages=2000, prefix=0, **kw):
    kc = torch.zeros(4, 16, 2, d, dtype=torch.bfloat16)
    table = torch.zeros(q.shape[0], pages, dtype=torch.int32)
    prefix_table = torch.zeros(-(-prefix // 16), dtype=torch.int32) if prefix else None
    return binding.paged_workspace_bytes(q, kc, table, prefix_table, prefix, **kw)


@pytest.mark.parametrize("prefix", [0, 500])
def test_queries_that_repeat_need_what_others_do(prefix):
    """One set of queries for the whole batch, or windows of one row: such a tensor can only be read, and the result is another."""
    whole = need(torch.zeros(3, 2, 8, 128, dtype=torch.bfloat16), prefix=prefix)
    assert whole > 0
    assert need(torch.zeros(1, 2, 8, 128, dtype=torch.bfloat16).expand(3, 2, 8, 128), prefix=prefix) == whole
    assert need(torch.zeros(64 * 128, dtype=torch.bfloat16).as_strided((3, 2, 8, 128), (1024, 1024, 128, 1)), prefix=prefix) == whole


def nowhere(*shape, dtype=torch.bfloat16):
    return torch.empty(*shape, dtype=dtype, device="meta")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv", [(32, 8), (28, 4), (8, 8), (7, 1)])
def test_bound(d, hq, hkv):
    """A row's unscaled result and its (m, l), 4 d + 8 bytes, once for each range that it is in.  A batch of `side` groups of 128 rows to
    a sequence is dealt to 512 / side workgroups and has a slot for each of them and each sequence: b * s * hq rows, and 512 groups of
    128 for the borders.  Behind a prefix the same again: its rows are everybody's, in parts of which 512 groups are made, or one part."""
    row, seen = 4 * d + 8, 0
    for b in (1, 2, 7, 16, 64, 256):
        for s in (1, 2, 5, 16, 64, 200, 512):
            for prefix, pages in ((0, 10), (0, 300), (0, 8192), (17, 10), (2000, 300), (131072, 10)):
                prefix_table = torch.zeros(-(-prefix // 16), dtype=torch.int32) if prefix else None
                got = binding.paged_workspace_bytes(nowhere(b, s, hq, d), nowhere(1, 16, hkv, d), nowhere(b, pages, dtype=torch.int32), prefix_table, prefix)
                most = (2 if prefix else 1) * (b * s * hq + 512 * 128) * row + 8 * b + 5 * 256
                assert got <= most, (b, s, prefix, pages, got, most)
                assert not prefix or got >= 2 * b * s * hq * row
                seen = max(seen, got)
    assert seen > 1 << 20


def test_sizes_of_large_batches_behind_a_prefix():
    """The figures that the documentation gives."""
    def mib(b, s):
        q, kc = nowhere(b, s, 32, 128), nowhere(4096, 16, 8, 128)
        return binding.paged_workspace_bytes(q, kc, nowhere(b, 64, dtype=torch.int32), torch.zeros(1000, dtype=torch.int32), 16000) / 2 ** 20

    assert round(mib(64, 200)) == 406 and round(mib(64, 512)) == 1040 and round(mib(4096, 4)) == 520
