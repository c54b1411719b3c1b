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
