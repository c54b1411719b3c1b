"""Host-side checks of the paged cache's entry points (no GPU): what they refuse, before touching a device; and the
oracle's own pins."""
import ctypes
import math
import os

import pytest
import torch

from oracle import paged_oracle
from paper_2512_07011_amd import binding

FAKE = ctypes.c_void_p(0x10000)      # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2512_07011_amd import build
        build.build_lib()
    return binding.lib()


def cache(**kw):
    c = binding.bsfa_cache(100, 16, 2, 128, 0, 16 * 256, 256, 128, 16 * 256, 256, 128, 0x10000, 0x10000)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def append(**kw):
    p = binding.bsfa_append(3, 4, 5, 2560, 512, 128, 1280, 256, 128, 1280, 256, 128, 2560, 512, 128, 1280, 256, 128,
                            None, 0x10000, 0x10000, 8, 8, 0x10000, 128, 128, 0)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def paged(**kw):
    p = binding.bsfa_paged(3, 4, 5, 2560, 512, 128, 2560, 512, 128, None, 0x10000, 0x10000, 8, 8, 0, None, 0, 0, 0x10000, 1 << 40)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


BAD_CACHE = [
    (dict(dtype=2), -3), (dict(n_pages=0), -2), (dict(n_kv_heads=0), -2), (dict(page_size=8), -2), (dict(page_size=48), -2),
    (dict(page_size=1 << 21), -2), (dict(page_size=0), -2), (dict(page_size=-16), -2), (dict(head_dim=96), -4), (dict(k_stride_n=250), -2), (dict(v_stride_h=64), -2),
    (dict(k_stride_page=-8), -2), (dict(v_stride_n=(1 << 25) + 8), -2), (dict(n_kv_heads=3), -2), (dict(k=None), -1), (dict(v=0x10008), -2),
]


@pytest.mark.parametrize("kw, code", BAD_CACHE + [(None, -1)])
def test_bad_caches(lib, kw, code):
    c = None if kw is None else ctypes.byref(cache(**kw))
    assert lib.bsfa_cache_append(c, ctypes.byref(append()), FAKE, FAKE, FAKE, FAKE, None, None) == code
    assert lib.bsfa_paged_attention(c, ctypes.byref(paged()), FAKE, 1, FAKE, None, None) == code
    assert lib.bsfa_last_error() != b""
    p = paged(prefix_table=0x10000, prefix_len=20, prefix_pages=2)
    assert lib.bsfa_prefix_attention(c, ctypes.byref(p), FAKE, 1, FAKE, None, None) == code
    if kw is None or not {"k", "v"} & set(kw):
        assert lib.bsfa_paged_workspace_bytes(c, ctypes.byref(paged())) == 0


@pytest.mark.parametrize("kw, code", [
    (dict(batch=0), -2), (dict(seqlen=0), -2), (dict(n_q_heads=3), -2), (dict(n_q_heads=0), -2), (dict(batch=1 << 20, seqlen=1 << 20), -2),
    (dict(q_stride_n=516), -2), (dict(k_stride_h=120), -2), (dict(v_stride_b=-8), -2), (dict(qo_stride_h=64), -2), (dict(ko_stride_n=4), -2),
    (dict(seqlens=0x10002), -2), (dict(start=None), -1), (dict(start=0x10001), -2), (dict(block_table=None), -1), (dict(table_pages=0), -2),
    (dict(table_pages=1 << 27), -2), (dict(table_stride_b=-1), -2), (dict(cos_sin=None), -1), (dict(cos_sin=0x10004), -2), (dict(n_positions=127), -2),
    (dict(rot_dim=0), -2), (dict(rot_dim=8), -2), (dict(rot_dim=72), -2), (dict(rot_dim=144), -2), (dict(interleaved=2), -2),
])
def test_bad_appends(lib, kw, code):
    c = cache()
    assert lib.bsfa_cache_append(ctypes.byref(c), ctypes.byref(append(**kw)), FAKE, FAKE, FAKE, FAKE, FAKE, None) == code, lib.bsfa_last_error()


def test_append_pointers(lib):
    c, p = ctypes.byref(cache()), ctypes.byref(append())
    odd = ctypes.c_void_p(0x10008)
    assert lib.bsfa_cache_append(c, None, FAKE, FAKE, FAKE, FAKE, None, None) == -1
    assert lib.bsfa_cache_append(c, p, FAKE, None, FAKE, FAKE, None, None) == -1
    assert lib.bsfa_cache_append(c, p, FAKE, FAKE, None, FAKE, None, None) == -1
    assert lib.bsfa_cache_append(c, p, FAKE, FAKE, FAKE, None, None, None) == -1
    for x in range(5):
        a = [FAKE] * 5
        a[x] = odd
        assert lib.bsfa_cache_append(c, p, *a, None) == -2


@pytest.mark.parametrize("kw, code", [
    (dict(batch=0), -2), (dict(seqlen=0), -2), (dict(n_q_heads=5), -2), (dict(batch=1 << 20, seqlen=1 << 20), -2), (dict(q_stride_b=-8), -2),
    (dict(batch=1 << 25, seqlen=1), -2), (dict(seqlen=1 << 25), -2), (dict(batch=1 << 20, seqlen=1, table_pages=1 << 11), -2),
    (dict(q_stride_h=4), -2), (dict(o_stride_n=120), -2), (dict(q_lens=0x10002), -2), (dict(cache_lens=None), -1), (dict(cache_lens=0x10003), -2),
    (dict(block_table=None), -1), (dict(table_pages=0), -2), (dict(table_pages=1 << 27), -2), (dict(table_stride_b=-8), -2), (dict(max_cache_len=-1), -2),
    (dict(workspace_bytes=-1), -5),
])
def test_bad_problems(lib, kw, code):
    c = ctypes.byref(cache())
    assert lib.bsfa_paged_attention(c, ctypes.byref(paged(**kw)), FAKE, 1, FAKE, None, None) == code, lib.bsfa_last_error()
    p = paged(prefix_table=0x10000, prefix_len=20, prefix_pages=2, **kw)
    assert lib.bsfa_prefix_attention(c, ctypes.byref(p), FAKE, 1, FAKE, None, None) == code


@pytest.mark.parametrize("kw, code", [(dict(prefix_len=0), -2), (dict(prefix_len=33), -2), (dict(prefix_table=None), -1), (dict(prefix_pages=0), -2),
                                      (dict(prefix_table=0x10002), -2), (dict(workspace=None), -5), (dict(workspace=0x10010), -5), (dict(workspace_bytes=100), -5)])
def test_bad_prefixes_and_workspaces(lib, kw, code):
    p = paged(**{**dict(prefix_table=0x10000, prefix_len=20, prefix_pages=2), **kw})
    assert lib.bsfa_prefix_attention(ctypes.byref(cache()), ctypes.byref(p), FAKE, 1, FAKE, None, None) == code, lib.bsfa_last_error()


def test_pointers(lib):
    c, p = ctypes.byref(cache()), ctypes.byref(paged())
    assert lib.bsfa_paged_attention(c, None, FAKE, 1, FAKE, None, None) == -1
    assert lib.bsfa_paged_attention(c, p, None, 1, FAKE, None, None) == -1
    assert lib.bsfa_paged_attention(c, p, FAKE, 1, None, None, None) == -1
    assert lib.bsfa_paged_attention(c, p, ctypes.c_void_p(0x10008), 1, FAKE, None, None) == -2
    assert lib.bsfa_paged_attention(c, p, FAKE, 1, ctypes.c_void_p(0x10002), None, None) == -2
    assert lib.bsfa_paged_attention(c, p, FAKE, 1, FAKE, ctypes.c_void_p(0x10002), None) == -2


def test_what_is_written_has_no_two_elements_in_one_place(lib):
    """A batch of one read tensor is fine (the check behind it answers), one of a written tensor is not."""
    c, still = ctypes.byref(cache()), dict(workspace=None, prefix_table=0x10000, prefix_len=20, prefix_pages=2)
    assert lib.bsfa_prefix_attention(c, ctypes.byref(paged(q_stride_b=0, **still)), FAKE, 1, FAKE, None, None) == -5
    assert lib.bsfa_prefix_attention(ctypes.byref(cache(k_stride_page=0)), ctypes.byref(paged(**still)), FAKE, 1, FAKE, None, None) == -5
    assert lib.bsfa_prefix_attention(c, ctypes.byref(paged(o_stride_b=0, **still)), FAKE, 1, FAKE, None, None) == -2
    for kw in (dict(qo_stride_b=0), dict(ko_stride_b=64)):
        assert lib.bsfa_cache_append(c, ctypes.byref(append(**kw)), FAKE, FAKE, FAKE, ctypes.c_void_p(0x20000), ctypes.c_void_p(0x30000), None) == -2
        assert b"_out" in lib.bsfa_last_error()
    for kw in (dict(k_stride_page=0), dict(v_stride_page=0)):
        assert lib.bsfa_cache_append(ctypes.byref(cache(**kw)), ctypes.byref(append()), FAKE, FAKE, FAKE, FAKE, None, None) == -2


def test_workspaces_of_the_binding_are_contiguous(monkeypatch):
    monkeypatch.setattr(binding, "_same_device", lambda *a: None)
    monkeypatch.setattr(binding, "_on_device", lambda *a: pytest.fail("launched"))
    q, kc = torch.zeros(2, 3, 4, 128, dtype=torch.bfloat16), torch.zeros(4, 16, 2, 128, dtype=torch.bfloat16)
    i, t = torch.zeros(2, dtype=torch.int32), torch.zeros(2, 100, dtype=torch.int32)
    with pytest.raises(TypeError):
        binding.bsfa_paged_attention(q, kc, kc, t, i, workspace=torch.zeros(1, dtype=torch.uint8).expand(1 << 24))


def test_workspace_follows_the_work(lib):
    """None where sequences are short by the host's knowledge; never more than a fixed number of ranges on top of the batch."""
    c = cache(n_pages=1 << 20)
    need = lambda **kw: lib.bsfa_paged_workspace_bytes(ctypes.byref(c), ctypes.byref(paged(**kw)))
    assert need() == 0 and need(table_pages=16) == 0 and need(table_pages=1000, max_cache_len=200) == 0
    assert 0 < need(seqlen=1, table_pages=1000) == need(seqlen=1, table_pages=100000) < 64 << 20
    assert need(prefix_table=0x10000, prefix_len=20, prefix_pages=2) > 0


def test_packed_descriptors_are_the_structures():
    """The binding packs the descriptors' members by format: at the places that the structures have them."""
    vals = iter(range(1, 200))
    for cls, pack in ((binding.bsfa_cache, binding._PACK_CACHE), (binding.bsfa_append, binding._PACK_APPEND), (binding.bsfa_paged, binding._PACK_PAGED)):
        v = [next(vals) for _ in cls._fields_]
        packed = pack(*v)
        assert bytes(cls(*v))[:len(packed)] == packed and ctypes.sizeof(cls) - len(packed) < 8


def test_binding_refuses():
    q = torch.zeros(1, 1, 2, 128, dtype=torch.bfloat16)
    kc = torch.zeros(4, 16, 2, 128, dtype=torch.bfloat16)
    i = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError):
        binding.bsfa_paged_attention(q, kc, kc, i[None], i)
    with pytest.raises(ValueError):
        binding.bsfa_cache_append(q, q, q, kc, kc, i[None], i)


def test_binding_checks_shapes_and_types(monkeypatch):
    """(no GPU: the check of the device is left out; nothing that is refused here reaches the library)"""
    monkeypatch.setattr(binding, "_same_device", lambda *a: None)
    monkeypatch.setattr(binding, "_on_device", lambda *a: pytest.fail("launched"))
    q, k = torch.zeros(2, 3, 4, 128, dtype=torch.bfloat16), torch.zeros(2, 3, 2, 128, dtype=torch.bfloat16)
    kc = torch.zeros(4, 16, 2, 128, dtype=torch.bfloat16)
    i, t = torch.zeros(2, dtype=torch.int32), torch.zeros(2, 1, dtype=torch.int32)
    cs = torch.zeros(16, 128)
    bad = [dict(q=q[..., :64]), dict(q=q[0]), dict(kc=kc[0]), dict(vc=kc[:2]), dict(t=t[:1]), dict(i=i[:1]), dict(vc=kc.half()), dict(q=q.half()), dict(t=t.long()),
           dict(i=i.float()), dict(q=q.transpose(2, 3)), dict(kc=kc.float(), vc=kc.float(), q=q.float())]
    for kw in bad:
        a = {**dict(q=q, kc=kc, vc=kc, t=t, i=i), **kw}
        with pytest.raises((ValueError, TypeError)):
            binding.bsfa_paged_attention(a["q"], a["kc"], a["vc"], a["t"], a["i"], workspace=None)
        with pytest.raises((ValueError, TypeError)):
            binding.bsfa_prefix_attention(a["q"], a["kc"], a["vc"], i, 16, a["t"], a["i"], workspace=None)
    for kw in (dict(q_lens=i[:1]), dict(out=q[:1]), dict(out=q.half()), dict(lse=torch.zeros(2, 3, 2)), dict(lse=torch.zeros(2, 3, 4, dtype=torch.float64))):
        with pytest.raises((ValueError, TypeError)):
            binding.bsfa_paged_attention(q, kc, kc, t, i, workspace=None, **kw)
    good = dict(q=q, k=k, v=k, k_cache=kc, v_cache=kc, block_table=t, start=i, cos_sin=cs)
    for kw in (dict(k=k[:1]), dict(v=k[:1]), dict(k=k[..., :1, :]), dict(q=q[:1]), dict(v=k.half()), dict(start=i[:1]), dict(start=i.long()), dict(block_table=t[0]), dict(cos_sin=cs.half()),
               dict(cos_sin=cs.t()), dict(cos_sin=None), dict(q_out=q[:1]), dict(k_out=q), dict(q=None, q_out=q), dict(seqlens=i[:1]), dict(seqlens=i.long()), dict(q=q.half())):
        with pytest.raises((ValueError, TypeError)):
            binding.bsfa_cache_append(**{**good, **kw})


# ---- the oracle ------------------------------------------------------------------------------------------
def test_oracle_attention_is_a_softmax_over_what_is_seen():
    g = torch.Generator().manual_seed(1)
    k, v, q = (torch.randn(3, 16, 1, 64, generator=g) for _ in range(2)), None, None
    kc, vc = k
    q = torch.randn(1, 3, 2, 64, generator=g)
    table = torch.tensor([[2, 0, -1]], dtype=torch.int32)
    out, lse, spread, _ = paged_oracle.attend(q, kc, vc, table, [20])
    keys, values = torch.cat([kc[2], kc[0]])[:, 0].double(), torch.cat([vc[2], vc[0]])[:, 0].double()
    for i in range(3):
        n = 18 + i
        s = torch.stack([sum(q[0, i, 1].double() * keys[t]) / 8 for t in range(n)])
        w = s.exp() / s.exp().sum()
        assert torch.allclose(out[0, i, 1], (w[:, None] * values[:n]).sum(0))
        assert torch.allclose(lse[0, i, 1], s.exp().sum().log())
        assert torch.allclose(spread[0, i, 1], (w[:, None] * values[:n].abs()).sum(0))
    whole, z, _, _ = paged_oracle.attend(q, kc, vc, table, [4], prefix_table=torch.tensor([2], dtype=torch.int32), prefix_len=16, causal=False)
    part = paged_oracle.attend(q, kc, vc, torch.tensor([[2, 2]], dtype=torch.int32), [20], causal=False)
    assert torch.allclose(whole, part[0]) and torch.allclose(z, part[1])
    empty = paged_oracle.attend(q, kc, vc, torch.tensor([[-1]], dtype=torch.int32), [16])
    assert (empty[0] == 0).all() and (empty[1] == -math.inf).all()


def test_oracle_rotation_keeps_lengths_and_relative_positions():
    """Products of rotated queries and keys depend on the difference of their positions alone."""
    g = torch.Generator().manual_seed(2)
    cs = binding.rotary_table(64, 64, device="cpu")
    q, k = torch.randn(1, 1, 1, 64, generator=g), torch.randn(1, 1, 1, 64, generator=g)
    z = torch.zeros(4, 16, 1, 64)
    for inter in (False, True):
        at = lambda x, pos: paged_oracle.append(x, x, z, z, torch.arange(4, dtype=torch.int32)[None], [pos], cs, x, interleaved=inter)
        dots = [(at(q, 5 + s)[2] * at(k, 2 + s)[3]).sum() for s in (0, 11, 40)]
        assert max(dots) - min(dots) < 1e-5
        kc, vc, qo, ko = at(k, 17)
        assert torch.allclose(ko.norm(), k.double().norm()) and torch.equal(kc[1, 1], ko[0, 0]) and torch.equal(vc[1, 1], k[0, 0].double())
        assert kc.count_nonzero() == 64 and torch.equal(at(k, 0)[3], k.double()) and torch.equal(qo, ko)
