"""The binding's calls of the paged cache that the documentation allows, or that it has to refuse (no GPU: the library is replaced by a
recorder)."""
import types

import pytest
import torch

from paper_2512_07011_amd import binding


class Recorder:
    def __init__(self):
        self.calls = []

    def bsfa_cache_append(self, *a):
        self.calls.append(a)
        return 0


@pytest.fixture
def recorded(monkeypatch):
    lib = Recorder()
    monkeypatch.setattr(binding, "lib", lambda: lib)
    monkeypatch.setattr(binding, "_same_device", lambda *a: None)
    monkeypatch.setattr(binding, "_on_device", lambda device, stream, call, *args: call(*args, 0))
    return lib


def tokens():
    q, k = torch.zeros(2, 3, 4, 128, dtype=torch.bfloat16), torch.zeros(2, 3, 2, 128, dtype=torch.bfloat16)
    kc = torch.zeros(4, 16, 2, 128, dtype=torch.bfloat16)
    i, t = torch.zeros(2, dtype=torch.int32), torch.zeros(2, 1, dtype=torch.int32)
    return q, k, k.clone(), kc, kc.clone(), t, i, torch.zeros(16, 128)


def test_rotated_keys_are_asked_for_or_not(recorded):
    """k_out True or a tensor: they are returned; None or False: they are not."""
    a = tokens()
    for k_out in (None, False):
        q, k = binding.bsfa_cache_append(*a, k_out=k_out)
        assert q.shape == a[0].shape and k is None and recorded.calls[-1][6] == 0
    q, k = binding.bsfa_cache_append(*a, k_out=True)
    assert k.shape == a[1].shape and recorded.calls[-1][6] == k.data_ptr()
    q, k = binding.bsfa_cache_append(*a, k_out=a[1])
    assert k is a[1] and recorded.calls[-1][6] == a[1].data_ptr()


def test_a_stream_of_another_device_is_refused(monkeypatch):
    """Kernels on it would run where the tensors are not."""
    monkeypatch.setattr(binding, "_current_device", lambda: 0)
    here, there = (types.SimpleNamespace(device=torch.device("cuda", x), cuda_stream=5 + x) for x in (0, 1))
    launched = []
    binding._on_device(torch.device("cuda", 0), here, lambda *a: launched.append(a), 1, 2)
    assert launched == [(1, 2, 5)]
    with pytest.raises(ValueError):
        binding._on_device(torch.device("cuda", 0), there, lambda *a: pytest.fail("launched"), 1, 2)


@pytest.mark.parametrize("rot", [0, -2, 1, 15, 63])
def test_rotation_tables_have_pairs(rot):
    """An odd width has no pairs: the table came out a column wider, for a rotation of other angles than the width says."""
    with pytest.raises(ValueError):
        binding.rotary_table(8, rot, device="cpu")
