"""More of what the paged cache's entry points refuse, and what they take, before touching a device (no GPU)."""
import ctypes

import pytest

from tests.test_paged_abi import FAKE, append, cache, lib, paged  # noqa: F401  (lib: a fixture)

OUT, KOUT = ctypes.c_void_p(0x20000), ctypes.c_void_p(0x30000)
# (behind every check of strides, before any launch: the workspace that is missing)
STOPS = dict(workspace=None, prefix_table=0x10000, prefix_len=20, prefix_pages=2)

# strides of three sequences of five tokens of four heads of width 128 (batch, token, head): is any place shared?
LAYOUTS = [((2560, 512, 128), False), ((2560, 128, 640), False), ((128, 1536, 384), False), ((512, 1536, 128), False), ((2568, 512, 128), False),
           ((128, 512, 128), True), ((2560, 128, 128), True), ((640, 128, 128), True), ((2552, 512, 128), True), ((2560, 504, 128), True),
           ((512, 512, 128), True), ((2560, 128, 632), True), ((256, 768, 192), True), ((1 << 61, 1 << 60, 1 << 59), True), ((1 << 62, 512, 128), True)]


@pytest.mark.parametrize("strides, shared", LAYOUTS)
def test_a_written_tensor_has_one_place_for_every_element(lib, strides, shared):
    if not shared and max(strides) < 1 << 40:                # (the table above, counted)
        at = {b * strides[0] + i * strides[1] + h * strides[2] for b in range(3) for i in range(5) for h in range(4)}
        order = sorted(at)
        assert len(at) == 60 and all(y - x >= 128 for x, y in zip(order, order[1:]))
    c = ctypes.byref(cache())
    o = dict(zip(("o_stride_b", "o_stride_n", "o_stride_h"), strides))
    assert lib.bsfa_prefix_attention(c, ctypes.byref(paged(**o, **STOPS)), FAKE, 1, FAKE, None, None) == (-2 if shared else -5), lib.bsfa_last_error()
    q = dict(zip(("q_stride_b", "q_stride_n", "q_stride_h"), strides))           # (what is read may repeat)
    assert lib.bsfa_prefix_attention(c, ctypes.byref(paged(**q, **STOPS)), FAKE, 1, FAKE, None, None) == -5
    for t in ("qo", "ko"):
        if t == "ko" and strides in ((2552, 512, 128), (2560, 504, 128)):
            continue                                         # (enough for two KV heads)
        p = append(interleaved=2, **dict(zip((t + "_stride_b", t + "_stride_n", t + "_stride_h"), strides)))
        assert lib.bsfa_cache_append(c, ctypes.byref(p), FAKE, FAKE, FAKE, OUT, KOUT, None) == -2        # (in the end by `interleaved`)
        assert ((t[0] + "_out").encode() in lib.bsfa_last_error()) == shared


@pytest.mark.parametrize("side", ["k", "v"])
@pytest.mark.parametrize("strides, shared", [((4096, 256, 128), False), ((4096, 128, 2048), False), ((128, 25600, 12800), False), ((128, 128, 128), True),
                                             ((4096, 128, 128), True), ((2048, 128, 128), True), ((4096, 256, 256), True), ((4088, 256, 128), True),
                                             ((4096, 128, 2040), True), ((128, 25600, 12672), True)])
def test_a_written_cache_has_one_place_for_every_element(lib, side, strides, shared):
    """100 pages of 16 tokens of two heads."""
    c = cache(**dict(zip((side + "_stride_page", side + "_stride_n", side + "_stride_h"), strides)))
    code = lib.bsfa_cache_append(ctypes.byref(c), ctypes.byref(append(interleaved=2)), FAKE, FAKE, FAKE, OUT, KOUT, None)
    assert code == -2 and ((side + " cache").encode() in lib.bsfa_last_error()) == shared            # (else what stops it: interleaved)
    assert lib.bsfa_prefix_attention(ctypes.byref(c), ctypes.byref(paged(**STOPS)), FAKE, 1, FAKE, None, None) == -5


@pytest.mark.parametrize("t, other", [("q", "qo"), ("k", "ko")])
def test_in_place_means_the_same_strides(lib, t, other):
    """A result at its input's address, laid out otherwise, would be written where other tokens are still to be read."""
    c, here = ctypes.byref(cache()), [FAKE, FAKE, FAKE, OUT, KOUT]
    here[3 if t == "q" else 4] = FAKE
    for x, strides in enumerate(((5120, 1024, 256), (2560, 128, 640), (2568, 512, 128))):
        p = append(interleaved=2, **dict(zip((other + "_stride_b", other + "_stride_n", other + "_stride_h"), strides)))
        assert lib.bsfa_cache_append(c, ctypes.byref(p), *here, None) == -2 and b"at the place of" in lib.bsfa_last_error()
        assert lib.bsfa_cache_append(c, ctypes.byref(p), FAKE, FAKE, FAKE, OUT, KOUT, None) == -2 and b"interleaved" in lib.bsfa_last_error()
    one = append(batch=1, interleaved=2, **{other + "_stride_b": 8})             # (never used: one element)
    assert lib.bsfa_cache_append(c, ctypes.byref(one), *here, None) == -2 and b"interleaved" in lib.bsfa_last_error()
    assert lib.bsfa_cache_append(c, ctypes.byref(append(interleaved=2)), *here, None) == -2 and b"interleaved" in lib.bsfa_last_error()
