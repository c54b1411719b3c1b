"""bsfa_prefix_attention against the 64-bit oracle where a sequence has more than 16 rows to a KV head: what small batches of single
tokens do not reach."""
import pytest

from tests.test_gpu_paged import run_case

pytestmark = pytest.mark.gpu


def _lens(b, most):
    return [(29 * i + 7) % (most + 1) if i != 2 else 0 for i in range(b)]


@pytest.mark.parametrize("s,hq,hkv", [(4, 64, 8), (4, 28, 4), (3, 7, 1), (8, 8, 2), (17, 2, 2)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_17_to_32_own_rows_behind_a_prefix_of_many(s, hq, hkv, d, dtype):
    """Own tokens streamed beside a prefix whose rows share tiles; the last sequences have fewer new tokens, or none."""
    for b, prefix, page in ((2, 61, 16), (5, 200, 32), (7, 1001, 64)):
        run_case(_lens(b, 300), s, hq, hkv, d, page, dtype, "hnd" if b == 5 else "nhd", prefix=prefix)
        run_case(_lens(b, 90), s, hq, hkv, d, page, dtype, "wide" if b == 5 else "nhd", prefix=prefix, q_lens=[max(0, s - x) for x in range(b)], causal=b != 7)


@pytest.mark.parametrize("s", [12, 25, 33, 40])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_many_own_rows_behind_a_prefix(s, d, dtype):
    for b, prefix, page in ((1, 65, 16), (3, 500, 128)):
        run_case(_lens(b, 400), s, 8, 2, d, page, dtype, "hnd" if b == 1 else "nhd", prefix=prefix)
        run_case(_lens(b, 50), s, 4, 1, d, page, dtype, "wide", prefix=prefix, q_lens=[s - 3 * x for x in range(b)], causal=b != 3)


@pytest.mark.parametrize("tiles", [1, 2, 3, 4, 5])
@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (64, "fp16"), (128, "bf16"), (128, "fp16")])
def test_even_and_odd_numbers_of_tiles_of_a_prefix(tiles, d, dtype):
    """Both kernels that multiply a prefix's tiles, with workgroups enough to fill the chip; a prefix that ends inside its last tile and
    one that fills it."""
    for end in (0, 13):
        run_case([5] * 30, 4, 64, 8, d, 16, dtype, prefix=64 * tiles - end, max_cache_len=16)
        run_case([70, 9, 40], 40, 16, 4, d, 64, dtype, prefix=64 * tiles - end)
