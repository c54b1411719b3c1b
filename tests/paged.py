"""Inputs and comparisons of the tests of the paged K/V cache."""
import math

import torch

from oracle import paged_oracle

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def half_step(dtype):
    """Largest relative error of one rounding to the type."""
    return torch.finfo(dtype).eps / 2


def pool(n_pages, page, hkv, d, dtype, layout, fill=math.nan):
    """One side of a cache, filled with NaN: what no token was written to must not matter."""
    if layout == "hnd":
        return torch.full((n_pages, hkv, page, d), fill, dtype=dtype).transpose(1, 2)
    if layout == "wide":                                     # slices of a larger tensor: no stride is the smallest possible
        return torch.full((n_pages, page + 3, hkv + 1, d + 8), fill, dtype=dtype)[:, 1:page + 1, 1:, 8:]
    return torch.full((n_pages, page, hkv, d), fill, dtype=dtype)


def filled(lens, page, hkv, d, dtype, layout, seed, spare=2, columns=None, prefix=0):
    """A cache that holds lens[b] tokens of each sequence (and a prefix) in scattered pages and NaN everywhere else:
    k_cache, v_cache, table (unused entries out of range), prefix_table."""
    g = torch.Generator().manual_seed(seed)
    need = [-(-n // page) for n in lens]
    shared = -(-prefix // page)
    ids = torch.randperm(sum(need) + shared + spare, generator=g)
    kc, vc = (pool(len(ids), page, hkv, d, dtype, layout) for _ in "kv")
    table = torch.full((len(lens), columns or max(need + [1]) + 1), 1 << 30, dtype=torch.int32)
    table[:, 1::2] = -7
    at = 0
    prefix_table = ids[:shared].int()
    at = shared
    rows = [(prefix_table, prefix)]
    for b, n in enumerate(need):
        table[b, :n] = ids[at:at + n]
        rows.append((table[b], lens[b]))
        at += n
    for row, n in rows:
        t = torch.arange(n)
        for c in (kc, vc):
            c[row.long()[t // page], t % page] = torch.randn(n, hkv, d, generator=g).to(dtype)
    return kc, vc, table, prefix_table


def check_attention(got, lse, ref, dtype, untouched):
    """Element by element against the oracle.  With u the half step of the type: the result is rounded once, u |o|; each
    probability is rounded once, off by u of itself, which moves the result by at most u times the mean of |v|.  A score is a
    sum of d products in 32 bits, off by (d + 2) 2^-24 of the sum of their sizes at most; its difference to the maximum and the
    base-2 exponential add 2^-22 of the score and 2^-22: e.  A relative error e of every weight moves the result by at most 2 e times
    the mean of |v| (numerator and normaliser), the log-sum-exp by e.  Sums over keys add n 2^-24 in the worst order, for which
    2^-14 is room up to a thousand keys to a lane (longer chains lie far below the worst order)."""
    out, z, spread, score = ref
    d = out.shape[3]
    u = half_step(dtype)
    e = ((d + 2) * 2.0 ** -24 + 2.0 ** -22) * score + 2.0 ** -22 + 2.0 ** -14
    there = ~out.isnan()
    got64 = got.double()
    tol = u * out.abs() + (u + 2 * e[..., None]) * spread * (1 + u) + torch.finfo(dtype).smallest_normal
    bad = there & ~((got64 - out).abs() <= tol)
    assert not bad.any(), "out: %d of %d off, the first at %s: %s instead of %s (tolerance %s)" % (
        bad.sum(), there.sum(), bad.nonzero()[0].tolist(), got64[bad][0].item(), out[bad][0].item(), tol[bad][0].item())
    assert (got[~there] == untouched).all()
    if lse is not None:
        rows = there[..., 0]
        empty = rows & (z == -math.inf)
        assert (lse.double()[empty] == -math.inf).all()
        seen = rows & ~empty
        off = (lse.double() - z).abs()[seen] - e[seen] - 2.0 ** -22 * z.abs()[seen]
        assert (off <= 0).all(), off.max()
        assert (lse[~rows] == untouched).all()


def run_oracle(q, kc, vc, table, lens, **kw):
    return paged_oracle.attend(q, kc, vc, table, lens, **kw)
