"""Batches over the 8-bit cache for its tests (no arithmetic of the method): lengths,
page tables in random order and caches as the oracle fills them."""
import numpy as np
import torch

from oracle import kv8_oracle as O

ORDER = ("Kc", "Vc", "Ks", "Vs")


def tables(r, lengths, slack=2, spare=3, fill=-1):
    """(table [B, most + slack], pages): every sequence's pages from a random order,
    `fill` behind them, `spare` pages no one's."""
    need = [-(-max(0, n) // O.PAGE) for n in lengths]
    pages = sum(need) + spare
    order = r.permutation(pages)
    table = np.full((len(lengths), max(need, default=0) + slack), fill, np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, pages


def rows_of(counts):
    return np.concatenate(([0], np.cumsum(counts))).astype(np.int32)


def heads_of(r, T, H, D, size=1.0):
    """fp16 [T, H, D] with a few large channels."""
    gain = np.where(r.random((H, D)) < 0.05, 8.0, 1.0) * size
    return (r.normal(size=(T, H, D)) * gain).astype(np.float16)


def filled(r, lengths, H, D, dirty=True, slack=2):
    """(cache, table): sequences of so many tokens, appended in one call to pages that
    hold what another program left there (bytes, and NaN as scales)."""
    table, pages = tables(r, lengths, slack)
    cache = O.empty_cache(pages, H, D, 0xA5 if dirty else 128, np.nan if dirty else 0.0)
    cu = rows_of(lengths)
    k, v = heads_of(r, cu[-1], H, D), heads_of(r, cu[-1], H, D, 0.5)
    O.append(cache, k, v, cu, np.array(lengths), table)
    return cache, table


def device(cache):
    return tuple(torch.from_numpy(cache[n]).cuda() for n in ORDER)


def host(tensors):
    return {n: t.cpu().numpy() for n, t in zip(ORDER, tensors)}


def ints(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def held(cache, table, lengths, D):
    """What of a cache's bytes and scales counts: (codes of keys, of values, scales) of
    every sequence's tokens and pages; codes under a scale of NaN, which stand for NaN
    whatever they are, as 0."""
    out = []
    for b, n in enumerate(lengths):
        for col in range(-(-n // O.PAGE)):
            p, m = int(table[b, col]), min(O.PAGE, n - col * O.PAGE)
            s = cache["Ks"][p], cache["Vs"][p]
            out += [np.where(np.isnan(s[0])[:, None, None], 0, cache["Kc"][p, :, :m, :D]),
                    np.where(np.isnan(s[1])[:, None, None], 0, cache["Vc"][p, :, :D, :m]), *s]
    return out


def assert_same_cache(got, want, table, lengths, D):
    for i, (a, b) in enumerate(zip(held(got, table, lengths, D), held(want, table, lengths, D))):
        if a.dtype == np.float32:
            assert np.array_equal(a, b, equal_nan=True), i
        else:
            assert np.array_equal(a, b), i
