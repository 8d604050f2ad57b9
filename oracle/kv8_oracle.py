"""The 8-bit key/value cache on the CPU: its codes and scales step by step as
include/ot.h defines them, and attention over the values that they stand for in
float64 (numpy).  None of the library's code is used.

A cache is a dict of Kc [pages, H, 64, Dp] and Vc [pages, H, Dp, 64] uint8 and Ks, Vs
[pages, H] float32."""
import numpy as np

PAGE = 64


def row_size(D):
    return next(w for w in (64, 96, 128, 192, 256) if w >= D)


def empty_cache(pages, H, D, fill=0, scale=0.0):
    Dp = row_size(D)
    return {"Kc": np.full((pages, H, PAGE, Dp), fill, np.uint8),
            "Vc": np.full((pages, H, Dp, PAGE), fill, np.uint8),
            "Ks": np.full((pages, H), scale, np.float32),
            "Vs": np.full((pages, H), scale, np.float32)}


def new_scale(most, old):
    """(scale, k) for new tokens of largest magnitude `most` (float32) in a page whose
    scale is `old` (None: no earlier token)."""
    most = np.float32(most)
    if old is not None and np.isnan(old) or not np.isfinite(most):
        return np.float32(np.nan), 0
    if old is None or not old > 0:
        return np.float32(most / np.float32(127)), 0
    fits, k = np.float32(np.float32(127.5) * np.float32(old)), 0
    while np.float64(fits) * 2.0 ** k < np.float64(most):
        k += 1
    return np.float32(np.float64(old) * 2.0 ** k), k


def codes(x, s):
    """Codes of float32 x under the scale s (nonzero and finite)."""
    inv = np.float32(np.float32(1) / np.float32(s))
    return np.clip(np.rint(np.float32(x) * inv), -127, 127)


def _append_one(C, S, x, keys, D):
    """x [tokens, D] (fp16) into the places lo.. of one page and head.  C: [64, Dp] or
    [Dp, 64] bytes; returns the scale."""
    lo, rows = x
    most = np.abs(rows.astype(np.float32)).max() if np.isfinite(rows).all() else np.float32(np.inf)
    s, k = new_scale(most, S if lo > 0 else None)
    page = C if keys else C.T
    if k:
        old = page[:lo].astype(np.float64) - 128
        page[:lo] = (np.rint(old * 2.0 ** -k) + 128).astype(np.uint8)
    if np.isfinite(s):
        c = codes(rows.astype(np.float32), s) if s > 0 else np.zeros(rows.shape)
        page[lo:lo + len(rows), :D] = (c + 128).astype(np.uint8)
    return s


def places(cu, start, table, pages, b):
    """(page or -1, first place, first row, rows) of each page that sequence b's rows
    from position start on touch."""
    row, end, pos = int(cu[b]), int(cu[b + 1]), int(start)
    out = []
    while row < end:
        n = min(PAGE - pos % PAGE, end - row)
        col = pos // PAGE
        page = int(table[b, col]) if 0 <= col < table.shape[1] else -1
        out.append((page if 0 <= page < pages else -1, pos % PAGE, row, n))
        row, pos = row + n, pos + n
    return out


def append(cache, k, v, cu, kv_len, table):
    """In place; k, v [T, H, D] fp16."""
    pages, H = cache["Ks"].shape
    for b in range(len(kv_len)):
        start = int(kv_len[b]) - int(cu[b + 1] - cu[b])
        for page, lo, row, n in places(cu, start, table, pages, b):
            if page < 0:
                continue
            for h in range(H):
                for x, C, S, keys in ((k, "Kc", "Ks", True), (v, "Vc", "Vs", False)):
                    cache[S][page, h] = _append_one(cache[C][page, h], cache[S][page, h],
                                                    (lo, x[row:row + n, h]), keys, k.shape[2])
    return cache


def page_values(cache, page, D):
    """float64 keys and values [H, 64, D] of a page."""
    k = (cache["Kc"][page, :, :, :D].astype(np.float64) - 128) * cache["Ks"][page][:, None, None]
    v = (cache["Vc"][page, :, :D].astype(np.float64) - 128) * cache["Vs"][page][:, None, None]
    return k, v.transpose(0, 2, 1)


def read(cache, cu, start, table, T, D):
    """fp16 k, v [T, H, D]; rows of no sequence are NaN."""
    pages, H = cache["Ks"].shape
    out = np.full((2, T, H, D), np.nan, np.float16)
    for b in range(len(start)):
        for page, lo, row, n in places(cu, start[b], table, pages, b):
            if page >= 0:
                for o, C, S, keys in ((out[0], "Kc", "Ks", True), (out[1], "Vc", "Vs", False)):
                    c = cache[C][page] if keys else cache[C][page].transpose(0, 2, 1)
                    c = c[:, lo:lo + n, :D].astype(np.float32) - np.float32(128)
                    with np.errstate(over="ignore"):
                        y = (c * cache[S][page][:, None, None]).astype(np.float16)
                    o[row:row + n] = y.transpose(1, 0, 2)
    return out[0], out[1]


def keys_values(cache, table, b, length, D):
    """float64 keys and values [H, length, D] of sequence b; NaN where it has no page."""
    pages, H = cache["Ks"].shape
    k, v = (np.full((H, length, D), np.nan) for _ in range(2))
    for col in range(-(-length // PAGE)):
        page = int(table[b, col]) if col < table.shape[1] else -1
        if 0 <= page < pages:
            kk, vv = page_values(cache, page, D)
            n = min(PAGE, length - col * PAGE)
            k[:, col * PAGE:col * PAGE + n] = kk[:, :n]
            v[:, col * PAGE:col * PAGE + n] = vv[:, :n]
    return k, v


def visible(n, length, causal, window):
    """Boolean [n, length]: which keys a sequence's rows see."""
    pos = length - n + np.arange(n)[:, None]
    j = np.arange(length)[None, :]
    see = np.ones((n, length), bool)
    if causal:
        see &= j <= pos
    if window:
        see &= j > pos - window
    return see


def attend(cache, q, cu, kv_len, table, scale, causal=True, window=0):
    """(Y, lse, tolerance of Y, tolerance of lse), float64 [T, Hq, D] and [T, Hq]; rows
    of no sequence are NaN, and so are both results of a row that sees a NaN.

    The tolerances, from the kernels' number formats (weights fp16, everything else
    fp32; p are the normalized weights, N the keys, x = scale q.k):
      dx   error of a score: D + 4 fp32 sums over exact products, each a step of 2^-23 of
           at most scale sum |q k|; the factors and the exponent's sums a few steps more
           of |x| and of the exponents (under 64: a scale's logarithm and the reference)
      w    a weight's relative error, dx (twice: against the reference too) + 2^-11 for
           fp16 (half a step) + 2^-21 for exp2
      Y    w sum p |v|  + the weights' sum's error dx |y| + N sums of 2^-23
           + half a step of fp16, and of its smallest number
      lse  dx + N 2^-23 + a few steps of |lse| and of the exponents"""
    T, Hq, D = q.shape
    H = cache["Ks"].shape[1]
    G = Hq // H
    Y, tol = (np.full((T, Hq, D), np.nan) for _ in range(2))
    lse, ltol = (np.full((T, Hq), np.nan) for _ in range(2))
    q = q.astype(np.float64)
    for b in range(len(kv_len)):
        r0, r1, length = int(cu[b]), int(cu[b + 1]), max(0, int(kv_len[b]))
        n = r1 - r0
        if n == 0:
            continue
        k, v = keys_values(cache, table, b, length, D)
        see = visible(n, length, causal, window)
        for g in range(Hq):
            kk, vv, qq = k[g // G], v[g // G], q[r0:r1, g]
            with np.errstate(all="ignore"):
                x = np.where(see, scale * (qq @ kk.T), -np.inf)
                size = np.where(see, abs(scale) * (np.abs(qq) @ np.abs(kk).T), 0.0)
                most = x.max(1, initial=-np.inf)
                safe = np.where(np.isneginf(most), 0.0, most)
                e = np.where(see, np.exp(x - safe[:, None]), 0.0)
                total = e.sum(1)
                p = e / total[:, None]
                y = np.zeros((n, D))
                spread = np.zeros((n, D))
                for i in range(n):
                    y[i] = p[i][see[i]] @ vv[see[i]]
                    spread[i] = p[i][see[i]] @ np.abs(vv[see[i]])
                step = 2.0 ** -23
                dx = ((D + 4) * size.max(1, initial=0.0) + 8 * np.abs(safe) + 8 * 64) * step
                w = 2 * dx + 2.0 ** -11 + 2.0 ** -21
                t = (w + length * step)[:, None] * spread + dx[:, None] * np.abs(y)
                t = t + np.abs(y) * 2.0 ** -11 + 2.0 ** -24
                some = see.any(1)
                Y[r0:r1, g] = np.where(some[:, None], y, 0.0)
                tol[r0:r1, g] = np.where(some[:, None], t, 0.0)
                ls = safe + np.log(total)
                ls = np.where((see & np.isnan(vv).any(1)).any(1), np.nan, ls)
                lse[r0:r1, g] = np.where(some, ls, -np.inf)
                ltol[r0:r1, g] = np.where(some, dx + (length + 8 + 8 * np.abs(ls)) * step, 0.0)
    return Y, lse, tol, ltol
