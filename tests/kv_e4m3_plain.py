"""Pages of 8-bit values and norms of heads by their definitions in 64 bits on the CPU, for the tests of the kernels.  Shares no code with the package;
pages are numpy byte arrays [page][layer][2 * kv_heads * page_tokens * (dim + 1)] in the layout that include/lora_kv.h documents."""
import numpy as np

import kv_plain

U = 16


def meant():
    """The 256 values of 8 bits."""
    code = np.arange(256)
    power, fraction = (code >> 3) & 15, code & 7
    size = np.where(power == 0, fraction * 2.0**-9, (1 + fraction / 8) * 2.0 ** (power - 7.0))
    size[(code & 127) == 127] = np.nan
    return np.where(code > 127, -size, size)


MEANT = meant()


def exponents(x):
    """x [..., dim] -> the smallest e, from -117 to 120, with which no finite value is over 448 * 2^e"""
    top = np.where(np.isfinite(x), np.abs(x), 0.0).max(-1)
    _f, e = np.frexp(top / 448.0)  # top / 448 = f * 2^e, f from 1/2 on (or 0)
    e = np.where(top <= 448.0 * 2.0 ** (e - 1.0), e - 1, e)
    return np.clip(np.where(top == 0, -117, e), -117, 120).astype(np.int64)


def to_bytes(x, e):
    """The nearest of 8 bits of x / 2^e, halves to even; what is infinite or no number is no number."""
    y = np.asarray(x, np.float64) / 2.0 ** np.asarray(e, np.float64)[..., None]
    with np.errstate(invalid="ignore"):
        size = np.abs(y)
        table = MEANT[:127]
        up = np.clip(np.searchsorted(table, size), 1, 126)
        lo, hi = table[up - 1], table[up]
        code = np.where(size - lo < hi - size, up - 1, np.where(size - lo > hi - size, up, np.where(up % 2 == 0, up, up - 1)))
    code = np.where(np.isfinite(y), code, 127)
    return (code | (np.signbit(y) << 7)).astype(np.uint8)


def places(table, page, dim, kv, head, n):
    """Where things of tokens 0 .. n - 1 lie: page numbers [n], bytes of keys [n][dim], of values [n][dim], of their exponents [n] each."""
    where, keys, vals = kv_plain.places(table, page, dim, U, n)
    off, half = np.arange(n) % page, kv * page * dim
    return where, head * page * dim + keys, half + head * page * dim + vals, 2 * half + head * page + off, 2 * half + (kv + head) * page + off


def read(pages, table, layer, head, kv, page, dim, n):
    """(keys, values) of one head, [n][dim] each, as what they stand for"""
    where, keys, vals, ke, ve = places(table, page, dim, kv, head, n)
    flat = pages[:, layer]
    unit = lambda at: 2.0 ** (flat[where, at].astype(np.float64) - 127)[:, None]  # noqa: E731
    return MEANT[flat[where[:, None], keys]] * unit(ke), MEANT[flat[where[:, None], vals]] * unit(ve)


def norm(x, weights, eps):
    """x [n][heads][dim], weights [dim] or [heads][dim]"""
    x = np.asarray(x, np.float64)
    return x / np.sqrt((x * x).mean(-1, keepdims=True) + float(np.float32(eps))) * np.asarray(weights, np.float64)
