"""The paged key-value cache's operators by their definitions in 64 bits on the CPU, for the tests of the kernels.
Shares no code with the package; pages are numpy arrays [page][layer][2][kv_head][page_tokens * dim] in the layout that
include/lora_kv.h documents."""
import numpy as np


def places(table, page_tokens, dim, u, n):
    """Where value d of tokens 0 .. n-1 of a sequence lies: page numbers [n], offsets of the keys [n][dim], of the values [n][dim]."""
    t, d = np.arange(n), np.arange(dim)
    off = t % page_tokens
    keys = ((d // u)[None, :] * page_tokens + off[:, None]) * u + d % u
    vals = ((off // u)[:, None] * dim + d[None, :]) * u + (off % u)[:, None]
    return np.asarray(table)[t // page_tokens], keys, vals


def read(pages, table, layer, kv_head, page_tokens, dim, u, n):
    """(keys, values) of one head, [n][dim] each."""
    where, keys, vals = places(table, page_tokens, dim, u, n)
    return (pages[where[:, None], layer, 0, kv_head, keys], pages[where[:, None], layer, 1, kv_head, vals])


def write(pages, table, layer, kv_head, page_tokens, dim, u, first, k, v):
    """Keys and values [m][dim] of tokens first .. first + m - 1."""
    m = len(k)
    where, keys, vals = (a[first:] for a in places(table, page_tokens, dim, u, first + m))
    pages[where[:, None], layer, 0, kv_head, keys] = k
    pages[where[:, None], layer, 1, kv_head, vals] = v


def attend(q, k, v, ctx, scale):
    """Rows q [n][dim] at positions ctx .. ctx + n - 1 over k, v [ctx + n][dim].
    -> outputs, sum of weight * |value| (what relative errors of weights are measured by), the largest scale * sum |q| |k| of a row."""
    out, mass, reach = np.zeros(q.shape), np.zeros(q.shape), np.zeros(len(q))
    q, k, v = (np.asarray(a, np.float64) for a in (q, k, v))
    for i in range(len(q)):
        kk, vv = k[: ctx + i + 1], v[: ctx + i + 1]
        s = scale * (kk @ q[i])
        w = np.exp(s - s.max())
        w /= w.sum()
        out[i], mass[i], reach[i] = w @ vv, w @ np.abs(vv), scale * (np.abs(kk) @ np.abs(q[i])).max()
    return out, mass, reach


def turn(x, pos, rope, neighbours):
    """x [n][heads][dim] at positions pos [n]; rope [positions][R]."""
    x = np.array(x, np.float64)
    r = rope.shape[1]
    c, s = rope[pos][:, None, : r // 2].astype(np.float64), rope[pos][:, None, r // 2 :].astype(np.float64)
    j = np.arange(r // 2)
    lo, hi = (2 * j, 2 * j + 1) if neighbours else (j, j + r // 2)
    a, b = x[..., lo].copy(), x[..., hi].copy()
    x[..., lo], x[..., hi] = a * c - b * s, b * c + a * s
    return x
