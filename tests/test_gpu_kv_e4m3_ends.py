"""Attention over 8-bit pages whose values have the largest and the smallest exponents, with keys and scores of ordinary sizes: weights keep their bits beside either."""
import math

import numpy as np
import pytest

import kv_e4m3_plain as plain
import kv_plain
import test_gpu_kv_e4m3 as e4m3
import test_gpu_kv_prefixes as prefixes

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def _values(host, kv, page, dim, exps, most, seed):
    """The values' half of pages [pages][layers][bytes] gets exponents exps[0] .. exps[1] - 1 and codes of at most `most` in size."""
    half, gen = kv * page * dim, torch.Generator().manual_seed(seed)
    x = (torch.randn(*host.shape[:2], half, generator=gen) * 100).clamp(-most, most)
    host[..., half : 2 * half] = x.to(torch.float8_e4m3fn).view(torch.uint8)
    host[..., 2 * half + kv * page :] = torch.randint(*exps, (*host.shape[:2], kv * page), generator=gen, dtype=torch.uint8)


def _compare(got, q, k, v, c, scale, few, lost=0.0):
    """One head of a segment, rows q [n][dim] behind c cached tokens; few: its weights have 16 bits; lost: what a value may be off by because it is too small"""
    dim, n = q.shape[1], len(q)
    want, mass, reach = kv_plain.attend(q, k, v, c, scale)
    # a score is off by dim products' roundings, sums over the tokens by two roundings a step, every weight by 2^-16 or 2^-8 of itself, and the output by half a step
    bound = mass * ((2 * dim + 8) * 2.0**-24 * reach[..., None] + (c + n + 32) * 2.0**-23 + (2.0**-16 if few else 2.0**-8)) + lost
    bound = bound + 2.0**-8 * (np.abs(want) + bound)
    over = np.abs(got - want) - bound
    assert np.isfinite(got).all() and (over <= 0).all(), (c, n, float((np.abs(got - want) / bound).max()))


# the values' exponents, and codes up to which they are finite in bf16: the largest and the smallest that append stores, and what a caller may put there
ENDS = [((244, 248), 240.0), ((10, 14), 448.0), ((253, 255), 0.9375), ((1, 5), 448.0)]


@pytest.mark.parametrize("exps,most", ENDS)
@pytest.mark.parametrize("segs,heads,kv,dim,page", [
    ([(90, 1), (700, 1), (33, 2), (0, 1)], 4, 2, 64, 32), ([(9001, 1)], 8, 1, 128, 64), ([(300, 1)] * 3, 6, 2, 256, 64), ([(20 + i, 1) for i in range(200)], 8, 8, 64, 64),
    ([(90, 60), (0, 150), (40, 1)], 4, 2, 128, 64), ([(4000, 40)], 8, 2, 64, 128)])
def test_values_of_the_largest_and_smallest_exponents(segs, heads, kv, dim, page, exps, most):
    s = e4m3.Setup(segs, heads, kv, dim, page=page, seed=41)
    try:
        _values(s.host, kv, page, dim, exps, most, 42)
        s.cache.pages.copy_(s.host)
        scale, out = 1.0 / math.sqrt(dim), torch.full(s.q.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
        s.cache.attend(s.batch, 0, s.q.cuda(), out, scale)
        got, q, pages = out.double().cpu().numpy(), s.q.double().numpy(), s.host.numpy()
        for i, (c, n) in enumerate(segs):
            rows = slice(int(s.offsets[i]), int(s.offsets[i + 1]))
            for h in range(0, heads, 3):
                k, v = plain.read(pages, s.tables[i], 0, h // (heads // kv), kv, page, dim, c + n)
                _compare(got[rows, h], q[rows, h], k, v, c, scale, n * (heads // kv) <= 16, 2.0**-126 if exps[0] < 10 else 0.0)
    finally:
        s.close()


@pytest.mark.parametrize("exps,most", ENDS)
@pytest.mark.parametrize("forks,tokens", [(3, 700), (40, 700), (4, 9000)])
def test_the_same_behind_shared_prefixes(forks, tokens, exps, most):
    t = prefixes.Tree(prefixes.forks(forks, tokens, lambda i: 7 * (i % 9)), 4, 2, 64, kind="e4m3", seed=43)
    try:
        assert t.info().n_segments == forks
        _values(t.host, 2, 64, 64, exps, most, 44)
        t.cache.pages.copy_(t.host)
        got, q = t.run().double().cpu().numpy(), t.q.double().numpy()
        for j, i in enumerate(t.ids):
            for h in range(4):
                k, v = t.keys_values(i, 0, h // 2, t.ctx[j] + 1)
                _compare(got[j : j + 1, h], q[j : j + 1, h], k, v, t.ctx[j], 1.0 / 8, True, 2.0**-126 if exps[0] < 10 else 0.0)
    finally:
        t.close()


@pytest.mark.parametrize("exps,most", ENDS)
@pytest.mark.parametrize("segs", [[(90, 1)], [(1000, 3)], [(3000, 1)], [(40, 60)], [(5000, 40)]])
def test_rows_beside_one_that_has_no_numbers(segs, exps, most):
    """Rows that are worked out again because a row beside them has no outputs keep their bits."""
    s = e4m3.Setup(segs, 4, 1, 64, seed=45)
    try:
        _values(s.host, 1, 64, 64, exps, most, 46)
        s.cache.pages.copy_(s.host)
        s.q[0, 0, 5] = float("nan")
        out = torch.full(s.q.shape, 0.0, dtype=torch.bfloat16, device="cuda")
        s.cache.attend(s.batch, 0, s.q.cuda(), out, 1.0 / 8)
        got, q = out.double().cpu().numpy(), s.q.double().numpy()
        (c, n), k_v = segs[0], plain.read(s.host.numpy(), s.tables[0], 0, 0, 1, 64, 64, sum(segs[0]))
        assert np.isnan(got[0, 0]).all()
        for h in (1, 3):
            _compare(got[:, h], q[:, h], *k_v, c, 1.0 / 8, n * 4 <= 16, 2.0**-126 if exps[0] < 10 else 0.0)
    finally:
        s.close()
