"""lora_kv_attend on batches that are cut and worked on in every way there is, against its definition in 64 bits: what one request holds leaves the others
alone, and a token's output does not depend on what is behind the token."""
import math

import numpy as np
import pytest

import kv_plain
from test_gpu_kv_attend import Setup

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def definition(s, scale, layer=0):
    """Setup.want in 64-bit matrix products on the GPU: outputs, sums of weight * |value|, the largest scale * sum |q| |k| of a row."""
    pages, q = s.host.float().numpy(), s.q.double()
    out, mass, reach = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape[:2])
    for i, (c, n) in enumerate(s.segs):
        rows = slice(int(s.offsets[i]), int(s.offsets[i + 1]))
        unseen = torch.arange(c + n, device="cuda") > c + torch.arange(n, device="cuda")[:, None]
        for h in range(s.heads if n else 0):
            k, v = (torch.from_numpy(a).cuda().double() for a in kv_plain.read(pages, s.tables[i], layer, h // (s.heads // s.kv), s.page, s.dim, s.u, c + n))
            x, kt = q[rows, h].cuda(), k.T.contiguous()
            w = torch.softmax((scale * (x @ kt)).masked_fill_(unseen, -math.inf), -1)
            out[rows, h], mass[rows, h] = (w @ v).cpu().numpy(), (w @ v.abs()).cpu().numpy()
            reach[rows, h] = (scale * (x.abs() @ kt.abs())).masked_fill_(unseen, 0).amax(-1).cpu().numpy()
    return out, mass, reach


def check(s, scale=None):
    scale = 1.0 / math.sqrt(s.dim) if scale is None else scale
    got = s.run(scale).float().cpu().numpy()
    out, mass, reach = definition(s, scale)
    over = np.abs(got - out) - s.bound(out, mass, reach)
    assert np.isfinite(got).all() and (over <= 0).all(), (s.segs, np.unravel_index(np.argmax(over), over.shape), float(over.max()))


def check_beside_no_number(s, which, at, kv_head, bad=float("nan")):
    """The key and value of token `at` of segment `which` are no numbers: rows of that segment and key-value head from that token on see them, all others do not."""
    scale = 1.0 / math.sqrt(s.dim)
    out, mass, reach = definition(s, scale)
    a = s.host.float().numpy()
    c, n = s.segs[which]
    k, v = kv_plain.read(a, s.tables[which], 0, kv_head, s.page, s.dim, s.u, c + n)
    k[at], v[at] = bad, bad
    kv_plain.write(a, s.tables[which], 0, kv_head, s.page, s.dim, s.u, 0, k, v)
    s.cache.pages.copy_(torch.from_numpy(a).to(s.dt))
    got, g = s.run(scale).float().cpu().numpy(), s.heads // s.kv
    clean = np.ones(got.shape, bool)
    clean[int(s.offsets[which]) + max(at - c, 0) : int(s.offsets[which + 1]), kv_head * g : (kv_head + 1) * g] = False
    over = np.where(clean, np.abs(got - out) - s.bound(out, mass, reach), 0)
    assert np.isfinite(got[clean]).all() and (over <= 0).all(), (s.segs, np.unravel_index(np.argmax(over), over.shape), float(over.max()))
    assert not np.isfinite(got[~clean]).any()


# Pieces of single tokens come before those of tiles and leave their partial results at no multiple of 32 rows
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("segs,which,at,heads,kv", [([(2500, 1), (2500, 60)], 1, 2530, 6, 2), ([(1700, 60), (3000, 3), (40, 70)], 0, 1701, 5, 1)])
def test_no_number_behind_a_token_of_a_cut_tile_beside_cut_rows(segs, which, at, heads, kv, dim, dtype):
    s = Setup(segs, heads, kv, dim, dtype=dtype, seed=21)
    try:
        check_beside_no_number(s, which, at, kv - 1)
    finally:
        s.close()


def info_of(s):
    from paper_2411_17741_amd import binding as B

    rc, info = B.lora_kv_batch_info(s.batch)
    assert rc == B.LORA_OK
    return info


PLAIN, MANY, PAIRS, TURNS = range(4)
# Each way of working on tiles: whole tiles and cut ones (with `joins`), broken last tiles, cached context, pages of every size, beside single tokens that are cut themselves;
# `which`, `at`: a token whose key and value can be no numbers
WAYS = [
    (TURNS, [(600, 1024)], 128, 16, 128, 32, 0, 0, 900),
    (TURNS, [(0, 2048)], 64, 64, 128, 256, 0, 0, 2047),
    (TURNS, [(611, 1013), (6000, 40)], 128, 16, 128, 64, 2, 1, 6003),
    (TURNS, [(2500, 1), (311, 1700), (6000, 50), (30, 7)], 80, 16, 128, 32, 2, 2, 6011),
    (TURNS, [(1000, 1), (2500, 300), (0, 1500)], 128, 8, 128, 128, 1, 1, 2600),
    (MANY, [(0, 60)] * 30 + [(700, 90)], 32, 32, 128, 64, 0, 30, 731),
    (MANY, [(0, 40)] * 30 + [(3600, 100), (2500, 1)], 32, 32, 128, 32, 2, 30, 3650),
    (PAIRS, [(3, 700), (12, 1), (900, 1), (0, 2)], 8, 4, 64, 32, 1, 0, 400),
    (PAIRS, [(2500, 1), (20, 1000), (0, 33)], 4, 4, 64, 128, 1, 1, 21),
    (PLAIN, [(0, 300), (70, 230), (0, 140)], 40, 40, 64, 64, 0, 1, 150),
    (PLAIN, [(2000, 900), (0, 900)], 6, 2, 128, 64, 2, 0, 2400),
    (PLAIN, [(1500, 300), (40, 50)], 4, 2, 256, 64, 1, 0, 1600),
]


@pytest.mark.parametrize("way,segs,heads,kv,dim,page,joins,which,at", WAYS)
def test_every_way_of_working_on_tiles(way, segs, heads, kv, dim, page, joins, which, at):
    s = Setup(segs, heads, kv, dim, page=page, seed=22, beyond=float("nan"))
    try:
        info = info_of(s)
        assert info.tiles_way == way and info.n_tile_items > 0 and info.n_joins >= joins
        check(s)
        first = s.run(0.1)
        assert torch.equal(s.run(0.1), first)
    finally:
        s.close()


@pytest.mark.parametrize("way,segs,heads,kv,dim,page,joins,which,at", WAYS)
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_no_number_behind_a_token_of_every_way(way, segs, heads, kv, dim, page, joins, which, at, bad):
    s = Setup(segs, heads, kv, dim, page=page, seed=23)
    try:
        assert info_of(s).tiles_way == way
        check_beside_no_number(s, which, at, kv // 2, bad)
    finally:
        s.close()


@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_scores_that_grow_along_prompts_in_turns(sign):
    """The running maximum moves in every stage, or never after the first."""
    s = Setup([(600, 1024)], 128, 16, 128, page=64, seed=24)
    try:
        assert info_of(s).tiles_way == TURNS
        a = s.host.float().numpy()
        for h in range(s.kv):
            k, v = kv_plain.read(a, s.tables[0], 0, h, s.page, s.dim, s.u, 1624)
            kv_plain.write(a, s.tables[0], 0, h, s.page, s.dim, s.u, 0, np.abs(k) * np.linspace(0.01, 4, 1624)[:, None], v)
        s.host = torch.from_numpy(a).to(s.dt)
        s.cache.pages.copy_(s.host)
        s.q = (s.q.float().abs() * sign).to(s.dt)
        check(s)
    finally:
        s.close()


# More short items than blocks are on the machine: a wavefront has one to itself; beside longer ones and tiles, with several tokens, in every length up to the longest short one
SHORT = [
    ([(i % 128, 1) for i in range(130)], 8, 8, 128, 64, 5, 5),
    ([(i % 120, 1 + i % 3) for i in range(80)] + [(300, 1), (0, 50), (2000, 1)], 32, 8, 128, 32, 77, 78),
    ([(100 + i, 1) for i in range(156)] + [(200, 4)] * 5, 16, 4, 64, 64, 156, 202),
    ([(i % 64, 1) for i in range(150)] + [(40, 3)], 4, 4, 256, 32, 150, 41),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("segs,heads,kv,dim,page,which,at", SHORT)
def test_short_items(segs, heads, kv, dim, page, which, at, dtype):
    s = Setup(segs, heads, kv, dim, page=page, dtype=dtype, seed=25, beyond=float("nan"))
    try:
        info = info_of(s)
        assert info.n_short_items * kv > 512 and info.n_row_items - info.n_short_items < 10
        check(s)
        s.host = torch.nan_to_num(s.host)
        check_beside_no_number(s, which, at, kv // 2)
    finally:
        s.close()


@pytest.mark.parametrize("segs", [[(0, 60)] * 30 + [(4000, 128)], [(0, 100)] * 40 + [(3969, 128)], [(0, 60)] * 30 + [(4000, 100), (2000, 1)]])
def test_a_last_piece_that_the_first_rows_of_its_tile_do_not_see(segs):
    """Three tiles on a compute unit, one query head to a key-value head: rows of a tile stand up to 127 tokens apart, its last piece has 32, 1 and 4 tokens."""
    s = Setup(segs, 32, 32, 128, seed=26, beyond=float("nan"))
    try:
        info = info_of(s)
        assert info.tiles_way == MANY and info.n_joins > 0
        check(s)
        s.host = torch.nan_to_num(s.host)
        which = next(i for i, (c, n) in enumerate(segs) if c and n > 1)
        check_beside_no_number(s, which, segs[which][0] + segs[which][1] - 1, 3)
    finally:
        s.close()


@pytest.mark.parametrize("segs", [[(300, 1)], [(900, 1), (40, 2), (0, 1)], [(20, 0)]])
def test_batches_without_tiles_take_no_way_of_theirs(segs):
    """Heads of 64: two groups of wavefronts to a tile are for batches that have tiles."""
    s = Setup(segs, 4, 4, 64, seed=27)
    try:
        info = info_of(s)
        assert info.tiles_way == PLAIN and info.n_tile_items == 0
        if s.T:
            check(s)
    finally:
        s.close()


# Batches whose single tokens, short segments and tiles are worked on and joined in every way
LARGE = [
    ([(5, 1), (300, 1), (0, 1), (40, 5)], 4, 2, 64, 0), ([(2500, 1), (4000, 2), (77, 1)], 8, 2, 128, 2), ([(1300, 1), (600, 3)], 2, 1, 256, 1),
    ([(i % 60, 1) for i in range(140)], 4, 4, 256, 0), ([(0, 70), (10, 200)], 4, 4, 64, 0), ([(2500, 60), (1800, 1)], 6, 2, 128, 2), ([(1500, 90)], 4, 2, 256, 1),
    ([(0, 60)] * 30 + [(1700, 100)], 32, 32, 128, 1), ([(600, 1024)], 128, 16, 128, 0), ([(2500, 1), (311, 1700), (6000, 50)], 80, 16, 128, 2),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", [1e33, 1e36, 2e37, 3e38])
@pytest.mark.parametrize("segs,heads,kv,dim,joins", LARGE)
def test_values_near_the_types_largest(segs, heads, kv, dim, joins, size, dtype):
    """Outputs are means of values: finite where those are, however close to the end of the type's range."""
    s = Setup(segs, heads, kv, dim, dtype=dtype, seed=28)
    try:
        assert info_of(s).n_joins >= joins
        host = s.host.float()
        sign = torch.where(torch.arange(dim) % 3 == 0, -1.0, 1.0).repeat_interleave(s.u).repeat(s.page // s.u)  # the values of a place have one sign: their sums grow
        host[:, :, 1] = (0.1 + 0.9 * torch.rand(host[:, :, 1].shape, generator=torch.Generator().manual_seed(1))) * size * sign
        s.host = host.to(s.dt)
        s.cache.pages.copy_(s.host)
        check(s)
    finally:
        s.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("segs,heads,kv,dim,joins", LARGE[:8])
def test_an_infinite_value_that_a_token_sees(segs, heads, kv, dim, joins, dtype):
    """One value of one token of each segment: that place of the outputs that see it is infinite, all others are as they were."""
    s = Setup(segs, heads, kv, dim, dtype=dtype, seed=29)
    try:
        scale, g = 1.0 / math.sqrt(dim), heads // kv
        out, mass, reach = definition(s, scale)
        a, inf = s.host.float().numpy(), np.zeros(out.shape, bool)
        for i, (c, n) in enumerate(segs):
            at, d, sign = (c + n) * 2 // 3, i % dim, 1 - 2 * (i % 2)
            k, v = kv_plain.read(a, s.tables[i], 0, kv - 1, s.page, dim, s.u, c + n)
            v[at, d] = sign * np.inf
            kv_plain.write(a, s.tables[i], 0, kv - 1, s.page, dim, s.u, 0, k, v)
            rows = slice(int(s.offsets[i]) + max(at - c, 0), int(s.offsets[i + 1]))
            inf[rows, (kv - 1) * g :, d] = True
            out[rows, (kv - 1) * g :, d] = sign * np.inf
        s.cache.pages.copy_(torch.from_numpy(a).to(s.dt))
        got = s.run(scale).float().cpu().numpy()
        assert np.array_equal(got[inf], out[inf])
        over = np.where(inf, 0, np.abs(np.where(inf, 0, got) - np.where(inf, 0, out)) - s.bound(np.where(inf, 0, out), mass, reach))
        assert np.isfinite(got[~inf]).all() and (over <= 0).all()
    finally:
        s.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("segs,heads,kv,dim,joins", LARGE)
def test_rows_all_of_whose_scores_are_minus_infinity(segs, heads, kv, dim, joins, dtype):
    """They have no softmax: no number, as the formula has it.  Rows that see one finite score are as if the others were not there."""
    s = Setup(segs, heads, kv, dim, dtype=dtype, seed=30)
    try:
        s.q, scale, g = s.q.abs() + 0.01, 1.0 / math.sqrt(dim), heads // kv
        a, none = s.host.float().numpy(), np.zeros((s.T, heads), bool)
        for i, (c, n) in enumerate(segs):
            upto = c + n // 2 if n > 1 else c + i % 2  # tokens of -inf: of half of a prompt's tokens, and of every other single token, all that they see
            k, v = kv_plain.read(a, s.tables[i], 0, 0, s.page, dim, s.u, c + n)
            k[:upto] = -np.inf
            kv_plain.write(a, s.tables[i], 0, 0, s.page, dim, s.u, 0, k, v)
            none[int(s.offsets[i]) : int(s.offsets[i]) + max(upto - c, 0), :g] = True
        s.host = torch.from_numpy(a).to(s.dt)
        s.cache.pages.copy_(s.host)
        got = s.run(scale).float().cpu().numpy()
        finite = s.host.clone()
        finite[torch.isneginf(finite)] = -1e4  # a weight of 0 too, and a bound on rounding that is a number
        s.host = finite
        out, mass, _reach = definition(s, scale)
        reach = np.full(none.shape, 6.0 * math.sqrt(dim))
        assert none.any() and np.isnan(got[none]).all()
        over = np.where(none[..., None], 0, np.abs(got - out) - s.bound(out, mass, reach))
        assert np.isfinite(got[~none]).all() and (over <= 0).all()
    finally:
        s.close()
