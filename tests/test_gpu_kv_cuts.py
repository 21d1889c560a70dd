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
