"""lora_kv_append against its definition: the pages' bits where tokens were put and nowhere else, turned keys and queries."""
import numpy as np
import pytest

import kv_plain

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

SEGS = [(0, 1), (7, 1), (8, 1), (0, 3), (5, 8), (0, 40), (61, 7), (64, 64), (31, 100), (10, 0), (0, 16)]


def _run(segs, heads, kv, dim, page, dtype, rope_dim, neighbours, with_q=True, strided=False, layers=2, layer=1):
    from paper_2411_17741_amd import binding as B
    from paper_2411_17741_amd.kv import KvCache

    dt, u = (torch.bfloat16, 8) if dtype == "bf16" else (torch.float32, 4)
    T = sum(n for _c, n in segs)
    cache = KvCache(layers, heads, kv, dim, sum(-(-(c + n) // page) for c, n in segs) + 2, page_tokens=page, max_seqs=len(segs), max_batch_seqs=len(segs),
                    max_batch_tokens=T, dtype=B.LORA_BF16 if dtype == "bf16" else B.LORA_F32)
    try:
        gen = torch.Generator().manual_seed(3)
        host = torch.randn(cache.pages.shape, generator=gen).to(dt)
        cache.pages.copy_(host)
        ids = np.arange(len(segs))
        cache.add(ids)
        cache.extend(ids, [c for c, _n in segs])
        off = np.concatenate([[0], np.cumsum([n for _c, n in segs])]).astype(np.int32)
        batch = cache.batch(ids, off)
        wide = torch.randn(T, heads + 2 * kv + 1, dim, generator=gen).to(dt)
        q, k, v = wide[:, :heads], wide[:, heads : heads + kv], wide[:, heads + kv : heads + 2 * kv]
        pos = np.concatenate([np.arange(c, c + n) for c, n in segs])
        rope = torch.randn(int(pos.max()) + 1, rope_dim, generator=gen) if rope_dim else None
        dev = wide.cuda()
        qd, kd, vd = dev[:, :heads], dev[:, heads : heads + kv], dev[:, heads + kv : heads + 2 * kv]
        if not strided:
            qd, kd, vd = qd.contiguous(), kd.contiguous(), vd.contiguous()
        q_out = torch.full((T, heads + 1, dim), 3.0, dtype=dt, device="cuda") if with_q else None
        cache.append(batch, layer, kd, vd, q=qd if with_q else None, q_out=q_out[:, :heads] if with_q else None, rope=None if rope is None else rope.cuda(), neighbours=neighbours)
        torch.cuda.synchronize()
        f = lambda t: t.float().numpy()  # noqa: E731
        turn = (lambda x: kv_plain.turn(f(x), pos, rope.numpy(), neighbours)) if rope_dim else (lambda x: f(x).astype(np.float64))
        # two products and a sum in fp32, then one rounding
        step = 2.0**-8 if dtype == "bf16" else 2.0**-22
        size = lambda x: (2.0 * np.abs(f(x)).max(-1, keepdims=True) * (float(rope.abs().max()) if rope_dim else 1.0))  # noqa: E731
        want_k, want_pages = turn(k), host.float().numpy().astype(np.float64)
        slack = np.zeros(want_pages.shape)
        for i, (c, n) in enumerate(segs):
            table, rows = cache.pages_of(i), slice(int(off[i]), int(off[i + 1]))
            for h in range(kv if n else 0):
                kv_plain.write(want_pages, table, layer, h, page, dim, u, c, want_k[rows, h], f(v)[rows, h])
                e = np.abs(want_k[rows, h]) * step + 2.0**-22 * size(k)[rows, h]
                e[:, rope_dim:] = 0  # not turned: the same bits
                kv_plain.write(slack, table, layer, h, page, dim, u, c, e, 0.0)
        got = cache.pages.float().cpu().numpy()
        assert (np.abs(got - want_pages) <= slack).all()
        if with_q:
            want_q, got_q = turn(q), q_out.float().cpu().numpy()
            e = np.abs(want_q) * step + 2.0**-22 * size(q)
            e[..., rope_dim:] = 0
            assert (np.abs(got_q[:, :heads] - want_q) <= e).all() and (got_q[:, heads] == 3).all()
            if not strided:  # in place
                cache.append(batch, layer, kd, vd, q=qd, rope=None if rope is None else rope.cuda(), neighbours=neighbours)
                assert torch.equal(qd, q_out[:, :heads])
        assert torch.equal(cache.pages.cpu(), torch.from_numpy(got).to(dt))
    finally:
        cache.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("dim,page,rope_dim", [(64, 32, 64), (128, 64, 128), (128, 128, 48), (256, 64, 256), (64, 256, 16), (64, 64, 0)])
def test_append(dim, page, rope_dim, neighbours, dtype):
    _run(SEGS, 6, 2, dim, page, dtype, rope_dim, neighbours)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_out_of_a_wider_buffer_and_without_queries(dtype):
    _run(SEGS, 5, 5, 128, 64, dtype, 128, False, strided=True)
    _run(SEGS, 8, 1, 64, 32, dtype, 64, True, with_q=False)
    _run([(999, 1)], 1, 1, 64, 64, dtype, 64, False)


@pytest.mark.parametrize("neighbours", [False, True])
def test_append_of_large_batches(neighbours):
    """Tokens times heads beyond the size from which a thread takes more heads, in numbers of heads that its share does not divide."""
    _run([(0, 2900), (5, 77), (64, 1)], 42, 7, 64, 64, "bf16", 64, neighbours, layers=1, layer=0)
    _run([(3, 2990)], 40, 4, 64, 32, "f32", 32, neighbours, strided=True, layers=1, layer=0)


def test_what_is_no_number_stays_where_it_was_put():
    """A NaN or infinity in one token changes that token's bits alone, and a value is stored as it is."""
    from paper_2411_17741_amd.kv import KvCache

    cache = KvCache(1, 2, 1, 64, 4, page_tokens=32, max_seqs=2, max_batch_seqs=2, max_batch_tokens=40)
    try:
        cache.pages.zero_()
        cache.add([0])
        b = cache.batch([0], [0, 20])
        k = torch.ones(20, 1, 64, device="cuda").bfloat16()
        k[7], k[9] = float("nan"), float("-inf")
        cache.append(b, 0, k, k)
        got = cache.pages[0].float().cpu().numpy()[None]
        keys, vals = kv_plain.read(got, [0], 0, 0, 32, 64, 8, 20)
        assert np.array_equal(keys, k[:, 0].float().cpu().numpy(), equal_nan=True) and np.array_equal(vals, keys, equal_nan=True)
    finally:
        cache.close()


def test_refusals():
    from paper_2411_17741_amd import binding as B
    from paper_2411_17741_amd.kv import KvCache

    cache = KvCache(2, 4, 2, 64, 8, page_tokens=32, max_seqs=2, max_batch_seqs=2, max_batch_tokens=40)
    try:
        cache.pages.zero_()
        cache.add([0])
        cache.extend([0], [30])
        b = cache.batch([0], [0, 5])
        k = torch.ones(5, 2, 64, device="cuda").bfloat16()
        q = torch.ones(5, 4, 64, device="cuda").bfloat16()
        rope = torch.ones(35, 64, device="cuda")
        torch.cuda.synchronize()
        kp, qp, rp = k.data_ptr(), q.data_ptr(), rope.data_ptr()
        good = dict(layer=0, k=kp, v=kp, k_stride=128, v_stride=128, q=qp, q_out=qp, q_stride=256, q_out_stride=256, rope=rp, rope_positions=35, rope_dim=64, rope_pairs=0)
        for kw in (dict(layer=2), dict(k=0), dict(v=0), dict(k=kp + 2), dict(k_stride=120), dict(v_stride=132), dict(q_out=0), dict(q=0), dict(q_out_stride=512),
                   dict(q_stride=0), dict(rope_positions=34), dict(rope_dim=80), dict(rope_dim=24), dict(rope_dim=0), dict(rope_pairs=2), dict(rope=rp + 4)):
            a = {**good, **kw}
            assert B.lora_kv_append(cache.handle, b, **a) == B.LORA_E_INVAL, kw
        torch.cuda.synchronize()
        assert not cache.pages.any() and bool((q == 1).all())
        assert B.lora_kv_append(cache.handle, b, **good) == B.LORA_OK
        with pytest.raises(ValueError):
            cache.append(b, 0, k, k, q_out=q)
        with pytest.raises(ValueError):
            cache.append(b, 0, k, k, rope=rope.double())
        with pytest.raises(ValueError):
            cache.append(b, 0, k[:4], k)
        cache.truncate([0], [31])
        assert B.lora_kv_append(cache.handle, b, **good) == B.LORA_E_STATE
        torch.cuda.synchronize()
    finally:
        cache.close()
