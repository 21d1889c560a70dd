"""Pages on the GPU: whatever is forked, copied on a write, cut back, freed and moved, every sequence reads the keys and values that were put in
for it; and the books give the pages that the host-only books give."""
import numpy as np
import pytest

import kv_plain

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("dtype,page,dim,layers,kv", [("bf16", 32, 64, 3, 2), ("f32", 64, 128, 1, 1), ("bf16", 128, 256, 2, 3)])
def test_sequences_keep_what_was_put_in_for_them(dtype, page, dim, layers, kv):
    from paper_2411_17741_amd import binding as B
    from paper_2411_17741_amd.kv import KvCache

    dt, u = (torch.bfloat16, 8) if dtype == "bf16" else (torch.float32, 4)
    rng, max_seqs, n_pages = np.random.default_rng(dim + kv), 12, 40
    cache = KvCache(layers, 2 * kv, kv, dim, n_pages, page_tokens=page, max_seqs=max_seqs, max_batch_seqs=max_seqs, max_batch_tokens=2000,
                    dtype=B.LORA_BF16 if dtype == "bf16" else B.LORA_F32)
    cache.pages.fill_(float("nan"))
    cfg = B.make_kv_config(layers, 2 * kv, kv, dim, page, n_pages, max_seqs, max_seqs, 2000, 1 << 20, 2, cache.cfg.dtype, B.LORA_KV_HOST_ONLY)
    rc, books = B.lora_kv_create(cfg, 0, 0, 0, 0)
    held = {}  # sequence -> [layers][2][kv][tokens][dim]
    moved = copied = 0

    def look():
        got = cache.pages.float().cpu().numpy()
        for i, want in held.items():
            table, n = cache.pages_of(i), want.shape[3]
            assert cache.length(i) == n and np.array_equal(table, B.lora_kv_seq_pages(books, i)[1])
            for layer in range(layers):
                for h in range(kv):
                    k, v = kv_plain.read(got, table, layer, h, page, dim, u, n)
                    assert np.array_equal(k, want[layer, 0, h]) and np.array_equal(v, want[layer, 1, h]), (i, layer, h)

    try:
        fresh = 0
        for step in range(160):
            what = rng.choice(["add", "fork", "batch", "batch", "batch", "truncate", "free", "compact"])
            alive = sorted(held)
            if what in ("add", "fork") and len(held) >= max_seqs - 1 or what != "add" and not held:
                continue
            if what == "add":
                cache.add(fresh), B.lora_kv_seq_add(books, fresh)
                held[fresh] = np.zeros((layers, 2, kv, 0, dim), np.float32)
                fresh += 1
            elif what == "fork":
                parent = int(rng.choice(alive))
                n = int(rng.integers(0, held[parent].shape[3] + 1))
                cache.fork(parent, [fresh], n), B.lora_kv_seq_fork(books, parent, [fresh], n)
                held[fresh] = held[parent][:, :, :, :n].copy()
                fresh += 1
            elif what == "batch":
                ids = rng.permutation(alive)[: rng.integers(1, 6)]
                lens = rng.integers(0, 2 * page, len(ids)) if rng.random() < 0.4 else np.ones(len(ids), np.int64)
                off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
                rc, batch = B.lora_kv_batch_create(cache.handle, ids, off, cache._stream(None))
                if rc == B.LORA_E_NOMEM:
                    assert B.lora_kv_seq_extend(books, ids, lens) == B.LORA_E_NOMEM
                    continue
                assert rc == 0 and B.lora_kv_seq_extend(books, ids, lens) == 0
                batch.n_tokens = int(off[-1])
                for layer in range(layers):
                    kvs = torch.randn(2, int(off[-1]), kv, dim, device="cuda").to(dt)
                    cache.append(batch, layer, kvs[0], kvs[1])
                    new = kvs.float().cpu().numpy()
                    for j, i in enumerate(ids.tolist()):
                        if layer == 0:
                            held[i] = np.concatenate([held[i], np.zeros((layers, 2, kv, lens[j], dim), np.float32)], 3)
                        if lens[j]:
                            held[i][layer, :, :, -lens[j] :] = new[:, off[j] : off[j + 1]].transpose(0, 2, 1, 3)
                cache.batch_destroy(batch)
            elif what == "truncate":
                i = int(rng.choice(alive))
                n = int(rng.integers(0, held[i].shape[3] + 1))
                cache.truncate(i, n), B.lora_kv_seq_truncate(books, i, n)
                held[i] = held[i][:, :, :, :n]
            elif what == "free":
                i = int(rng.choice(alive))
                cache.free(i), B.lora_kv_seq_free(books, i)
                del held[i]
            else:
                n = cache.compact()
                assert n == B.lora_kv_compact(books)[1]
                moved += n
                assert cache.stats().pages_end == cache.stats().pages_used
            look()
        copied = cache.stats().pages_copied - moved
        assert moved > 0 and copied > 0
    finally:
        cache.close()
        B.lora_kv_destroy(books)


def test_many_pages_move_in_one_call():
    """More copies than one launch takes, for continuations and together."""
    from paper_2411_17741_amd.kv import KvCache

    n = 300
    cache = KvCache(2, 1, 1, 64, 2 * n + 10, page_tokens=32, max_seqs=n + 1, max_batch_seqs=n, max_batch_tokens=n)
    try:
        cache.pages.zero_()
        cache.add(0)
        cache.extend(0, 50)
        table = cache.pages_of(0)
        cache.pages[table[1]] = torch.randn_like(cache.pages[table[1]])
        ids = np.arange(1, n + 1)
        cache.fork(0, ids)
        batch = cache.batch(ids, np.arange(n + 1))
        torch.cuda.synchronize()
        want = cache.pages[table[1]].clone()
        assert cache.stats().pages_copied == n
        assert all(torch.equal(cache.pages[cache.pages_of(int(i))[1]], want) for i in ids)
        cache.batch_destroy(batch)
        cache.free(ids[0::2])
        cache.pages[int(table[1]) + 1 :: 2] = float("nan")  # what was given back
        torch.cuda.synchronize()
        kept = {int(i): cache.pages[cache.pages_of(int(i))[1]].clone() for i in ids[1::2]}
        moved = cache.compact()
        torch.cuda.synchronize()
        st = cache.stats()
        assert moved > 0 and st.pages_end == st.pages_used == 2 + n // 2
        assert all(torch.equal(cache.pages[cache.pages_of(i)[1]], v) or bool(torch.isnan(v.float()).any()) for i, v in kept.items())
        cache.set_limit(st.pages_end)
        from paper_2411_17741_amd import binding as B
        assert B.lora_kv_seq_extend(cache.handle, [2], [64]) == B.LORA_E_NOMEM
    finally:
        cache.close()


def test_batches_at_their_limits():
    from paper_2411_17741_amd import binding as B
    from paper_2411_17741_amd.kv import KvCache

    cache = KvCache(1, 2, 2, 64, 10, page_tokens=32, max_seqs=4, max_batch_seqs=3, max_batch_tokens=100, max_batch_pages=6, n_batches=2)
    try:
        cache.add([1, 2, 3, 4])
        make = lambda ids, off: B.lora_kv_batch_create(cache.handle, ids, off, 0)  # noqa: E731
        for ids, off, rc in (([1, 2], [0, 1, 102], B.LORA_E_NOMEM), ([1, 2, 3, 4], [0, 1, 2, 3, 4], B.LORA_E_NOMEM), ([1, 1], [0, 1, 2], B.LORA_E_INVAL), ([1, 9], [0, 1, 2], B.LORA_E_NOTFOUND),
                             ([1, 2], [0, 3, 2], B.LORA_E_INVAL), ([1], [1, 2], B.LORA_E_INVAL), ([1], [0, -1], B.LORA_E_INVAL)):
            assert make(ids, off)[0] == rc, (ids, off)
            assert cache.stats().pages_used == 0
        one, two = make([1, 2], [0, 100, 100]), make([1, 3], [0, 28, 60])  # 4 + 0 pages, then 4 + 1
        assert one[0] == two[0] == 0
        assert make([4], [0, 1])[0] == B.LORA_E_NOMEM  # two are alive
        assert B.lora_kv_batch_destroy(cache.handle, one[1]) == 0
        assert make([1, 2], [0, 1, 70])[0] == B.LORA_E_NOMEM  # 5 + 3 pages
        assert make([4, 2], [0, 64, 70])[0] == 0 and cache.stats().pages_used == 8
        assert B.lora_kv_seq_extend(cache.handle, [4, 2], [64, 64]) == B.LORA_E_NOMEM and cache.stats().pages_used == 8
        info = B.lora_kv_batch_info(two[1])[1]
        assert (info.n_tokens, info.n_segments, info.n_pages) == (60, 2, 5)
    finally:
        cache.close()


def test_a_captured_stream_takes_no_batch():
    from paper_2411_17741_amd import binding as B
    from paper_2411_17741_amd.kv import KvCache

    cache = KvCache(1, 2, 2, 64, 10, page_tokens=32, max_seqs=4)
    try:
        cache.add([1])
        cache.extend([1], [5])
        x = torch.zeros(8, device="cuda")
        torch.cuda.synchronize()
        graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        with torch.cuda.graph(graph, stream=stream):
            x.add_(1)
            got = [B.lora_kv_batch_create(cache.handle, [1], [0, 1], stream.cuda_stream)[0], B.lora_kv_seq_extend(cache.handle, [1], [1], stream.cuda_stream)]
        assert got == [B.LORA_E_STATE, B.LORA_E_STATE] and cache.length(1) == 5
        graph.replay()
        torch.cuda.synchronize()
        assert bool((x == 1).all())
    finally:
        cache.close()


def test_pages_are_given_out_behind_the_work_that_reads_them():
    """A request ends while its attention is still to come on one stream; its pages are filled for another request, or put to another use behind a limit, on a second stream."""
    from paper_2411_17741_amd.kv import KvCache

    cache = KvCache(1, 4, 2, 64, 20, page_tokens=32, max_seqs=4, max_batch_seqs=2, max_batch_tokens=8)
    try:
        one, two = torch.cuda.Stream(), torch.cuda.Stream()
        q = torch.randn(1, 4, 64, device="cuda").bfloat16()
        for use in ("extend", "compact"):
            cache.pages.normal_()
            cache.add([0])
            cache.extend([0], [600])
            batch = cache.batch([0], [0, 1])
            want, out = torch.empty_like(q), torch.empty_like(q)
            cache.attend(batch, 0, q, want, 0.1)
            torch.cuda.synchronize()
            with torch.cuda.stream(one):
                torch.cuda._sleep(20_000_000)
            cache.attend(batch, 0, q, out, 0.1, stream=one)
            cache.batch_destroy(batch)
            cache.free([0])
            if use == "extend":
                cache.add([1])
                cache.extend([1], [640], stream=two)
                taken = torch.from_numpy(cache.pages_of(1).astype("int64")).cuda()
                cache.free([1])
            else:
                assert cache.compact(stream=two) == 0
                cache.set_limit(0)
                taken = torch.arange(20, device="cuda")
                cache.set_limit(20)
            with torch.cuda.stream(two):
                two.wait_stream(torch.cuda.default_stream())
                cache.pages[taken] = float("nan")
            torch.cuda.synchronize()
            assert torch.equal(out, want), use
    finally:
        cache.close()


def test_no_call_joins_a_capture_of_another_stream():
    """The latest call's stream is being captured: a call on another cannot wait for it, and is refused before it changes anything."""
    from paper_2411_17741_amd import binding as B
    from paper_2411_17741_amd.kv import KvCache

    cache = KvCache(1, 4, 2, 64, 20, page_tokens=32, max_seqs=4, max_batch_seqs=3, max_batch_tokens=100)
    try:
        cache.pages.normal_()
        q = torch.randn(3, 4, 64, device="cuda").bfloat16()
        out, other_out, k = torch.zeros_like(q), torch.zeros_like(q), torch.randn(3, 2, 64, device="cuda").bfloat16()
        graph, stream, other = torch.cuda.CUDAGraph(), torch.cuda.Stream(), torch.cuda.Stream()
        torch.cuda.synchronize()
        cache.add([0, 1])
        cache.extend([0, 1], [70, 70], stream=stream)
        cache.fork(1, [2])
        cache.free([0])  # (something to move)
        batch = cache.batch([1, 2], [0, 1, 3], stream=stream)
        cache.attend(batch, 0, q, out, 0.1, stream=stream)
        pages, before, row, h, o = [cache.pages_of(i).tolist() for i in (1, 2)], cache.stats(), 4 * 64, cache.handle, other.cuda_stream
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            cache.attend(batch, 0, q, out, 0.1, stream=stream)
            got = [B.lora_kv_batch_create(h, [1], [0, 1], o)[0], B.lora_kv_seq_extend(h, [1, 2], [40, 1], o), B.lora_kv_compact(h, o)[0],
                   B.lora_kv_append(h, batch, 0, k.data_ptr(), k.data_ptr(), 128, 128, stream=o),
                   B.lora_kv_attend(h, batch, 0, q.data_ptr(), row, other_out.data_ptr(), row, 0.1, o)]
        assert got == [B.LORA_E_STATE] * 5
        after = cache.stats()
        assert [cache.pages_of(i).tolist() for i in (1, 2)] == pages and all(getattr(after, n) == getattr(before, n) for n, _t in before._fields_)
        assert cache.length(1) == 71 and cache.length(2) == 72
        # afterwards they go through, and the graph holds its own call alone
        cache.attend(batch, 0, q, other_out, 0.1, stream=other)
        torch.cuda.synchronize()
        want = other_out.clone()
        for _ in range(3):
            out.zero_(), other_out.zero_()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want) and not other_out.any()
        assert B.lora_kv_batch_create(h, [1], [0, 1], o)[0] == B.LORA_OK and cache.compact(stream=other) > 0
    finally:
        cache.close()


def test_a_destroyed_batch_stays_one():
    """Its lists serve other batches later; its handle is refused for good, and does nothing to them."""
    from paper_2411_17741_amd import binding as B
    from paper_2411_17741_amd.kv import KvCache

    make = lambda: KvCache(1, 2, 2, 64, 10, page_tokens=32, max_seqs=4, n_batches=2)  # noqa: E731
    cache, other = make(), make()
    try:
        q = torch.zeros(1, 2, 64, device="cuda").bfloat16()
        k, out, h = torch.zeros_like(q), torch.zeros_like(q), cache.handle
        for c in (cache, other):
            c.add([1])
        first = other.batch([1], [0, 1])
        old = []
        for i in range(12):
            batch = cache.batch([1], [0, 1])
            for b in old[-9:] + [first]:
                assert B.lora_kv_batch_destroy(h, b) == B.LORA_E_INVAL
                assert B.lora_kv_attend(h, b, 0, q.data_ptr(), 128, out.data_ptr(), 128, 0.1) == B.LORA_E_INVAL
                assert B.lora_kv_append(h, b, 0, k.data_ptr(), k.data_ptr(), 128, 128) == B.LORA_E_INVAL
            assert all(B.lora_kv_batch_info(b)[0] == B.LORA_E_INVAL for b in old)
            rc, info = B.lora_kv_batch_info(batch)
            assert rc == 0 and info.n_tokens == 1 and B.lora_kv_batch_info(first)[0] == 0
            cache.append(batch, 0, k, k)
            cache.attend(batch, 0, q, out, 0.1)
            cache.batch_destroy(batch)
            old.append(batch)
        torch.cuda.synchronize()
        assert cache.length(1) == 12
        assert B.lora_kv_batch_info(None)[0] == B.LORA_E_INVAL
        other.batch_destroy(first)
    finally:
        cache.close()
        other.close()
    assert all(B.lora_kv_batch_info(b)[0] == B.LORA_E_INVAL for b in old + [first])


def test_a_batch_of_many_forks_of_a_long_prefix():
    """Its sequences name each page of the prefix: many times as many as there are, all of which are there."""
    from paper_2411_17741_amd import binding as B
    from paper_2411_17741_amd.kv import KvCache

    n, prefix, page = 50, 2048, 32
    cache = KvCache(1, 1, 1, 64, prefix + n + 2, page_tokens=page, max_seqs=n + 1, max_batch_tokens=n)
    try:
        cache.pages.normal_()
        ids = np.arange(1, n + 1)
        cache.add(0)
        cache.extend(0, prefix * page - 5)
        cache.fork(0, ids)
        batch = cache.batch(ids, np.arange(n + 1))
        assert B.lora_kv_batch_info(batch)[1].n_pages == n * prefix
        q = torch.randn(1, 1, 64, device="cuda").bfloat16().expand(n, 1, 64).contiguous()
        k = torch.randn(1, 1, 64, device="cuda").bfloat16().expand(n, 1, 64).contiguous()
        out = torch.empty_like(q)
        cache.append(batch, 0, k, k)
        cache.attend(batch, 0, q, out, 0.125)
        torch.cuda.synchronize()
        host, table, total = cache.pages.float().cpu().numpy(), cache.pages_of(n), prefix * page - 4
        keys, vals = kv_plain.read(host, table, 0, 0, page, 64, 8, total)
        want, mass, _reach = kv_plain.attend(q[:1, 0].float().cpu().numpy(), keys, vals, total - 1, 0.125)
        got = out.float().cpu().numpy()
        # weights of 16 significant bits, one rounding of the output to 8
        assert (np.abs(got[:, 0] - want) <= 2.0**-8 * np.abs(want) + 2.0**-12 * mass).all() and all(np.array_equal(g, got[0]) for g in got)
    finally:
        cache.close()


def test_pages_that_move_are_the_ones_that_were_kept():
    """More moves than one launch takes; every kept page is told apart by its bits, and none of them is a NaN."""
    from paper_2411_17741_amd.kv import KvCache

    n = 600
    cache = KvCache(2, 1, 1, 64, 2 * n + 10, page_tokens=32, max_seqs=n + 1, max_batch_seqs=n, max_batch_tokens=n)
    try:
        ids = np.arange(1, n + 1)
        cache.add(0)
        cache.extend(0, 50)
        cache.fork(0, ids)
        batch = cache.batch(ids, np.arange(n + 1))
        cache.batch_destroy(batch)
        torch.cuda.synchronize()
        cache.pages.copy_(torch.randn(cache.pages.shape, generator=torch.Generator().manual_seed(1)))
        before = cache.pages.clone()
        tables = {int(i): cache.pages_of(int(i)) for i in ids}
        cache.free(ids[0::2])
        cache.pages[torch.as_tensor([int(tables[int(i)][1]) for i in ids[0::2]], device="cuda")] = float("nan")  # what was given back
        torch.cuda.synchronize()
        moved = cache.compact()
        torch.cuda.synchronize()
        st = cache.stats()
        assert moved > 128 and st.pages_end == st.pages_used == 2 + n // 2
        assert not torch.isnan(cache.pages[: st.pages_end]).any()
        for i in ids[1::2].tolist():
            now = cache.pages_of(i)
            assert all(torch.equal(cache.pages[int(a)], before[int(b)]) for a, b in zip(now, tables[i]))
    finally:
        cache.close()
