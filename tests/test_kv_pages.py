"""Sequences and pages of the key-value cache against plain books: a dict of lists, the free pages in a set.  Host only, no kernel is launched."""
import numpy as np
import pytest

from paper_2411_17741_amd import binding as B


class Books:
    """The dumbest model: a sequence is its length and its list of pages; a page's holders are counted by looking."""

    def __init__(self, page, n_pages, max_seqs):
        self.page, self.n_pages, self.max_seqs, self.limit = page, n_pages, max_seqs, n_pages
        self.seqs, self.copied = {}, 0

    def holders(self, p):
        return sum(pages.count(p) for _n, pages in self.seqs.values())

    def free(self):
        used = {p for _n, pages in self.seqs.values() for p in pages}
        return [p for p in range(self.limit) if p not in used]

    def add(self, ids):
        if len(self.seqs) + len(ids) > self.max_seqs:
            return B.LORA_E_NOMEM
        if any(i in self.seqs for i in ids) or len(set(ids)) < len(ids):
            return B.LORA_E_STATE
        self.seqs.update({i: (0, []) for i in ids})
        return 0

    def fork(self, parent, ids, n):
        if parent not in self.seqs:
            return B.LORA_E_NOTFOUND
        length, pages = self.seqs[parent]
        if n > length:
            return B.LORA_E_INVAL
        n = length if n < 0 else n
        rc = self.add(ids)
        if rc == 0:
            self.seqs.update({i: (n, pages[: -(-n // self.page)]) for i in ids})
        return rc

    def extend(self, ids, counts):
        before, copied = {k: (n, list(p)) for k, (n, p) in self.seqs.items()}, self.copied
        done = set()
        for i, c in zip(ids, counts):
            if i not in self.seqs or i in done or c < 0:
                self.seqs, self.copied = before, copied
                return B.LORA_E_NOTFOUND if i not in before else B.LORA_E_INVAL
            done.add(i)
        for i, c in zip(ids, counts):
            n, pages = self.seqs[i]
            pages = list(pages)
            want = -(-(n + c) // self.page)
            take = []
            if c and n % self.page and self.holders(pages[-1]) > 1:
                pages.pop()
                take.append(None)
                self.copied += 1
            fresh = self.free()[: want - len(pages)]
            if len(fresh) < want - len(pages):
                self.seqs, self.copied = before, copied
                return B.LORA_E_NOMEM
            # the copy is taken before the old page is let go
            self.seqs[i] = (n + c, pages + fresh)
        return 0

    def truncate(self, ids, counts):
        for k, (i, c) in enumerate(zip(ids, counts)):
            if i not in self.seqs:
                return B.LORA_E_NOTFOUND
            if i in ids[:k] or not 0 <= c <= self.seqs[i][0]:
                return B.LORA_E_INVAL
        for i, c in zip(ids, counts):
            self.seqs[i] = (c, self.seqs[i][1][: -(-c // self.page)])
        return 0

    def release(self, ids):
        for k, i in enumerate(ids):
            if i not in self.seqs:
                return B.LORA_E_NOTFOUND
            if i in ids[:k]:
                return B.LORA_E_INVAL
        for i in ids:
            del self.seqs[i]
        return 0

    def compact(self):
        used = sorted({p for _n, pages in self.seqs.values() for p in pages})
        holes = [p for p in range(len(used)) if p not in used]
        to = dict(zip([p for p in used if p >= len(used)], holes))
        self.seqs = {i: (n, [to.get(p, p) for p in pages]) for i, (n, pages) in self.seqs.items()}
        self.copied += len(to)
        return len(to)

    def set_limit(self, limit):
        if not 0 <= limit <= self.n_pages:
            return B.LORA_E_INVAL
        if any(p >= limit for _n, pages in self.seqs.values() for p in pages):
            return B.LORA_E_STATE
        self.limit = limit
        return 0


def _cache(page=32, n_pages=70, max_seqs=9, **kw):
    cfg = B.make_kv_config(kw.get("layers", 2), kw.get("heads", 4), kw.get("kv", 2), kw.get("dim", 64), page, n_pages, max_seqs, max_seqs, 4096, 4096,
                           2, B.LORA_BF16, B.LORA_KV_HOST_ONLY)
    rc, h = B.lora_kv_create(cfg, 0, 0, 0, 0)
    assert rc == B.LORA_OK
    return h


def _same(h, books):
    for i, (n, pages) in books.seqs.items():
        rc, info = B.lora_kv_seq_info(h, i)
        assert rc == 0 and (info.n_tokens, info.n_pages, info.n_shared) == (n, len(pages), sum(books.holders(p) > 1 for p in pages))
        assert B.lora_kv_seq_pages(h, i)[1].tolist() == pages
    rc, st = B.lora_kv_stats(h)
    used = {p for _n, pages in books.seqs.values() for p in pages}
    assert (st.limit, st.pages_used, st.pages_free, st.seqs, st.pages_copied) == (books.limit, len(used), len(books.free()), len(books.seqs), books.copied)
    assert st.pages_shared == sum(books.holders(p) > 1 for p in used) and st.pages_end == max(used, default=-1) + 1


@pytest.mark.parametrize("seed", range(8))
@pytest.mark.parametrize("page,n_pages,max_seqs", [(32, 70, 9), (64, 13, 5), (32, 300, 40)])
def test_books_agree(page, n_pages, max_seqs, seed):
    rng = np.random.default_rng(seed)
    h, books = _cache(page, n_pages, max_seqs), Books(page, n_pages, max_seqs)
    some = lambda: [int(v) for v in rng.integers(0, 2 * max_seqs, rng.integers(1, 4))]  # noqa: E731
    alive = lambda: [int(v) for v in rng.choice(sorted(books.seqs), min(len(books.seqs), int(rng.integers(1, 4))), replace=bool(rng.random() < 0.1))] if books.seqs else some()  # noqa: E731
    refused = 0
    for _ in range(300):
        what = rng.choice(["add", "fork", "extend", "extend", "extend", "truncate", "free", "compact", "limit"])
        if what == "add":
            ids = some()
            got, want = B.lora_kv_seq_add(h, ids), books.add(ids)
        elif what == "fork":
            parent, ids = alive()[0], some()
            n = int(rng.integers(-1, 1 + (books.seqs[parent][0] if parent in books.seqs else 5) * 5 // 4 + 1))
            got, want = B.lora_kv_seq_fork(h, parent, ids, n), books.fork(parent, ids, n)
        elif what == "extend":
            ids = alive() if rng.random() < 0.9 else some()
            counts = [int(v) for v in rng.integers(-1 if rng.random() < 0.05 else 0, 3 * page, len(ids))]
            got, want = B.lora_kv_seq_extend(h, ids, counts), books.extend(ids, counts)
        elif what == "truncate":
            ids = alive()
            counts = [int(rng.integers(0, 2 + (books.seqs[i][0] if i in books.seqs else 3))) for i in ids]
            got, want = B.lora_kv_seq_truncate(h, ids, counts), books.truncate(ids, counts)
        elif what == "free":
            ids = alive()[:2]
            got, want = B.lora_kv_seq_free(h, ids), books.release(ids)
        elif what == "compact":
            got, want = B.lora_kv_compact(h), (0, books.compact())
        else:
            limit = int(rng.integers(-1, n_pages + 2)) if rng.random() < 0.5 else n_pages
            got, want = B.lora_kv_set_limit(h, limit), books.set_limit(limit)
        assert got == want, (what, got, want)
        refused += what != "compact" and want != 0
        _same(h, books)
    assert refused > 5
    assert B.lora_kv_destroy(h) == 0


def test_a_shared_page_is_copied_for_all_but_its_last_holder():
    h = _cache()
    assert B.lora_kv_seq_add(h, [1]) == 0 and B.lora_kv_seq_extend(h, [1], [40]) == 0
    assert B.lora_kv_seq_fork(h, 1, [2, 3]) == 0
    assert B.lora_kv_seq_extend(h, [1, 2, 3], [1, 1, 1]) == 0
    rows = [B.lora_kv_seq_pages(h, i)[1].tolist() for i in (1, 2, 3)]
    assert rows == [[0, 2], [0, 3], [0, 1]] and B.lora_kv_stats(h)[1].pages_copied == 2
    # full pages are never written again
    assert B.lora_kv_seq_fork(h, 1, [4], 32) == 0 and B.lora_kv_seq_extend(h, [4], [1]) == 0
    assert B.lora_kv_seq_pages(h, 4)[1].tolist() == [0, 4] and B.lora_kv_stats(h)[1].pages_copied == 2
    B.lora_kv_destroy(h)


def test_configs_are_checked():
    good = dict(n_layers=2, n_heads=8, n_kv_heads=2, head_dim=128, page_tokens=64, n_pages=10, max_seqs=4, max_batch_seqs=4, max_batch_tokens=64,
                max_batch_pages=40, n_batches=1, dtype=B.LORA_BF16)
    cfg = B.make_kv_config(**good)
    page = 2 * 2 * 2 * 64 * 128 * 2
    assert B.lora_kv_page_bytes(cfg) == page and B.lora_kv_pages_bytes(cfg) == 10 * page and B.lora_kv_work_bytes(cfg) > 0
    assert B.lora_kv_page_bytes(B.make_kv_config(**{**good, "dtype": B.LORA_F32})) == 2 * page
    for kw in (dict(n_layers=0), dict(n_heads=0), dict(n_kv_heads=0), dict(n_kv_heads=3), dict(n_heads=1), dict(head_dim=96), dict(head_dim=0), dict(page_tokens=16),
               dict(page_tokens=48), dict(page_tokens=512), dict(n_pages=0), dict(max_seqs=0), dict(max_batch_seqs=0), dict(max_batch_tokens=-1), dict(max_batch_pages=0),
               dict(n_batches=0), dict(dtype=2), dict(flags=2)):
        bad = B.make_kv_config(**{**good, **kw})
        assert B.lora_kv_page_bytes(bad) == 0 and B.lora_kv_work_bytes(bad) == 0
        assert B.lora_kv_create(bad, 256, 1 << 40, 256, 1 << 40)[0] == B.LORA_E_INVAL, kw
    # device memory that is missing, too small or not aligned
    n, w = B.lora_kv_pages_bytes(cfg), B.lora_kv_work_bytes(cfg)
    for args, rc in (((0, n, 256, w), B.LORA_E_INVAL), ((256, n, 0, w), B.LORA_E_INVAL), ((128, n, 256, w), B.LORA_E_INVAL), ((256, n, 16, w), B.LORA_E_INVAL),
                     ((256, n - 1, 256, w), B.LORA_E_NOMEM), ((256, n, 256, w - 1), B.LORA_E_NOMEM)):
        assert B.lora_kv_create(cfg, *args)[0] == rc, args


def test_handles_and_lists_are_checked():
    h = _cache()
    assert B.lora_kv_seq_add(None, [1]) == B.LORA_E_INVAL and B.lora_kv_destroy(None) == B.LORA_E_INVAL
    assert B._lib.lora_kv_seq_add(h, 1, None) == B.LORA_E_INVAL and B._lib.lora_kv_seq_add(h, -1, None) == B.LORA_E_INVAL
    assert B.lora_kv_seq_add(h, []) == 0
    assert B.lora_kv_seq_info(h, 5)[0] == B.LORA_E_NOTFOUND and B.lora_kv_seq_pages(h, 5)[0] == B.LORA_E_NOTFOUND
    assert B.lora_kv_seq_add(h, [5]) == 0
    assert B.lora_kv_seq_extend(h, [5], [B.LORA_KV_MAX_TOKENS]) == B.LORA_E_NOMEM and B.lora_kv_seq_extend(h, [5], [2**31 - 1]) == B.LORA_E_NOMEM
    assert B.lora_kv_batch_create(h, [5], [0, 1])[0] == B.LORA_E_STATE  # host only: no device to run a batch on
    assert B.lora_kv_batch_create(h, [5], [1, 1])[0] == B.LORA_E_INVAL and B.lora_kv_batch_create(None, [5], [0, 1])[0] == B.LORA_E_INVAL
    with pytest.raises(ValueError):
        B.lora_kv_seq_extend(h, [5], [1, 2])
    with pytest.raises(ValueError):
        B.lora_kv_batch_create(h, [5], [0])
    B.lora_kv_destroy(h)


def test_tensors_of_another_gpu_are_refused(monkeypatch):
    """Keys, values, queries, outputs and tables of angles have to lie on the cache's device: any other's address means nothing there.  Host only: tensors that
    say where they lie, and calls that say that they were made."""
    torch = pytest.importorskip("torch")
    from types import SimpleNamespace

    from paper_2411_17741_amd.kv import KvCache

    class On:
        def __init__(self, device, *shape, dtype=torch.bfloat16):
            t = torch.empty(shape, dtype=dtype)
            self.shape, self.dtype, self.is_cuda, self.device = t.shape, dtype, True, torch.device("cuda", device)
            self.stride, self.dim, self.is_contiguous = t.stride, t.dim, t.is_contiguous

        def get_device(self):
            return self.device.index

        def data_ptr(self):
            return 4096

    calls = []
    for name in ("lora_kv_append", "lora_kv_attend"):
        monkeypatch.setattr(B, name, lambda *a, name=name, **kw: calls.append(name) or 0)
    cache = KvCache.__new__(KvCache)
    cache.handle, cache.device, cache._index = None, torch.device("cuda", 0), 0
    cache.n_heads, cache.n_kv_heads, cache.head_dim, cache.dtype = 4, 2, 64, torch.bfloat16
    batch, stream = SimpleNamespace(n_tokens=3), SimpleNamespace(cuda_stream=0)

    def call(**other):
        on = lambda name: other.get(name, 0)  # noqa: E731
        cache.append(batch, 0, On(on("k"), 3, 2, 64), On(on("v"), 3, 2, 64), q=On(on("q"), 3, 4, 64), q_out=On(on("q_out"), 3, 4, 64), rope=On(on("rope"), 9, 64, dtype=torch.float32), stream=stream)
        cache.attend(batch, 0, On(on("aq"), 3, 4, 64), On(on("out"), 3, 4, 64), 0.1, stream=stream)

    call()
    assert calls == ["lora_kv_append", "lora_kv_attend"]
    for name in ("k", "v", "q", "q_out", "rope", "aq", "out"):
        with pytest.raises(ValueError, match="cuda:0"):
            call(**{name: 1})
    cache.handle = None
