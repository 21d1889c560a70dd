"""Pages of 8-bit values, norms and reads: what is refused on the host, without a GPU.  No kernel is launched."""
from types import SimpleNamespace

import numpy as np
import pytest

import kv_e4m3_plain as plain
from paper_2411_17741_amd import binding as B

GOOD = dict(n_layers=2, n_heads=8, n_kv_heads=2, head_dim=128, page_tokens=64, n_pages=10, max_seqs=4, max_batch_seqs=4, max_batch_tokens=64,
            max_batch_pages=40, n_batches=1, dtype=B.LORA_BF16)


def test_pages_take_a_byte_for_each_value_and_one_for_each_token_and_head():
    for dim, page, kv in ((128, 64, 2), (64, 32, 1), (256, 256, 2)):
        cfg = B.make_kv_config(**{**GOOD, "head_dim": dim, "page_tokens": page, "n_kv_heads": kv, "flags": B.LORA_KV_PAGES_E4M3})
        assert B.lora_kv_page_bytes(cfg) == 2 * 2 * kv * page * (dim + 1) and B.lora_kv_work_bytes(cfg) > 0


def test_configs_are_checked():
    for kw in (dict(dtype=B.LORA_F32, flags=B.LORA_KV_PAGES_E4M3), dict(flags=B.LORA_KV_PAGES_E4M3 | 2), dict(flags=8), dict(head_dim=96, flags=B.LORA_KV_PAGES_E4M3)):
        cfg = B.make_kv_config(**{**GOOD, **kw})
        assert B.lora_kv_page_bytes(cfg) == 0 and B.lora_kv_create(cfg, 256, 1 << 40, 256, 1 << 40)[0] == B.LORA_E_INVAL, kw


def test_reads_and_norms_are_checked():
    cfg = B.make_kv_config(**{**GOOD, "flags": B.LORA_KV_PAGES_E4M3 | B.LORA_KV_HOST_ONLY})
    rc, h = B.lora_kv_create(cfg, 0, 0, 0, 0)
    assert rc == B.LORA_OK
    assert B.lora_kv_seq_add(h, [1]) == 0 and B.lora_kv_seq_extend(h, [1], [70]) == 0
    assert B.lora_kv_seq_read(h, [1], [0], [70], 0, 256, 256, 256, 256, 70) == B.LORA_E_STATE  # host only
    assert B.lora_kv_seq_read(None, [1], [0], [70], 0, 256, 256, 256, 256, 70) == B.LORA_E_INVAL
    assert B.lora_kv_seq_read(h, [1], [0], [70], 2, 256, 256, 256, 256, 70) == B.LORA_E_INVAL
    assert B._lib.lora_kv_seq_read(h, -1, None, None, None, 0, 256, 256, 256, 256, 70, None) == B.LORA_E_INVAL
    assert B._lib.lora_kv_seq_read(h, 1, None, None, None, 0, 256, 256, 256, 256, 70, None) == B.LORA_E_INVAL
    with pytest.raises(ValueError):
        B.lora_kv_seq_read(h, [1], [0, 0], [70], 0, 256, 256, 256, 256, 70)
    assert B.lora_kv_append_norm(h, None, 0, 256, 256, 256, 256, k_norm=256) == B.LORA_E_INVAL
    B.lora_kv_destroy(h)


def test_tensors_of_another_gpu_are_refused(monkeypatch):
    torch = pytest.importorskip("torch")
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
    for name in ("lora_kv_append_norm", "lora_kv_seq_read"):
        monkeypatch.setattr(B, name, lambda *a, name=name, **kw: calls.append(name) or 0)
    cache = KvCache.__new__(KvCache)
    cache.handle, cache.device, cache._index = None, torch.device("cuda", 0), 0
    cache.n_heads, cache.n_kv_heads, cache.head_dim, cache.dtype = 4, 2, 64, torch.bfloat16
    batch, stream = SimpleNamespace(n_tokens=3), SimpleNamespace(cuda_stream=0)

    def call(**other):
        on = lambda name: other.get(name, 0)  # noqa: E731
        cache.append(batch, 0, On(0, 3, 2, 64), On(0, 3, 2, 64), q=On(0, 3, 4, 64), q_norm=On(on("q_norm"), 64, dtype=torch.float32),
                     k_norm=On(on("k_norm"), 2, 64, dtype=torch.float32), stream=stream)
        cache.read([5], 0, On(on("k"), 3, 2, 64), On(on("v"), 3, 2, 64), first=[0], n_tokens=[3], stream=stream)

    call()
    assert calls == ["lora_kv_append_norm", "lora_kv_seq_read"]
    for name in ("q_norm", "k_norm", "k", "v"):
        with pytest.raises(ValueError, match="cuda:0"):
            call(**{name: 1})


def test_the_plain_definition_of_8_bits():
    """The oracle against torch's own conversion, and its exponents against their definition by trial."""
    torch = pytest.importorskip("torch")
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(plain.MEANT, want, equal_nan=True)
    rng = np.random.default_rng(0)
    x = rng.normal(size=(300, 40)) * np.exp2(rng.integers(-140, 120, (300, 1)))
    x[0] = 0
    x[1], x[2] = 448.0, 449.0
    e = plain.exponents(x)
    for row, exp in zip(np.abs(x).max(-1), e):
        fits = [k for k in range(-117, 121) if row <= 448 * 2.0**k]
        assert exp == min(fits)
    y = np.clip(x / 2.0 ** e[:, None], -448, 448)
    assert np.array_equal(plain.to_bytes(x, e), torch.from_numpy(y).to(torch.float8_e4m3fn).view(torch.uint8).numpy())
