"""Norms of heads where values, weights and eps are so large or small that products of two of them leave the normal fp32 numbers, while the results do not."""
import numpy as np
import pytest

import kv_e4m3_plain
import kv_plain

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("size,weight,eps", [
    (1e36, 1e-8, 1e-5), (1e30, 1e-14, 1e-5), (1e-15, 1e28, 1e-30),  # the factor of a head times a weight leaves them
    (1e17, 1.0, float(np.finfo(np.float32).max)), (1e10, 1e6, 1e38)])  # the mean of the squares and eps do
def test_results_in_range_of_what_is_not(size, weight, eps, dim, kind):
    from paper_2411_17741_amd import binding as B
    from paper_2411_17741_amd.kv import KvCache

    T, heads, kv = 50, 6, 2
    dt, u, half = (torch.bfloat16, 8, 2.0**-8) if kind == "bf16" else (torch.float32, 4, 2.0**-24)
    cache = KvCache(1, heads, kv, dim, 2, page_tokens=32, max_seqs=1, max_batch_seqs=1, max_batch_tokens=T, dtype=B.LORA_BF16 if kind == "bf16" else B.LORA_F32)
    try:
        gen = torch.Generator().manual_seed(7)
        x = (size * torch.randn(T, heads + kv, dim, generator=gen).clamp(-3, 3)).to(dt)
        w = weight * (1 + 0.5 * torch.rand(dim, generator=gen))
        cache.pages.zero_()
        cache.add(0)
        batch = cache.batch([0], [0, T])
        q, k = x[:, :heads].cuda(), x[:, heads:].cuda()
        cache.append(batch, 0, k, k, q=q, q_norm=w.cuda(), k_norm=w.cuda(), eps=eps)
        want = kv_e4m3_plain.norm(x.double().numpy(), w.double().numpy(), eps)
        # three roundings of a value's products, 14 of the sum, the root and the quotient, and the output's
        bound = 19 * 2.0**-24 * np.abs(want)
        bound = bound + half * (np.abs(want) + bound)
        assert 1e-20 < np.abs(want).max() < 1e30  # of the test's own numbers
        got = q.double().cpu().numpy()
        assert (np.abs(got - want[:, :heads]) <= bound[:, :heads]).all(), float(np.abs(got / want[:, :heads] - 1).max())
        pages = cache.pages.float().cpu().numpy()
        for h in range(kv):
            keys, _v = kv_plain.read(pages, cache.pages_of(0), 0, h, 32, dim, u, T)
            assert (np.abs(keys - want[:, heads + h]) <= bound[:, heads + h]).all()
    finally:
        cache.close()
