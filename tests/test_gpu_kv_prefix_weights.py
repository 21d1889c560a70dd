"""The weights of segments with up to 16 rows keep 16 bits in bf16, whether their tokens are shared or not (lora_kv.h: lora_kv_attend,
lora_kv_batch_create_shared)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

SCALE = 0.69120 / 1771.5  # scores of -1772 and -1771 have weights of 0.50083 and 0.50102: on both sides of the middle, 0.50098, of two neighbouring bf16 numbers


def _cache(heads, kv, dim, tokens, forks, page, e4m3):
    """A request of `tokens` tokens and forks of it: every 32nd key is 0, the others have scores -1772 and -1771 in turn with queries that begin 1, 1, 1; their values
    are 1 and -1 and nearly cancel.  All numbers are exact in bf16 and in 8 bits."""
    from paper_2411_17741_amd.kv import KvCache

    step = 4096
    cache = KvCache(1, heads, kv, dim, -(-tokens // page) + forks + 4, page_tokens=page, max_seqs=forks + 2, max_batch_seqs=forks + 2, max_batch_tokens=step, e4m3=e4m3)
    cache.add(0)
    t = torch.arange(tokens, device="cuda")
    k = torch.zeros(tokens, kv, dim, device="cuda")
    v = torch.zeros(tokens, kv, dim, device="cuda")
    some = t % 32 != 0
    k[some, :, 0], k[some, :, 1] = -1664, -104
    k[:, :, 2] = torch.where(some, torch.where(t % 2 == 0, -4.0, -3.0), 0.0)[:, None]
    v[:] = torch.where(some, torch.where(t % 2 == 0, 1.0, -1.0), 0.0)[:, None, None]
    k, v = k.bfloat16(), v.bfloat16()
    for at in range(0, tokens, step):
        n = min(step, tokens - at)
        b = cache.batch([0], [0, n])
        cache.append(b, 0, k[at : at + n], v[at : at + n])
        cache.batch_destroy(b)
    cache.fork(0, np.arange(1, forks + 1))
    return cache


def _want(tokens):
    """of the prefix and a token of key and value 0 behind it"""
    t = np.arange(tokens)
    s = np.where(t % 32 == 0, 0.0, np.where(t % 2 == 0, -1772.0, -1771.0)) * float(np.float32(SCALE))
    v = np.where(t % 32 == 0, 0.0, np.where(t % 2 == 0, 1.0, -1.0))
    p = np.exp(s)
    return (p * v).sum() / (p.sum() + 1)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize(
    "heads,kv,dim,tokens,forks,page",
    [
        (4, 1, 128, 640, 20, 64),
        (4, 4, 64, 640, 20, 32),
        (4, 2, 256, 640, 20, 64),
        (8, 1, 64, 1920, 150, 128),
        (32, 8, 128, 1280, 130, 64),
        (32, 8, 128, 40000, 64, 64),  # tiles of 256 rows
        (16, 16, 256, 640, 300, 32),  # tiles and rows in launches of their own
        (16, 1, 64, 64, 1, 64),       # as many rows as a row item has
    ],
)
def test_weights_of_few_rows_keep_their_bits(heads, kv, dim, tokens, forks, page, e4m3):
    from paper_2411_17741_amd import binding as B

    cache = _cache(heads, kv, dim, tokens, forks, page, e4m3)
    try:
        q = torch.zeros(forks, heads, dim, device="cuda", dtype=torch.bfloat16)
        q[:, :, :3] = 1
        none = torch.zeros(forks, kv, dim, device="cuda", dtype=torch.bfloat16)
        want = _want(tokens)
        for shared in (False, 64):
            ids = np.arange(1, forks + 1)
            batch = cache.batch(ids, np.arange(forks + 1), shared=shared)
            info, prefixes = B.lora_kv_batch_info(batch)[1], B.lora_kv_batch_prefixes(batch)[1]
            assert prefixes.n_prefixes == int(bool(shared) and forks > 1)
            assert info.n_tile_items == 0 or shared
            if shared and forks > 1:
                assert prefixes.n_tile_items and prefixes.n_tokens == tokens
                assert (info.tiles_way == B.LORA_KV_TILES_TURNS) == (tokens == 40000)
            cache.append(batch, 0, none, none)
            out = torch.full_like(q, float("nan"))
            cache.attend(batch, 0, q, out, SCALE)
            torch.cuda.synchronize()
            # Relative to the sum of the weights: weights in two bf16 parts are off by 2^-16, in fp32 (scores of 1.0 in units of log2, exponentials of an ulp) by 2^-21; partial sums, of
            # terms that cancel two by two, by 2^-24 of a few terms.  The sum of weights is off by 2^-24 at each of its steps.  Rounded to bf16 at the end
            bound = 2.0**-16 + 2.0**-20 + abs(want) * tokens * 2.0**-24
            bound += 2.0**-8 * (abs(want) + bound)
            off = (out.double() - want).abs().max().item()
            assert off <= bound, (shared, off, bound)
            cache.batch_destroy(batch)
            cache.truncate(ids, np.full(forks, tokens))
    finally:
        cache.close()
