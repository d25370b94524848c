"""cache_restore: without lengths, and of so many results in the 16-bit types that they go past the caches."""
import numpy as np
import pytest
import torch

import paper_2402_02361_amd as P
import test_gpu_token_cache as caches

pytestmark = pytest.mark.gpu
BF, HALF, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.mark.parametrize("dtype", [BF, HALF, F32])
def test_without_lengths_all_tokens_are_there(dtype):
    m = caches.Model(51, 3, 4, 2, 48, 16)
    k = caches._new(m.rng, BF, 3, 64, 2, 48)
    m.append(k, k * 2, None, None)
    for tokens in (64, 37, 1, 0):
        n = caches._ints([tokens] * 3)
        for a, b in zip(P.cache_restore(m.cache, tokens, None, dtype), P.cache_restore(m.cache, tokens, n, dtype)):
            assert a.shape == (3, tokens, 2, 48) and torch.equal(a, b)
    row = P.new_cache(13, 2, 48, 4, 16)   # (a page is left over)
    P.cache_append(row, k, k * 2)
    for a, b in zip(P.cache_restore(row, 64, None, dtype), P.cache_restore(m.cache, 64, None, dtype)):
        assert torch.equal(a, b)
    with pytest.raises(P.PrunerError):
        P.cache_restore(row, 65, None, dtype)


@pytest.mark.parametrize("dtype", [BF, HALF])
@pytest.mark.parametrize("page_tokens", [32, 64])
def test_more_than_the_caches_are_good_for(dtype, page_tokens):
    """2 (keys, values) x 2 x 17000 x 4 x 128 x 2 bytes are 70 MB, beyond the 64 MB from which on results go past the caches: the same as parts of them, whose calls are small."""
    rng = np.random.default_rng(52)
    seq_pages = -(-17000 // page_tokens)
    pages = 2 * seq_pages + 9
    cache = P.new_cache(pages, 4, 128, caches._ints(rng.permutation(pages)[:2 * seq_pages].reshape(2, seq_pages)), page_tokens)
    for t, lo, hi in zip(cache[:4], (0, 0, 110, 110), (120, 120, 130, 130)):
        t.copy_(torch.from_numpy(rng.integers(lo, hi, t.shape, dtype=np.uint8)))
    n = caches._ints([17000, 9001])
    whole = P.cache_restore(cache, 17000, n, dtype)
    for b in range(2):
        one = cache._replace(table=cache.table[b:b + 1].contiguous())
        for first in (0, 8960, 17000 - 17000 % page_tokens - 5 * page_tokens):
            of = one._replace(table=one.table[:, first // page_tokens:].contiguous())
            tokens = min(700, 17000 - first)
            part = P.cache_restore(of, tokens, (n[b:b + 1] - first).clamp(min=0), dtype)
            for x, y in zip(part, whole):
                assert torch.equal(x[0], y[b, first:first + tokens])
    assert not whole[0][1, 9001:].any() and whole[0][1, 9000].any() and not whole[1][1, 9001:].any() and whole[1][0, 16999].any()


def test_a_cache_is_any_five():
    """A plain tuple of the same."""
    cache = P.new_cache(4, 2, 32, 2, 16)
    k = torch.randn(2, 20, 2, 32, device="cuda", dtype=BF)
    P.cache_append(tuple(cache), k, k)
    n = caches._ints([20, 7])
    for lengths in (n, None):
        for a, b in zip(P.cache_restore(tuple(cache), 20, lengths, BF), P.cache_restore(cache, 20, lengths, BF)):
            assert torch.equal(a, b)
    assert torch.equal(P.cache_attention(k, tuple(cache), k_len=n), P.cache_attention(k, cache, k_len=n))
