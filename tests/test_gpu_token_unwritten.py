"""cache_attention where pages hold nothing of a sequence: those that are reserved and not yet written, and those that are not there.  Their memory holds anything, exponent bytes that no append makes
among it, and none of it reaches a result."""
import numpy as np
import pytest
import torch

import paper_2402_02361_amd as P
import test_gpu_token_attention as attention

pytestmark = pytest.mark.gpu
BF, HALF = torch.bfloat16, torch.float16


def _with_bytes(cache, k_len, byte):
    """The same cache, in a pool whose page 0 and whose other pages without tokens have codes that are NaN and `byte` for exponents of keys and values."""
    pages, page_tokens = cache.k_codes.shape[0], cache.k_codes.shape[3]
    table = cache.table.cpu().numpy()
    moved = np.where((table >= 0) & (table < pages), table + 1, np.where(table == pages, pages + 1, table)).astype(np.int32)
    unused = np.ones(pages + 1, bool)
    for b, n in enumerate(k_len):
        inside = moved[b, :-(-n // page_tokens)]
        unused[inside[(inside >= 0) & (inside <= pages)]] = False
    assert unused[0] and unused.sum() > 1
    at = torch.from_numpy(unused).cuda()
    pool = [torch.cat([t[:1], t]) for t in cache[:4]]
    for t, fill in zip(pool, (255, 255, byte, byte)):
        t[at] = fill
    return P.Cache(*pool, torch.from_numpy(moved).cuda())


@pytest.mark.parametrize("byte", [255, 0])
@pytest.mark.parametrize("missing", [False, True])
@pytest.mark.parametrize("page_tokens", [16, 32, 64, 128])
@pytest.mark.parametrize("dtype,q_tokens,head_dim", [(BF, 1, 64), (HALF, 1, 128), (HALF, 20, 32), (BF, 5, 80), (BF, 100, 64), (HALF, 100, 128), (BF, 70, 32)])
def test_what_pages_without_tokens_hold_does_not_matter(dtype, q_tokens, head_dim, page_tokens, missing, byte):
    """The same bits as with other bytes there, which are checked against the definition."""
    k_len = [400, 20, 321, 130]
    gone = [(0, 0), (0, 2), (0, 9), (2, 1), (2, 320 // page_tokens)] + [(3, i) for i in range(26)]
    missing = [g for g in gone if g[1] < -(-401 // page_tokens)] if missing else ()
    q, cache, table, kw, o, lse = attention._check(dtype, 4, q_tokens, 401, 4, 2, head_dim, page_tokens, 1, k_len=k_len, seed=21, missing=missing)
    q = torch.nan_to_num(q)
    other = _with_bytes(cache, k_len, byte)
    got, got_lse = P.cache_attention(q, other, table, attention.E, want_lse=True, k_tokens=401, **kw)
    assert torch.equal(got, o) and torch.equal(got_lse, lse)


@pytest.mark.parametrize("page_tokens", [16, 32, 64])
@pytest.mark.parametrize("q_tokens", [1, 20, 60])
def test_a_new_cache_over_memory_that_held_ones(q_tokens, page_tokens):
    """Sequences in pages of their own, in a row: the bytes of pages that nothing was stored in are 255."""
    gen = torch.Generator().manual_seed(22)
    k, v = (torch.randn(2, 100, 2, 64, generator=gen).to(BF).cuda() for _ in range(2))
    q = torch.randn(2, q_tokens, 8, 64, generator=gen).to(BF).cuda()
    n = torch.tensor([70, 65], dtype=torch.int32).cuda()
    made = []
    for fill in (255, 120):
        cache = P.new_cache(2 * 128 // page_tokens, 2, 64, 128 // page_tokens, page_tokens)
        for t in cache[:4]:
            t.fill_(fill)
        P.cache_append(cache, k[:, :70], v[:, :70], n, n)
        made.append(P.cache_attention(q, cache, k_len=n))
    assert torch.isfinite(made[0]).all() and torch.equal(*made)
