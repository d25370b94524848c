"""cache_attention of few columns (up to 32 queries of heads that share a key head): what a result loses beside its own rounding."""
import numpy as np
import pytest
import torch

import block_reference as block
import paper_2402_02361_amd as P
import test_gpu_token_attention as attention
import token_reference as ref

pytestmark = pytest.mark.gpu
BF, HALF = torch.bfloat16, torch.float16


def _bound(want, dtype):
    """Half a step of the result (1 % for roundings on the way to it), a weight's two bfloat16 terms (2^-8 of 2^-8) and binary32's share of a weight."""
    return 1.01 * ref.UNIT[dtype] * np.abs(want["o"]) + (2.0 ** -16 + block.EXP) * want["o_abs"] + ref.TINY[dtype]


@pytest.mark.parametrize("dtype", [BF, HALF])
@pytest.mark.parametrize("batch,q_tokens,k_tokens,q_heads,kv_heads,head_dim,page_tokens,sides", [
    (2, 1, 300, 8, 8, 64, 64, 0), (1, 1, 9000, 16, 2, 128, 128, 0), (2, 5, 2000, 8, 2, 80, 16, 1), (1, 8, 700, 4, 1, 128, 64, 1), (1, 30, 500, 1, 1, 32, 16, 0), (3, 2, 90, 3, 3, 96, 32, 0)])
def test_weights_keep_their_digits(dtype, batch, q_tokens, k_tokens, q_heads, kv_heads, head_dim, page_tokens, sides):
    q, cache, table, kw, o, _ = attention._check(dtype, batch, q_tokens, k_tokens, q_heads, kv_heads, head_dim, page_tokens, sides, seed=41)
    k, v = (ref.cpu(t) for t in P.cache_restore(cache, k_tokens, kw["k_len"], torch.float32))
    want = block.attention(ref.cpu(q), k, v, ref.cpu(table), attention.E, [q_tokens] * batch, [k_tokens] * batch, True, kw["scale"])
    worst = np.abs(ref.cpu(o) - want["o"]) / _bound(want, dtype)
    assert (worst <= 1).all(), f"{worst.max():.3g} of its bound"


@pytest.mark.parametrize("dtype", [BF, HALF])
@pytest.mark.parametrize("q_tokens,heads", [(1, 1), (1, 20)])
def test_many_small_weights(dtype, q_tokens, heads):
    """One key takes nearly all of the weight and has a value of 0; 20000 others have exp(-18) each, below binary16's smallest numbers, and values of 1: the result is their sum."""
    n = 20000
    k, v = torch.zeros(1, n, 1, 32, device="cuda"), torch.ones(1, n, 1, 32, device="cuda")
    k[0, 5, 0, 3], v[0, 5] = 18.0, 0.0
    cache = P.new_cache(-(-n // 64), 1, 32, -(-n // 64), 64)
    P.cache_append(cache, k, v)
    q = torch.zeros(1, q_tokens, heads, 32, dtype=dtype, device="cuda")
    q[..., 3] = 1.0
    o = P.cache_attention(q, cache, k_len=torch.tensor([n], dtype=torch.int32).cuda(), scale=1.0)
    small = (n - 1) * np.exp(-18.0)
    want = small / (1 + small)
    assert np.abs(ref.cpu(o) - want).max() <= (1.01 * ref.UNIT[dtype] + 2.0 ** -16 + block.EXP) * want
