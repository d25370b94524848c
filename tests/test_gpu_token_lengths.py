"""Lengths outside their range mean the same to every call of a token step: rotary turns a token for the place where cache_append stores it and where cache_attention has its query stand."""
import numpy as np
import pytest
import torch

import paper_2402_02361_amd as P
import test_gpu_token_rotary as rotary
import token_reference as ref

pytestmark = pytest.mark.gpu
F32 = torch.float32


def _ints(*n):
    return torch.tensor(n, dtype=torch.int32).cuda()


@pytest.mark.parametrize("interleaved", [False, True])
def test_new_tokens_outside_their_range_are_clamped(interleaved):
    gen = torch.Generator().manual_seed(31)
    q, k = rotary._randn(gen, 5, 10, 2, 32, dtype=F32), rotary._randn(gen, 5, 10, 1, 32, dtype=F32)
    k_len, q_len = np.array([40, 12, 7, 2 ** 31 - 1, 0]), np.array([11, -5, 2 ** 31 - 1, -2 ** 31, 10])
    at = (k_len - np.clip(q_len, 0, 10))[:, None] + np.arange(10)[None]
    at = (at + 2 ** 31) % 2 ** 32 - 2 ** 31   # (positions have 32 bits)
    rotary._check(q, k, P.rotary_frequencies(32), at, interleaved, k_len=_ints(*k_len), q_len=_ints(*q_len))


def test_tokens_are_turned_for_the_places_where_they_are_stored():
    """One row of ones as every key, turned and stored with such lengths: the cache's token t is that row turned for t."""
    freqs, tokens = P.rotary_frequencies(64), 6
    q_len, k_len = _ints(9, 4, -2), _ints(20, 20, 20)
    k = torch.ones(3, tokens, 1, 64, device="cuda")
    turned = P.rotary(k, None, freqs, q_len=q_len, k_len=k_len)[0]
    cache = P.new_cache(6, 1, 64, 2, 16)
    for t in cache[:4]:
        t.fill_(120)
    P.cache_append(cache, turned, turned, q_len=q_len, k_len=k_len)
    got = ref.cpu(P.cache_restore(cache, 20, k_len, F32)[0])
    for b, first in ((0, 14), (1, 16)):
        at = np.arange(first, 20)
        want, _ = ref.rotary(np.ones((1, len(at), 1, 64)), freqs, at[None])
        # (e4m3: half a step, 2^-4 of a value, or of its smallest steps under a page's largest: sizes are at most sqrt(2) = 1.41 < 448 x 2^-8, whose smallest steps are 2^-9 x 2^-8)
        assert (np.abs(got[b, first:] - want[0]) <= 2.0 ** -4 * np.abs(want[0]) + 2.0 ** -17).all()
