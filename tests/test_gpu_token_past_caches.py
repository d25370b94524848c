"""Rotary of more than the caches are good for, where results go past them: what is written there lies in whole lines."""
import pytest
import torch

import paper_2402_02361_amd as P

pytestmark = pytest.mark.gpu
BF, HALF, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype,tokens,heads,head_dim,rotary_dim", [(F32, 18001, 15, 128, 128), (HALF, 18001, 31, 128, 128), (BF, 36001, 15, 128, 64), (F32, 18001, 20, 96, 96), (HALF, 18001, 45, 90, 90), (F32, 18001, 19, 100, 36)])
def test_the_same_bits_as_parts_of_it(dtype, tokens, heads, head_dim, rotary_dim, interleaved):
    gen = torch.Generator(device="cuda").manual_seed(tokens + heads)
    q = torch.randn(1, tokens, heads, head_dim, generator=gen, device="cuda").to(dtype)
    assert q.numel() * q.element_size() > 128 << 20
    freqs = P.rotary_frequencies(rotary_dim)
    whole = P.rotary(q, None, freqs, interleaved=interleaved)[0]
    other = P.rotary_grad(q, None, freqs, interleaved=interleaved)[0]
    parts = []
    for lo in (0, 1000, tokens - 77):
        n = torch.tensor([lo + 77], dtype=torch.int32).cuda()
        parts.append(P.rotary(q[:, lo:lo + 77], None, freqs, k_len=n, interleaved=interleaved)[0])
        assert torch.equal(parts[-1], whole[:, lo:lo + 77])
        assert torch.equal(P.rotary_grad(q[:, lo:lo + 77], None, freqs, k_len=n, interleaved=interleaved)[0], other[:, lo:lo + 77])
    P.rotary(q, None, freqs, interleaved=interleaved, out=(q, None))   # in place
    assert torch.equal(q, whole)
