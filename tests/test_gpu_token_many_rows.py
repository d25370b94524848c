"""Rotary of more tokens than one launch has workgroups for."""
import numpy as np
import pytest
import torch

import paper_2402_02361_amd as P
import test_gpu_token_rotary as rotary
import token_reference as ref

pytestmark = pytest.mark.gpu


def test_more_tokens_than_a_launch_holds():
    """2^28 tokens and some, sixteen to a workgroup, of heads of two columns (1 GB): the first ones, those about each launch's end (2^23 workgroups) and the last ones."""
    tokens = (1 << 28) + 1003
    gen = torch.Generator(device="cuda").manual_seed(61)
    q = torch.randn(1, tokens, 1, 2, generator=gen, device="cuda", dtype=torch.bfloat16)
    freqs = P.rotary_frequencies(2)
    got = P.rotary(q, None, freqs)[0]
    for first in (0, (1 << 27) - 40, (1 << 28) - 40, tokens - 80):
        at = first + np.arange(80)
        want, size = ref.rotary(ref.cpu(q[:, first:first + 80]), freqs, at[None])
        assert (np.abs(ref.cpu(got[:, first:first + 80]) - want) <= rotary._bound(want, size, torch.bfloat16)).all()
    back = P.rotary_grad(got, None, freqs, out=(got, None))[0]
    assert torch.isfinite(back).all()
    for first in range(0, tokens, 1 << 26):   # (two roundings to bfloat16, of each of the pair)
        a, b = q[:, first:first + (1 << 26)].float(), back[:, first:first + (1 << 26)].float()
        assert ((a - b).abs() <= 2.0 ** -8 * 1.05 * (a.abs() + 2 * (a[..., :1].abs() + a[..., 1:].abs()))).all()
