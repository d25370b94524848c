"""rel_attention_grad in binary16 where the output's gradient is small, as an averaged loss gives it, or of very different sizes in a sequence: a score's gradient
is about a row's length smaller still, and no digit of it may be lost for that.

The bound is that of block_reference.attention_bounds without what it grants a score's gradient below binary16's smallest step: a rounding of the result (half a
step of 2^-24 at least), one of every weight and score gradient, relative, and binary32's."""
import numpy as np
import pytest
import torch

import block_reference as ref
import paper_2402_02361_amd as P

pytestmark = pytest.mark.gpu
HALF = torch.float16


def _randn(gen, *shape, scale=1.0):
    return (torch.randn(*shape, generator=gen) * scale).to(HALF).cuda()


def _check(q, k, v, do, causal, table=None, edges=()):
    want = ref.attention(ref.cpu(q), ref.cpu(k), ref.cpu(v), ref.cpu(table), edges, causal=causal, do=ref.cpu(do))
    for n in ("dq_tiny", "dk_tiny"):
        want[n] = np.zeros_like(want[n])
    bound = ref.attention_bounds(want, HALF)
    o, lse = torch.from_numpy(want["o"]).to(HALF).cuda(), torch.from_numpy(want["lse"]).float().cuda()
    got = P.rel_attention_grad(do, q, k, v, o, lse, table, edges if table is not None else None, causal=causal)
    for name, t in zip(("dq", "dk", "dv"), got):
        g = ref.cpu(t)
        worst = np.abs(g - want[name]) / bound[name]
        assert np.isfinite(g).all() and (worst <= 1).all(), f"{name}: {worst.max():.3g} of its bound"


SHAPES = [  # batch, q_tokens, k_tokens, q_heads, kv_heads, head_dim
    (1, 2100, 2100, 2, 1, 64), (1, 130, 4000, 2, 1, 128), (1, 700, 2500, 1, 1, 32), (3, 30, 60, 4, 2, 64), (2, 20, 64, 4, 2, 128), (2, 32, 50, 1, 1, 32)]


@pytest.mark.parametrize("size", [200.0, 1e-3, 1e-4, 1e-5])
@pytest.mark.parametrize("shape", SHAPES)
def test_small_and_large_output_gradients(shape, size):
    batch, lq, lk, hq, hk, d = shape
    gen = torch.Generator().manual_seed(sum(shape))
    q, k, v = _randn(gen, batch, lq, hq, d), _randn(gen, batch, lk, hk, d), _randn(gen, batch, lk, hk, d)
    _check(q, k, v, _randn(gen, batch, lq, hq, d, scale=size), causal=lq % 4 == 0)


@pytest.mark.parametrize("falling", [False, True])
@pytest.mark.parametrize("shape", [(1, 520, 700, 2, 1, 64), (1, 300, 300, 2, 2, 128), (2, 32, 64, 2, 1, 64)])
def test_sizes_that_change_along_a_sequence(shape, falling):
    """From tile to tile the score gradients of a key grow, or fall, by up to 10^5, those of a query by up to 300."""
    batch, lq, lk, hq, hk, d = shape
    gen = torch.Generator().manual_seed(lq)
    by_query, by_key = torch.logspace(-4, 1, lq)[None, :, None, None], torch.logspace(-1, 1.5, lk)[None, :, None, None]
    if falling:
        by_query, by_key = by_query.flip(1), by_key.flip(1)
    q, k = _randn(gen, batch, lq, hq, d), _randn(gen, batch, lk, hk, d)
    v, do = _randn(gen, batch, lk, hk, d, scale=by_key), _randn(gen, batch, lq, hq, d, scale=by_query)
    edges = np.array([1, 2, 5, 30], np.int32)
    _check(q, k, v, do, False, _randn(gen, 10, hq), edges)


def test_a_gradient_of_zero():
    gen = torch.Generator().manual_seed(1)
    q, k, v = (_randn(gen, 1, 200, 2, 64) for _ in range(3))
    o, lse = P.rel_attention(q, k, v, want_lse=True)
    got = P.rel_attention_grad(torch.zeros_like(q), q, k, v, o, lse)
    assert all(not t.any() for t in got[:3])
