"""rel_attention and its gradients where a whole row's biases are large: masks of the type's lowest value or of -1e9 that a row sees nothing but, and biases whose sum with
a score keeps few digits in binary32.  A row's weights sum to 1 in the backward pass as in the forward pass, whatever binary32 keeps of log sum exp.

Bounds are block_reference.attention_bounds', and where scores are not lost beside the bias altogether, of every weight what two roundings of its score in binary32 make."""
import numpy as np
import pytest
import torch

import block_reference as ref
import paper_2402_02361_amd as P

pytestmark = pytest.mark.gpu
BF, HALF = torch.bfloat16, torch.float16
E = np.array([1, 2, 3, 4, 6, 9, 14, 22], np.int32)
SHAPES = [  # batch, q_tokens, k_tokens, q_heads, kv_heads, head_dim
    (2, 20, 20, 2, 2, 64), (1, 32, 60, 4, 2, 128), (1, 150, 150, 2, 1, 64), (1, 333, 500, 2, 2, 128), (1, 90, 700, 2, 1, 32), (1, 700, 40, 2, 2, 64)]


def _randn(gen, dtype, *shape, scale=1.0):
    return (torch.randn(*shape, generator=gen) * scale).to(dtype).cuda()


def _within(got, want, bound, what):
    g = ref.cpu(got)
    worst = np.abs(g - want) / np.maximum(bound, 1e-300)
    assert np.isfinite(g).all() and (worst <= 1).all(), f"{what}: {worst.max():.3g} of its bound at {np.unravel_index(worst.argmax(), worst.shape)}"


def _check(dtype, shape, sides, causal, change, score=0.0, still=False):
    """change(table) makes some biases large; score: the largest size of a score that is not lost beside them; still: queries are zero (scores then are the biases)."""
    batch, lq, lk, hq, hk, d = shape
    gen = torch.Generator().manual_seed(sum(shape) + sides)
    q, k, v, do = (_randn(gen, dtype, batch, n, h, d) for n, h in ((lq, hq), (lk, hk), (lk, hk), (lq, hq)))
    if still:
        q.zero_()
    table = _randn(gen, dtype, sides * (len(E) + 1), hq, scale=0.7)
    change(table)
    want = ref.attention(*(ref.cpu(t) for t in (q, k, v, table)), E, causal=causal, do=ref.cpu(do))
    bound = ref.attention_bounds(want, dtype)
    lost = 2 * ref.F32 * score   # of a weight, by two roundings of its score
    bound["o"] += lost * want["o_abs"]
    for n in ("dq", "dk", "dv", "dtable"):
        bound[n] += 2 * lost * want[n + "_abs"]
    o, lse = P.rel_attention(q, k, v, table, E, causal=causal, want_lse=True)
    _within(o, want["o"], bound["o"], "o")
    none = np.isinf(want["lse"])
    assert np.array_equal(np.isinf(ref.cpu(lse)), none)
    o64, lse64 = torch.from_numpy(want["o"]).to(dtype).cuda(), torch.from_numpy(want["lse"]).float().cuda()
    got = P.rel_attention_grad(do, q, k, v, o64, lse64, table, E, causal=causal)
    for name, t in zip(("dq", "dk", "dv", "dtable"), got):
        _within(t, want[name], bound[name], name)


def _all(value):
    def change(table):
        table[:, 0] = value
    return change


def _near(value):   # the distances below 6 at or behind the query
    def change(table):
        table[:5] = value
    return change


@pytest.mark.parametrize("sides,causal", [(1, True), (2, False), (2, True), (1, False)])
@pytest.mark.parametrize("dtype", [BF, HALF])
@pytest.mark.parametrize("shape", SHAPES)
class TestMasks:
    def test_a_head_of_the_lowest_value(self, shape, dtype, sides, causal):
        lowest = torch.finfo(dtype).min
        _check(dtype, shape, sides, causal, _all(lowest), score=65504.0 if dtype == HALF else 0.0)

    def test_rows_that_see_only_the_lowest_value(self, shape, dtype, sides, causal):
        lowest = torch.finfo(dtype).min
        _check(dtype, shape, sides, causal, _near(lowest), score=65504.0 if dtype == HALF else 0.0)

    def test_a_bias_that_leaves_scores_some_digits(self, shape, dtype, sides, causal):
        _check(dtype, shape, sides, causal, _all(-3000.0), score=3000.0)
        _check(dtype, shape, sides, causal, _near(5000.0), score=5000.0)


@pytest.mark.parametrize("sides,causal", [(1, True), (2, False)])
@pytest.mark.parametrize("value", [-1e9, -1e5, 1e7])
@pytest.mark.parametrize("shape", SHAPES)
def test_large_biases_alone(shape, value, sides, causal):
    _check(BF, shape, sides, causal, _all(value), still=True)
    _check(BF, shape, sides, causal, _near(value), still=True)
