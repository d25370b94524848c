"""rotary and rotary_grad against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2402_02361_amd as P
import token_reference as ref

pytestmark = pytest.mark.gpu
BF, HALF, F32 = torch.bfloat16, torch.float16, torch.float32

# Sine and cosine: the reduced angle (at most pi / 4) has three roundings, 2.4 x 2^-24, the series two or three of a value of at most 1, the amplitude one: below 7 x 2^-24 of each
# term's size; the two products and their sum round once each.  The result is then rounded to the type, half a step.
SUM = 9 * ref.F32


def _randn(gen, *shape, dtype):
    return torch.randn(*shape, generator=gen).to(dtype).cuda()


def _bound(want, size, dtype):
    return SUM * size + (ref.UNIT[dtype] if dtype != F32 else 0) * (np.abs(want) + SUM * size) + ref.TINY[dtype] + 1e-40


def _check(q, k, freqs, at, interleaved=False, amplitude=1.0, **kw):
    amplitude32 = float(np.float32(amplitude))
    for back, call in ((False, P.rotary), (True, P.rotary_grad)):
        got = call(q, k, freqs, interleaved=interleaved, amplitude=amplitude, **kw)
        for x, y in zip((q, k), got):
            if x is None:
                assert y is None
                continue
            want, size = ref.rotary(ref.cpu(x), freqs, at, interleaved, amplitude32, back)
            g = ref.cpu(y)
            worst = np.abs(g - want) / _bound(want, size, x.dtype)
            assert y.dtype == x.dtype and y.is_contiguous() and np.isfinite(g).all() and (worst <= 1).all(), f"{worst.max():.3g} of its bound at {np.unravel_index(worst.argmax(), worst.shape)}"
            assert np.array_equal(g[..., 2 * len(freqs):], ref.cpu(x)[..., 2 * len(freqs):])


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [BF, HALF, F32])
@pytest.mark.parametrize("batch,tokens,q_heads,kv_heads,head_dim,rotary_dim", [
    (1, 1, 1, 1, 2, 2), (1, 1, 32, 8, 128, 128), (3, 7, 4, 2, 64, 32), (2, 33, 5, 1, 80, 80), (1, 130, 3, 3, 100, 36), (2, 5, 2, 1, 37, 22), (1, 3, 1, 1, 512, 256), (2, 300, 12, 3, 96, 6),
    (1, 9, 9, 2, 65, 64), (4, 1, 7, 7, 18, 18)])
def test_shapes(dtype, interleaved, batch, tokens, q_heads, kv_heads, head_dim, rotary_dim):
    gen = torch.Generator().manual_seed(head_dim)
    q, k = _randn(gen, batch, tokens, q_heads, head_dim, dtype=dtype), _randn(gen, batch, tokens, kv_heads, head_dim, dtype=dtype)
    k_len = torch.randint(tokens, 5000, (batch,), generator=gen, dtype=torch.int32)
    at = k_len.numpy()[:, None] - tokens + np.arange(tokens)
    _check(q, k, P.rotary_frequencies(rotary_dim), at, interleaved, 1.25 if rotary_dim % 4 else 1.0, k_len=k_len.cuda())


def test_where_tokens_stand():
    gen = torch.Generator().manual_seed(1)
    q, k = _randn(gen, 3, 10, 2, 32, dtype=F32), _randn(gen, 3, 10, 1, 32, dtype=F32)
    freqs, rows = P.rotary_frequencies(32, factor=4.0), np.arange(10)[None, :]
    ints = lambda *n: torch.tensor(n, dtype=torch.int32).cuda()  # noqa: E731
    _check(q, k, freqs, rows + np.zeros((3, 1)))
    _check(q, k, freqs, np.array([[5], [0], [7]]) - 10 + rows, k_len=ints(5, 0, 7))                       # (before the first place: negative)
    _check(q, k, freqs, np.array([[5 - 2], [0], [7 - 9]]) + rows, k_len=ints(5, 0, 7), q_len=ints(2, 0, 9))
    far = np.stack([2 ** 31 - 11 + np.arange(10), -2 ** 31 + np.arange(10), np.arange(10)[::-1] * 12345])
    _check(q, k, freqs, far, positions=torch.from_numpy(far.astype(np.int32)).cuda())
    _check(q, None, freqs, rows + np.zeros((3, 1)))


@pytest.mark.parametrize("f", [0.0, 64.0, -1.0, 1e-12, 2 * np.pi, np.pi / 4, np.pi / 2])
def test_frequencies_of_any_size(f):
    """A frequency of exactly a quarter of a turn has its quadrants' borders at every position."""
    gen = torch.Generator().manual_seed(2)
    q = _randn(gen, 1, 500, 1, 16, dtype=F32)
    freqs = np.array([f, f / 3, 1.0, f, 0.5, f, f, 2.0 ** -20])
    _check(q, None, freqs, 1000000 + np.arange(500)[None], k_len=torch.tensor([1000500], dtype=torch.int32).cuda())


@pytest.mark.parametrize("dtype", [BF, HALF, F32])
@pytest.mark.parametrize("interleaved", [False, True])
def test_strides_orders_and_in_place(dtype, interleaved):
    """Parts of a fused projection, heads before tokens, rows that begin anywhere, an expanded input, outputs over their inputs: the same bits."""
    gen = torch.Generator().manual_seed(3)
    qkv = _randn(gen, 2, 40, 9, 81, dtype=dtype)
    q, k = qkv[:, :, :4, 1:], qkv[:, :, 5:7, 1:]
    freqs = P.rotary_frequencies(44)
    want = P.rotary(q.contiguous(), k.contiguous(), freqs, interleaved=interleaved)
    got = P.rotary(q, k, freqs, interleaved=interleaved)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    heads_first = lambda t: t.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)  # noqa: E731
    out = (heads_first(torch.zeros_like(q)), heads_first(torch.zeros_like(k)))
    got = P.rotary(heads_first(q), heads_first(k), freqs, interleaved=interleaved, out=out)
    assert got[0] is out[0] and all(torch.equal(a, b) for a, b in zip(want, got))
    one = P.rotary(q[:1, :1].expand(2, 40, 4, 80), None, freqs, interleaved=interleaved)[0]
    assert torch.equal(one, P.rotary(q[:1, :1].expand(2, 40, 4, 80).contiguous(), None, freqs, interleaved=interleaved)[0])
    before = qkv.clone()
    got = P.rotary(q, k, freqs, interleaved=interleaved, out=(q, k))
    assert got[0] is q and torch.equal(q, want[0]) and torch.equal(k, want[1])
    assert torch.equal(qkv[..., 0], before[..., 0]) and torch.equal(qkv[:, :, 4], before[:, :, 4]) and torch.equal(qkv[:, :, 7:], before[:, :, 7:])
    # one in place, one not
    q2, k2 = q.contiguous(), torch.zeros_like(k)
    again = P.rotary(q, k, freqs, interleaved=interleaved)
    P.rotary(q2, k, freqs, interleaved=interleaved, out=(q2, k2))
    assert torch.equal(q2, again[0]) and torch.equal(k2, again[1])


@pytest.mark.parametrize("interleaved", [False, True])
def test_gradients_are_those_of_differences(interleaved):
    """The operator is linear in its inputs: <dy, R(x + h e) - R(x)> / h is <R'(dy), e> up to the roundings of two results."""
    gen = torch.Generator().manual_seed(4)
    x, dy, e = (_randn(gen, 1, 6, 2, 24, dtype=F32) for _ in range(3))
    freqs = P.rotary_frequencies(20)
    kw = dict(interleaved=interleaved, amplitude=1.5, k_len=torch.tensor([100], dtype=torch.int32).cuda())
    up, down = P.rotary(x + e, None, freqs, **kw)[0], P.rotary(x - e, None, freqs, **kw)[0]
    left, right = (ref.cpu(dy) * (ref.cpu(up) - ref.cpu(down))).sum() / 2, (ref.cpu(P.rotary_grad(dy, None, freqs, **kw)[0]) * ref.cpu(e)).sum()
    size = np.abs(ref.cpu(dy)).sum() * 1.5 * 2 * np.abs(ref.cpu(x)).max() + np.abs(ref.cpu(e)).sum() * 1.5 * 2 * np.abs(ref.cpu(dy)).max()
    assert abs(left - right) <= 4 * SUM * size
    back = P.rotary_grad(P.rotary(x, None, freqs, **kw)[0], None, freqs, **kw)[0]
    assert (back[..., :20] - 2.25 * x[..., :20]).abs().max() <= 4 * SUM * 2.25 * 4 * x.abs().max()


def test_nan_and_infinity_stay_in_their_pair():
    x = torch.ones(1, 2, 1, 32, device="cuda")
    x[0, 0, 0, 3], x[0, 1, 0, 20] = float("nan"), float("inf")
    y = P.rotary(x, None, P.rotary_frequencies(32))[0]
    bad = ~torch.isfinite(y)
    assert bad[0, 0, 0].nonzero().flatten().tolist() == [3, 19] and bad[0, 1, 0].nonzero().flatten().tolist() == [4, 20]


def test_many_rows():
    """More rows than one thread's heads: every head group and the last rows."""
    gen = torch.Generator().manual_seed(5)
    q, k = _randn(gen, 2, 3001, 20, 64, dtype=BF), _randn(gen, 2, 3001, 3, 64, dtype=BF)
    freqs = P.rotary_frequencies(64)
    got = P.rotary(q, k, freqs)
    some = np.unique(np.concatenate([np.arange(0, 3001, 97), np.arange(2980, 3001)]))
    at = torch.from_numpy(some).cuda()
    for x, y in zip((q, k), got):
        want, size = ref.rotary(ref.cpu(x[:, at]), freqs, np.stack([some, some]))
        assert (np.abs(ref.cpu(y[:, at]) - want) <= _bound(want, size, BF)).all()


def test_empty_and_streams_and_graphs():
    gen = torch.Generator().manual_seed(6)
    q, k = _randn(gen, 2, 70, 4, 64, dtype=BF), _randn(gen, 2, 70, 2, 64, dtype=BF)
    freqs = P.rotary_frequencies(64)
    for a, b in ((q[:0], k[:0]), (q[:, :0], k[:, :0]), (q[:, :, :0], k[:, :, :0])):
        x, y = P.rotary(a, b, freqs)
        assert x.shape == a.shape and y.shape == b.shape
    want = P.rotary(q, k, freqs)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = P.rotary(q, k, freqs, stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = P.rotary(q, k, freqs)
    for n in range(3):
        for t in got:
            t.fill_(7.0)
        q.mul_(2 if n else 1), k.mul_(2 if n else 1)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(P.rotary(q, k, freqs), got))


def test_refusals_of_the_binding():
    q, k, freqs = torch.zeros(2, 3, 4, 16, device="cuda"), torch.zeros(2, 3, 2, 16, device="cuda"), P.rotary_frequencies(16)
    for bad in (dict(k=k.half()), dict(k=k[:, :2]), dict(k=k[..., :8]), dict(freqs=P.rotary_frequencies(18)), dict(freqs=freqs[:0]), dict(positions=torch.zeros(2, 3, dtype=torch.int64).cuda()),
                dict(positions=torch.zeros(2, 4, dtype=torch.int32).cuda()), dict(q_len=torch.zeros(3, dtype=torch.int32).cuda()), dict(out=(q, None)), dict(out=(q[:1], k)), dict(q=q.cpu()),
                dict(q=q.transpose(2, 3))):
        with pytest.raises(AssertionError):
            P.rotary(**{**dict(q=q, k=k, freqs=freqs), **bad})
    for bad in (dict(amplitude=float("inf")), dict(freqs=freqs * 100), dict(q=q.double(), k=k.double()), dict(freqs=freqs * np.nan)):
        with pytest.raises(P.PrunerError):
            P.rotary(**{**dict(q=q, k=k, freqs=freqs), **bad})
