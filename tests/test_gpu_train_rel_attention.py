"""rel_attention and rel_attention_grad against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

import block_reference as ref
import paper_2402_02361_amd as P

pytestmark = pytest.mark.gpu
BF, HALF = torch.bfloat16, torch.float16


def _randn(gen, *shape, dtype, scale=1.0):
    return (torch.randn(*shape, generator=gen) * scale).to(dtype).cuda()


def _inputs(dtype, batch, lq, lk, hq, hk, d, sides, edges, seed=0, fused=False):
    gen = torch.Generator().manual_seed(seed)
    if fused:
        qkv = _randn(gen, batch, lq, hq + 2 * hk, d, dtype=dtype)
        q, k, v = qkv[:, :, :hq], qkv[:, :, hq:hq + hk], qkv[:, :, hq + hk:]
    else:
        q, k, v = _randn(gen, batch, lq, hq, d, dtype=dtype), _randn(gen, batch, lk, hk, d, dtype=dtype), _randn(gen, batch, lk, hk, d, dtype=dtype)
    table = _randn(gen, sides * (len(edges) + 1), hq, dtype=dtype, scale=0.7) if sides else None
    return q, k, v, table, _randn(gen, batch, lq, hq, d, dtype=dtype)


def _lengths(n):
    return None if n is None else torch.tensor(n, dtype=torch.int32).cuda()


def _within(got, want, bound, what):
    g = ref.cpu(got)
    assert np.isfinite(g).all(), what
    worst = np.abs(g - want) / np.maximum(bound, 1e-300)
    assert (worst <= 1).all(), f"{what}: {worst.max():.3g} of its bound at {np.unravel_index(worst.argmax(), worst.shape)}"


def _check(q, k, v, table, do, edges, q_len=None, k_len=None, causal=False, scale=None, grads=True):
    kw = dict(q_len=_lengths(q_len), k_len=_lengths(k_len), causal=causal, scale=scale)
    o, lse = P.rel_attention(q, k, v, table, edges, want_lse=True, **kw)
    clean = lambda t, n: ref.cpu(t) if n is None else np.where(np.arange(t.shape[1])[None, :, None, None] < np.asarray(n)[:, None, None, None], ref.cpu(t), 0.0)  # noqa: E731
    want = ref.attention(clean(q, q_len), clean(k, k_len), clean(v, k_len), ref.cpu(table), [] if edges is None else edges, q_len, k_len, causal, scale,
                         clean(do, q_len) if grads else None)
    bound = ref.attention_bounds(want, q.dtype)
    _within(o, want["o"], bound["o"], "o")
    g = ref.cpu(lse)
    none = np.isinf(want["lse"])
    assert np.array_equal(none, np.isinf(g)) and (np.abs(g - want["lse"])[~none] <= 1e-5 + 2e-6 * np.abs(want["lse"][~none])).all()
    if not grads:
        return o, lse
    o64 = torch.from_numpy(want["o"]).to(q.dtype).cuda()
    lse64 = torch.from_numpy(want["lse"]).float().cuda()
    got = P.rel_attention_grad(do, q, k, v, o64, lse64, table, edges, **kw)
    for name, t in zip(("dq", "dk", "dv", "dtable"), got):
        if name == "dtable" and table is None:
            assert t is None
        else:
            _within(t, want[name], bound[name], name)
    return o, lse, got


E = np.array([1, 2, 3, 4, 6, 9, 14, 22], np.int32)
SHAPES = [  # batch, q_tokens, k_tokens, q_heads, kv_heads, head_dim
    (3, 1, 1, 2, 1, 64), (2, 8, 8, 1, 1, 64), (5, 32, 32, 3, 3, 32), (1, 33, 33, 2, 2, 64), (2, 31, 64, 4, 2, 128), (1, 65, 65, 8, 2, 80), (2, 129, 129, 3, 1, 64),
    (1, 300, 300, 2, 1, 128), (1, 257, 130, 8, 8, 8), (2, 40, 200, 14, 2, 96), (1, 7, 513, 8, 2, 64), (1, 200, 70, 1, 1, 32), (1, 150, 1300, 1, 1, 64)]


@pytest.mark.parametrize("causal,sides", [(False, 2), (True, 1), (False, 0), (False, 1), (True, 2)])
@pytest.mark.parametrize("shape", SHAPES)
def test_shapes(shape, causal, sides):
    dtype = (BF, HALF)[(sum(shape) + sides) % 2]
    _check(*_inputs(dtype, *shape, sides, E, fused=shape[1] == shape[2]), E, causal=causal)


@pytest.mark.parametrize("dtype", [BF, HALF])
@pytest.mark.parametrize("q_len,k_len", [([0, 5, 40, 17], [0, 5, 40, 17]), ([9, 40, 3, 0], [4, 0, 40, 12]), ([40, 40, 1, 20], [10, 39, 1, 40])])
@pytest.mark.parametrize("tokens", [40, 24])
def test_lengths_leave_rows_empty_and_padding_does_not_matter(dtype, q_len, k_len, tokens):
    """Queries before the first key (more queries than keys under the causal mask) and empty sequences; what the padding holds is NaN and infinity."""
    q_len, k_len = [min(n, tokens) for n in q_len], [min(n, tokens) for n in k_len]
    q, k, v, table, do = _inputs(dtype, 4, tokens, tokens, 4, 2, 64, 2, E, seed=1)
    for b in range(4):
        for t, n in ((q, q_len), (do, q_len), (k, k_len), (v, k_len)):
            t[b, n[b]:] = float("nan")
            if n[b] + 1 < t.shape[1]:
                t[b, n[b] + 1] = float("inf")
    for causal in (False, True):
        _check(q, k, v, table, do, E, q_len, k_len, causal)


def test_lengths_outside_are_clamped():
    q, k, v, table, do = _inputs(BF, 3, 20, 50, 2, 2, 32, 1, E, seed=2)
    a = P.rel_attention(q, k, v, table, E, q_len=_lengths([-4, 99, 7]), k_len=_lengths([50, 1000, -1]), causal=True)
    b = P.rel_attention(q, k, v, table, E, q_len=_lengths([0, 20, 7]), k_len=_lengths([50, 50, 0]), causal=True)
    assert torch.equal(a, b) and not a[0].any() and not a[2].any()


@pytest.mark.parametrize("q_tokens,k_tokens,q_heads,kv_heads,head_dim,batch", [
    (1, 2000, 8, 1, 128, 3), (1, 70, 8, 8, 64, 2), (2, 3001, 12, 3, 64, 1), (4, 900, 16, 2, 80, 2), (1, 5000, 32, 1, 32, 1), (3, 65, 7, 1, 128, 4), (1, 1, 4, 2, 64, 5)])
@pytest.mark.parametrize("dtype", [BF, HALF])
def test_few_tokens_against_a_cache(q_tokens, k_tokens, q_heads, kv_heads, head_dim, batch, dtype):
    q, k, v, table, do = _inputs(dtype, batch, q_tokens, k_tokens, q_heads, kv_heads, head_dim, 1, P.relative_edges(16, 128) if k_tokens > 128 else E, seed=3)
    edges = P.relative_edges(16, 128) if k_tokens > 128 else E
    table = torch.randn(len(edges) + 1, q_heads, generator=torch.Generator().manual_seed(5)).to(dtype).cuda()
    k_len = [max(q_tokens, k_tokens - 61 * b) if b % 2 == 0 else max(1, k_tokens // (b + 1)) for b in range(batch)]
    _check(q, k, v, table, do, edges, [q_tokens] * batch, k_len, causal=True, grads=k_tokens < 1000)


def test_the_rows_before_a_token_do_not_change_its_result():
    """Scoring a sequence at once and token by token agree to the type's rounding."""
    q, k, v, table, _ = _inputs(BF, 1, 90, 90, 4, 2, 64, 1, E, seed=4)
    whole = P.rel_attention(q, k, v, table, E, causal=True)
    for t in (0, 1, 40, 89):
        one = P.rel_attention(q[:, t:t + 1], k, v, table, E, q_len=_lengths([1]), k_len=_lengths([t + 1]), causal=True)
        assert (one - whole[:, t:t + 1]).abs().max() <= 2.0 ** -7 * whole[:, t].abs().max()


@pytest.mark.parametrize("far", [1, 40, 500, 1024])
@pytest.mark.parametrize("sides", [1, 2])
def test_long_distances(far, sides):
    edges = P.relative_edges(min(far, 20), far)
    q, k, v, table, do = _inputs(BF, 1, 700, 700, 2, 1, 32, sides, edges, seed=6)
    _check(q, k, v, table, do, edges, causal=sides == 1)


def test_no_edges():
    for sides, causal in ((1, True), (2, False)):
        q, k, v, table, do = _inputs(HALF, 2, 70, 70, 2, 2, 64, sides, (), seed=7)
        _check(q, k, v, table, do, None, causal=causal)


@pytest.mark.parametrize("tokens", [20, 150])
def test_masks_through_the_table(tokens):
    """A bias of minus infinity removes its pairs (and a row whose pairs are all removed is empty); the type's lowest value leaves a row's weights
    as they are where all of the row has it."""
    for value in (float("-inf"), torch.finfo(BF).min):
        q, k, v, table, do = _inputs(BF, 1, tokens, tokens, 2, 2, 64, 2, E, seed=8)
        table[:5, 0] = value                # head 0: distances below 6 behind or at the query
        table[:, 1] = value                 # head 1: everything
        o, lse, got = None, None, None
        o, lse = P.rel_attention(q, k, v, table, E, want_lse=True)
        want = ref.attention(ref.cpu(q), ref.cpu(k), ref.cpu(v), ref.cpu(table), E)
        assert torch.isfinite(o).all()
        _within(o[:, :, 0], want["o"][:, :, 0], ref.attention_bounds(want, BF)["o"][:, :, 0], "o")
        grads = P.rel_attention_grad(do, q, k, v, o, lse, table, E)
        assert all(torch.isfinite(g).all() for g in grads)
        if value == float("-inf"):
            assert not o[:, :, 1].any() and torch.isinf(lse[:, 1]).all() and not grads[0][:, :, 1].any() and not grads[2][:, :, 1].any()
            assert not grads[3][:5, 0].any()
        else:   # scores vanish beside the lowest value: every key counts alike
            mean = ref.cpu(v)[:, :, 1].mean(1)
            assert np.abs(ref.cpu(o)[:, :, 1] - mean[:, None]).max() <= 2.0 ** -7 * np.abs(ref.cpu(v)).max()


def test_nan_in_a_key_that_is_seen_reaches_the_queries_that_see_it():
    q, k, v, table, _ = _inputs(BF, 1, 100, 100, 1, 1, 64, 1, E, seed=9)
    k[0, 60] = float("nan")
    o = P.rel_attention(q, k, v, table, E, causal=True)
    assert torch.isfinite(o[0, :60]).all() and torch.isnan(o[0, 60:]).all()


def test_strides_and_orders():
    """Heads before tokens, tokens apart, an output of its own order: the same bits as contiguous tensors."""
    q, k, v, table, do = _inputs(BF, 2, 70, 70, 4, 2, 64, 1, E, seed=10)
    want, lse = P.rel_attention(q, k, v, table, E, causal=True, want_lse=True)
    heads_first = lambda t: t.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)  # noqa: E731
    wide = lambda t: torch.cat([t, t + 1], 3)[..., :t.shape[3]]  # noqa: E731
    o = torch.empty(2, 4, 70, 64, dtype=BF, device="cuda").permute(0, 2, 1, 3)
    got = P.rel_attention(heads_first(q), wide(k), heads_first(v), table, E, causal=True, o=o)
    assert got is o and torch.equal(got, want)
    a = P.rel_attention_grad(do, q, k, v, want, lse, table, E, causal=True)
    b = P.rel_attention_grad(wide(do), heads_first(q), wide(k), heads_first(v), o, lse, table, E, causal=True)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    with pytest.raises(P.PrunerError):
        P.rel_attention(torch.cat([q, q], 3)[..., 4:68], k, v, table, E)   # rows that begin between multiples of 16 bytes


def test_offsets_beyond_32_bits():
    """A cache whose tokens are 2^17 bytes apart and more than 2^32 bytes long."""
    tokens, apart = 40000, 1 << 16
    room = torch.empty(tokens * apart, dtype=BF, device="cuda")
    k = room.as_strided((1, tokens, 1, 64), (0, apart, 64, 1))
    v = room.as_strided((1, tokens, 1, 64), (0, apart, 64, 1), 64)
    gen = torch.Generator().manual_seed(11)
    k.copy_(_randn(gen, 1, tokens, 1, 64, dtype=BF))
    v.copy_(_randn(gen, 1, tokens, 1, 64, dtype=BF))
    for rows in (1, 40):
        q = _randn(gen, 1, rows, 1, 64, dtype=BF)
        near = P.rel_attention(q, k.contiguous(), v.contiguous(), q_len=_lengths([rows]), causal=True)
        assert torch.equal(P.rel_attention(q, k, v, q_len=_lengths([rows]), causal=True), near)


def test_the_same_bits_every_time_and_on_another_stream():
    q, k, v, table, do = _inputs(BF, 3, 333, 333, 6, 2, 64, 2, E, seed=12)
    first = None
    for n in range(4):
        stream = torch.cuda.Stream() if n % 2 else None
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        o, lse = P.rel_attention(q, k, v, table, E, want_lse=True, stream=stream)
        got = (o, lse, *P.rel_attention_grad(do, q, k, v, o, lse, table, E, stream=stream))
        torch.cuda.synchronize()
        assert first is None or all(torch.equal(a, b) for a, b in zip(first, got))
        first = got


def test_in_a_graph():
    """Captured and replayed with other work between, the calls give what they give outside."""
    q, k, v, table, do = _inputs(BF, 2, 200, 200, 4, 1, 64, 1, E, seed=13)
    kw = dict(causal=True)
    o, lse = P.rel_attention(q, k, v, table, E, want_lse=True, **kw)
    want = (o, lse, *P.rel_attention_grad(do, q, k, v, o, lse, table, E, **kw))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o, lse = P.rel_attention(q, k, v, table, E, want_lse=True, **kw)
        got = (o, lse, *P.rel_attention_grad(do, q, k, v, o, lse, table, E, **kw))
    for _ in range(3):
        for t in got:
            t.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_empty_calls():
    q, k, v, table, do = _inputs(BF, 2, 10, 10, 2, 2, 32, 1, E, seed=14)
    none = k[:, :0]
    o, lse = P.rel_attention(q, none, none, table, E, want_lse=True)
    assert not o.any() and torch.isinf(lse).all()
    dq, dk, dv, dt = P.rel_attention_grad(do, q, none, none, o, lse, table, E)
    assert not dq.any() and dk.shape[1] == 0 and not dt.any()
    o, lse = P.rel_attention(q[:, :0], k, v, table, E, want_lse=True)
    dq, dk, dv, dt = P.rel_attention_grad(do[:, :0], q[:, :0], k, v, o, lse, table, E)
    assert o.shape[1] == 0 and not dk.any() and not dv.any() and not dt.any()
    o, lse = P.rel_attention(q[:0], k[:0], v[:0], table, E, want_lse=True)
    assert not P.rel_attention_grad(do[:0], q[:0], k[:0], v[:0], o, lse, table, E)[3].any()


def test_refusals_of_the_binding():
    q, k, v, table, do = _inputs(BF, 2, 10, 10, 2, 2, 32, 1, E, seed=15)
    for bad in (dict(k=k.half()), dict(table=table.float()), dict(table=table[:5]), dict(v=v[:, :5]), dict(q_len=torch.ones(2, dtype=torch.int64).cuda())):
        with pytest.raises(AssertionError):
            P.rel_attention(**{**dict(q=q, k=k, v=v, table=table, edges=E), **bad})
    for bad in (dict(scale=0.0), dict(edges=E[::-1].copy()), dict(q=q[:, :, :1].expand(2, 10, 3, 32), table=None)):
        with pytest.raises(P.PrunerError):
            P.rel_attention(**{**dict(q=q, k=k, v=v, table=table, edges=E), **bad})
    with pytest.raises(P.PrunerError):
        P.rel_attention(q, k, v, table, E, workspace=torch.empty(0, dtype=torch.uint8, device="cuda"), scale=-1.0)
