"""cache_append and cache_restore against a model of a cache that is written token by token in 64 bits: codes and exponents are equal."""
import numpy as np
import pytest
import torch

import paper_2402_02361_amd as P
import token_reference as ref

pytestmark = pytest.mark.gpu
BF, HALF, F32 = torch.bfloat16, torch.float16, torch.float32


def _ints(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def _table(rng, batch, seq_pages, spare=3):
    total = batch * seq_pages + spare
    return rng.permutation(total)[:batch * seq_pages].reshape(batch, seq_pages).astype(np.int32), total


class Model:
    """A Cache and its model side by side; unused memory holds random bytes."""

    def __init__(self, seed, batch, seq_pages, heads, head_dim, page_tokens, table=None, pages=None):
        self.rng = np.random.default_rng(seed)
        if table is None:
            table, pages = _table(self.rng, batch, seq_pages)
        self.table = table
        self.cache = P.new_cache(pages, heads, head_dim, _ints(table), page_tokens)
        for t, first, last in zip(self.cache[:4], (0, 0, 1, 1), (255, 255, 254, 254)):   # (exponent bytes are 1 .. 254)
            t.copy_(torch.from_numpy(self.rng.integers(first, last + 1, t.shape, dtype=np.uint8)))
        self.read()

    def read(self):
        k, v, ke, ve = (t.cpu().numpy() for t in self.cache[:4])
        self.k, self.v, self.ke, self.ve = ref.keys_of(k), ref.values_of(v), ke.copy(), ve.copy()

    def append(self, k, v, q_len, k_len, **kw):
        P.cache_append(self.cache, k, v, q_len=None if q_len is None else _ints(q_len), k_len=None if k_len is None else _ints(k_len), **kw)
        batch, tokens = k.shape[:2]
        n = [tokens] * batch if q_len is None else q_len
        kl = n if k_len is None else k_len
        for codes, exps, x in ((self.k, self.ke, k), (self.v, self.ve, v)):
            ref.append(codes, exps, self.table, ref.cpu(x), n, kl)
        self.check()

    def check(self):
        k, v, ke, ve = (t.cpu().numpy() for t in self.cache[:4])
        k, v = ref.keys_of(k), ref.values_of(v)
        assert np.array_equal(ke, self.ke) and np.array_equal(ve, self.ve)
        for got, want in ((k, self.k), (v, self.v)):
            nan = (want & 127) == 127
            assert np.array_equal(got[~nan], want[~nan]) and ((got[nan] & 127) == 127).all()

    def restored(self, tokens, k_len, dtype):
        k, v = P.cache_restore(self.cache, tokens, _ints(k_len), dtype)
        for got, codes, exps in ((k, self.k, self.ke), (v, self.v, self.ve)):
            want, there = ref.dense(codes, exps, self.table, tokens, np.clip(k_len, 0, tokens))
            want = torch.from_numpy(want).to(dtype).double().numpy()   # (exact within the type's range)
            assert got.shape == want.shape and np.array_equal(ref.cpu(got), want, equal_nan=True)
        return k, v


def _new(rng, dtype, *shape, scale=1.0):
    x = rng.standard_normal(shape) * np.exp(rng.standard_normal(shape[:2] + (1, 1))) * np.exp(0.7 * rng.standard_normal((1, 1) + shape[2:])) * scale
    return torch.from_numpy(x).to(dtype).cuda()


@pytest.mark.parametrize("dtype", [BF, HALF, F32])
@pytest.mark.parametrize("batch,heads,head_dim,page_tokens,tokens,before", [
    (1, 1, 16, 16, 1, 0), (3, 2, 64, 64, 1, 100), (2, 3, 128, 32, 70, 5), (2, 1, 80, 16, 33, 15), (1, 2, 32, 128, 300, 127), (4, 1, 48, 256, 2, 255), (1, 8, 128, 64, 64, 64), (2, 2, 112, 16, 16, 8)])
def test_append_and_restore(dtype, batch, heads, head_dim, page_tokens, tokens, before):
    m = Model(tokens + head_dim, batch, -(-(before + 2 * tokens + 2) // page_tokens), heads, head_dim, page_tokens)
    if before:
        m.append(_new(m.rng, dtype, batch, before, heads, head_dim), _new(m.rng, dtype, batch, before, heads, head_dim), None, None)
    n = [max(0, before - 3 * b) for b in range(batch)]   # (shorter sequences write over what is behind them)
    for scale in (1.0, 30.0):   # the second time exponents grow
        m.append(_new(m.rng, dtype, batch, tokens, heads, head_dim, scale=scale), _new(m.rng, dtype, batch, tokens, heads, head_dim, scale=scale), None, [x + tokens for x in n])
        n = [x + tokens for x in n]
    m.restored(max(n), n, dtype)
    m.restored(max(n) + 1, [x - 1 for x in n], F32)


def test_token_by_token():
    """Sixty steps of sequences of different lengths, of one to three tokens each, sizes that grow and shrink by large factors."""
    m = Model(1, 3, 6, 2, 32, 16)
    n = np.array([0, 5, 17])
    m.append(_new(m.rng, BF, 3, 17, 2, 32), _new(m.rng, BF, 3, 17, 2, 32), n, n)
    for step in range(30):
        new = m.rng.integers(0, 4, 3)
        n = n + new
        scale = 2.0 ** m.rng.integers(-12, 12)
        m.append(_new(m.rng, BF, 3, 3, 2, 32, scale=scale), _new(m.rng, BF, 3, 3, 2, 32, scale=1 / scale), new, n)
    m.restored(int(n.max()), n, F32)


def test_lengths_outside_and_tokens_that_have_no_place():
    """q_len is clamped; tokens before the first place or behind the last page are left out, the others are stored."""
    m = Model(2, 6, 3, 1, 16, 16)
    k, v = _new(m.rng, F32, 6, 20, 1, 16), _new(m.rng, F32, 6, 20, 1, 16)
    m.append(k, v, [-3, 99, 20, 20, 20, 0], [5, 20, 10, 58, 400, 30])
    m.append(k, v, [20, 20, 20, 3, 1, 1], [-7, 2 ** 31 - 1, 48, 49, 0, 1])
    m.restored(48, [48, -3, 1000, 47, 0, 33], BF)


def test_pages_that_are_not_there():
    table = np.array([[0, -1, 2, 7], [5, 4, 1 << 30, -2 ** 31], [-1, -1, -1, 3]], np.int32)
    m = Model(3, 3, 4, 2, 64, 16, table=table, pages=7)
    m.append(_new(m.rng, BF, 3, 64, 2, 64), _new(m.rng, BF, 3, 64, 2, 64), None, None)
    m.restored(64, [64, 64, 64], BF)


def test_infinities_and_nan_are_their_own():
    """They become NaN where they stand; the page's exponent is that of what is finite, or the smallest one."""
    m = Model(4, 2, 1, 1, 32, 32)
    k, v = _new(m.rng, F32, 2, 20, 1, 32), _new(m.rng, F32, 2, 20, 1, 32)
    k[0, 3, 0, 4], k[0, 5, 0, 5], v[0, 19, 0, 31], v[0, 0, 0, 0] = float("inf"), float("nan"), float("-inf"), float("nan")
    k[1], v[1] = float("nan"), float("inf")
    m.append(k, v, None, None)
    assert m.ke[m.table[1, 0], 0] == 1
    k = _new(m.rng, F32, 2, 2, 1, 32)
    m.append(k, k, None, [22, 22])   # (older tokens that are NaN stay so when the exponent grows)
    m.restored(22, [22, 22], F32)


@pytest.mark.parametrize("dtype,values", [(F32, [0.0, 1e-45, 1e-38, 448.0, 448.1, 1.75 * 2.0 ** 100, 3.4e38, 3e-39]), (BF, [0.0, 9.2e-41, 448.0, 450.0, 3.38e38, 1e-30]), (HALF, [0.0, 6e-8, 448.0, 448.5, 65504.0, 1e-4])])
def test_the_largest_and_the_smallest(dtype, values):
    for x in values:
        m = Model(5, 1, 1, 1, 16, 16)
        t = torch.full((1, 3, 1, 16), x, dtype=dtype).cuda()
        t[0, 0, 0, ::2] *= -0.37
        m.append(t, t, None, None)
        m.restored(3, [3], F32)


def test_strides():
    """Parts of a fused projection, heads before tokens, rows that begin anywhere: the same bytes."""
    rng = np.random.default_rng(6)
    kv = _new(rng, BF, 2, 40, 7, 67)
    k, v = kv[:, :, :2, 1:65], kv[:, :, 4:6, 3:67]
    heads_first = lambda t: t.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)  # noqa: E731
    table, pages = _table(rng, 2, 3)
    want = None
    for a, b in ((k.contiguous(), v.contiguous()), (k, v), (heads_first(k), heads_first(v))):
        cache = P.new_cache(pages, 2, 64, _ints(table), 16)
        for t in cache[:4]:
            t.zero_()
        P.cache_append(cache, a, b)
        want = want or cache
        assert all(torch.equal(x, y) for x, y in zip(cache[:4], want[:4]))


@pytest.mark.parametrize("page_tokens", [16, 64])
def test_sequences_that_share_a_full_page(page_tokens):
    """The same as sequences with that page's tokens for themselves."""
    rng = np.random.default_rng(17)
    n, heads, d = page_tokens + 5, 2, 48
    k, v = _new(rng, BF, 2, n, heads, d), _new(rng, BF, 2, n, heads, d)
    k[1, :page_tokens], v[1, :page_tokens] = k[0, :page_tokens], v[0, :page_tokens]
    shared, own = P.new_cache(4, heads, d, _ints([[2, 0], [2, 3]]), page_tokens), P.new_cache(4, heads, d, 2, page_tokens)
    P.cache_append(own, k, v)
    P.cache_append(shared, k[:, :page_tokens], v[:, :page_tokens], _ints([page_tokens, 0]), _ints([page_tokens, 0]))
    P.cache_append(shared, k[:, page_tokens:], v[:, page_tokens:], None, _ints([n, n]))
    lengths = _ints([n, n - 2])
    for x, y in zip(P.cache_restore(shared, n, lengths, BF), P.cache_restore(own, n, lengths, BF)):
        assert torch.equal(x, y)
    for tokens in (1, 17, 40):   # (two rows to a key head, so few columns, and many)
        q = _new(rng, BF, 2, tokens, 4, d)
        assert torch.equal(P.cache_attention(q, shared, k_len=lengths), P.cache_attention(q, own, k_len=lengths))


def test_the_end_of_binary16s_range():
    """Values from 31/32 of 2^16 on round to 2^16, which binary16 does not have; what lies below rounds down to 15/16 of it."""
    for x, want in ((65504.0, float("inf")), (63488.0, float("inf")), (63456.0, 61440.0)):
        cache = P.new_cache(1, 1, 16, 1, 16)
        t = torch.full((1, 1, 1, 16), x, dtype=HALF).cuda()
        P.cache_append(cache, t, -t)
        k, v = P.cache_restore(cache, 1, _ints([1]), HALF)
        assert (k == want).all() and (v == -want).all()


def test_pages_in_a_row_without_a_table():
    """A number of pages for a table: the same as the table that says so."""
    rng = np.random.default_rng(7)
    k, v = _new(rng, HALF, 3, 50, 2, 32), _new(rng, HALF, 3, 50, 2, 32)
    got, want = P.new_cache(13, 2, 32, 4, 16), P.new_cache(13, 2, 32, _ints(np.arange(12).reshape(3, 4)), 16)
    for cache in (got, want):
        for t in cache[:4]:
            t.zero_()
        P.cache_append(cache, k, v)
    assert all(torch.equal(a, b) for a, b in zip(got[:4], want[:4]))
    n = _ints([50, 7, 64])
    assert all(torch.equal(a, b) for a, b in zip(P.cache_restore(got, 60, n, HALF), P.cache_restore(want, 60, n, HALF)))


def test_a_pool_beyond_4_gib():
    """Pages at its end are written and read where they are."""
    pages, heads, d, t = 2 ** 32 // (64 * 128 * 8) + 1000, 8, 128, 64
    cache = P.new_cache(pages, heads, d, _ints([[3, pages - 1], [pages - 2, 7]]), t)
    rng = np.random.default_rng(8)
    k, v = _new(rng, BF, 2, 100, heads, d), _new(rng, BF, 2, 100, heads, d)
    P.cache_append(cache, k, v)
    small = P.new_cache(4, heads, d, _ints([[0, 1], [2, 3]]), t)
    P.cache_append(small, k, v)
    n = _ints([100, 100])
    for a, b in zip(P.cache_restore(cache, 100, n, BF), P.cache_restore(small, 100, n, BF)):
        assert torch.equal(a, b)
    q = _new(rng, BF, 2, 1, 16, d)
    assert torch.equal(P.cache_attention(q, cache, k_len=n), P.cache_attention(q, small, k_len=n))
    q = _new(rng, BF, 2, 40, 16, d)
    assert torch.equal(P.cache_attention(q, cache, k_len=n), P.cache_attention(q, small, k_len=n))


def test_empty_calls_and_a_pool_without_pages():
    m = Model(9, 2, 2, 2, 32, 16)
    k = _new(m.rng, BF, 2, 5, 2, 32)
    m.append(k[:, :0], k[:, :0], None, [5, 5])
    m.append(k, k, [0, 0], [5, 40])
    k0, v0 = P.cache_restore(m.cache, 0, _ints([1, 1]), BF)
    assert k0.shape == (2, 0, 2, 32)
    none = P.new_cache(0, 2, 32, _ints([[0], [0]]), 16)
    P.cache_append(none, k, k)
    got, _ = P.cache_restore(none, 16, _ints([5, 5]), BF)
    assert not got.any()
    assert not P.cache_attention(k, none, k_len=_ints([5, 5])).any()
    empty = P.new_cache(3, 2, 32, torch.zeros(2, 0, dtype=torch.int32, device="cuda"), 16)
    P.cache_append(empty, k, k)
    assert not P.cache_attention(k, empty).any()


def test_streams_and_graphs():
    """Captured steps, replayed with new tokens in place, leave what eager steps leave."""
    rng = np.random.default_rng(10)
    a, b = (P.new_cache(8, 2, 32, _ints([[1, 3, 5], [0, 6, 2]]), 16) for _ in range(2))
    for t, u in zip(a[:4], b[:4]):
        t.zero_(), u.zero_()
    k, v, n = _new(rng, BF, 2, 1, 2, 32), _new(rng, BF, 2, 1, 2, 32), _ints([1, 1])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.cache_append(a, k, v, k_len=n)
        got = P.cache_restore(a, 48, n, BF)
    for step in range(20):
        k.copy_(_new(rng, BF, 2, 1, 2, 32, scale=2.0 ** (step % 7))), v.copy_(_new(rng, BF, 2, 1, 2, 32))
        n.fill_(step + 1)
        graph.replay()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        P.cache_append(b, k, v, k_len=n, stream=side)
        want = P.cache_restore(b, 48, n, BF, stream=side)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(a[:4], b[:4])) and all(torch.equal(x, y) for x, y in zip(got, want))


def test_refusals_of_the_binding():
    cache = P.new_cache(4, 2, 32, _ints([[0, 1], [2, 3]]), 16)
    k = torch.zeros(2, 5, 2, 32, dtype=BF, device="cuda")
    for bad in (dict(k=k[:, :, :1]), dict(v=k.half()), dict(v=k[:, :4]), dict(k=k[:1], v=k[:1]), dict(cache=cache._replace(k_exps=cache.k_exps[:3])), dict(cache=cache._replace(v_codes=cache.k_codes)),
                dict(cache=cache._replace(table=cache.table.long())), dict(q_len=torch.zeros(3, dtype=torch.int32).cuda()), dict(k=k.cpu(), v=k.cpu()), dict(k=k.transpose(2, 3), v=k.transpose(2, 3))):
        with pytest.raises(AssertionError):
            P.cache_append(**{**dict(cache=cache, k=k, v=k), **bad})
    with pytest.raises(AssertionError):
        P.new_cache(4, 2, 40, 2)
    with pytest.raises(P.PrunerError):
        P.cache_append(cache, k.double(), k.double())
    with pytest.raises(P.PrunerError):
        P.cache_restore(cache, 33, _ints([1, 1]), BF)
    with pytest.raises(P.PrunerError):
        P.cache_append(cache._replace(table=3), k, k)   # four pages are not two times three
