"""The operators of a token step together, as a served model uses them: against the definitions in 64 bits, with what each step rounds; captured and replayed; what calls on a given stream
allocate; the kernels that only large calls reach."""
import os
import sys

import numpy as np
import pytest
import torch

import block_reference as block
import paper_2402_02361_amd as P
import token_reference as ref

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu
BF, HALF, F32 = torch.bfloat16, torch.float16, torch.float32


def _ints(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


class Layer:
    """A layer's attention as it is served: a packed projection, rotary positions, the cache, attention, a packed projection back."""

    def __init__(self, seed, dim, q_heads, kv_heads, head_dim, batch, seq_pages, page_tokens, dtype):
        gen = torch.Generator().manual_seed(seed)
        self.q_heads, self.kv_heads, self.head_dim, self.dtype = q_heads, kv_heads, head_dim, dtype
        self.wide = P.weights_pack((torch.randn((q_heads + 2 * kv_heads) * head_dim, dim, generator=gen) * dim ** -0.5).cuda(), 64)
        self.back = P.weights_pack((torch.randn(dim, q_heads * head_dim, generator=gen) * (q_heads * head_dim) ** -0.5).cuda(), 32)
        self.freqs = P.rotary_frequencies(head_dim, factor=4.0, trained=64)
        order = np.random.default_rng(seed).permutation(batch * seq_pages + 2)[:batch * seq_pages].reshape(batch, seq_pages)
        self.cache = P.new_cache(batch * seq_pages + 2, kv_heads, head_dim, _ints(order), page_tokens)

    def step(self, x, q_len, k_len, **kw):
        """x [batch, tokens, dim]: the layer's output, and what it was made from."""
        batch, tokens, dim = x.shape
        qkv = P.weights_linear(x.reshape(-1, dim), self.wide, **kw).view(batch, tokens, -1, self.head_dim)
        hq, hk = self.q_heads, self.kv_heads
        q, k = P.rotary(qkv[:, :, :hq], qkv[:, :, hq:hq + hk], self.freqs, q_len=q_len, k_len=k_len, **kw)
        P.cache_append(self.cache, k, qkv[:, :, hq + hk:], q_len=q_len, k_len=k_len, **kw)
        o = P.cache_attention(q, self.cache, q_len=q_len, k_len=k_len, **kw)
        return P.weights_linear(o.view(batch * tokens, hq * self.head_dim), self.back, **kw).view(batch, tokens, dim), (qkv, q, k, o)


def _check_step(layer, x, q_len, k_len, room):
    """Each operator against its definition on what the one before gave."""
    y, (qkv, q, k, o) = layer.step(x, q_len, k_len)
    hq, hk, dt, u = layer.q_heads, layer.kv_heads, layer.dtype, ref.UNIT[layer.dtype]
    batch, tokens, dim = x.shape
    ql, kl = q_len.cpu().numpy(), k_len.cpu().numpy()
    for a, w, out in ((x.reshape(-1, dim), layer.wide, qkv), (o.reshape(batch * tokens, -1), layer.back, y)):
        dense = ref.cpu(P.weights_restore(w, F32))
        want, size = ref.cpu(a) @ dense.T, np.abs(ref.cpu(a)) @ np.abs(dense).T
        # (bfloat16: sums of terms of up to 136 |x| times a group's scale, of which a weight is at most 7: 136 sum |x| scale <= 136 x groups' largest; taken as 2^-14 of the terms' size and of |x|'s)
        spread = np.abs(ref.cpu(a)).sum(1)[:, None] * np.abs(dense).max(1)[None, :]
        assert (np.abs(ref.cpu(out).reshape(want.shape) - want) <= 1.01 * u * np.abs(want) + 2.0 ** -14 * size + 2.0 ** -15 * spread + ref.TINY[dt]).all()
    at = (kl - ql)[:, None] + np.arange(tokens)[None, :]
    for a, b in ((qkv[:, :, :hq], q), (qkv[:, :, hq:hq + hk], k)):
        want, size = ref.rotary(ref.cpu(a), layer.freqs, at)
        assert (np.abs(ref.cpu(b) - want) <= 1.01 * u * np.abs(want) + 10 * ref.F32 * size + ref.TINY[dt]).all()
    kk, vv = (ref.cpu(t) for t in P.cache_restore(layer.cache, room, k_len, F32))
    for b in range(batch):   # the new tokens are the rounded ones: half a step of e4m3, or of its smallest one under the page's largest
        new, got = ref.cpu(k)[b, :ql[b]], kk[b, kl[b] - ql[b]:kl[b]]
        assert (np.abs(got - new) <= 2.0 ** -4 * np.abs(new) + 2.0 ** -10 * np.abs(kk[b]).max() / 200).all()
    want = block.attention(ref.cpu(q), kk, vv, q_len=ql, k_len=kl, causal=True)
    bound = block.attention_bounds(want, dt)["o"]
    assert (np.abs(ref.cpu(o) - want["o"]) <= bound).all()
    return y


@pytest.mark.parametrize("dtype", [BF, HALF])
@pytest.mark.parametrize("dim,q_heads,kv_heads,head_dim,page_tokens", [(200, 4, 2, 64, 16), (96, 8, 1, 32, 64), (300, 6, 3, 128, 32)])
def test_a_prompt_and_then_token_by_token(dtype, dim, q_heads, kv_heads, head_dim, page_tokens):
    gen = torch.Generator().manual_seed(dim)
    layer = Layer(dim, dim, q_heads, kv_heads, head_dim, 3, -(-120 // page_tokens), page_tokens, dtype)
    n = np.array([60, 1, 33])
    x = torch.randn(3, 60, dim, generator=gen).to(dtype).cuda()
    _check_step(layer, x, _ints(n), _ints(n), 60)
    for new in ([1, 1, 1], [1, 1, 1], [3, 0, 2], [1, 1, 1], [20, 31, 9]):
        n = n + np.array(new)
        x = torch.randn(3, max(new), dim, generator=gen).to(dtype).cuda()
        _check_step(layer, x, _ints(new), _ints(n), int(n.max()))


def test_captured_and_replayed():
    """A step in a graph, its inputs changed in place between replays, leaves the bits that eager steps leave; two graphs of two layers share nothing."""
    gen = torch.Generator().manual_seed(1)
    dim, batch = 128, 2
    layers = [Layer(s, dim, 4, 2, 64, batch, 60, 16, BF) for s in (1, 1, 2, 2)]   # each one twice: replayed and eager
    for layer in layers:
        for t in layer.cache[:4]:
            t.zero_()
    x, k_len, q_len = torch.zeros(batch, 1, dim, dtype=BF, device="cuda"), _ints([1, 1]), _ints([1, 1])
    warm = Layer(1, dim, 4, 2, 64, batch, 60, 16, BF)
    warm.step(x, q_len, k_len)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for layer in (layers[0], layers[2]):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(layer.step(x, q_len, k_len)[0])
    for n in range(40):
        x.copy_(torch.randn(batch, 1, dim, generator=gen))
        k_len.copy_(torch.tensor([n + 1, 900 if n == 39 else 2 * n + 1], dtype=torch.int32))
        for g in graphs:
            g.replay()
        want = [layer.step(x, q_len, k_len)[0] for layer in (layers[1], layers[3])]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
        for a, b in ((0, 1), (2, 3)):
            assert all(torch.equal(s, t) for s, t in zip(layers[a].cache[:4], layers[b].cache[:4]))


def test_on_a_given_stream():
    """What calls on a given stream allocate is not given away while that stream still works with it."""
    gen = torch.Generator().manual_seed(2)
    layer, other = (Layer(3, 256, 8, 2, 64, 2, 100, 64, BF) for _ in range(2))
    x, n = torch.randn(2, 3, 256, generator=gen).to(BF).cuda(), _ints([3, 3])
    long = _ints([6400, 5000])
    filled = torch.randn(2, 6400, 2, 64, generator=gen).to(BF).cuda()
    for one in (layer, other):
        P.cache_append(one.cache, filled, filled)
    want = layer.step(x, n, long)[0]
    a = torch.randn(4096, 4096, device="cuda", dtype=BF)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(60):   # (several milliseconds before the call's first launch)
            a @ a
    got = other.step(x, n, long, stream=side)[0]
    junk = [torch.full((1 << b,), float("nan"), device="cuda") for b in range(22, 6, -1) for _ in range(3)]
    torch.cuda.synchronize()
    assert torch.equal(got, want) and all(j.isnan().all() for j in junk)


def test_the_example_of_a_sequence_that_grows():
    """With weights that 4 bits hold exactly, what is left between the example's two ways are roundings of keys and values to 8 bits: half a step, 2^-4, of a value and of a score's terms."""
    from flow_block import FlowModel, synthetic
    model = FlowModel(seed=7)
    for name in ("embed", "qkv"):
        packed = P.weights_pack(model.weight(name))
        model.p[name].copy_(P.weights_restore(packed, BF))
        # (restored values round to bfloat16, so packing them again may differ by that: 2^-8 of a weight)
    flows = synthetic(5, 8, 8)[0]
    small = model.grow_small(flows)
    for i in range(5):
        want = model.grow(flows[i]).float()
        assert (small[i].float() - want).abs().max() <= 0.25 * want.abs().max() and (small[i].float() - want).norm() <= 0.1 * want.norm()


# ---- kernels that only large calls reach

def test_rotary_past_the_caches():
    """Inputs of more than 128 MB: the same bits as parts of them."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    for dtype, tokens, heads, head_dim in ((BF, 18001, 30, 128), (F32, 32001, 11, 100), (HALF, 20001, 44, 90)):
        q = torch.randn(1, tokens, heads, head_dim, generator=gen, device="cuda").to(dtype)
        for interleaved in (False, True):
            freqs = P.rotary_frequencies(head_dim // 4 * 2)
            whole = P.rotary(q, None, freqs, interleaved=interleaved)[0]
            for lo in (0, 1000, tokens - 77):
                part = P.rotary(q[:, lo:lo + 77], None, freqs, k_len=_ints([lo + 77]), interleaved=interleaved)[0]
                assert torch.equal(part, whole[:, lo:lo + 77])


@pytest.mark.parametrize("q_tokens,group", [(1, 1), (4, 4), (5, 4)])
def test_attention_past_the_caches(q_tokens, group):
    """More room than the caches hold, short sequences: the same as with less room, whatever the parts (each row's sum is of the same terms)."""
    gen = torch.Generator().manual_seed(4)
    batch, hk, d, t, seq_pages = 3, 2, 128, 64, 3000
    k, v = (torch.randn(batch, 700, hk, d, generator=gen).to(BF).cuda() for _ in range(2))
    q = torch.randn(batch, q_tokens, hk * group, d, generator=gen).to(BF).cuda()
    n = _ints([700, 5, 333])
    pages = np.full((batch, seq_pages), -1, np.int32)
    pages[:, :11] = np.random.default_rng(5).permutation(33).reshape(3, 11)
    large = P.new_cache(33, hk, d, _ints(pages), t)
    P.cache_append(large, k, v)
    small = large._replace(table=_ints(pages[:, :11]))
    a, b = (P.cache_attention(q, c, k_len=n, want_lse=True) for c in (large, small))
    kk, vv = (ref.cpu(x) for x in P.cache_restore(small, 700, n, F32))
    ql = [q_tokens] * batch
    want = block.attention(ref.cpu(q), kk, vv, q_len=ql, k_len=[700, 5, 333], causal=True)
    for o, lse in (a, b):
        assert (np.abs(ref.cpu(o) - want["o"]) <= block.attention_bounds(want, BF)["o"]).all()
        assert np.allclose(ref.cpu(lse), want["lse"], atol=1e-5, rtol=2e-6)


def test_restore_past_the_caches():
    """Results of more than 128 MB: the same as parts of them."""
    rng = np.random.default_rng(6)
    cache = P.new_cache(300, 4, 128, _ints(rng.permutation(300)[:280].reshape(2, 140)), 64)
    for t, lo, hi in zip(cache[:4], (0, 0, 100, 100), (120, 120, 130, 130)):
        t.copy_(torch.from_numpy(rng.integers(lo, hi, t.shape, dtype=np.uint8)))
    n = _ints([8900, 4001])
    for dtype in (F32, BF):   # (146 MB, and half of it)
        whole = P.cache_restore(cache, 8900, n, dtype)
        for b in range(2):
            one = cache._replace(table=cache.table[b:b + 1].contiguous())
            for i in (0, 1):
                assert torch.equal(P.cache_restore(one, 900, n[b:b + 1], dtype)[i][0], whole[i][b, :900])
        assert not whole[0][1, 4001:].any() and whole[0][1, 4000].any()


def test_weights_past_the_caches():
    """More codes than 96 MB: outputs are those of the rows' own packed weights."""
    w = torch.randn(16384, 13000, generator=torch.Generator(device="cuda").manual_seed(7), device="cuda", dtype=BF)
    x = torch.randn(5, 13000, generator=torch.Generator(device="cuda").manual_seed(8), device="cuda", dtype=BF)
    y = P.weights_linear(x, P.weights_pack(w, 128))
    for lo in (0, 8192, 16384 - 512 * 16):
        assert torch.equal(P.weights_linear(x, P.weights_pack(w[lo:lo + 8192], 128)), y[:, lo:lo + 8192])
