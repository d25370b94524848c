"""The block's operators where a call is large enough for the forms that small ones do not reach: large tiles of the weight gradient, norms whose workgroups take several rows in
turn, long axes cut into parts and their joins, diagonals of many workgroups; lengths and padding on every route; the backward pass from the forward pass's own results;
graphs."""
import numpy as np
import pytest
import torch

import block_reference as ref
import paper_2402_02361_amd as P
from test_gpu_train_checkpoint import _wgrad
from test_gpu_train_gated_norm import _inputs as norm_inputs, _within as norm_within
from test_gpu_train_rel_attention import E, _check, _inputs, _lengths, _randn

pytestmark = pytest.mark.gpu
BF, HALF, F32 = torch.bfloat16, torch.float16, torch.float32


# ---- the weight gradient: sizes for which one workgroup takes 256 x 256, in parts and not, aligned and odd (the bound is that of the small sizes' test)
@pytest.mark.parametrize("dtype,rows,n_out,dim", [(BF, 8192, 2048, 1024), (HALF, 8190, 2000, 1000), (HALF, 2000, 1601, 903), (BF, 4001, 1031, 1000), (BF, 500, 4096, 4096), (HALF, 130, 4095, 4093)])
def test_weight_gradient_by_large_tiles(dtype, rows, n_out, dim):
    dy, kept, want, size = _wgrad(dtype, rows, n_out, dim, seed=rows)
    bound = (rows / 8 + 8) * ref.F32 * size
    got = P.checkpoint_wgrad(dy, kept)
    assert (np.abs(ref.cpu(got) - want) <= bound).all()
    again = P.checkpoint_wgrad(dy, kept)
    assert torch.equal(got, again)
    P.checkpoint_wgrad(dy, kept, dw=again, accumulate=True)
    assert (np.abs(ref.cpu(again) - 2 * want) <= 2 * bound + 2 * ref.F32 * np.abs(want)).all()


# ---- norms: more rows than the device's workgroups take at once, for rows of part of a wavefront, of two, of three, of ten and of sixteen, in eights and from anywhere
NORM_SHAPES = [(40000, 96), (40000, 99), (9000, 1024), (9000, 1021), (4000, 1104), (4000, 1101), (1500, 5000), (1500, 5001), (700, 8192), (700, 8189)]


@pytest.mark.parametrize("rows,dim", NORM_SHAPES)
def test_norms_of_many_rows(rows, dim):
    dtype, gate, center = ((BF, "rows", False), (HALF, "vector", True), (F32, "rows", True))[(rows + dim) % 3]
    x, f, dh, dy, w1, w2, g = norm_inputs(dtype, rows, dim, gate, seed=dim)
    h, y, kept = P.gated_norm(x, f, w1, w2, gate=g, alpha=0.7, center=center, checkpoint=True)
    got = P.gated_norm_grad(dh, dy, x, f, w1, w2, gate=g, alpha=0.7, center=center)
    # rows are each for itself: a sample of them, the last ones among it
    some = np.unique(np.concatenate([np.arange(0, rows, max(1, rows // 400)), np.arange(rows - 40, rows)]))
    pick = lambda t: t[torch.from_numpy(some).cuda()]  # noqa: E731
    rows_gate = gate == "rows"
    want = ref.norm(*(ref.cpu(t) for t in (pick(x), pick(f), w1, w2, pick(g) if rows_gate else g)), float(np.float32(0.7)), float(np.float32(1e-6)), center, ref.cpu(pick(dh)), ref.cpu(pick(dy)))
    norm_within(pick(h), want["h"], want["h_abs"], dtype, "h")
    norm_within(pick(y), want["y"], want["y_abs"], dtype, "y")
    norm_within(pick(got[0]), want["dx"], want["dx_abs"], dtype, "dx")
    norm_within(pick(got[1]), want["df"], want["df_abs"], dtype, "df")
    if rows_gate:
        norm_within(pick(got[2]), want["dgate"], want["dgate_abs"], dtype, "dgate")
    codes, exps = ref.pack(ref.cpu(pick(y)[-60:]))
    assert np.array_equal(codes, pick(kept.codes)[-60:].cpu().numpy()) and np.array_equal(exps, pick(kept.exps)[-60:].cpu().numpy())


@pytest.mark.parametrize("rows,dim", NORM_SHAPES)
def test_sums_over_many_rows_have_every_row(rows, dim):
    """All gradients but those of sixty rows, the last ones among them, are zero: the sums over the rows are those rows' sums."""
    x, f, dh, dy, w1, w2, g = norm_inputs(F32, rows, dim, "vector", seed=dim + 1)
    rng = np.random.default_rng(rows)
    some = np.unique(np.concatenate([rng.integers(0, rows, 50), np.arange(rows - 10, rows)]))
    at = torch.from_numpy(some).cuda()
    only = torch.zeros(rows, 1, device="cuda").index_fill_(0, at, 1.0)
    _, _, dgate, dw1, dw2 = P.gated_norm_grad(dh * only, dy * only, x, f, w1, w2, gate=g)
    want = ref.norm(*(ref.cpu(t) for t in (x[at], f[at], w1, w2, g)), 1.0, float(np.float32(1e-6)), False, ref.cpu(dh[at]), ref.cpu(dy[at]))
    norm_within(dw1, want["dw_post"], want["dw_post_abs"], F32, "dw_post", len(some))
    norm_within(dw2, want["dw_pre"], want["dw_pre_abs"], F32, "dw_pre", len(some))
    norm_within(dgate, want["dgate"].sum(0), want["dgate_abs"].sum(0), F32, "dgate", len(some))


# ---- attention: many workgroups' diagonals, and long axes in parts
@pytest.mark.parametrize("shape,sides", [((70, 8, 8, 2, 1, 32), 2), ((40, 30, 60, 1, 1, 64), 1), ((33, 130, 130, 1, 1, 32), 2), ((1, 1500, 1500, 2, 1, 32), 1), ((2, 520, 2600, 1, 1, 64), 2),
                                         ((1, 2000, 300, 2, 2, 128), 2), ((1, 40, 6000, 2, 1, 128), 1), ((1, 130, 9000, 1, 1, 64), 2)])
@pytest.mark.parametrize("causal", [False, True])
def test_many_workgroups_and_long_axes(shape, sides, causal):
    dtype = (BF, HALF)[(sum(shape) + causal) % 2]
    _check(*_inputs(dtype, *shape, sides, E, seed=sum(shape), fused=shape[1] == shape[2]), E, causal=causal)


# ---- lengths and padding, on the routes by shared tiles of every width and by few tokens: what the padding holds is NaN and infinity
@pytest.mark.parametrize("dtype", [BF, HALF])
@pytest.mark.parametrize("head_dim", [24, 32, 64, 80, 128])
@pytest.mark.parametrize("q_tokens,k_tokens", [(300, 300), (24, 60), (150, 700)])
def test_padding_does_not_matter(head_dim, q_tokens, k_tokens, dtype):
    q_len, k_len = [q_tokens, 0, q_tokens // 3 + 1, q_tokens - 1], [k_tokens - 1, k_tokens, k_tokens // 2 - 3, 1]
    q, k, v, table, do = _inputs(dtype, 4, q_tokens, k_tokens, 4, 2, head_dim, 2, E, seed=head_dim)
    _poison(((q, q_len), (do, q_len), (k, k_len), (v, k_len)))
    for causal in (False, True):
        _check(q, k, v, table, do, E, q_len, k_len, causal)


@pytest.mark.parametrize("dtype", [BF, HALF])
@pytest.mark.parametrize("head_dim", [24, 64, 80, 128])
@pytest.mark.parametrize("k_tokens", [70, 1300])
def test_padding_of_a_cache_does_not_matter(k_tokens, head_dim, dtype):
    q_len, k_len = [3, 2, 0, 1, 3], [k_tokens, 1, k_tokens - 1, k_tokens // 2 + 5, 2]
    q, k, v, table, do = _inputs(dtype, 5, 3, k_tokens, 8, 2, head_dim, 1, E, seed=head_dim + 1)
    _poison(((q, q_len), (do, q_len), (k, k_len), (v, k_len)))
    _check(q, k, v, table, do, E, q_len, k_len, causal=True, grads=k_tokens < 1000)


def _poison(tensors):
    for t, lengths in tensors:
        for b, n in enumerate(lengths):
            t[b, n:] = float("nan")
            if n + 1 < t.shape[1]:
                t[b, n + 1] = float("inf")


# ---- the forward pass's own results in the backward pass
@pytest.mark.parametrize("dtype", [BF, HALF])
@pytest.mark.parametrize("shape,causal", [((3, 8, 8, 2, 1, 64), False), ((2, 30, 60, 4, 2, 128), True), ((1, 300, 300, 4, 2, 64), True), ((2, 129, 400, 2, 1, 80), False), ((1, 1, 500, 8, 2, 128), True)])
def test_gradients_from_the_forward_pass(shape, causal, dtype):
    """o is off by a rounding of itself and of its weights, and delta with it; lse by 1e-5 and 2e-6 of itself (as test_gpu_train_rel_attention allows), and with it every weight."""
    q, k, v, table, do = _inputs(dtype, *shape, 2, E, seed=sum(shape) + 1)
    o, lse = P.rel_attention(q, k, v, table, E, causal=causal, want_lse=True)
    got = P.rel_attention_grad(do, q, k, v, o, lse, table, E, causal=causal)
    args = [ref.cpu(t) for t in (q, k, v, table)]
    want = ref.attention(*args, E, causal=causal, do=ref.cpu(do))
    # (what the weights' rounding adds to delta: that of o with |v| for v, whose sum over a row bounds it; the reference's own is of |o|)
    wide = ref.attention(args[0], args[1], np.abs(args[2]), args[3], E, causal=causal, do=np.abs(ref.cpu(do)))
    bound = ref.attention_bounds(want, dtype)
    lse_off = 1e-5 + 2e-6 * np.abs(want["lse"][np.isfinite(want["lse"])]).max()
    for name, t in zip(("dq", "dk", "dv", "dtable"), got):
        slip = 0 if name == "dv" else (ref.UNIT[dtype] + ref.EXP) * wide[name + "_delta"]
        b = bound[name] + slip + 2 * lse_off * want[name + "_abs"]
        g = ref.cpu(t)
        worst = np.abs(g - want[name]) / np.maximum(b, 1e-300)
        assert np.isfinite(g).all() and (worst <= 1).all(), f"{name}: {worst.max():.3g} of its bound"


# ---- graphs
def _norm_calls():
    x, f, dh, dy, w1, w2, g = norm_inputs(BF, 3000, 320, "rows", seed=3)

    def call():
        h, y, kept = P.gated_norm(x, f, w1, w2, gate=g, checkpoint=True)
        return (h, y, *kept, *P.gated_norm_grad(dh, dy, x, f, w1, w2, gate=g))

    return call


def _checkpoint_calls():
    gen = torch.Generator().manual_seed(4)
    x, dy = _randn(gen, 6000, 136, dtype=BF), _randn(gen, 6000, 200, dtype=BF)

    def call():
        kept = P.checkpoint_pack(x)
        return (*kept, P.checkpoint_restore(kept, F32), P.checkpoint_wgrad(dy, kept))

    return call


def _few_tokens():
    q, k, v, table, _ = _inputs(HALF, 2, 1, 3000, 8, 2, 64, 1, E, seed=5)
    one, n = _lengths([1, 1]), _lengths([3000, 1700])
    return lambda: P.rel_attention(q, k, v, table, E, q_len=one, k_len=n, causal=True, want_lse=True)


@pytest.mark.parametrize("make", [_norm_calls, _checkpoint_calls, _few_tokens])
def test_in_a_graph(make):
    """Captured and replayed with other work between, the calls give what they give outside."""
    call = make()
    want = [t.clone() for t in call()]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call()
    for _ in range(3):
        for t in got:
            t.fill_(7)
        (torch.ones(1000, 1000, device="cuda") @ torch.ones(1000, 1000, device="cuda")).sum().item()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))
