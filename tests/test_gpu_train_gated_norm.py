"""gated_norm and gated_norm_grad against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

import block_reference as ref
import paper_2402_02361_amd as P

pytestmark = pytest.mark.gpu
# a value is a chain of at most some forty binary32 operations, and sums over a row of up to 8192 values by a tree of 13 levels over
# eight in turn: 64 roundings of the terms' sizes cover both
STEPS = 64 * ref.F32


def _inputs(dtype, rows, dim, gate, seed=0):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    x, f, dh, dy = (r(rows, dim).to(dtype).cuda() for _ in range(4))
    g = None if gate is None else r(rows, dim).to(dtype).cuda() if gate == "rows" else r(dim).cuda()
    return x, f, dh, dy, (1 + 0.3 * r(dim)).cuda(), (1 + 0.3 * r(dim)).cuda(), g


def _within(got, want, size, dtype, what, rows=1):
    u = ref.UNIT[dtype] if got.dtype == dtype else 0.0
    bound = u * np.abs(want) * 1.01 + (STEPS + rows * ref.F32) * size + ref.TINY[dtype] + 1e-30
    g = ref.cpu(got)
    worst = np.abs(g - want) / bound
    assert np.isfinite(g).all() and (worst <= 1).all(), f"{what}: {worst.max():.3g} of its bound"


def _check(x, f, dh, dy, w1, w2, gate, alpha=1.0, center=False, eps=1e-6, checkpoint=False):
    dtype = x.dtype
    h, y, kept = P.gated_norm(x, f, w1, w2, gate=gate, alpha=alpha, eps=eps, center=center, checkpoint=True)
    f_in = f
    if checkpoint:
        f_in = P.checkpoint_pack(f)
        f = P.checkpoint_restore(f_in, torch.float32)
    args = [ref.cpu(t) for t in (x, f, w1, w2, gate)]
    alpha, eps = float(np.float32(alpha)), float(np.float32(eps))
    want = ref.norm(*args, alpha, eps, center, ref.cpu(dh), ref.cpu(dy))
    if not checkpoint:
        _within(h, want["h"], want["h_abs"], dtype, "h")
        _within(y, want["y"], want["y_abs"], dtype, "y")
    codes, exps = ref.pack(ref.cpu(y))   # the checkpoint is that of y as it came out, exactly
    assert np.array_equal(codes, kept.codes.cpu().numpy()) and np.array_equal(exps, kept.exps.cpu().numpy())
    dx, df, dgate, dw1, dw2 = P.gated_norm_grad(dh, dy, x, f_in, w1, w2, gate=gate, alpha=alpha, eps=eps, center=center)
    rows = x.shape[0]
    _within(dx, want["dx"], want["dx_abs"], dtype, "dx")
    _within(dw2, want["dw_pre"], want["dw_pre_abs"], torch.float32, "dw_pre", rows)
    if f is None:
        assert df is None and dgate is None and dw1 is None
        return
    _within(df, want["df"], want["df_abs"], dtype, "df")
    _within(dw1, want["dw_post"], want["dw_post_abs"], torch.float32, "dw_post", rows)
    if gate is None:
        assert dgate is None
    elif gate.dim() == 1:
        _within(dgate, want["dgate"].sum(0), want["dgate_abs"].sum(0), torch.float32, "dgate", rows)
    else:
        _within(dgate, want["dgate"], want["dgate_abs"], dtype, "dgate")


@pytest.mark.parametrize("dim", [1, 3, 24, 32, 33, 100, 256, 300, 512, 513, 672, 1024, 1100, 2048, 2052, 4096, 5000, 8192])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_widths(dim, dtype):
    gate = ("rows", "vector", None)[dim % 3]
    _check(*_inputs(dtype, 7, dim, gate, seed=dim), alpha=0.7, center=dim % 2 == 1 and dim > 1, checkpoint=dim % 4 == 0)


@pytest.mark.parametrize("rows", [1, 2, 9, 333, 5000])
@pytest.mark.parametrize("gate", [None, "rows", "vector"])
@pytest.mark.parametrize("center", [False, True])
def test_rows(rows, gate, center):
    _check(*_inputs(torch.bfloat16, rows, 96, gate, seed=rows), center=center, checkpoint=gate == "rows")


def test_without_a_block_before():
    x, _, dh, dy, _, w2, _ = _inputs(torch.float32, 50, 200, None)
    _check(x, None, dh, dy, None, w2, None, alpha=1.3)
    _check(x, None, None, dy, None, w2, None)


def test_without_a_gradient_of_the_residual_stream():
    x, f, _, dy, w1, w2, gate = _inputs(torch.float16, 50, 200, "rows")
    _check(x, f, None, dy, w1, w2, gate)


def test_without_a_norm_after():
    x, f, _, _, w1, w2, gate = _inputs(torch.bfloat16, 30, 640, "rows")
    h, y, kept = P.gated_norm(x, f, w1, None, gate=gate)
    assert y is None and kept is None and torch.equal(h, P.gated_norm(x, f, w1, w2, gate=gate)[0])


def test_rows_apart_and_odd_places():
    """Rows further apart than their width, and rows that begin at odd places: the same bits, by narrower accesses."""
    x, f, dh, dy, w1, w2, gate = _inputs(torch.bfloat16, 20, 136, "rows")
    want = P.gated_norm(x, f, w1, w2, gate=gate, checkpoint=True)
    grads = P.gated_norm_grad(dh, dy, x, f, w1, w2, gate=gate)
    for left, right in ((0, 8), (0, 4), (1, 0), (4, 4)):
        apart = lambda t: torch.cat([t[:, :left] + 9, t, t[:, :right] + 9], 1)[:, left:left + 136]  # noqa: E731
        got = P.gated_norm(apart(x), f, w1, w2, gate=apart(gate), checkpoint=True)
        assert all(torch.equal(a, b) for a, b in zip((want[0], want[1], *want[2]), (got[0], got[1], *got[2])))
        got = P.gated_norm_grad(apart(dh), apart(dy), x, apart(f), w1, w2, gate=gate)
        assert all(torch.equal(a, b) for a, b in zip(grads, got))


def test_zero_rows_and_large_values():
    x, f, dh, dy, w1, w2, gate = _inputs(torch.float32, 6, 64, "rows")
    x[0], f[0] = 0, 0                   # both norms see zeros
    f[1], gate[2], gate[3] = 0, 200, -200
    x[4], f[4] = x[4] * 1e15, f[4] * 1e15
    _check(x, f, dh, dy, w1, w2, gate)
    h, y, _ = P.gated_norm(x[1:], f[1:], w1, w2, gate=gate[1:], eps=0.0)   # five rows: the workgroup's other rows are padding
    assert torch.isfinite(y[1:]).all()
    g = P.gated_norm_grad(dh[2:], dy[2:], x[2:], f[2:], w1, w2, gate=gate[2:], eps=0.0)
    assert all(torch.isfinite(t).all() for t in g)


def test_no_rows():
    x, f, dh, dy, w1, w2, gate = _inputs(torch.bfloat16, 4, 64, "vector")
    h, y, kept = P.gated_norm(x[:0], f[:0], w1, w2, gate=gate, checkpoint=True)
    assert h.shape == y.shape == (0, 64)
    g = P.gated_norm_grad(dh[:0], dy[:0], x[:0], f[:0], w1, w2, gate=gate)
    assert all(not t.any() for t in g[2:])


def test_the_same_bits_every_time():
    args = _inputs(torch.bfloat16, 3000, 320, "vector", seed=5)
    x, f, dh, dy, w1, w2, gate = args
    runs = [P.gated_norm_grad(dh, dy, x, f, w1, w2, gate=gate) for _ in range(3)]
    assert all(torch.equal(a, b) for r in runs[1:] for a, b in zip(runs[0], r))
