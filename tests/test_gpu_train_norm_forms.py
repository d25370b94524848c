"""gated_norm without a norm after it (the last block of a model): its gradients against the definition in 64 bits, and what goes together in a call."""
import numpy as np
import pytest
import torch

import block_reference as ref
import paper_2402_02361_amd as P
from test_gpu_train_gated_norm import _inputs, _within

pytestmark = pytest.mark.gpu


def _check(dtype, rows, dim, gate, center=False, alpha=1.0, checkpoint=False, block=True):
    x, f, dh, dy, w1, _, gate = _inputs(dtype, rows, dim, gate, seed=rows + dim)
    if not block:
        f = w1 = gate = None
    h, y, kept = P.gated_norm(x, f, w1, None, gate=gate, alpha=alpha, center=center)
    assert y is None and kept is None
    f_in = f
    if checkpoint:
        f_in = P.checkpoint_pack(f)
        f = P.checkpoint_restore(f_in, torch.float32)
    one = np.ones(dim)
    # the reference's y takes no part where its gradient is zero
    args = [ref.cpu(t) for t in (x, f, w1)]
    want = ref.norm(*args, one, ref.cpu(gate), float(np.float32(alpha)), float(np.float32(1e-6)), center, ref.cpu(dh), np.zeros((rows, dim)))
    dx, df, dgate, dw1, dw2 = P.gated_norm_grad(dh, None, x, f_in, w1, None, gate=gate, alpha=alpha, center=center)
    assert dw2 is None
    if block and not checkpoint:
        _within(h, want["h"], want["h_abs"], dtype, "h")
    _within(dx, want["dx"], want["dx_abs"], dtype, "dx")
    if not block:
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


@pytest.mark.parametrize("checkpoint", [False, True])
@pytest.mark.parametrize("gate", [None, "rows", "vector"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("rows,dim", [(1, 40), (33, 256), (700, 100), (60, 1111), (20, 2048), (9, 6000)])
def test_without_a_norm_after(rows, dim, dtype, gate, checkpoint):
    _check(dtype, rows, dim, gate, center=rows % 2 == 1 and dim > 100, alpha=0.7, checkpoint=checkpoint)


def test_without_a_norm_after_and_a_block_before():
    _check(torch.bfloat16, 50, 200, None, alpha=1.3, block=False)


def test_a_loss_of_the_output_by_differences():
    """The gradient of sum(h dh) by x, f, the gate and w_post, binary32, against differences of the forward pass in 64 bits."""
    x, f, dh, _, w1, _, gate = _inputs(torch.float32, 3, 10, "rows", seed=9)
    got = P.gated_norm_grad(dh, None, x, f, w1, None, gate=gate)
    base = [ref.cpu(t) for t in (x, f, gate, w1)]
    loss = lambda x, f, g, w: (ref.norm(x, f, w, np.ones(10), g)["h"] * ref.cpu(dh)).sum()  # noqa: E731
    rng = np.random.default_rng(1)
    for n, t in zip(range(4), (got[0], got[1], got[2], got[3])):
        for _ in range(5):
            i = tuple(int(rng.integers(s)) for s in base[n].shape)
            up, down = [a.copy() for a in base], [a.copy() for a in base]
            up[n][i] += 1e-5
            down[n][i] -= 1e-5
            # (binary32: some forty roundings of terms of a few units)
            assert abs((loss(*up) - loss(*down)) / 2e-5 - float(t[i])) < 1e-4


def test_no_rows():
    x, f, dh, _, w1, _, gate = _inputs(torch.bfloat16, 4, 64, "vector")
    _, _, dgate, dw1, dw2 = P.gated_norm_grad(dh[:0], None, x[:0], f[:0], w1, None, gate=gate)
    assert not dgate.any() and not dw1.any() and dw2 is None


def test_what_goes_together():
    x, f, dh, dy, w1, w2, _ = _inputs(torch.bfloat16, 4, 64, None)
    for a in ((None, None, x, f, w1, None), (dh, dy, x, f, w1, None), (dh, None, x, f, w1, w2), (None, None, x, f, w1, w2)):
        with pytest.raises(AssertionError):
            P.gated_norm_grad(*a)


@pytest.mark.parametrize("size", [1e-17, 1e-18, 1e-19, 3e-20, 1e-20])
def test_tiny_values_without_eps(size):
    """Mean squares below binary32's smallest normal number: they keep a step of 2^-149, of which a value's square is off by half, beside the usual roundings."""
    gen = torch.Generator().manual_seed(1)
    f, dh = torch.randn(5, 200, generator=gen).cuda() * size, torch.randn(5, 200, generator=gen).cuda()
    w, x = torch.ones(200, device="cuda"), torch.zeros(5, 200, device="cuda")
    h, _, _ = P.gated_norm(x, f, w, None, eps=0.0)
    _, df, _, dw, _ = P.gated_norm_grad(dh, None, x, f, w, None, eps=0.0)
    want = ref.norm(*(ref.cpu(t) for t in (x, f, w, w)), eps=0.0, dh=ref.cpu(dh), dy=np.zeros((5, 200)))
    off = 2.0 ** -149 / size ** 2 + 64 * ref.F32
    assert (np.abs(ref.cpu(h) - want["h"]) <= off * np.abs(want["h"])).all()
    # (twice for r and z, and as much again for <d z>)
    assert (np.abs(ref.cpu(df) - want["df"]) <= 4 * off * want["df_abs"]).all()
    assert (np.abs(ref.cpu(dw) - want["dw_post"]) <= off * want["dw_post_abs"]).all()
