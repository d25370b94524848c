"""Checkpoints in 8 bits, and the weight gradient taken from them."""
import numpy as np
import pytest
import torch

import block_reference as ref
import paper_2402_02361_amd as P

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16, torch.float32]


def _check(x):
    kept = P.checkpoint_pack(x)
    codes, exps = ref.pack(ref.cpu(x))
    assert np.array_equal(exps, kept.exps.cpu().numpy()) and np.array_equal(codes, kept.codes.cpu().numpy())
    for dtype in TYPES:
        want = torch.from_numpy(ref.restore(codes, exps)).to(dtype)
        got = P.checkpoint_restore(kept, dtype).cpu()
        assert torch.equal(torch.nan_to_num(got, 7.5), torch.nan_to_num(want, 7.5))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,dim", [(1, 1), (3, 5), (2, 31), (4, 32), (5, 33), (7, 100), (3, 164), (2, 1100), (65, 96)])
def test_shapes(dtype, rows, dim):
    gen = torch.Generator().manual_seed(rows * dim)
    _check((torch.randn(rows, dim, generator=gen) * torch.exp(3 * torch.randn(rows, 1, generator=gen))).to(dtype).cuda())


@pytest.mark.parametrize("dtype", TYPES)
def test_values_at_the_edges(dtype):
    x = torch.zeros(10, 64)
    x[1, 3], x[2, 3], x[3, 5] = 127.0, 128.0, 127.5            # just in, just out of a power's range, and between
    x[4, :4] = torch.tensor([64.0, 0.5, 1.5, 2.5])             # ties go to the even code
    x[5, 40], x[6, 2], x[7, 33] = float("inf"), float("nan"), float("-inf")
    x[8] = torch.finfo(dtype).max if dtype != torch.float32 else 3.0e38
    x[9] = torch.finfo(dtype).tiny
    _check(x.to(dtype).cuda())
    if dtype != torch.float16:
        _check((x * 0 + torch.arange(64) * 2.0 ** -133).nan_to_num(0).to(dtype).cuda())   # below the smallest power
    _check(-x.to(dtype).cuda())


def test_restored_values_are_within_half_a_code():
    x = torch.randn(50, 320, generator=torch.Generator().manual_seed(2)).cuda()
    kept = P.checkpoint_pack(x)
    step = 2.0 ** (kept.exps.float() - 127).repeat_interleave(32, 1)
    assert ((P.checkpoint_restore(kept, torch.float32) - x).abs() <= step / 2).all()
    # the largest of a group takes at least half of the codes
    assert (kept.codes.abs().view(50, 10, 32).amax(-1) >= 63).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_apart(dtype):
    gen = torch.Generator().manual_seed(3)
    x = torch.randn(9, 72, generator=gen).to(dtype).cuda()
    want = P.checkpoint_pack(x)
    for left, right in ((0, 8), (8, 0), (4, 0), (1, 2)):
        wide = torch.randn(9, left + 72 + right, generator=gen).to(dtype).cuda()
        wide[:, left:left + 72] = x
        got = P.checkpoint_pack(wide[:, left:left + 72])
        assert torch.equal(want.codes, got.codes) and torch.equal(want.exps, got.exps)
        before = wide.clone()
        P.checkpoint_restore(want, x=wide[:, left:left + 72])
        assert torch.equal(wide[:, left:left + 72], P.checkpoint_restore(want, dtype))
        assert torch.equal(wide[:, :left], before[:, :left]) and torch.equal(wide[:, left + 72:], before[:, left + 72:])


def _wgrad(dtype, rows, n_out, dim, seed=0):
    gen = torch.Generator().manual_seed(seed)
    dy = torch.randn(rows, n_out, generator=gen).to(dtype).cuda()
    kept = P.checkpoint_pack(torch.randn(rows, dim, generator=gen).cuda())
    x = ref.restore(kept.codes.cpu().numpy(), kept.exps.cpu().numpy())
    return dy, kept, ref.cpu(dy).T @ x, np.abs(ref.cpu(dy)).T @ np.abs(x)


# every restored value is exact in either type, products are exact in binary32's sums: what differs is the sums' roundings, one per 8 rows
# at the most, and one per part
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,n_out,dim", [(1, 1, 1), (3, 154, 44), (64, 128, 128), (65, 129, 130), (200, 40, 300), (1000, 256, 164), (3000, 100, 33), (5000, 8, 1000), (1500, 300, 7)])
def test_weight_gradient(dtype, rows, n_out, dim):
    dy, kept, want, size = _wgrad(dtype, rows, n_out, dim, seed=rows)
    bound = (rows / 8 + 8) * ref.F32 * size
    got = P.checkpoint_wgrad(dy, kept)
    assert (np.abs(ref.cpu(got) - want) <= bound).all()
    again = P.checkpoint_wgrad(dy, kept)
    assert torch.equal(got, again)
    P.checkpoint_wgrad(dy, kept, dw=again, accumulate=True)
    assert (np.abs(ref.cpu(again) - 2 * want) <= 2 * bound + 2 * ref.F32 * np.abs(want)).all()


def test_weight_gradient_of_rows_apart():
    dy, kept, _, _ = _wgrad(torch.bfloat16, 700, 136, 96)
    want = P.checkpoint_wgrad(dy, kept)
    for left, right in ((0, 8), (8, 16), (4, 0), (1, 0)):
        wide = torch.full((700, left + 136 + right), float("nan"), dtype=dy.dtype, device="cuda")
        wide[:, left:left + 136] = dy
        assert torch.equal(P.checkpoint_wgrad(wide[:, left:left + 136], kept), want)


def test_weight_gradient_of_a_checkpoint_with_an_infinity():
    x = torch.randn(100, 64, generator=torch.Generator().manual_seed(4)).cuda()
    x[50, 40] = float("inf")
    dw = P.checkpoint_wgrad(torch.ones(100, 16, dtype=torch.bfloat16, device="cuda"), P.checkpoint_pack(x))
    assert torch.isfinite(dw[:, :32]).all() and torch.isnan(dw[:, 32:]).all()


def test_no_rows():
    dy, kept, _, _ = _wgrad(torch.bfloat16, 4, 24, 40)
    none = P.Checkpoint(kept.codes[:0], kept.exps[:0])
    assert not P.checkpoint_wgrad(dy[:0], none).any()
    dw = torch.ones(24, 40, device="cuda")
    assert (P.checkpoint_wgrad(dy[:0], none, dw=dw, accumulate=True) == 1).all()
    assert P.checkpoint_restore(P.checkpoint_pack(torch.empty(0, 40, device="cuda")), torch.float32).shape == (0, 40)
