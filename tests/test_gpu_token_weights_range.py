"""weights_linear where every sum is exact, so that one wrong code or input shows; and with inputs at the end of the type's range, and infinities."""
import numpy as np
import pytest
import torch

import paper_2402_02361_amd as P
import test_gpu_token_weights as weights
import token_reference as ref

pytestmark = pytest.mark.gpu
BF, HALF, F32 = torch.bfloat16, torch.float16, torch.float32

ROUTES = [(1, 50, 300), (16, 33, 1100), (6, 8200, 130), (17, 100, 97), (40, 16400, 200)]   # a tile of outputs and rows of a wavefront, two tiles, two by two, four by two


def _exact_weights(rng, n_out, dim, group):
    """Weights (code - 8) 2^e whose groups have a 7 or a -7 each, so that packing gives just these."""
    codes = rng.integers(-7, 8, (n_out, dim))
    codes[:, ::group] = np.where(codes[:, ::group] < 0, -7, 7)
    return codes * np.repeat(2.0 ** rng.integers(-3, 4, (n_out, -(-dim // group))), group, axis=1)[:, :dim]


def _on_gpu(w, dtype=F32):
    return torch.from_numpy(np.ascontiguousarray(w)).to(dtype).cuda()


@pytest.mark.parametrize("dtype", [BF, HALF])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("rows,n_out,dim", ROUTES)
def test_exact_sums(dtype, group, rows, n_out, dim):
    """Integers below 2^24 eighths: a group's sums are at most 128 x 143 x 3, all groups' 1100 x 56 x 3 eighths x 8.  What is left is the result's rounding, to the nearest, ties to even."""
    rng = np.random.default_rng(rows + dim + group)
    w, x = _exact_weights(rng, n_out, dim, group), rng.integers(-3, 4, (rows, dim)).astype(np.float64)
    packed = P.weights_pack(_on_gpu(w), group)
    assert np.array_equal(ref.cpu(P.weights_restore(packed, F32)), w)
    bias = rng.integers(-50, 50, n_out).astype(np.float64)
    want = torch.from_numpy(x @ w.T + bias).to(F32).to(dtype)
    assert torch.equal(P.weights_linear(_on_gpu(x, dtype), packed, bias=_on_gpu(bias)).cpu(), want)


@pytest.mark.parametrize("dtype", [BF, HALF])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dim", [128, 129, 161, 200, 255])
def test_rows_that_pick_one_input(dtype, group, dim):
    rng = np.random.default_rng(dim)
    w = _exact_weights(rng, 37, dim, group)
    y = P.weights_linear(torch.eye(dim, dtype=dtype, device="cuda"), P.weights_pack(_on_gpu(w), group))
    assert np.array_equal(ref.cpu(y), w.T)
    for i in (0, dim - 1):
        one = torch.zeros(1, dim, dtype=dtype, device="cuda")
        one[0, i] = 1
        assert np.array_equal(ref.cpu(P.weights_linear(one, P.weights_pack(_on_gpu(w), group)))[0], w[:, i])


def _by_definition(x, w):
    """x w^T term by term: infinities of one sign give one, of both a NaN, and so does an infinity times 0."""
    with np.errstate(invalid="ignore"):
        return np.stack([np.add.reduce(x[None, r] * w, axis=1) for r in range(x.shape[0])])


@pytest.mark.parametrize("dtype", [BF, HALF])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("rows,n_out,dim", [r for r in ROUTES if r[0] > 4])
def test_infinities_are_those_of_the_definition(dtype, group, rows, n_out, dim):
    rng = np.random.default_rng(rows)
    w = _exact_weights(rng, n_out, dim, group)
    w[3, 40], w[5, 96] = 0.0, 0.0
    packed = P.weights_pack(_on_gpu(w), group)
    w = ref.cpu(P.weights_restore(packed, F32))
    x = rng.standard_normal((rows, dim))
    clean = P.weights_linear(_on_gpu(x, dtype), packed)
    x[0, 40], x[1, 7], x[1, 96], x[2, 50], x[4, 96] = np.inf, np.inf, -np.inf, np.nan, -np.inf
    y = P.weights_linear(_on_gpu(x, dtype), packed)
    want = _by_definition(ref.cpu(_on_gpu(x, dtype)), w)
    got, bad = ref.cpu(y), [0, 1, 2, 4]
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[np.isinf(want)], want[np.isinf(want)])
    assert np.isinf(want[0]).any() and np.isnan(want[0, 3]) and np.isnan(want[2]).all() and not np.isfinite(got[bad]).any()
    others = [i for i in range(rows) if i not in bad]
    assert torch.equal(y[others], clean[others])


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("rows,n_out,dim", ROUTES)
def test_inputs_at_the_end_of_bfloat16s_range(rows, n_out, dim, group):
    """Inputs up to 2^127.9 with weights small enough for finite results; also beside weights of 0, where the others' sum is left."""
    rng = np.random.default_rng(dim)
    w = _exact_weights(rng, n_out, dim, group) * 2.0 ** -20
    w[1] = 0.0
    w[1, 0] = 7 * 2.0 ** -20
    packed = P.weights_pack(_on_gpu(w), group)
    w = ref.cpu(P.weights_restore(packed, F32))
    codes, scales = ref.pack_weights(w, group)
    x = rng.standard_normal((rows, dim))
    x[0] = rng.uniform(-1, 1, dim) * 3.3e38
    x[0, 0] = 1.0
    if rows > 2:
        x[2, dim // 2] = -3.3e38
    given = _on_gpu(x, BF)
    want = ref.cpu(given) @ w.T
    y = P.weights_linear(given, packed)
    assert (np.abs(ref.cpu(y) - want) <= weights._linear_bound(ref.cpu(given), codes, scales, group, want, BF, None)).all()
    assert float(y[0, 1]) == 7 * 2.0 ** -20
    if rows > 2:
        small = x.copy()
        small[0], small[2] = 0.0, 0.0
        others = [i for i in range(rows) if i not in (0, 2)]
        assert torch.equal(y[others], P.weights_linear(_on_gpu(small, BF), packed)[others])
