"""weights_pack, weights_restore and weights_linear against their definitions."""
import numpy as np
import pytest
import torch

import paper_2402_02361_amd as P
import token_reference as ref

pytestmark = pytest.mark.gpu
BF, HALF, F32 = torch.bfloat16, torch.float16, torch.float32


def _weights(rng, dtype, n_out, dim):
    w = rng.standard_normal((n_out, dim)) * np.exp(rng.standard_normal((n_out, 1)))
    return torch.from_numpy(w).to(dtype).cuda()


def _dense(codes, scales, group):
    return (codes - 8) * np.repeat(scales, group, axis=1)[:, :codes.shape[1]]


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", [BF, HALF, F32])
@pytest.mark.parametrize("n_out,dim", [(1, 1), (16, 128), (17, 129), (5, 31), (33, 300), (100, 64), (16, 97)])
def test_pack_and_restore(dtype, group, n_out, dim):
    rng = np.random.default_rng(n_out + dim)
    w = _weights(rng, dtype, n_out, dim)
    if n_out > 4 and dim > 8:
        w[2, 5], w[3], w[4, 8:] = float("nan"), 0.0, float("inf")
        w[1, ::3] = 0.0
    packed = P.weights_pack(w, group)
    codes, scales = ref.pack_weights(ref.cpu(w), group)
    words, laid = ref.lay_weights(codes, scales, group)
    assert np.array_equal(packed.codes.cpu().numpy(), words) and np.array_equal(ref.cpu(packed.scales), laid, equal_nan=True)
    want = _dense(codes, scales, group)
    for out in (F32, BF, HALF):
        assert np.array_equal(ref.cpu(P.weights_restore(packed, out)), torch.from_numpy(want.astype(np.float32)).to(out).double().numpy(), equal_nan=True)
    wide = torch.full((n_out, dim + 5), 7.0, dtype=dtype, device="cuda")   # rows further apart: what is between them stays
    P.weights_restore(packed, w=wide[:, :dim])
    assert (wide[:, dim:] == 7.0).all() and np.array_equal(ref.cpu(wide[:, :dim]), torch.from_numpy(want.astype(np.float32)).to(dtype).double().numpy(), equal_nan=True)
    wide[:, :dim] = w
    again = P.weights_pack(wide[:, :dim], group)
    assert torch.equal(again.codes, packed.codes) and torch.equal(again.scales.view(torch.int16), packed.scales.view(torch.int16))


def test_the_smallest_and_the_largest_weights():
    w = torch.tensor([[3e38, -1e38], [1e-45, 2e-45], [1e-38, -1e-39], [0.0, -0.0]], device="cuda")
    packed = P.weights_pack(w)
    codes, scales = ref.pack_weights(ref.cpu(w), 32)
    words, laid = ref.lay_weights(codes, scales, 32)
    assert np.array_equal(packed.codes.cpu().numpy(), words) and np.array_equal(ref.cpu(packed.scales), laid)


# A product with a code is exact; in bfloat16 it is of x times 128 + code, and a group's sum starts from -136 times the sum of x: of `group` inputs there are 2 group additions of terms of at most 271 |x|,
# each half a step of binary32 of the sum so far or less (truncated: one step), which is off by 2 group 2^-24 x 271 sum |x| at most (binary16: group 2^-24 x 8 sum |x|); groups, their scales and the
# wavefronts' parts round once more each; the result rounds to the type.
def _linear_bound(x, codes, scales, group, want, dtype, bias):
    groups = scales.shape[1]
    size = np.zeros(want.shape)
    terms = np.zeros(want.shape)
    for g in range(groups):
        part = slice(g * group, min((g + 1) * group, codes.shape[1]))
        each = np.abs(x[:, part]).sum(1)[:, None] * np.abs(scales[:, g])[None, :]
        size += each * (2 * group * 271 if dtype == BF else group * 8) * 2 * ref.F32
        terms += np.abs(x[:, part]) @ np.abs(codes[:, part] - 8).T * np.abs(scales[:, g])[None, :]
    b = size + (groups + 40) * ref.F32 * (terms + (0 if bias is None else np.abs(bias)[None, :]))
    return 1.01 * ref.UNIT[dtype] * np.abs(want) + b + ref.TINY[dtype]


def _check(dtype, rows, n_out, dim, group, bias=False, seed=0, pad=0):
    rng = np.random.default_rng(seed)
    packed = P.weights_pack(_weights(rng, F32, n_out, dim), group)
    w = P.weights_restore(packed, F32)
    codes, scales = ref.pack_weights(ref.cpu(_weights(np.random.default_rng(seed), F32, n_out, dim)), group)
    assert np.array_equal(ref.cpu(w), _dense(codes, scales, group).astype(np.float32))
    room = torch.full((rows, dim + pad), float("nan"), dtype=dtype, device="cuda")
    x = room[:, pad:] if pad % 2 else room[:, :dim]
    x.copy_(torch.from_numpy(rng.standard_normal((rows, dim)) + 0.5))
    b = torch.from_numpy(rng.standard_normal(n_out)).float().cuda() if bias else None
    out = torch.full((rows, n_out + pad), 3.0, dtype=dtype, device="cuda")
    got = P.weights_linear(x, packed, bias=b, y=out[:, :n_out]) if pad else P.weights_linear(x, packed, bias=b)
    want = ref.cpu(x) @ _dense(codes, scales, group).T + (ref.cpu(b) if bias else 0.0)
    bound = _linear_bound(ref.cpu(x), codes, scales, group, want, dtype, ref.cpu(b) if bias else None)
    worst = np.abs(ref.cpu(got) - want) / bound
    assert (worst <= 1).all(), f"{worst.max():.3g} of its bound at {np.unravel_index(worst.argmax(), worst.shape)}"
    assert (out[:, n_out:] == 3.0).all()
    return x, packed, got


@pytest.mark.parametrize("dtype", [BF, HALF])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("rows,n_out,dim", [(1, 1, 1), (1, 16, 128), (1, 50, 300), (3, 17, 129), (16, 100, 1100), (17, 33, 260), (1, 1603, 1101), (33, 40, 97), (70, 20, 64), (2, 5, 2049), (12, 96, 512)])
def test_linear(dtype, group, rows, n_out, dim):
    _check(dtype, rows, n_out, dim, group, bias=bool(n_out % 2), seed=rows + dim, pad=(rows + n_out) % 4)


@pytest.mark.parametrize("dtype,rows,n_out,dim,group", [(BF, 1, 20000, 2000, 128), (HALF, 5, 17001, 700, 32), (BF, 40, 16400, 300, 64), (BF, 1, 64, 40000, 32), (HALF, 300, 600, 500, 128)])
def test_many_outputs_inputs_and_rows(dtype, rows, n_out, dim, group):
    _check(dtype, rows, n_out, dim, group, bias=True, seed=1)


def test_inputs_below_the_smallest_normal_number():
    """binary16 below 2^-14, and sums of them that are normal: nothing is taken for 0."""
    rng = np.random.default_rng(9)
    packed = P.weights_pack(torch.from_numpy(rng.standard_normal((64, 256)) * 300).float().cuda())
    x = torch.from_numpy(rng.integers(-1000, 1000, (3, 256)) * 2.0 ** -24).half().cuda()
    dense = ref.cpu(P.weights_restore(packed, F32))
    want, size = ref.cpu(x) @ dense.T, np.abs(ref.cpu(x)) @ np.abs(dense).T
    assert (np.abs(ref.cpu(P.weights_linear(x, packed)) - want) <= 1.01 * ref.UNIT[HALF] * np.abs(want) + 256 * 2 * ref.F32 * size + ref.TINY[HALF]).all()


def test_rows_are_each_for_itself():
    """The same bits whatever the other rows are, up to the rows that a workgroup takes: one row of sixteen, a NaN among the others."""
    x, packed, y = _check(BF, 16, 100, 600, 64, seed=2)
    z = x.clone()
    z[3] = float("nan")
    z[7] = float("inf")
    got = P.weights_linear(z, packed)
    others = [i for i in range(16) if i not in (3, 7)]
    assert torch.equal(got[others], y[others]) and got[3].isnan().all() and not torch.isfinite(got[7]).any()
    for i in (0, 5):
        assert torch.equal(P.weights_linear(x[i:i + 1], packed), y[i:i + 1])


def test_a_group_that_is_not_a_number_reaches_its_output_alone():
    w = torch.randn(40, 300, generator=torch.Generator().manual_seed(3)).cuda()
    w[5, 100] = float("nan")
    y = P.weights_linear(torch.ones(2, 300, dtype=HALF, device="cuda"), P.weights_pack(w))
    bad = ~torch.isfinite(y)
    assert bad[:, 5].all() and bad.sum() == 2


def test_the_same_bits_every_time_on_another_stream_and_in_a_graph():
    x, packed, want = _check(HALF, 9, 500, 900, 32, seed=4)
    for n in range(3):
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = P.weights_linear(x, packed, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = P.weights_linear(x, packed)
    for n in range(3):
        got.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want)


def test_no_rows():
    packed = P.weights_pack(torch.randn(20, 40).cuda())
    assert P.weights_linear(torch.zeros(0, 40, dtype=BF, device="cuda"), packed).shape == (0, 20)


def test_refusals_of_the_binding():
    packed = P.weights_pack(torch.randn(20, 40).cuda())
    x = torch.zeros(3, 40, dtype=BF, device="cuda")
    for bad in (dict(x=x[:, :39]), dict(x=x.t()), dict(x=x.cpu()), dict(packed=packed._replace(group=48)), dict(packed=packed._replace(scales=packed.scales.half())), dict(packed=packed._replace(n_out=40)),
                dict(packed=packed._replace(codes=packed.codes.long())), dict(bias=torch.zeros(19, device="cuda")), dict(bias=torch.zeros(20, device="cuda", dtype=BF)),
                dict(y=torch.zeros(3, 20, device="cuda")), dict(y=torch.zeros(3, 21, dtype=BF, device="cuda"))):
        with pytest.raises(AssertionError):
            P.weights_linear(**{**dict(x=x, packed=packed), **bad})
    with pytest.raises(P.PrunerError):
        P.weights_linear(x.float(), packed)
    with pytest.raises(AssertionError):
        P.weights_pack(torch.zeros(40, 20, device="cuda").t())
    with pytest.raises(P.PrunerError):
        P.weights_pack(torch.zeros(4, 20, device="cuda", dtype=torch.float64))
