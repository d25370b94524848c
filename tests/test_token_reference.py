"""What the 64-bit definitions of the token step's operators say on cases small enough to know (no GPU), and the binding's helpers."""
import math

import numpy as np
import pytest
import torch

import paper_2402_02361_amd as P
import paper_2402_02361_amd.binding as B
import token_reference as ref


def test_packed_structs_are_the_structs():
    rotation = (1, 2, 3, 4, 5, 6, 7, 1, 0.5, 0x10, 0x20, 0x30, 0x40)
    assert B._PACK_ROTATION.pack(*rotation) == bytes(B.CRotation(*rotation))
    cache = (0x10, 0x20, 0x30, 0x40, 0x50, 1, 2, 3, 4, 5)
    assert B._PACK_CACHE.pack(*cache) == bytes(B.CCache(*cache))
    assert B._PACK_WEIGHTS.pack(0x10, 0x20, 1, 2, 3) == bytes(B.CWeights(0x10, 0x20, 1, 2, 3))


def test_e4m3_is_the_type_that_torch_calls_so():
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(ref.e4m3(codes), want, equal_nan=True)
    x = np.concatenate([np.linspace(-448, 448, 20011), np.linspace(-0.05, 0.05, 20011), 2.0 ** np.arange(-14, 9), ref.VALUES, (ref.VALUES[1:] + ref.VALUES[:-1]) / 2]).astype(np.float32)
    got = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(ref.to_e4m3(x.astype(np.float64)) & 127, got & 127)
    assert ref.to_e4m3(np.array([np.nan, np.inf, -np.inf])).tolist() == [127] * 3


def test_exponents():
    assert [ref.exponent(t) for t in (448.0, 448.1, 1.75, 1.7501, 1.0, 0.0, 2.0 ** -130)] == [0, 1, -8, -7, -8, -126, -126]


def test_a_page_rounds_older_tokens_again():
    page = ref.Page(np.zeros((16, 16), np.uint8), 200)
    page.append(0, np.full((2, 16), 1.0))                 # e = -8: 1 = 256 x 2^-8
    assert page.byte == 119 and (page.values()[:2] == 1.0).all()
    page.append(2, np.full((1, 16), 1000.0))              # e = 2: 1 / 4 is a value, 1000 / 4 = 250 rounds to 256
    assert page.byte == 129 and (page.values()[:2] == 1.0).all() and (page.values()[2] == 1024.0).all()
    page.append(3, np.full((1, 16), 0.001))               # the exponent does not shrink: 0.001 / 4 is below half of the smallest step
    assert page.byte == 129 and not page.values()[3].any()
    page.append(0, np.full((1, 16), 0.001))               # a page that begins again has no older tokens
    assert page.byte < 119


def test_rotary_turns_pairs():
    x = np.arange(8.0).reshape(1, 1, 1, 8)
    f = np.array([math.pi / 2, math.pi])
    y, _ = ref.rotary(x, f, np.ones((1, 1)))
    assert np.allclose(y[0, 0, 0], [-2, -1, 0, -3, 4, 5, 6, 7], atol=1e-12)      # (0, 2) by a quarter, (1, 3) by half a turn
    y, _ = ref.rotary(x, f, np.ones((1, 1)), interleaved=True, amplitude=2.0)
    assert np.allclose(y[0, 0, 0], [-2, 0, -4, -6, 4, 5, 6, 7], atol=1e-12)
    z, _ = ref.rotary(y, f, np.ones((1, 1)), interleaved=True, amplitude=0.5, back=True)
    assert np.allclose(z, x, atol=1e-12)
    # far positions: whole turns of a frequency that is a fraction of one
    y, _ = ref.rotary(x, np.array([2 * math.pi / 64]), np.full((1, 1), 64 * 10 ** 6 + 16), interleaved=True)
    assert np.allclose(y[0, 0, 0, :2], [-1, 0], atol=1e-6)


def test_frequencies():
    assert np.allclose(P.rotary_frequencies(8), [1, 0.1, 0.01, 0.001])
    assert np.allclose(P.rotary_frequencies(8, base=16.0, factor=4.0), np.array([1, 0.5, 0.25, 0.125]) / 4)
    f = P.rotary_frequencies(64, factor=8.0, trained=4096)
    plain, turns = P.rotary_frequencies(64), 4096 * P.rotary_frequencies(64) / (2 * math.pi)
    assert np.array_equal(f[turns >= 4], plain[turns >= 4]) and np.allclose(f[turns <= 1], plain[turns <= 1] / 8)
    mid = (turns > 1) & (turns < 4)
    assert mid.any() and np.allclose(f[mid] / plain[mid], (turns[mid] - 1) / 3 + (1 - (turns[mid] - 1) / 3) / 8)
    for bad in (dict(rotary_dim=7), dict(rotary_dim=0), dict(rotary_dim=258), dict(rotary_dim=8, factor=0.0), dict(rotary_dim=8, trained=10, low=2.0, high=2.0)):
        with pytest.raises(AssertionError):
            P.rotary_frequencies(**bad)


def test_weights_lie_as_documented():
    codes = np.arange(17 * 130).reshape(17, 130) % 16
    words, scales = ref.lay_weights(codes, np.arange(17 * 3).reshape(17, 3) + 1.0, 64)
    assert words.shape == (2, 2, 4, 16, 4) and scales.shape == (2, 2, 4, 2, 4)
    # output 5, input 77 = 32 * 2 + 8 * 1 + 5: bit 4 * 2 + 16
    assert (int(words[0, 0, 1, 5, 2]) >> 24) & 15 == codes[5, 77]
    assert (int(words[1, 1, 0, 0, 0]) >> 16) & 15 == codes[16, 129] and (int(words[1, 1, 0, 0, 0]) >> 4) & 15 == 8
    assert scales[0, 0, 1, 1, 1] == 5 * 3 + 1 + 1 and scales[1, 1, 0, 0, 0] == 16 * 3 + 2 + 1 and scales[1, 1, 0, 1, 0] == 0


def test_packing_a_group():
    w = np.zeros((1, 64))
    w[0, :4] = [7.0, -7.0, 3.5, 0.25]
    w[0, 32:34] = [np.inf, 1.0]
    codes, scales = ref.pack_weights(w, 32)
    assert scales[0, 0] == 1.0 and codes[0, :5].tolist() == [15, 1, 12, 8, 8] and np.isnan(scales[0, 1])   # (3.5 is halfway: to the even 4)
