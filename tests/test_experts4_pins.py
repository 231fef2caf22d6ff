"""Experts in 4 bits, host side: the oracle's format against its definition, sizes, scale order, refusals without a GPU."""
import ctypes
import itertools

import numpy as np
import pytest
import torch

import oracle
from paper_2506_07366_b200 import binding, build


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding._lib()


def test_codes_are_the_nearest_values():
    """Every magnitude on a grid of sixteenths up to 6, with a 6 in its block so that the scale is 1."""
    grid = np.arange(0, 97) / 16.0
    for v, sign in itertools.product(grid, (1, -1)):
        w = np.zeros((1, 32))
        w[0, 0], w[0, 1] = 6.0, sign * v
        code, scale = oracle.weights4_encode(w)
        assert scale[0, 0] == 127 and code.shape == (1, 128) and (code[0, 32:] == 0).all() and (scale[0, 1:] == 0).all()
        got = oracle.weights4_decode(code, scale, 32)[0, 1]
        off = np.abs(oracle.experts4.VALUES - v)
        assert np.abs(got - sign * v) == off.min()
        if (off == off.min()).sum() == 2:                # a tie
            assert code[0, 1] & 1 == 0


@pytest.mark.parametrize("top,k", [(6.0, 0), (6.0625, 1), (3.0, -1), (3.03125, 0), (0.0, -127), (2.0 ** -133, -127),
                                   (6 * 2.0 ** -127, -127), (6.0625 * 2.0 ** -127, -126), (1.5 * 2.0 ** 127, 125),
                                   (1.9921875 * 2.0 ** 127, 125)])
def test_scale_is_the_smallest_that_fits(top, k):
    w = np.zeros((1, 32))
    w[0, 7] = -top
    code, scale = oracle.weights4_encode(w)
    assert scale[0, 0] == k + 127
    back = oracle.weights4_decode(code, scale, 32)[0, 7]
    assert abs(back + top) <= max(2.0 ** k * (1.0 if k < 125 else 2.0), 0)
    if k < 125:
        again, scale2 = oracle.weights4_encode(oracle.weights4_decode(code, scale, 32))
        assert oracle.weights4_decode(again, scale2, 32)[0, 7] == back


def test_blocks_that_are_not_finite():
    w = np.ones((2, 64))
    w[0, 3], w[1, 40] = np.inf, np.nan
    code, scale = oracle.weights4_encode(w)
    back = oracle.weights4_decode(code, scale, 64)
    assert np.isnan(back[0, :32]).all() and (back[0, 32:] == 1).all() and (back[1, :32] == 1).all() and np.isnan(back[1, 32:]).all()


@pytest.mark.parametrize("E,N,C", [(1, 1, 32), (2, 130, 136), (3, 128, 256), (1, 257, 1000)])
def test_scale_order(E, N, C):
    rng = np.random.default_rng(N)
    code, scale = oracle.weights4_encode(rng.standard_normal((E, N, C)) * np.exp(rng.standard_normal((E, N, 1))))
    _, packed = oracle.weights4_pack(code, scale)
    blocks = (C + 31) // 32                              # a checkpoint has no blocks for the filling
    got = binding.w4_scale_tiles(torch.from_numpy(scale[..., :blocks].copy()))
    assert np.array_equal(got.numpy(), packed)


def test_sizes(lib):
    for s in (binding.Shape(5, 136, 264, 3, 2, 4), binding.Shape(1, 4096, 14336, 8, 2, 8), binding.Shape(0, 8, 8, 1, 1, 1)):
        c = s.c_struct()
        for down in (False, True):
            codes, scales = s.w4_shapes(down)
            assert lib.moegps_weights4_bytes(ctypes.byref(c), int(down)) == np.prod(codes)
            assert lib.moegps_weights4_scale_bytes(ctypes.byref(c), int(down)) == np.prod(scales)
        d4, f4 = (s.D + 127) // 128 * 128, (s.F + 127) // 128 * 128
        least = 2 * s.Rcap * (d4 + f4) * 33 // 32        # two terms, a byte for each value and one for 32
        assert least <= binding.expert_ffn4_workspace_bytes(s)
    bad = binding.Shape(5, 130, 264, 3, 2, 4)
    c = bad.c_struct()
    assert lib.moegps_weights4_bytes(ctypes.byref(c), 0) == lib.moegps_weights4_scale_bytes(ctypes.byref(c), 1) == 0
    assert binding.expert_ffn4_workspace_bytes(bad) == 0


def test_null_context(lib):
    p = 4096
    assert lib.moegps_weights_quantize4(None, p, 0, p, p, None) == binding.ERR_INVALID_ARG
    assert lib.moegps_weights_dequantize4(None, p, p, 0, p, None) == binding.ERR_INVALID_ARG
    assert lib.moegps_expert_ffn4(None, *[p] * 11, None) == binding.ERR_INVALID_ARG


# ------------------------------------------------------------------------------------------- rows in two terms
def two_terms(v, top):
    """fp64 v, |v| <= top, as the products take them: two e4m3 terms with a power of two each, by the largest of the block."""
    mantissa, e = np.frexp(top)
    k = max(int(e) - 9 + int(mantissa > 0.875), -127)    # smallest with top <= 448 * 2^k
    k2 = max(k - 4, -127)
    e4m3 = lambda a: torch.from_numpy(a).float().to(torch.float8_e4m3fn).double().numpy()  # noqa: E731
    first = e4m3(v * 2.0 ** -k) * 2.0 ** k
    return first + e4m3((v - first) * 2.0 ** -k2) * 2.0 ** k2


ALL_BF16 = (torch.arange(0, 0x7f80, dtype=torch.int32) << 16).view(torch.float32).double().numpy()       # 0 and up


@pytest.mark.parametrize("unit", [1.0, 2.0 ** -100, 2.0 ** 110])
def test_bf16_in_two_terms(unit):
    """Every bf16 beside every largest value that has the same scale: exact from 2^-13 of it on, 2^-21 of it off at most below."""
    largest_off = 0.0
    for top in ALL_BF16[(ALL_BF16 > 224 * unit) & (ALL_BF16 <= 448 * unit)]:
        v = ALL_BF16[ALL_BF16 <= top]
        off = np.abs(two_terms(v, top) - v)
        assert (off[v >= 2.0 ** -13 * top] == 0).all() and off.max() <= 2.0 ** -21 * top
        largest_off = max(largest_off, v[off > 0].max() / top)
    assert largest_off > 2.0 ** -14                      # 2^-14 would be too much to promise


def test_smallest_bf16_in_two_terms():
    for top in (2.0 ** -116, 2.0 ** -118, 1.5 * 2.0 ** -120, 2.0 ** -126, 2.0 ** -133):
        v = ALL_BF16[ALL_BF16 <= top]
        assert np.array_equal(two_terms(v, top), v)


@pytest.mark.parametrize("top", [224.0 + 2.0 ** -16, 300.0, 448.0])
@pytest.mark.parametrize("unit", [1.0, 2.0 ** 100])
def test_fp32_in_two_terms(top, unit):
    """2^-9 relative or 2^-21 of the largest; the first alone does not hold."""
    rng = np.random.default_rng(int(top))
    v = rng.uniform(0.5, 1.0, 400000) * 2.0 ** -rng.integers(0, 26, 400000) * top
    v = v.astype(np.float32).astype(np.float64) * unit
    off = np.abs(two_terms(v, top * unit) - v)
    assert (off <= np.maximum(2.0 ** -9 * v, 2.0 ** -21 * top * unit)).all()
    assert (off <= 2.0 ** -9 * v)[v >= 2.0 ** -12 * top * unit].all() and (off > 2.0 ** -9 * v).any()
