"""Microscaled 4-bit operators without a GPU: pins of the oracle, refusals of the ABI and of the binding."""
import ctypes

import numpy as np
import pytest

from oracle import mx4_oracle as mo
from paper_2309_15531_amd import binding as B
from tests.test_abi_cpu import A16, ODD, ctx  # noqa: F401  (the fixture)

F16, BF16, F32, MX4 = B.TYPE_F16, B.TYPE_BF16, B.TYPE_F32, B.TYPE_MX4
BYTE = ctypes.c_void_p(0x1001)


# ------------------------------------------------------------------------------------------ the oracle
def test_a_block_by_hand():
    """amax 7: 2^2 <= 7 < 2^3, so the scale is 2^0 and 7 is cut to 6."""
    x = np.zeros((1, 32))
    x[0, :10] = [7, 0.25, 0.75, -1.25, 1.75, 2.5, -3.5, 5, 0.26, -0.1]
    codes, scales = mo.quantize(x)
    assert scales.shape == (1, 1, 4) and scales[0, 0].tolist() == [127, 127, 127, 127]
    low, high = codes[0, :5] & 15, codes[0, :5] >> 4
    #        7  .75  1.75 -3.5  .26           .25 -1.25  2.5   5   -.1
    assert low.tolist() == [7, 2, 4, 8 + 6, 1] and high.tolist() == [0, 8 + 2, 4, 6, 8]
    assert codes[0, 5:].tolist() == [0] * 59
    assert mo.values(codes, scales, 10)[0].tolist() == [6, 0, 1, -1, 2, 2, -4, 4, 0.5, 0]


def test_every_value_of_the_grid_is_kept():
    for e in (-127, -100, -3, 0, 5, 124):
        x = np.ldexp(np.tile(mo.VALUES, 2), e)[None]
        codes, scales = mo.quantize(x)
        assert scales[0, 0, 0] == e + 127
        assert np.array_equal(mo.values(codes, scales, 32), x)


@pytest.mark.parametrize("cols", [1, 31, 32, 100, 128, 300])
def test_nearest_and_within_half_a_step(cols):
    x = np.random.default_rng(cols).standard_normal((9, cols)) * np.exp2(np.arange(9) - 4)[:, None]
    codes, scales = mo.quantize(x)
    v = mo.values(codes, scales, cols)
    s = np.ldexp(1.0, scales.transpose(1, 0, 2).reshape(9, -1).astype(int) - 127).repeat(32, 1)[:, :cols]
    m = np.abs(x) / s
    assert np.all(m < 8) and np.all(m.max() >= 4)
    grid = s[..., None] * np.array(mo.GRID)
    assert np.allclose(np.abs(np.abs(x) - np.abs(v)), np.abs(np.abs(x)[..., None] - grid).min(-1), atol=0, rtol=1e-12)


def test_bad_and_empty_blocks():
    x = np.ones((3, 128))
    x[0, 40], x[1, 64], x[2, 96:] = np.nan, -np.inf, 0
    codes, scales = mo.quantize(x)
    assert scales[0].tolist() == [[125, 255, 125, 125], [125, 125, 255, 125], [125, 125, 125, 127]]
    v = mo.values(codes, scales, 128)
    assert np.isnan(v[0, 32:64]).all() and np.isnan(v[1, 64:96]).all() and (v[2, 96:] == 0).all() and np.isnan(v).sum() == 64


def test_route_by_hand():
    inf, nan = np.inf, np.nan
    l = np.array([[1, 3, 3, 2], [-inf, 0, nan, -inf], [nan, -inf, -inf, nan], [0, 0, 0, inf]])
    r = mo.route(l, 2, True)
    assert r["chosen"].tolist() == [[1, 2], [1, -1], [-1, -1], [3, 0]]
    assert r["weights"].tolist() == [[0.5, 0.5], [1, 0], [0, 0], [1, 0]]
    assert r["offsets"].tolist() == [0, 1, 3, 4, 5] and r["rows"].tolist() == [3, 0, 1, 0, 3, -1, -1, -1]
    assert r["slots"].tolist() == [[1, 3], [2, -1], [-1, -1], [4, 0]]
    all_ = mo.route(l[:1], 2, False)["weights"][0]
    assert np.allclose(all_, 1 / (2 + np.exp(-1) + np.exp(-2)))


# ------------------------------------------------------------------------------------------ refusals
def test_sizes_of_the_arrays(ctx):
    lib = B.load_library()
    for rows, cols in ((1, 1), (3, 128), (5, 129), (70, 4096)):
        c, s = B.mx4_shapes(rows, cols)
        assert lib.adadim_mx4_code_bytes(rows, cols) == np.prod(c) and lib.adadim_mx4_scale_bytes(rows, cols) == np.prod(s)
    assert lib.adadim_mx4_code_bytes(0, 5) == 0 and lib.adadim_mx4_scale_bytes(5, -1) == 0


def test_quantize_refusals(ctx):
    q = lambda *a: ctx.raw("adadim_mx4_quantize", *a)
    none = (None, 0, None)
    assert q(None, F16, 4, 128, 128, A16, A16, *none) == B.ENULL
    assert q(A16, F16, 4, 128, 128, None, A16, *none) == B.ENULL
    assert q(A16, F16, 4, 128, 128, A16, None, *none) == B.ENULL
    assert q(A16, MX4, 4, 128, 128, A16, A16, *none) == B.EINVAL
    assert "x_type" in ctx.last_error()
    assert q(A16, F16, -1, 128, 128, A16, A16, *none) == B.EINVAL
    assert q(A16, F16, 4, 0, 128, A16, A16, *none) == B.EINVAL
    assert q(A16, F16, 4, 128, 127, A16, A16, *none) == B.EINVAL
    assert q(A16, F16, 1 << 30, 1 << 24, 1 << 24, A16, A16, *none) == B.EINVAL           # more workgroups than a launch has
    assert q(BYTE, F16, 4, 128, 128, A16, A16, *none) == B.EALIGN
    assert q(A16, F16, 4, 128, 128, ODD, A16, *none) == B.EALIGN
    assert q(A16, F16, 4, 128, 128, A16, BYTE, *none) == B.EALIGN
    assert q(A16, F16, 4, 128, 128, A16, A16, A16, 9, None) == B.EINVAL
    assert q(A16, F16, 4, 128, 128, A16, A16, A16, B.DW_F16_SCALED, None) == B.ENULL
    assert q(A16, F16, 4, 128, 128, A16, A16, BYTE, B.DW_F32, None) == B.EALIGN
    assert q(None, F16, 0, 128, 128, None, None, *none) == B.OK                          # no rows: nothing to do
    d = lambda *a: ctx.raw("adadim_mx4_dequantize", *a)
    assert d(A16, A16, 4, 128, A16, MX4, 128) == B.EINVAL
    assert d(A16, A16, 4, 128, A16, F16, 100) == B.EINVAL
    assert d(A16, None, 4, 128, A16, F16, 128) == B.ENULL
    assert d(ODD, A16, 4, 128, A16, F16, 128) == B.EALIGN
    assert d(None, None, 0, 128, None, F16, 128) == B.OK


def test_matmul_refusals(ctx):
    m = lambda *a: ctx.raw("adadim_mx4_matmul", *a)
    w = (A16, A16, 64, 128)
    assert m(A16, None, F32, 4, 128, *w, A16, F16, 64) == B.EINVAL
    assert "x_type" in ctx.last_error()
    assert m(A16, None, F16, 4, 128, *w, A16, MX4, 64) == B.EINVAL
    assert m(A16, None, F16, -4, 128, *w, A16, F16, 64) == B.EINVAL
    assert m(A16, None, F16, 4, 127, *w, A16, F16, 64) == B.EINVAL
    assert m(A16, None, F16, 4, 128, *w, A16, F16, 63) == B.EINVAL
    assert m(A16, None, F16, 4, 128, A16, A16, 0, 128, A16, F16, 64) == B.EINVAL
    assert m(A16, None, F16, 4, 128, A16, A16, 64, 0, A16, F16, 64) == B.EINVAL
    assert m(None, None, F16, 4, 128, *w, A16, F16, 64) == B.ENULL
    assert m(A16, None, MX4, 4, 0, *w, A16, F16, 64) == B.ENULL                          # x_scales
    assert m(A16, None, F16, 4, 128, None, A16, 64, 128, A16, F16, 64) == B.ENULL
    assert m(A16, None, F16, 4, 128, *w, None, F16, 64) == B.ENULL
    assert m(BYTE, None, F16, 4, 128, *w, A16, F16, 64) == B.EALIGN
    assert m(ODD, A16, MX4, 4, 0, *w, A16, F16, 64) == B.EALIGN
    assert m(A16, None, F16, 4, 128, ODD, A16, 64, 128, A16, F16, 64) == B.EALIGN
    assert m(None, None, F16, 0, 128, None, None, 64, 128, None, F16, 64) == B.OK
    e = lambda *a: ctx.raw("adadim_mx4_matmul_experts", *a)
    x = (A16, None, F16, 4, 128)
    y = (*w, A16, F16, 64)
    assert e(*x, A16, 8, None, 2, *y) == B.ENULL
    assert e(*x, A16, 8, A16, 0, *y) == B.EINVAL
    assert e(*x, A16, 8, A16, 1025, *y) == B.EINVAL
    assert e(*x, None, 8, A16, 2, *y) == B.EINVAL                                        # 8 rows of Y, 4 of X, no rows[]
    assert e(*x, A16, -8, A16, 2, *y) == B.EINVAL
    assert e(*x, A16, 8, BYTE, 2, *y) == B.EALIGN
    assert e(*x, BYTE, 8, A16, 2, *y) == B.EALIGN
    assert e(*x, A16, 0, A16, 2, *y) == B.OK


def test_route_and_combine_refusals(ctx):
    r = lambda *a: ctx.raw("adadim_expert_route", *a)
    o = (A16,) * 5
    assert r(A16, MX4, 4, 8, 8, 2, 1, *o) == B.EINVAL
    assert r(A16, F32, 4, 7, 8, 2, 1, *o) == B.EINVAL
    assert r(A16, F32, -4, 8, 8, 2, 1, *o) == B.EINVAL
    assert r(A16, F32, 4, 8, 8, 0, 1, *o) == B.EINVAL
    assert r(A16, F32, 4, 8, 8, 9, 1, *o) == B.EINVAL
    assert r(A16, F32, 4, 64, 64, 33, 1, *o) == B.EINVAL
    assert r(A16, F32, 4, 1025, 1025, 2, 1, *o) == B.EINVAL
    assert r(A16, F32, 1 << 27, 32, 32, 16, 1, *o) == B.EINVAL                           # 2^31 places
    assert r(A16, F32, 4, 8, 8, 2, 2, *o) == B.EINVAL
    assert r(None, F32, 4, 8, 8, 2, 1, *o) == B.ENULL
    for i in range(5):
        assert r(A16, F32, 4, 8, 8, 2, 1, *o[:i], None, *o[i + 1:]) == B.ENULL
        assert r(A16, F32, 4, 8, 8, 2, 1, *o[:i], BYTE, *o[i + 1:]) == B.EALIGN
    c = lambda *a: ctx.raw("adadim_expert_combine", *a)
    assert c(A16, MX4, 8, 64, 64, A16, A16, 4, 2, A16, F16, 64) == B.EINVAL
    assert c(A16, F16, 8, 64, 63, A16, A16, 4, 2, A16, F16, 64) == B.EINVAL
    assert c(A16, F16, 8, 64, 64, A16, A16, 4, 0, A16, F16, 64) == B.EINVAL
    assert c(A16, F16, 8, 64, 64, A16, A16, 4, 2, A16, F16, 63) == B.EINVAL
    assert c(None, F16, 8, 64, 64, A16, A16, 4, 2, A16, F16, 64) == B.ENULL
    assert c(A16, F16, 8, 64, 64, None, A16, 4, 2, A16, F16, 64) == B.ENULL
    assert c(BYTE, F16, 8, 64, 64, A16, A16, 4, 2, A16, F16, 64) == B.EALIGN
    assert c(None, F16, 0, 64, 64, None, None, 0, 2, None, F16, 64) == B.OK


class Tensor:
    """On the device, as far as the binding looks."""
    is_cuda = True

    def __init__(self, dtype, *shape, pitch=None):
        self.dtype, self.shape, self._pitch = "torch." + dtype, shape, pitch

    def dim(self):
        return len(self.shape)

    def numel(self):
        return int(np.prod(self.shape))

    def stride(self, d=None):
        st = [int(np.prod(self.shape[i + 1:])) for i in range(len(self.shape))]
        if self._pitch:
            st[0] = self._pitch
        return st if d is None else st[d]

    def is_contiguous(self):
        return not self._pitch

    def data_ptr(self):
        return 0x1000


def test_the_binding_checks_shapes():
    class Fake(B.Context):
        def __init__(self):
            self._lib = self._h = None
    f = Fake()
    x, u8, i32 = (lambda t: lambda *s, **k: Tensor(t, *s, **k))("float16"), (lambda *s: Tensor("uint8", *s)), (lambda *s: Tensor("int32", *s))
    (c, s) = B.mx4_shapes(64, 200)
    assert (c, s) == ((64, 128), (2, 64, 4))
    with pytest.raises(ValueError, match="codes"):
        f.adadim_mx4_quantize(x(64, 200), u8(64, 64), u8(*s))
    with pytest.raises(ValueError, match="scales"):
        f.adadim_mx4_quantize(x(64, 200), u8(*c), u8(64, 2, 4))
    with pytest.raises(TypeError, match="X"):
        f.adadim_mx4_quantize(i32(64, 200), u8(*c), u8(*s))
    with pytest.raises(ValueError, match="dW"):
        f.adadim_mx4_quantize(x(64, 200), u8(*c), u8(*s), dW=Tensor("float32", 64, 100))
    with pytest.raises(ValueError, match="two axes"):
        f.adadim_mx4_dequantize(u8(*c), u8(*s), x(200))
    with pytest.raises(ValueError, match="rows"):
        f.adadim_mx4_matmul(x(5, 200), u8(*c), u8(*s), x(6, 64))
    with pytest.raises(ValueError, match="columns"):
        f.adadim_mx4_matmul(x(5, 200), u8(*c), u8(*s), x(5, 64), in_f=100)
    with pytest.raises(ValueError, match="in_f"):
        f.adadim_mx4_matmul(u8(5, 128), u8(*c), u8(*s), x(5, 64))
    with pytest.raises(ValueError, match="x_scales"):
        f.adadim_mx4_matmul(x(5, 200), u8(*c), u8(*s), x(5, 64), x_scales=u8(2, 5, 4))
    with pytest.raises(ValueError, match="codes"):
        f.adadim_mx4_matmul_experts(x(5, 200), u8(3, *c), u8(3, *s), i32(5), x(8, 64), rows=i32(8))
    with pytest.raises(ValueError, match="without rows"):
        f.adadim_mx4_matmul_experts(x(5, 200), u8(3, *c), u8(3, *s), i32(4), x(8, 64))
    with pytest.raises(ValueError, match="rows"):
        f.adadim_mx4_matmul_experts(x(5, 200), u8(3, *c), u8(3, *s), i32(4), x(8, 64), rows=i32(7))
    with pytest.raises(ValueError, match="offsets"):
        f.adadim_expert_route(x(5, 8), i32(5, 2), Tensor("float32", 5, 2), i32(8), i32(10), i32(5, 2))
    with pytest.raises(ValueError, match="Y"):
        f.adadim_expert_combine(x(10, 64), i32(5, 2), Tensor("float32", 5, 2), x(5, 63))
