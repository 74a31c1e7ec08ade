"""Attention over the mx4 cache where scores are large: against the oracle, through the C ABI.

All scores here are sums of two products that fp32 holds, so the differences between them are exact and a row's weights are known whatever the scores' size.
Tolerance, with y = sum_j w_j v_j, A = sum_j w_j |v_j| and n positions; a weight counts down to 2^-33 of the row's largest, of an exponent 33 at the most:
  exponent   scale log2(e) is a constant's rounding and a product's, (score - largest) times it two more, and the join of waves and of shares two
             each: 8 x 33 x 2^-24, which comes back by log 2; a weight and the sum it is divided by: twice that, 2^-15
  2^x        2^-22 of itself, and as much again from the raised maxima's factors: 2^-16 at the most
  fp16       half a step of 11 bits, 2^-11; what is smaller than its subnormals is lost: n 2^-32 max |v|, with half a step for where the maximum lies
  sums       n terms in fp32 for the numerator and for the sum: 4 n 2^-24
  result     half a unit of its type, and of fp16's smallest subnormal
"""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as co
from paper_2309_15531_amd import binding as B
from test_gpu_cache import batch, ints
from test_gpu_mx4 import TINY, TYPES, UNIT, host

pytestmark = pytest.mark.gpu

PAGE = 64
CONSTANT = 2.0 ** 15                              # of the keys' element 0; their element 32 is one of E2M1's values


@pytest.fixture(scope="module")
def ctx():
    c = B.Context()
    yield c
    c.close()


def attend(ctx, r, q0, q1, k1, group, dim, scale, x, y="f32", window=0):
    """Row i of head h has the scores  q0[i, h] 2^15 + q1[i, h] k1[j]."""
    added, n = len(q0), len(k1)
    pages = -(-n // PAGE)
    table = batch(r, [n], PAGE, pages, pages)
    k, v = np.zeros((n, 1, dim)), r.standard_normal((n, 1, dim))
    k[:, 0, 0], k[:, 0, 32] = CONSTANT, k1
    c = np.zeros(B.mx4_cache_shape(pages, PAGE, 1, dim), np.uint8)
    co.store(c, k, v, table[0][np.arange(n) // PAGE] * PAGE + np.arange(n) % PAGE)
    q = np.zeros((added, group, dim))
    q[..., 0], q[..., 32] = q0, q1
    qd = torch.from_numpy(q.reshape(added, -1)).to(TYPES[x])
    assert bool((qd.double().numpy() == q.reshape(added, -1)).all())
    s = q0[..., None] * CONSTANT + q1[..., None] * k1
    assert bool((s == s.astype(np.float32)).all())
    yd = torch.full((added, group * dim), float("nan"), dtype=TYPES[y], device="cuda")
    ctx.adadim_mx4_attention(qd.cuda(), torch.from_numpy(c).cuda(), ints(table), ints([0, added]), ints([n]), yd, dim, scale=scale, window=window, max_new=added,
                             max_length=n)
    got = host(yd).astype(np.float64).reshape(q.shape)
    want, weight, _ = co.attention(q, c, table, [0, added], [n], dim, float(np.float32(scale)), window=window)
    vmax = np.abs(co.load(c, np.arange(pages * PAGE), dim)[1]).max()
    tol = weight * (2.0 ** -15 + 2.0 ** -16 + 2.0 ** -11 + 4 * n * 2.0 ** -24) + n * 2.0 ** -32 * vmax
    tol = tol * (1 + UNIT[y]) + np.abs(want) * UNIT[y] + TINY[y]
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (f"{bad.any(-1).sum()} of {added * group} rows", np.argwhere(bad)[:3], got[bad][:3], want[bad][:3])


GRID = np.array([0, .5, 1, 1.5, 2, 3, 4, 6, -.5, -1, -1.5, -2, -3, -4, -6])
# new tokens, query heads, positions, window: few rows, few in shares, many, many in shares; records that some rows of a wave do not see
FORMS = [(3, 5, 200, 0), (1, 7, 2100, 0), (300, 1, 320, 50), (140, 2, 1100, 0)]


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("form", range(len(FORMS)))
@pytest.mark.parametrize("scale", [0.125, 1.0, 1024.0, 1e12, 2e38])
def test_large_scores_beside_ordinary_ones(ctx, dim, form, scale):
    """Rows of scores from 1 to 2^27, positive and negative, side by side in a wave."""
    added, group, n, window = FORMS[form]
    r = np.random.default_rng([41, dim, form])
    a = r.integers(-15, 13, (added, group))
    q0 = np.exp2(a) * r.choice([-1.0, 1.0], a.shape)
    q1 = np.exp2(np.minimum(a - 7 + r.integers(0, 13, a.shape), 15))
    x = "f16" if form % 2 else "bf16"
    attend(ctx, r, q0, q1, r.choice(GRID, n), group, dim, scale, x, "f32" if dim == 64 else x, window)


@pytest.mark.parametrize("form,dim", [(0, 64), (1, 256), (2, 128), (3, 256)])
@pytest.mark.parametrize("power", [18, 20, 21, 25, 30])
@pytest.mark.parametrize("order", ["rising", "falling", "mixed"])
def test_maxima_on_both_sides_of_a_power_of_two(ctx, form, dim, power, order):
    """Scores whose products with scale log2(e) lie on both sides of 2^20, where sums that count are carried on from one way of weighing to the other;
    and around a multiple of other powers of two, by a factor that leaves no product exact."""
    added, group, n, window = FORMS[form]
    r = np.random.default_rng([42, dim, form, power])
    k1 = np.sort(r.choice(GRID, n))
    k1 = k1 if order == "rising" else k1[::-1] if order == "falling" else r.permutation(k1)
    q0 = 4096.0 * r.choice([-1.0, 1.0], (added, group))                # 2^27
    q1 = np.exp2(r.integers(5, 11, (added, group)))
    attend(ctx, r, q0, q1, k1.copy(), group, dim, 2.0 ** (power - 27) * (np.log(2.0) if power == 20 else 0.7137), "f16", window=window)


@pytest.mark.parametrize("form", range(len(FORMS)))
@pytest.mark.parametrize("scale", [1e-45, 1e-38, 2.2e-38, 3e-38])
def test_the_smallest_scales(ctx, form, scale):
    """Scores beyond 2^126, whose products with the smallest scales are a few; 7 / (scale log2(e)), or a score and that, is beyond fp32."""
    added, group, n, window = FORMS[form]
    r = np.random.default_rng([43, form])
    a = r.integers(100, 112, (added, group))
    q0 = np.exp2(a) * r.choice([-1.0, 1.0], a.shape)
    q1 = np.exp2(a + r.integers(0, 13, a.shape))
    attend(ctx, r, q0, q1, r.choice(GRID, n), group, 128, scale, "bf16", "bf16", window)
