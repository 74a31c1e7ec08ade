"""Edges of the microscaled operators and of the routing that other tests do not reach."""
import numpy as np
import pytest
import torch

from paper_2309_15531_amd import binding as B
from test_gpu_mx4 import TYPES, mx4, rng, spread

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = B.Context()
    yield c
    c.close()


@pytest.mark.parametrize("x", ["f16", "bf16", "mx4"])
@pytest.mark.parametrize("rows,out,inn", [(3, 40, 200), (90, 40, 200), (900, 270, 136), (700, 520, 1024)])
def test_experts_without_tokens(ctx, x, rows, out, inn):
    """rows[] can name no row of X then: the groups' rows are zeros, the others stay."""
    codes, scales = (torch.stack([t, t, t]) for t in mx4(ctx, spread(rng(rows, out), out, inn)))
    c, s = B.mx4_shapes(0, inn)
    X = torch.empty(c, dtype=torch.uint8, device="cuda") if x == "mx4" else torch.empty((0, inn), dtype=TYPES[x], device="cuda")
    xs = torch.empty(s, dtype=torch.uint8, device="cuda") if x == "mx4" else None
    offsets = torch.tensor([1, 2, 2, rows - 1], dtype=torch.int32, device="cuda")
    named = torch.from_numpy(rng(rows).integers(-1, 5, rows).astype(np.int32)).cuda()
    Y = torch.full((rows, out + 2), 9.0, device="cuda")
    ctx.adadim_mx4_matmul_experts(X, codes, scales, offsets, Y[:, :out], in_f=inn, x_scales=xs, rows=named)
    assert bool((Y[1:rows - 1, :out] == 0.0).all())
    assert bool((Y[0] == 9.0).all()) and bool((Y[rows - 1] == 9.0).all()) and bool((Y[:, out:] == 9.0).all())
