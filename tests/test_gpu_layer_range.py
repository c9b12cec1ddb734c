"""Activations and their slopes over their whole range, where only a relative bound says something: near zero
and in the tails.

u is half a step of the rounding of a result, relative to it: 2^-8 for bf16, 2^-24 for fp32.
"""
import numpy as np
import pytest
import torch

import paper_2309_15275_b200 as lbp
from oracle import layer_oracle as Y

pytestmark = pytest.mark.gpu

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
DTYPES = [torch.bfloat16, torch.float32]
ACTS = ["relu", "gelu", "gelu_tanh", "silu"]
# rows, Cin, Cout: every form of lbp_linear.  bf16: up to 8 and 16 tokens, a CTA a tile, K shared among four and two CTAs of a
# cluster, CTA pairs; fp32: few tokens, one tile and several to a CTA.
FORMS = [(5, 64, 128), (12, 64, 128), (100, 128, 192), (100, 1024, 192), (1000, 2304, 768), (1000, 128, 64), (1000, 192, 512),
         (20000, 64, 128)]


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    return torch.device("cuda:0")


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def _picks(Cin, Cout, dtype):
    """A weight that picks a channel of x for each output: z = x[:, c % Cin]."""
    w = torch.zeros(Cout, Cin, dtype=dtype)
    w[torch.arange(Cout), torch.arange(Cout) % Cin] = 1.0
    return w.cuda()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("a", ACTS)
@pytest.mark.parametrize("rows,Cin,Cout", FORMS)
def test_activations_near_zero(dev, dtype, a, rows, Cin, Cout):
    """act(0) is 0, and for z from x of 2^-118 to 2^-6 there is no absolute error: u and, of the activation itself, 2^-12 (bf16; the
    largest is that of GELU's polynomial, 3.7e-5 < 2^-14, of half of z) or 2^-20 (fp32: 3.9e-7 < 2^-21 of the
    same, and a few units of 2^-23 of the exponential and the reciprocal), times what drop() scales by."""
    g = torch.Generator().manual_seed(rows + Cin)
    size = torch.exp2(-6 - 112 * torch.rand(rows, Cin, generator=g, dtype=torch.float64))
    x = (size * (1 - 2 * torch.randint(0, 2, (rows, Cin), generator=g))).to(dtype)
    x[rows // 2] = 0.0
    x[:, 3] = -0.0
    x, w = x.cuda(), _picks(Cin, Cout, dtype)
    picked = f64(x)[:, np.arange(Cout) % Cin]
    for p in (0.0, 0.25):
        y, z = lbp.lbp_linear(x, w, activation=a, p=p, seed=7, offset=4, save_z=True)
        z = f64(z)   # (exactly what the activation is taken of: x of bf16 passes unrounded)
        assert np.all(np.abs(z - picked) <= (0.0 if dtype == torch.bfloat16 else Cin * 2.0 ** -23) * np.abs(picked))
        want = Y.drop(Y.act(z, a), Y.row_numbers(rows, Cout), p, 7, 4)
        off, own = np.abs(f64(y) - want), HALF[dtype] + (2.0 ** -12 if dtype == torch.bfloat16 else 2.0 ** -20)
        assert np.all(off <= own * np.abs(want)), (p, float(np.max(off / np.maximum(np.abs(want), 1e-300))))
        assert torch.equal(lbp.lbp_linear(x, w, activation=a, p=p, seed=7, offset=4), y)


@pytest.mark.parametrize("dtype", DTYPES)
def test_slope_of_gelu_in_its_negative_tail(dev, dtype):
    """Phi(z) + z phi(z) for -12 <= z <= -1, away from its zero at -0.75: no absolute error.

    It is exp(-a^2/2) (Q - a / sqrt(2 pi)).  Q is off by at most 4e-7 (fp32) or 3.7e-5 (bf16) of itself, which at -1, where
    the difference is smallest beside Q (0.137 and 0.262), is 2^-20 and 2^-13.7 of the result; the exponent's two roundings are
    at most a^2 2^-24, the constant's and the exponential's own a^2 2^-25 and 2^-22."""
    z = torch.linspace(-12, -1, 49152 * 8, dtype=torch.float64).view(-1, 512).to(dtype)
    g = torch.where(torch.arange(z.numel()).view_as(z) % 3 == 0, -0.75, 1.0).to(dtype)
    zz = f64(z)
    for p in (0.0, 0.4):
        want = Y.drop(f64(g), Y.row_numbers(*z.shape), p, 3, 8) * Y.act_slope(zz, "gelu")
        got = f64(lbp.lbp_linear_grad(g.cuda(), z.cuda(), activation="gelu", p=p, seed=3, offset=8))
        own = 2.0 ** -12 if dtype == torch.bfloat16 else 2.0 ** -19 * (1 + zz * zz)
        off = np.abs(got - want)
        assert np.all(off <= (HALF[dtype] + own) * np.abs(want)), (p, float(np.max(off / np.maximum(np.abs(want), 1e-300))))
        assert np.all(got[want != 0] != 0)
