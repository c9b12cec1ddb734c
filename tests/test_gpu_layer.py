"""A layer's epilogue, its gradients and dropout against the fp64 oracle.

Bounds, element by element (u = 2^-8 for bf16, 2^-24 for fp32: half a step of the rounding of
a result, relative to it):
  z     u |z| + K 2^-23 S, with S the sum of |x w| over the K terms and |b|: fp32 sums of K + 1 terms are off
        by at most K 2^-24 S when each addition rounds, and the tensor cores' additions cut, which is
        twice that
  y     u |y| + s (1.13 dz + da) + 2^-23 (|r| + |d|): dz the second part of z's bound (1.13 bounds the
        activations' slopes), da the error of the activation itself, s the scale of drop(), the rest the sum
        with the residual.  da: 2^-13 |act| + 2^-20 for bf16 data, whose GELU is approximated to 3.7e-5 of Phi(-|z|)
        and the others to a few units of 2^-22, 2^-20 (1 + z^2) |act| + 2^-24 for
        fp32 (a few units of 2^-22, and of 2^-24 times z^2 for the rounding of the exponent)
  g_z   (u + 2^-21) |g_z| + s |g_y| ds, ds = 2^-14 (bf16), 2^-19 (fp32) the error of a slope (the parts of a
        slope are at most z^2 exp(-z^2/2) times a rounding of 2^-24 each)
"""
import numpy as np
import pytest
import torch

import paper_2309_15275_b200 as lbp
from oracle import lbp_oracle as O
from oracle import layer_oracle as Y

pytestmark = pytest.mark.gpu

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
DTYPES = [torch.bfloat16, torch.float32]
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    return torch.device("cuda:0")


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def _normal(shape, std, dtype, seed):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * std).to(dtype).cuda()


def _inputs(rows, Cin, Cout, dtype, seed=0):
    return (_normal((rows, Cin), 1.0, dtype, 3 * seed), _normal((Cout, Cin), Cin ** -0.5, dtype, 3 * seed + 1),
            _normal((Cout,), 0.3, dtype, 3 * seed + 2))


def _scale(p):
    t = Y.threshold(p)
    return 65536.0 / (65536 - t) if t < 65536 else 1.0


def _want_linear(x, W, b, a, res, p, seed, offset, first=0, step=0):
    """z, y and their bounds."""
    x, W = x.double(), W.double()
    z = x @ W.t()
    S = x.abs() @ W.abs().t()
    if b is not None:
        z, S = z + b.double(), S + b.double().abs()
    z, dz = f64(z), x.shape[1] * 2.0 ** -23 * f64(S)
    v = Y.act(z, a)
    d = Y.drop(v, Y.row_numbers(*z.shape, first, step), p, seed, offset)
    r = 0.0 if res is None else f64(res)
    return z, d + r, dz, v, np.abs(r) + np.abs(d)


def _check_linear(dtype, got_y, got_z, want, p, fast=None):
    z, y, dz, v, parts = want
    u = HALF[dtype]
    if got_z is not None:
        assert np.all(np.abs(f64(got_z) - z) <= u * np.abs(z) + dz), "z"
    if dtype == torch.bfloat16:
        da = 2.0 ** -13 * np.abs(v) + 2.0 ** -20
    else:
        da = 2.0 ** -20 * (1 + z * z) * np.abs(v) + 2.0 ** -24
    bound = u * np.abs(y) + _scale(p) * (1.13 * dz + da) + 2.0 ** -23 * parts
    off = np.abs(f64(got_y) - y)
    assert np.all(off <= bound), ("y", float(np.max(off / bound)))


# One token, the borders of the tiles and of the forms for few rows, odd and long ones.
ROWS = [1, 2, 5, 8, 9, 16, 17, 32, 33, 64, 65, 127, 128, 129, 197, 256, 257, 300, 515]
SIZES = [(8, 8), (48, 192), (192, 48), (72, 264), (768, 768), (1032, 24), (64, 520), (2304, 136)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("i,rows", list(enumerate(ROWS)))
def test_linear_over_rows_and_widths(dev, dtype, i, rows):
    for j, (Cin, Cout) in enumerate(SIZES):
        n = i + j
        x, W, b = _inputs(rows, Cin, Cout, dtype, n)
        a, p = ACTS[n % 5], (0.0, 0.1, 0.5)[n % 3]
        res = _normal((rows, Cout), 1.0, dtype, 900 + n) if n % 2 else None
        bias = b if n % 4 else None
        y, z = lbp.lbp_linear(x, W, bias, activation=a, residual=res, p=p, seed=n * 2 ** 33 + 5, offset=4 * n, save_z=True)
        _check_linear(dtype, y, z, _want_linear(x, W, bias, a, res, p, n * 2 ** 33 + 5, 4 * n), p)
        # without z the same y, bit for bit, and again the same
        again = lbp.lbp_linear(x, W, bias, activation=a, residual=res, p=p, seed=n * 2 ** 33 + 5, offset=4 * n)
        assert torch.equal(again, y)


@pytest.mark.parametrize("Cin,Cout", [(4, 4), (12, 20), (52, 100), (100, 52), (4, 1028)])
@pytest.mark.parametrize("rows", [1, 3, 31, 130])
def test_linear_fp32_at_channels_of_four(dev, rows, Cin, Cout):
    x, W, b = _inputs(rows, Cin, Cout, torch.float32, rows)
    y, z = lbp.lbp_linear(x, W, b, activation="gelu", p=0.3, seed=11, offset=8, save_z=True)
    _check_linear(torch.float32, y, z, _want_linear(x, W, b, "gelu", None, 0.3, 11, 8), 0.3)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("a", ACTS)
@pytest.mark.parametrize("rows,p", [(6, 0.0), (6, 0.25), (40, 0.0), (700, 0.25), (700, 1.0)])
def test_linear_activations_and_dropout(dev, dtype, a, rows, p):
    x, W, b = _inputs(rows, 256, 384, dtype, rows)
    x = x * 3      # pre-activations from -10 to 10
    res = _normal((rows, 384), 1.0, dtype, 5)
    for r in (None, res):
        y, z = lbp.lbp_linear(x, W, b, activation=a, residual=r, p=p, seed=77, offset=2 ** 40 + 4, save_z=True)
        _check_linear(dtype, y, z, _want_linear(x, W, b, a, r, p, 77, 2 ** 40 + 4), p)


@pytest.mark.parametrize("rows,Cin,Cout,dtype", [(32768, 768, 3072, torch.bfloat16), (8192, 3072, 768, torch.bfloat16),
                                                 (50176, 48, 192, torch.bfloat16), (3136, 448, 1792, torch.float32),
                                                 (1025, 4096, 1024, torch.bfloat16)])
def test_linear_at_the_sizes_of_the_configurations(dev, rows, Cin, Cout, dtype):
    x, W, b = _inputs(rows, Cin, Cout, dtype, 1)
    y, z = lbp.lbp_linear(x, W, b, activation="gelu", p=0.1, seed=3, offset=0, save_z=True)
    # rows from all over; the oracle takes a while over all of them
    pick = torch.unique(torch.cat([torch.arange(40), torch.randint(0, rows, (400,), generator=torch.Generator().manual_seed(1)),
                                   torch.arange(rows - 40, rows)])).cuda()
    xs = x[pick].double()
    zw = f64(xs @ W.double().t() + b.double())
    dz = Cin * 2.0 ** -23 * f64(xs.abs() @ W.double().abs().t() + b.double().abs())
    v = Y.act(zw, "gelu")
    numbers = f64(pick)[:, None].astype(np.int64) * Cout + np.arange(Cout)[None, :]
    d = Y.drop(v, numbers, 0.1, 3, 0)
    _check_linear(dtype, y[pick], z[pick], (zw, d, dz, v, np.abs(d)), 0.1)
    # every row, against the library's own product as torch has it: no tile is missing
    ref = (x.float() @ W.float().t() + b.float())
    assert float((z.float() - ref).norm() / ref.norm()) < (3e-3 if dtype == torch.bfloat16 else 2e-6)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", [3, 50, 300])
def test_linear_views(dev, dtype, rows):
    """Channel slices and tokens of wider tensors: strided in place, and nothing is written beside them."""
    Cin, Cout, n = 64, 128, (8 if dtype == torch.bfloat16 else 4)
    wide = _normal((rows, Cin + 3 * n), 1.0, dtype, 1)
    x = wide[:, n:n + Cin]
    _, W, b = _inputs(rows, Cin, Cout, dtype, 2)
    res = _normal((rows, Cout + n), 1.0, dtype, 4)[:, :Cout]
    outs = [torch.full((rows + 2, Cout + 2 * n), 7.0, dtype=dtype, device=dev) for _ in range(2)]
    y, z = (o[1:-1, n:n + Cout] for o in outs)
    got = lbp.lbp_linear(x, W, b, activation="silu", residual=res, p=0.2, seed=1, offset=4, out=y, z=z)
    assert got[0].data_ptr() == y.data_ptr() and got[1].data_ptr() == z.data_ptr()
    _check_linear(dtype, y, z, _want_linear(x, W, b, "silu", res, 0.2, 1, 4), 0.2)
    for o in outs:
        o[1:-1, n:n + Cout] = 7.0
        assert bool((o == 7.0).all())
    # onto the residual itself
    acc = res.clone(memory_format=torch.contiguous_format)
    same = lbp.lbp_linear(x, W, b, residual=acc, p=0.2, seed=1, offset=4)
    lbp.lbp_linear(x, W, b, residual=acc, p=0.2, seed=1, offset=4, out=acc)
    assert torch.equal(acc, same)
    # leading dimensions
    x3 = x.contiguous().view(1, rows, 1, Cin)
    assert lbp.lbp_linear(x3, W, b).shape == (1, rows, 1, Cout)
    with pytest.raises(ValueError, match="distance"):
        lbp.lbp_linear(_normal((4, 6, Cin), 1.0, dtype, 0)[:, :3], W, b)
    with pytest.raises(ValueError, match="contiguous"):
        lbp.lbp_linear(_normal((Cin, rows), 1.0, dtype, 0).t(), W, b)
    with pytest.raises(ValueError, match="overlap"):
        lbp.lbp_linear(_normal((1, Cin), 1.0, dtype, 0).expand(5, Cin), W, b)
    with pytest.raises(ValueError, match="overlap"):
        lbp.lbp_linear(x, W, b, residual=b.expand(rows, Cout))


@pytest.mark.parametrize("dtype", DTYPES)
def test_calls_without_tokens(dev, dtype):
    x, W, b = _inputs(4, 64, 32, dtype)
    y, z = lbp.lbp_linear(x[:0], W, b, activation="gelu", save_z=True)
    assert y.shape == z.shape == (0, 32)
    assert lbp.lbp_dropout(x[:0], 0.5).shape == (0, 64)
    assert lbp.lbp_linear_grad(x[:0], x[:0], activation="relu").shape == (0, 64)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", [4, 200])
def test_values_that_are_not_finite(dev, dtype, rows):
    """They stay in their rows, activations go to their limits, and a dropped one is zero."""
    x, W, b = _inputs(rows, 64, 128, dtype, 9)
    x[1, 3] = float("inf")
    x[2, 5] = float("nan")
    p, seed, offset = 0.5, 9, 16
    kept = torch.from_numpy(Y.keep(Y.row_numbers(rows, 128), p, seed, offset)).to(dev)
    for a in ACTS:
        clean = x.clone()
        clean[1, 3] = clean[2, 5] = 0
        y, z = lbp.lbp_linear(x, W, b, activation=a, p=p, seed=seed, offset=offset, save_z=True)
        yc = lbp.lbp_linear(clean, W, b, activation=a, p=p, seed=seed, offset=offset)
        others = [r for r in range(rows) if r not in (1, 2)]
        assert torch.equal(y[others], yc[others])
        assert bool(torch.isinf(z[1]).all()) and bool(torch.isnan(z[2]).all())
        assert bool((y[~kept] == 0).all())
        up, down = kept[1] & (z[1] > 0), kept[1] & (z[1] < 0)
        assert bool((y[1][up] == float("inf")).all())
        assert bool((y[1][down] == (float("-inf") if a == "none" else 0.0)).all())
        assert bool(torch.isnan(y[2][kept[2]]).all())
        # and their gradients
        g = torch.ones_like(z)
        gz = lbp.lbp_linear_grad(g, z, activation=a, p=p, seed=seed, offset=offset)
        assert bool((gz[~kept] == 0).all())
        if a != "none":
            assert bool((gz[1][up] == 2).all()) and bool((gz[1][down] == 0).all())
            assert bool(torch.isnan(gz[2][kept[2]]).all())
    r = torch.full((rows, 64), 2.0, dtype=dtype, device=dev)
    bad = torch.full((rows, 64), float("nan"), dtype=dtype, device=dev)
    assert torch.equal(lbp.lbp_dropout(bad, 1.0, seed=1, residual=r), r)


# ------------------------------------------------------------------ pointwise calls ----
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,Cc", [(1, 8), (1, 768), (3, 24), (7, 1000), (197, 768), (1031, 48), (4099, 264)])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.75, 1.0])
def test_dropout(dev, dtype, rows, Cc, p):
    x, r = _normal((rows, Cc), 1.0, dtype, 1), _normal((rows, Cc), 1.0, dtype, 2)
    seed, offset = 2 ** 63 + 17, 2 ** 35 + 12
    n = Y.row_numbers(rows, Cc)
    d = Y.drop(f64(x), n, p, seed, offset)
    for res in (None, r):
        want = d if res is None else d + f64(res)
        got = lbp.lbp_dropout(x, p, seed=seed, offset=offset, residual=res)
        parts = np.abs(d) + (0 if res is None else np.abs(f64(res)))
        assert np.all(np.abs(f64(got) - want) <= HALF[dtype] * np.abs(want) + 2.0 ** -23 * parts)
        # in place
        for target in (x.clone(),) if res is None else (x.clone(), r.clone()):
            src = target if res is None or torch.equal(target, x) else x
            rr = None if res is None else (target if src is x else r)
            assert torch.equal(lbp.lbp_dropout(src, p, seed=seed, offset=offset, residual=rr, out=target), got)
    if p > 0:   # what is zero is what the oracle drops
        assert np.array_equal(f64(lbp.lbp_dropout(torch.ones_like(x), p, seed=seed, offset=offset)) == 0,
                              ~Y.keep(n, p, seed, offset))
    # the backward pass: the same choice on the gradient
    g = _normal((rows, Cc), 1.0, dtype, 3)
    assert torch.equal(lbp.lbp_linear_grad(g, p=p, seed=seed, offset=offset), lbp.lbp_dropout(g, p, seed=seed, offset=offset))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("a", ACTS)
@pytest.mark.parametrize("rows,Cc,p", [(1, 64, 0.0), (49, 1792, 0.0), (197, 768, 0.1), (1030, 200, 0.6)])
def test_linear_grad(dev, dtype, a, rows, Cc, p):
    g, z = _normal((rows, Cc), 0.7, dtype, 1), _normal((rows, Cc), 3.0, dtype, 2)
    want = Y.drop(f64(g), Y.row_numbers(rows, Cc), p, 5, 4) * Y.act_slope(f64(z), a)
    got = lbp.lbp_linear_grad(g, z, activation=a, p=p, seed=5, offset=4)
    ds = 2.0 ** -14 if dtype == torch.bfloat16 else 2.0 ** -19
    bound = (HALF[dtype] + 2.0 ** -21) * np.abs(want) + _scale(p) * np.abs(f64(g)) * ds
    assert np.all(np.abs(f64(got) - want) <= bound)
    for target in (g.clone(), z.clone()):
        args = (target, z) if torch.equal(target, g) else (g, target)
        assert torch.equal(lbp.lbp_linear_grad(*args, activation=a, p=p, seed=5, offset=4, out=target), got)
    if p == 0 and dtype == torch.float32:
        # differences of the forward call itself: fp32, step h = 2^-6: h^2/6 |f'''| and rounding 2^-22 |f| / h
        h = 2.0 ** -6
        eye = torch.eye(Cc, device=dev)
        f = lambda v: f64(lbp.lbp_linear(v, eye, activation=a))  # noqa: E731
        slope = (f(z + h) - f(z - h)) / (2 * h)
        away = np.abs(f64(z)) > h if a == "relu" else np.ones(z.shape, bool)
        assert np.all((np.abs(slope * f64(g) - f64(got)) <= np.abs(f64(g)) * (h * h + 2.0 ** -22 * 16 / h + ds))[away])


@pytest.mark.parametrize("dtype", DTYPES)
def test_pointwise_views(dev, dtype):
    n = 8 if dtype == torch.bfloat16 else 4
    g = _normal((6, 10, 96 + 2 * n), 1.0, dtype, 1)[:, :, n:n + 96]
    z = _normal((6, 10, 96 + n), 1.0, dtype, 2)[:, :, :96]
    whole = torch.full((60, 96 + n), 7.0, dtype=dtype, device=dev)
    out = whole.view(6, 10, 96 + n)[:, :, :96]
    got = lbp.lbp_linear_grad(g, z, activation="gelu", p=0.3, seed=1, out=out)
    assert torch.equal(got, lbp.lbp_linear_grad(g.contiguous(), z.contiguous(), activation="gelu", p=0.3, seed=1))
    assert bool((whole[:, 96:] == 7.0).all())
    whole.fill_(7.0)
    got = lbp.lbp_dropout(g, 0.3, seed=1, residual=z, out=out)
    assert torch.equal(got, lbp.lbp_dropout(g.contiguous(), 0.3, seed=1, residual=z.contiguous()))
    assert bool((whole[:, 96:] == 7.0).all())


def test_numbers_past_32_bits(dev):
    """Element numbers past 2^35 (groups past 32 bits) and strides of the numbering, through the C ABI."""
    from paper_2309_15275_b200 import binding as B
    x = torch.ones(5, 64, dtype=torch.bfloat16, device=dev)
    out = torch.empty_like(x)
    e = B._epilogue(None, 0.5, 3, 8, None, x.device)
    e.first, e.number = 2 ** 36 + 16, B.View(0, 0, 4096)
    assert B._lib().lbp_dropout(x.data_ptr(), None, out.data_ptr(), 5, 64, lbp.LBP_BF16, None, e, B._stream()) == 0
    want = Y.keep(Y.row_numbers(5, 64, 2 ** 36 + 16, 4096), 0.5, 3, 8)
    assert np.array_equal(f64(out) != 0, want)


def test_large_tensors_past_2_31_elements(dev):
    """Offsets past 32 bits: 2^31 + 2^22 elements of bf16, the far end against the oracle."""
    rows, Cc = (2 ** 31 + 2 ** 22) // 4096, 4096
    x = torch.ones(rows, Cc, dtype=torch.bfloat16, device=dev)
    y = lbp.lbp_dropout(x, 0.5, seed=21, offset=4)
    want = Y.keep(Y.row_numbers(8, Cc, (rows - 8) * Cc), 0.5, 21, 4)
    assert np.array_equal(f64(y[-8:]) != 0, want)
    W = torch.zeros(8, Cc, dtype=torch.bfloat16, device=dev)
    W[:, 7] = torch.arange(8, dtype=torch.bfloat16, device=dev)
    x[-3, 7] = 5.0
    y = lbp.lbp_linear(x, W)
    assert torch.equal(y[-3], 5 * W[:, 7]) and torch.equal(y[-2], W[:, 7]) and torch.equal(y[0], W[:, 7])


# ---------------------------------------------------------------------- projection ----
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("k,H,W,r", [(8, 16, 16, 8), (8, 7, 7, 10), (4, 14, 9, 3), (4, 8, 8, 15), (16, 20, 33, 6), (8, 24, 16, 40),
                                     (8, 8, 8, 64), (16, 16, 16, 60)])
def test_project_grad(dev, dtype, k, H, W, r):
    Cc, B, p = 200, 3, 0.2
    bases = O.select_bases(k, O.RULE_PREFIX, r)
    g, z = _normal((B, H, W, Cc), 1.0, dtype, 1), _normal((B, H, W, Cc), 2.0, dtype, 2)
    n = Y.row_numbers(B * H * W, Cc).reshape(B, H, W, Cc)
    for a, q in (("gelu", p), ("none", p), ("silu", 0.0), ("relu", 0.0), ("gelu_tanh", p)):
        gz = Y.drop(f64(g), n, q, 9, 12) * Y.act_slope(f64(z), a)
        want = O.project_padded(gz, k, bases)
        got = lbp.lbp_project_grad(g, None if a == "none" else z, k, bases, activation=a, p=q, seed=9, offset=12)
        assert got.shape == want.shape
        # every g_z is off by its bound (test_linear_grad) and rounded once more to bf16 on the way into the
        # products; a coefficient is 1/k times a signed sum of k^2 of them, in fp32, and rounded
        u = HALF[dtype]
        ds = 2.0 ** -14 if dtype == torch.bfloat16 else 2.0 ** -19
        each = (u + 2.0 ** -21) * np.abs(gz) + _scale(q) * np.abs(f64(g)) * ds
        total = O.project_padded(np.abs(gz) * 2.0 ** -24 * k * k + each, k, [(0, 0)])
        assert np.all(np.abs(f64(got) - want) <= u * np.abs(want) + total), (a, q)


def test_project_grad_of_a_strided_sequence(dev):
    """The tokens of a (B, 1 + H*W, C) sequence behind its class token, numbered as the sequence is."""
    from paper_2309_15275_b200 import binding as B
    Bn, H, W, Cc, k = 2, 14, 14, 128, 8
    bases = O.select_bases(k, O.RULE_PREFIX, 8)
    seq_g, seq_z = (_normal((Bn, 1 + H * W, Cc), 1.0, torch.bfloat16, s) for s in (1, 2))
    g, z = (t.as_strided((Bn, H, W, Cc), ((1 + H * W) * Cc, W * Cc, Cc, 1), Cc) for t in (seq_g, seq_z))
    e = B._epilogue("gelu", 0.3, 4, 8, None, g.device)
    e.first, e.number = Cc, B.View((1 + H * W) * Cc, W * Cc, Cc)
    view = B.View((1 + H * W) * Cc, W * Cc, Cc)
    out = torch.empty((Bn, 2, 2, 8, Cc), dtype=torch.bfloat16, device=dev)
    ws = torch.empty(lbp.lbp_project_grad_workspace_bytes(Bn, H, W, Cc, k, 8, lbp.LBP_BF16), dtype=torch.uint8, device=dev)
    assert B._lib().lbp_project_grad(g.data_ptr(), z.data_ptr(), out.data_ptr(), Bn, H, W, Cc, k, B._bases(bases), 8,
                                     lbp.LBP_BF16, view, e, ws.data_ptr(), ws.numel(), B._stream()) == 0
    assert lbp.lbp_poll_status(ws) == 0
    whole = lbp.lbp_linear_grad(seq_g, seq_z, activation="gelu", p=0.3, seed=4, offset=8)
    ref = lbp.lbp_project(whole[:, 1:].reshape(Bn, H, W, Cc).contiguous(), k, bases)
    # the two may round g_z at different places: each coefficient within the sum of half steps of its 64 terms
    each = np.abs(f64(whole[:, 1:].reshape(Bn, H, W, Cc))) * 2.0 ** -7
    bound = O.project_padded(each, k, [(0, 0)]) + 2.0 ** -7 * np.abs(f64(ref))
    assert np.all(np.abs(f64(out) - f64(ref)) <= bound)
    # a strided call through the binding
    got = lbp.lbp_project_grad(g, z, k, bases, activation="gelu")
    dense = lbp.lbp_project_grad(g.contiguous(), z.contiguous(), k, bases, activation="gelu")
    assert torch.equal(got, dense)


# ------------------------------------------------------------------ backward, as a whole ----
def _rel(a, b):
    return float((a.double() - b.double()).norm() / b.double().norm())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("k,r,H,W", [(8, 8, 16, 16), (8, 10, 7, 7), (4, 3, 14, 14), (8, 64, 8, 8), (8, 50, 16, 8)])
def test_backward_act_is_the_backward_pass_of_its_gradient(dev, dtype, k, r, H, W):
    B, Cin, Cout = 4, 192, 256
    bases = O.select_bases(k, O.RULE_PREFIX, r)
    x, g, z = (_normal((B, H, W, c), s, dtype, i) for i, (c, s) in enumerate(((Cin, 1.0), (Cout, 0.1), (Cout, 1.5))))
    w = _normal((Cout, Cin), Cin ** -0.5, dtype, 7)
    gb, gb2 = (torch.empty(Cout, device=dev) for _ in range(2))
    for a, p in (("gelu", 0.1), ("none", 0.3), ("relu", 0.0)):
        zz = None if a == "none" else z
        gx, gw = lbp.lbp_backward_act(x, g, zz, w, k, bases, activation=a, p=p, seed=5, offset=4, g_bias=gb)
        gz = lbp.lbp_linear_grad(g, zz, activation=a, p=p, seed=5, offset=4)
        rx, rw = lbp.lbp_backward_ex(x, gz, w, k, bases, g_bias=gb2)
        # the same but for where g_z and its coefficients round: 2^-9 a rounding in the mean, three of them (bf16)
        tol = 3 * 2.0 ** -9 if dtype == torch.bfloat16 else 1e-5
        assert max(_rel(gx, rx), _rel(gw, rw), _rel(gb, gb2)) <= tol, (a, p)
        # x_hat instead, accumulating
        xh = lbp.lbp_project(x, k, bases)
        acc = torch.ones_like(gw)
        px, pw = lbp.lbp_backward_act(None, g, zz, w, k, bases, activation=a, p=p, seed=5, offset=4, x_hat=xh, beta=1.0, g_W=acc)
        assert max(_rel(px, rx), _rel(pw - 1, rw)) <= (tol if dtype == torch.bfloat16 else 3e-5)


@pytest.mark.parametrize("n_cls", [0, 1, 2])
@pytest.mark.parametrize("dtype", DTYPES)
def test_a_vit_mlp_trains_as_its_formulas_say(dev, dtype, n_cls):
    """fc1 with GELU and dropout, fc2 with dropout onto the residual stream, forward and backward through
    autograd, against the oracle fed with the same numbers (full rank: exact gradients)."""
    B, H, W, d, k, p = 2, 14, 14, 64, 8, 0.2
    grid = (H, W) if n_cls else None
    bases = O.select_bases(k, O.RULE_PREFIX, k * k)
    torch.manual_seed(5)
    make = lambda i, o, **m: lbp.LbpLinear(i, o, k, bases, device=dev, dtype=dtype, bias=True, grid=grid, dropout=p, **m)  # noqa: E731
    fc1, fc2 = make(d, 4 * d, activation="gelu"), make(4 * d, d)
    with torch.no_grad():
        fc1.bias.normal_(0, 0.1)
        fc2.bias.normal_(0, 0.1)
    shape = (B, n_cls + H * W, d) if n_cls else (B, H, W, d)
    x = _normal(shape, 1.0, dtype, 3).requires_grad_()
    res = _normal(shape, 1.0, dtype, 4).requires_grad_()
    torch.manual_seed(99)
    first = torch.cuda.default_generators[0].get_offset()
    y = fc2(fc1(x), residual=res)
    seed = torch.cuda.initial_seed()
    g = _normal(shape, 0.5, dtype, 6)
    params = (x, res, fc1.weight, fc1.bias, fc2.weight, fc2.bias)
    got = torch.autograd.grad(y, params, g)

    rows = lambda t: f64(t).reshape(-1, t.shape[-1])  # noqa: E731
    X, R, G, W1, b1, W2, b2 = rows(x), rows(res), rows(g), *(f64(q) for q in (fc1.weight, fc1.bias, fc2.weight, fc2.bias))
    z1 = X @ W1.T + b1
    n1, n2 = Y.row_numbers(*z1.shape), Y.row_numbers(*R.shape)
    h = Y.drop(Y.act(z1, "gelu"), n1, p, seed, first)
    want_y = R + Y.drop(h @ W2.T + b2, n2, p, seed, first + 4)
    gz2 = Y.drop(G, n2, p, seed, first + 4)
    gh = gz2 @ W2
    gz1 = Y.drop(gh, n1, p, seed, first) * Y.act_slope(z1, "gelu")
    want = (gz1 @ W1, G, gz1.T @ X, gz1.sum(0), gz2.T @ h, gz2.sum(0))
    rel = lambda a, b: np.linalg.norm(rows(a).reshape(-1) - b.reshape(-1)) / np.linalg.norm(b)  # noqa: E731
    # a chain of at most five roundings to bf16 of 2^-9 each in the mean; fp32: as the other parity tests
    tol = 5 * 2.0 ** -9 if dtype == torch.bfloat16 else 1e-5
    assert rel(y, want_y) <= tol
    for name, a, b in zip(("x", "res", "W1", "b1", "W2", "b2"), got, want):
        assert a.shape == {"x": x, "res": res, "W1": fc1.weight, "b1": fc1.bias, "W2": fc2.weight, "b2": fc2.bias}[name].shape
        assert rel(a, b) <= tol, name
    # answering: no dropout, nothing drawn
    fc1.eval(), fc2.eval()
    before = torch.cuda.default_generators[0].get_offset()
    with torch.no_grad():
        y = fc2(fc1(x), residual=res)
    assert torch.cuda.default_generators[0].get_offset() == before
    assert rel(y, R + Y.act(z1, "gelu") @ W2.T + b2) <= tol


def test_module_with_saved_projection_and_low_rank(dev):
    B, H, W, Cin, Cout, k, r = 4, 16, 16, 128, 192, 8, 8
    bases = O.select_bases(k, O.RULE_PREFIX, r)
    layer = lbp.LbpLinear(Cin, Cout, k, bases, device=dev, dtype=torch.bfloat16, bias=True, save_projected=True,
                          activation="gelu", dropout=0.1)
    x = _normal((B, H, W, Cin), 1.0, torch.bfloat16, 1).requires_grad_()
    torch.manual_seed(1)
    off = torch.cuda.default_generators[0].get_offset()
    y = layer(x)
    g = _normal(y.shape, 0.1, torch.bfloat16, 2)
    gx, gw, gb = torch.autograd.grad(y, (x, layer.weight, layer.bias), g)
    z = lbp.lbp_linear(x.detach(), layer.weight.detach(), layer.bias.detach())
    gz = lbp.lbp_linear_grad(g, z, activation="gelu", p=0.1, seed=torch.cuda.initial_seed(), offset=off)
    ref_b = torch.empty(Cout, device=dev)
    rx, rw = lbp.lbp_backward_ex(x.detach(), gz, layer.weight.detach(), k, bases, g_bias=ref_b)
    assert max(_rel(gx, rx), _rel(gw, rw), _rel(gb, ref_b)) <= 3 * 2.0 ** -9
    # under autocast everything is of its type
    wide = lbp.LbpLinear(Cin, Cout, k, bases, device=dev, dtype=torch.float32, bias=True, activation="gelu")
    xf = x.detach().float().requires_grad_()
    with torch.autocast("cuda", dtype=torch.bfloat16):
        y = wide(xf)
    assert y.dtype == torch.bfloat16
    y.backward(g)
    assert xf.grad.dtype == torch.float32 and wide.weight.grad.dtype == torch.float32
    with torch.autocast("cuda", dtype=torch.float16), pytest.raises(ValueError):
        wide(xf)
    with pytest.raises(ValueError):
        wide(xf.detach(), residual=torch.zeros(1, device=dev))


# --------------------------------------------------------------- streams, graphs, devices ----
def test_calls_on_another_stream_and_two_at_once(dev):
    x, W, b = _inputs(4000, 256, 512, torch.bfloat16)
    want = [lbp.lbp_linear(x, W, b, activation="gelu", p=0.1, seed=s) for s in (1, 2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(lbp.lbp_linear(x, W, b, activation="gelu", p=0.1, seed=i + 1))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(t, want[i]) for t in got[i])


def test_captured_calls_draw_new_numbers_at_each_replay(dev):
    for rows in (4, 100, 600):
        x, W, b = _inputs(rows, 64, 128, torch.bfloat16)
        rng = torch.tensor([41, 8], dtype=torch.int64, device=dev)
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            lbp.lbp_linear(x, W, b, activation="gelu", p=0.5, rng=rng, save_z=True)
            lbp.lbp_project_grad(x.view(1, 2, rows // 2, 64), None, 8, [(0, 0)], p=0.5, rng=rng)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y, z = lbp.lbp_linear(x, W, b, activation="gelu", p=0.5, rng=rng, save_z=True)
            gz = lbp.lbp_linear_grad(y, z, activation="gelu", p=0.5, rng=rng)
            d = lbp.lbp_dropout(x, 0.5, rng=rng, offset=4)
            t = lbp.lbp_project_grad(x.view(1, 2, rows // 2, 64), None, 8, [(0, 0)], p=0.5, rng=rng)
        seen = []
        for offset in (8, 16, 8):
            rng[1] = offset
            graph.replay()
            torch.cuda.synchronize()
            ref, rz = lbp.lbp_linear(x, W, b, activation="gelu", p=0.5, seed=41, offset=offset, save_z=True)
            assert torch.equal(y, ref) and torch.equal(z, rz)
            assert torch.equal(gz, lbp.lbp_linear_grad(ref, rz, activation="gelu", p=0.5, seed=41, offset=offset))
            assert torch.equal(d, lbp.lbp_dropout(x, 0.5, seed=41, offset=offset + 4))
            assert torch.equal(t, lbp.lbp_project_grad(x.view(1, 2, rows // 2, 64), None, 8, [(0, 0)], p=0.5, seed=41, offset=offset))
            seen.append(y.clone())
        assert torch.equal(seen[0], seen[2]) and not torch.equal(seen[0], seen[1])


def test_a_captured_training_step(dev):
    """Forward and backward of the module in one graph: every replay draws anew, and its backward pass
    sees the forward pass's choice."""
    B, H, W, d, k = 2, 8, 8, 64, 8
    bases = O.select_bases(k, O.RULE_PREFIX, 8)
    layer = lbp.LbpLinear(d, 2 * d, k, bases, device=dev, dtype=torch.bfloat16, bias=True, dropout=0.5)
    x = _normal((B, H, W, d), 1.0, torch.bfloat16, 1).requires_grad_()
    g = torch.ones(B, H, W, 2 * d, dtype=torch.bfloat16, device=dev)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            torch.autograd.grad(layer(x), (x, layer.weight, layer.bias), g)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = layer(x)
        gx, gw, gb = torch.autograd.grad(y, (x, layer.weight, layer.bias), g)
    masks = []
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        kept = (y != 0)     # (a bias and products of normal numbers are not zero)
        masks.append(kept.clone())
        gz = kept.to(torch.bfloat16) * 2
        ref_b = torch.empty(2 * d, device=dev)
        rx, rw = lbp.lbp_backward_ex(x.detach(), gz, layer.weight.detach(), k, bases, g_bias=ref_b)
        assert max(_rel(gx, rx), _rel(gw, rw), _rel(gb, ref_b)) <= 2 * 2.0 ** -9
    assert not torch.equal(masks[0], masks[1]) and not torch.equal(masks[1], masks[2])


def test_tensors_of_another_device_are_refused(dev):
    if torch.cuda.device_count() < 2:
        pytest.skip("one device")
    x, W, b = (t.to("cuda:1") for t in _inputs(4, 64, 32, torch.bfloat16))
    for call in (lambda: lbp.lbp_linear(x, W, b), lambda: lbp.lbp_dropout(x, 0.5), lambda: lbp.lbp_linear_grad(x)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("rows,Cin,Cout", [(100, 128, 192), (1000, 128, 64), (1000, 192, 512)])
def test_expired_wait_is_reported_and_the_next_call_is_clean(dev, rows, Cin, Cout):
    """No load is issued (one CTA a tile, and pairs): the call reports it, and the next one on the same workspace is right."""
    x, W, b = _inputs(rows, Cin, Cout, torch.bfloat16)
    res = _normal((rows, Cout), 1.0, torch.bfloat16, 8)
    ws = torch.zeros(lbp.lbp_linear_workspace_bytes(rows, Cin, Cout, lbp.LBP_BF16), dtype=torch.uint8, device=dev)
    lbp.lbp_test_stall_products(True, linear=True)
    try:
        lbp.lbp_linear(x, W, b, residual=res, ws=ws)
    finally:
        lbp.lbp_test_stall_products(False)
    assert lbp.lbp_poll_status(ws) == 10
    assert lbp.lbp_poll_status(ws) == 0
    y = lbp.lbp_linear(x, W, b, residual=res, ws=ws)
    assert lbp.lbp_poll_status(ws) == 0
    _check_linear(torch.bfloat16, y, None, _want_linear(x, W, b, "none", res, 0.0, 0, 0), 0.0)


def test_expired_wait_in_the_projection_of_a_gradient(dev):
    """No box is fetched: the warps that form the gradient give up too, the call reports it, the next one is right."""
    g, z = (_normal((2, 16, 24, 256), 1.0, torch.bfloat16, s) for s in (1, 2))
    bases = O.select_bases(8, O.RULE_PREFIX, 6)
    ws = torch.zeros(lbp.lbp_project_grad_workspace_bytes(2, 16, 24, 256, 8, 6, lbp.LBP_BF16), dtype=torch.uint8, device=dev)
    lbp.lbp_test_stall_products(True, projection=True)
    try:
        lbp.lbp_project_grad(g, z, 8, bases, activation="gelu", p=0.2, ws=ws)
    finally:
        lbp.lbp_test_stall_products(False)
    assert lbp.lbp_poll_status(ws) == 10
    got = lbp.lbp_project_grad(g, z, 8, bases, activation="gelu", p=0.2, ws=ws)
    assert lbp.lbp_poll_status(ws) == 0
    # the gradient is formed and rounded as lbp_linear_grad has it, and projected as lbp_project does
    gz = lbp.lbp_linear_grad(g, z, activation="gelu", p=0.2)
    assert torch.equal(got, lbp.lbp_project(gz, 8, bases))


@pytest.mark.parametrize("k,H,W,r", [(4, 9, 22, 3), (4, 16, 16, 16), (8, 23, 17, 8), (8, 16, 16, 40), (16, 20, 33, 6), (16, 16, 32, 48)])
@pytest.mark.parametrize("Cc", [8, 72, 640])
def test_projected_gradient_is_the_projection_of_the_gradient(dev, k, H, W, r, Cc):
    """Bit for bit: formed on the way into the projection or written out first."""
    bases = O.select_bases(k, O.RULE_LINF if r == k * k else O.RULE_PREFIX, k if r == k * k else r)
    g, z = _normal((5, H, W, Cc), 1.0, torch.bfloat16, 1), _normal((5, H, W, Cc), 2.0, torch.bfloat16, 2)
    for a in ACTS:
        for p in (0.0, 0.3, 0.7, 1.0):
            zz = None if a == "none" else z
            gz = lbp.lbp_linear_grad(g, zz, activation=a, p=p, seed=3, offset=4)
            got = lbp.lbp_project_grad(g, zz, k, bases, activation=a, p=p, seed=3, offset=4)
            assert torch.equal(got, lbp.lbp_project(gz, k, bases)), (a, p)


def test_backward_act_without_the_mean_basis_and_on_views(dev):
    """A list without (0, 0) cannot give the bias's sum; gradients with strides of a wider tensor; both as on the written gradient."""
    B, H, W, Cin, Cout, k = 3, 16, 16, 128, 192, 8
    x = _normal((B, H, W, Cin), 1.0, torch.bfloat16, 1)
    wide = _normal((2, B, H, W, Cout + 64), 1.0, torch.bfloat16, 2)
    g, z = wide[0, ..., 64:], wide[1, ..., 64:]
    w = _normal((Cout, Cin), Cin ** -0.5, torch.bfloat16, 3)
    for bases in ([(1, 0), (0, 1), (2, 2)], O.select_bases(k, O.RULE_PREFIX, 5)):
        for bias in (False, True):
            gb, gb2 = (torch.empty(Cout, device=dev) if bias else None for _ in range(2))
            gx, gw = lbp.lbp_backward_act(x, g, z, w, k, bases, activation="gelu", p=0.4, seed=1, offset=8, g_bias=gb)
            gz = lbp.lbp_linear_grad(g, z, activation="gelu", p=0.4, seed=1, offset=8)
            rx, rw = lbp.lbp_backward_ex(x, gz, w, k, bases, g_bias=gb2)
            assert torch.equal(gx, rx) and torch.equal(gw, rw)
            if bias:
                assert torch.equal(gb, gb2)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", [5, 300])
def test_all_tensors_in_columns_of_one_matrix(dev, dtype, rows):
    Cin, Cout = 64, 96
    wide = _normal((rows, Cin + 3 * Cout), 1.0, dtype, 1)
    x, r, y, z = wide[:, :Cin], *(wide[:, Cin + i * Cout:Cin + (i + 1) * Cout] for i in range(3))
    _, W, b = _inputs(rows, Cin, Cout, dtype, 2)
    before = wide.clone()
    ry, rz = lbp.lbp_linear(x.contiguous(), W, b, activation="gelu", residual=r.contiguous(), p=0.2, seed=1, save_z=True)
    lbp.lbp_linear(x, W, b, activation="gelu", residual=r, p=0.2, seed=1, out=y, z=z)
    assert torch.equal(y, ry) and torch.equal(z, rz) and torch.equal(wide[:, :Cin + Cout], before[:, :Cin + Cout])
    want = lbp.lbp_linear_grad(ry, rz, activation="gelu", p=0.2, seed=1)
    lbp.lbp_linear_grad(y, z, activation="gelu", p=0.2, seed=1, out=r)
    assert torch.equal(r, want) and torch.equal(wide[:, :Cin], before[:, :Cin])


def test_a_module_stored_without_an_epilogue_loads(dev, tmp_path):
    layer = lbp.LbpLinear(64, 32, 8, [(0, 0)], device=dev, dtype=torch.bfloat16)
    del layer.__dict__["activation"], layer.__dict__["dropout"]
    torch.save(layer, tmp_path / "layer.pt")
    back = torch.load(tmp_path / "layer.pt", weights_only=False)
    x = _normal((1, 8, 8, 64), 1.0, torch.bfloat16, 1)
    assert torch.equal(back(x), layer(x))


def test_dropout_repeats_under_checkpointing(dev):
    """torch's checkpoint puts the generator back for the second forward pass: the same elements are dropped."""
    from torch.utils.checkpoint import checkpoint
    layer = lbp.LbpLinear(64, 64, 8, O.select_bases(8, O.RULE_PREFIX, 64), device=dev, dtype=torch.float32, activation="silu", dropout=0.4)
    x = _normal((2, 8, 8, 64), 1.0, torch.float32, 1).requires_grad_()
    grads = []
    for run in (lambda: layer(layer(x)), lambda: checkpoint(lambda v: layer(layer(v)), x, use_reentrant=False)):
        torch.manual_seed(3)
        y = run()
        grads.append(torch.autograd.grad(y.square().sum(), (x, layer.weight)))
    assert all(torch.equal(a, b) for a, b in zip(*grads))


@pytest.mark.parametrize("dtype", DTYPES)
def test_without_activation_and_dropout_it_is_the_plain_call(dev, dtype):
    """The same launches, so the same bits; of a module too, with any number of class tokens."""
    x, g = _normal((4, 16, 16, 192), 1.0, dtype, 0), _normal((4, 16, 16, 256), 0.1, dtype, 1)
    w, bases = _normal((256, 192), 0.07, dtype, 2), O.select_bases(8, O.RULE_PREFIX, 8)
    gb, gb2 = (torch.empty(256, device=dev) for _ in range(2))
    gx, gw = lbp.lbp_backward_act(x, g, None, w, 8, bases, p=2.0 ** -18, g_bias=gb)
    n = lbp.lbp_launch_count()
    rx, rw = lbp.lbp_backward_ex(x, g, w, 8, bases, g_bias=gb2)
    plain = lbp.lbp_launch_count() - n
    n = lbp.lbp_launch_count()
    lbp.lbp_backward_act(x, g, None, w, 8, bases, p=0.0, g_bias=gb)
    assert lbp.lbp_launch_count() - n == plain
    assert torch.equal(gx, rx) and torch.equal(gw, rw) and torch.equal(gb, gb2)
    for cls in (0, 1, 2):
        layer = lbp.LbpLinear(192, 256, 8, bases, bias=True, device=dev, dtype=dtype, grid=(16, 16))
        s = _normal((4, cls + 256, 192), 1.0, dtype, 3).requires_grad_()
        r = _normal((4, cls + 256, 256), 1.0, dtype, 4).requires_grad_()
        gy = _normal((4, cls + 256, 256), 0.1, dtype, 5)
        got = torch.autograd.grad(layer(s, residual=r), (s, r, layer.weight, layer.bias), gy)
        want = torch.autograd.grad(layer(s), (s, layer.weight, layer.bias), gy)
        assert torch.equal(got[1], gy)
        assert all(torch.equal(a, b) for a, b in zip((got[0],) + got[2:], want))


def test_expanded_operands_of_the_backward_pass_are_refused(dev):
    """Their strides of zero would read as those of a dense tensor."""
    w, bases = _normal((64, 64), 0.1, torch.bfloat16, 0), O.select_bases(8, O.RULE_PREFIX, 8)
    one, full = _normal((1, 1, 1, 64), 1.0, torch.bfloat16, 1), _normal((2, 8, 8, 64), 1.0, torch.bfloat16, 2)
    for x, g in ((one.expand(2, 8, 8, 64), full), (full, one.expand(2, 8, 8, 64))):
        with pytest.raises(ValueError):
            lbp.lbp_backward_ex(x, g, w, 8, bases)
        with pytest.raises(ValueError):
            lbp.lbp_backward_act(x, g, full, w, 8, bases, activation="gelu")
    with pytest.raises(ValueError):
        lbp.lbp_project_grad(one.expand(2, 8, 8, 64), full, 8, bases, activation="gelu")


@pytest.mark.parametrize("rows,Cin,Cout", [
    (620000, 8, 8),      # more tiles than the SMs take in 32 turns each, a block of K to a tile
    (20000, 4, 4),       # few terms
    (40000, 200, 72), (3300, 448, 1792), (9000, 64, 260),
])
def test_linear_fp32_of_many_tiles(dev, rows, Cin, Cout):
    """A CTA has several tiles; y is the residual itself, and what is not finite stays in its rows."""
    x, W, b = _inputs(rows, Cin, Cout, torch.float32, 4)
    res = _normal((rows, Cout), 1.0, torch.float32, 6)
    y, z = res.clone(), torch.empty_like(res)
    lbp.lbp_linear(x, W, b, activation="gelu", residual=y, out=y, z=z, p=0.25, seed=5, offset=12)
    bad = torch.tensor([0, rows // 3, rows // 3 + 1, rows // 2, rows - 1])
    pick = torch.unique(torch.cat([bad + 2, torch.arange(130), torch.randint(0, rows, (300,), generator=torch.Generator().manual_seed(2)),
                                   torch.arange(rows - 130, rows)]).clamp(max=rows - 1)).cuda()
    zw = x[pick].double() @ W.double().t() + b.double()
    dz = Cin * 2.0 ** -23 * f64(x[pick].double().abs() @ W.double().abs().t() + b.double().abs())
    v = Y.act(f64(zw), "gelu")
    d = Y.drop(v, f64(pick)[:, None].astype(np.int64) * Cout + np.arange(Cout)[None, :], 0.25, 5, 12)
    r = f64(res[pick])
    _check_linear(torch.float32, y[pick], z[pick], (f64(zw), d + r, dz, v, np.abs(r) + np.abs(d)), 0.25)
    ref = x.double() @ W.double().t() + b.double()
    S = x.double().abs() @ W.double().abs().t() + b.double().abs()
    assert bool(((z.double() - ref).abs() <= 2.0 ** -24 * ref.abs() + Cin * 2.0 ** -23 * S).all())
    # rows that are not finite, in several tiles
    xb = x.clone()
    xb[bad, 1] = float("nan")
    xb[rows // 2, 1] = float("inf")
    yb, zb = res.clone(), torch.empty_like(res)
    lbp.lbp_linear(xb, W, b, activation="gelu", residual=yb, out=yb, z=zb, p=0.25, seed=5, offset=12)
    others = torch.ones(rows, dtype=torch.bool, device=dev)
    others[bad] = False
    assert torch.equal(yb[others], y[others]) and torch.equal(zb[others], z[others])
    assert not bool(torch.isfinite(zb[bad]).any())
    numbers = np.asarray(bad, dtype=np.int64)[:, None] * Cout + np.arange(Cout)[None, :]
    kept = torch.from_numpy(Y.keep(numbers, 0.25, 5, 12)).to(dev)
    assert torch.equal(yb[bad][~kept], res[bad][~kept])
    # a column of W that is not finite: its channel alone
    Wb = W.clone()
    Wb[3, 0] = float("nan")
    zc = torch.empty_like(res)
    lbp.lbp_linear(x, Wb, b, z=zc, save_z=True)
    assert bool(torch.isnan(zc[:, 3]).all())
    keep = [c for c in range(Cout) if c != 3]
    assert bool(((zc.double() - ref).abs() <= 2.0 ** -24 * ref.abs() + Cin * 2.0 ** -23 * S)[:, keep].all())


@pytest.mark.parametrize("dtype", DTYPES)
def test_backward_act_of_a_sequence_by_either_way_into_the_library(dev, dtype, monkeypatch):
    """The native binding and the one by ctypes: the same bits, and the same refusals."""
    from paper_2309_15275_b200 import binding
    B, H, Cin, Cout = 3, 8, 64, 96
    bases = O.select_bases(8, O.RULE_PREFIX, 8)
    seq = [_normal((B, 1 + H * H, c), 1.0, dtype, i) for i, c in enumerate((Cin, Cout, Cout))]
    x, g, z = (t[:, 1:].unflatten(1, (H, H)) for t in seq)
    w = _normal((Cout, Cin), 0.1, dtype, 5)

    def call(**more):
        gxe, gb = torch.empty(B, Cin, dtype=dtype, device=dev), torch.empty(Cout, device=dev)
        kw = dict(activation="silu", p=0.3, seed=7, offset=4, g_bias=gb, x_extra=seq[0][:, 0], gy_extra=seq[1][:, 0],
                  z_extra=seq[2][:, 0], gx_extra=gxe, first=Cout, number=((1 + H * H) * Cout, H * Cout, Cout),
                  number_extra=(1 + H * H) * Cout)
        gx, gw = lbp.lbp_backward_act(x, g, more.pop("z", z), w, 8, bases, **{**kw, **more})
        return gx, gw, gb, gxe

    bad = [dict(z=None), dict(z=z.contiguous()), dict(z_extra=seq[2][:, 0].contiguous()), dict(activation="tanh"), dict(p=1.5),
           dict(seed=-1), dict(rng=torch.zeros(2, device=dev)), dict(first=-8), dict(number=(0, 0, -8))]
    native = call()
    gz = lbp.lbp_linear_grad(seq[1], seq[2], activation="silu", p=0.3, seed=7, offset=4)
    gxe, gb = torch.empty(B, Cin, dtype=dtype, device=dev), torch.empty(Cout, device=dev)
    gx, gw = lbp.lbp_backward_ex(x, gz[:, 1:].unflatten(1, (H, H)), w, 8, bases, g_bias=gb, x_extra=seq[0][:, 0], gy_extra=gz[:, 0],
                                 gx_extra=gxe)
    tol = 3 * 2.0 ** -9 if dtype == torch.bfloat16 else 1e-5
    assert max(_rel(a, b) for a, b in zip(native, (gx, gw, gb, gxe))) <= tol
    for kw in bad:
        with pytest.raises((ValueError, RuntimeError)):
            call(**kw)
    module = binding._native()

    class Without:
        def __getattr__(self, name):
            return (lambda *a: None) if name == "backward_act" else getattr(module, name)

    monkeypatch.setattr(binding, "_native", lambda: Without())
    assert all(torch.equal(a, b) for a, b in zip(native, call()))
    for kw in bad:
        with pytest.raises((ValueError, RuntimeError)):
            call(**kw)
