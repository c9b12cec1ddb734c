"""LbpLinear with an epilogue among torch's own mechanisms: autocast and forward-mode derivatives."""
import pytest
import torch

import paper_2309_15275_b200 as lbp
from oracle import lbp_oracle as O

pytestmark = pytest.mark.gpu

K, BASES = 8, O.select_bases(8, O.RULE_PREFIX, 8)
EPILOGUES = [dict(activation="gelu", dropout=0.2), dict(dropout=0.3), dict(activation="silu"), dict()]


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    return torch.device("cuda:0")


def _normal(shape, std, dtype, seed):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * std).to(dtype).cuda()


@pytest.mark.parametrize("epilogue", EPILOGUES)
@pytest.mark.parametrize("cls", [None, 0, 1, 2])
def test_a_residual_stream_keeps_its_type_under_autocast(dev, epilogue, cls):
    """torch's rule for the sum: fp32 onto bf16 is fp32, with not a bit of the stream lost.  The terms are those of the call
    without a residual, so y, and every gradient, is what torch's own sum behind that call gives."""
    seq = () if cls is None else (cls + 64,)
    shape = (3, 8, 8) if cls is None else (3,) + seq
    layer = lbp.LbpLinear(64, 96, K, BASES, device=dev, dtype=torch.float32, bias=True, grid=None if cls is None else (8, 8), **epilogue)
    with torch.no_grad():
        layer.bias.normal_(0, 0.3)
    x = _normal(shape + (64,), 1.0, torch.float32, 1).requires_grad_()
    r = _normal(shape + (96,), 1.0, torch.float32, 2).requires_grad_()
    g = _normal(shape + (96,), 1.0, torch.float32, 3)
    leaves = (x, layer.weight, layer.bias, r)

    def run(step):
        torch.manual_seed(11)
        with torch.autocast("cuda", dtype=torch.bfloat16):
            y = step()
        return y, torch.autograd.grad(y, leaves, g)

    want, want_grads = run(lambda: r + layer(x))
    y, grads = run(lambda: layer(x, residual=r))
    assert want.dtype == y.dtype == torch.float32 and torch.equal(y, want)
    assert torch.equal(grads[3], g) and all(torch.equal(a, b) for a, b in zip(grads, want_grads))
    with torch.no_grad():     # and where nothing is to be differentiated
        torch.manual_seed(11)
        with torch.autocast("cuda", dtype=torch.bfloat16):
            assert torch.equal(layer(x, residual=r), want)
            # a residual of autocast's own type still rides in the epilogue
            low = layer(x, residual=r.bfloat16())
            assert low.dtype == torch.bfloat16 and low.shape == y.shape
            for bad in (r[..., :1], r[:1], r.long(), r.cpu()):
                with pytest.raises(ValueError):
                    layer(x, residual=bad)
    with pytest.raises(ValueError):   # without autocast one dtype, as before
        layer(x, residual=r.bfloat16())


@pytest.mark.parametrize("epilogue", EPILOGUES)
@pytest.mark.parametrize("frozen", [False, True])
@pytest.mark.parametrize("with_grad", [False, True])
def test_tangents_are_refused_and_not_lost(dev, epilogue, frozen, with_grad):
    """There is no forward-mode derivative; a call that went on without the tangent would answer zero for it."""
    from torch.autograd import forward_ad
    layer = lbp.LbpLinear(64, 64, K, BASES, device=dev, dtype=torch.float32, bias=True, **epilogue)
    layer.requires_grad_(not frozen)
    x, r = (_normal((1, 8, 8, 64), 1.0, torch.float32, s) for s in (1, 2))
    before = torch.cuda.default_generators[0].get_offset()
    with torch.set_grad_enabled(with_grad), forward_ad.dual_level():
        dual = forward_ad.make_dual(x, torch.ones_like(x))
        for call in (lambda: layer(dual), lambda: layer(dual, residual=r), lambda: layer(x, residual=dual)):
            with pytest.raises(RuntimeError, match="forward-mode|jvp"):
                call()
            with torch.autocast("cuda", dtype=torch.bfloat16), pytest.raises(RuntimeError, match="forward-mode|jvp"):
                call()
        assert layer(x, residual=r).shape == x.shape     # without one it goes on as ever
    assert torch.cuda.default_generators[0].get_offset() == before + (4 if epilogue.get("dropout") else 0)


def test_save_z_is_any_truth_value(dev):
    """A 1 or a numpy truth value asks for z as True does (and is not answered with y alone, which unpacks into rows)."""
    import numpy as np
    x, w = _normal((2, 64), 1.0, torch.float32, 1), _normal((32, 64), 1.0, torch.float32, 2)
    y, z = lbp.lbp_linear(x, w, activation="relu", save_z=True)
    for yes in (1, np.True_):
        got = lbp.lbp_linear(x, w, activation="relu", save_z=yes)
        assert isinstance(got, tuple) and torch.equal(got[0], y) and torch.equal(got[1], z)
    for no in (0, np.False_, None):
        assert torch.equal(lbp.lbp_linear(x, w, activation="relu", save_z=no), y)


AUTOCAST = [(b, i) for b in (None, torch.bfloat16, torch.float32) for i in (torch.bfloat16, torch.float32)]


@pytest.mark.parametrize("bias,dtype", AUTOCAST)
@pytest.mark.parametrize("epilogue", EPILOGUES)
@pytest.mark.parametrize("cls", [None, 1, 2])
def test_a_residual_stream_under_autocast_with_any_bias_and_input(dev, epilogue, cls, bias, dtype):
    """An fp32 stream onto a layer of fp32 weights: whatever the layer's input and bias are, it is torch's sum of the two."""
    shape = (3, 8, 8) if cls is None else (3, cls + 64)
    layer = lbp.LbpLinear(64, 96, K, BASES, device=dev, dtype=torch.float32, bias=bias is not None,
                          grid=None if cls is None else (8, 8), **epilogue)
    if bias is not None:
        layer.bias = torch.nn.Parameter(_normal((96,), 0.3, bias, 9))
    x = _normal(shape + (64,), 1.0, dtype, 1).requires_grad_()
    r = _normal(shape + (96,), 1.0, torch.float32, 2).requires_grad_()
    g = _normal(shape + (96,), 1.0, torch.float32, 3)
    leaves = (x, r) + tuple(layer.parameters())

    def run(step):
        torch.manual_seed(11)
        with torch.autocast("cuda", dtype=torch.bfloat16):
            y = step()
        return y, torch.autograd.grad(y, leaves, g)

    want, want_grads = run(lambda: r + layer(x))
    y, grads = run(lambda: layer(x, residual=r))
    assert y.dtype == torch.float32 and torch.equal(y, want)
    assert torch.equal(grads[1], g) and all(torch.equal(a, b) and a.dtype == v.dtype for a, b, v in zip(grads, want_grads, leaves))


@pytest.mark.parametrize("bias,dtype", AUTOCAST)
@pytest.mark.parametrize("cls,projected", [(None, False), (None, True), (1, False), (2, False)])
def test_the_plain_layer_trains_under_autocast_with_any_bias_and_input(dev, cls, projected, bias, dtype):
    """y is torch's: the product in bf16, the bias added by torch's rules.  The backward pass is the library's on operands of
    y's type."""
    shape = (3, 8, 8) if cls is None else (3, cls + 64)
    layer = lbp.LbpLinear(64, 96, K, BASES, device=dev, dtype=torch.float32, bias=bias is not None, save_projected=projected,
                          grid=None if cls is None else (8, 8))
    if bias is not None:
        layer.bias = torch.nn.Parameter(_normal((96,), 0.3, bias, 9))
    x = _normal(shape + (64,), 1.0, dtype, 1).requires_grad_()
    with torch.autocast("cuda", dtype=torch.bfloat16):
        y = layer(x)
        want = torch.matmul(x, layer.weight.t())
        want = want if bias is None else want + layer.bias
    assert y.dtype == want.dtype and torch.equal(y, want)
    g = _normal(y.shape, 1.0, y.dtype, 3)
    grads = torch.autograd.grad(y, (x,) + tuple(layer.parameters()), g)
    same = lbp.LbpLinear(64, 96, K, BASES, device=dev, dtype=y.dtype, bias=bias is not None, save_projected=projected, grid=layer.grid)
    same.load_state_dict({n: v.to(y.dtype) for n, v in layer.state_dict().items()})
    xs = x.detach().to(y.dtype).requires_grad_()
    ref = torch.autograd.grad(same(xs), (xs,) + tuple(same.parameters()), g)
    for a, b, v in zip(grads, ref, (x,) + tuple(layer.parameters())):
        assert a.dtype == v.dtype and torch.equal(a, b.to(v.dtype))


@pytest.mark.parametrize("epilogue", EPILOGUES)
@pytest.mark.parametrize("bias", [False, True])
def test_a_look_without_gradients_first_loses_none_under_autocast(dev, epilogue, bias):
    """In one autocast context: evaluation under no_grad, then a training step of the same layer."""
    layer = lbp.LbpLinear(64, 96, K, BASES, device=dev, dtype=torch.float32, bias=bias, **epilogue)
    x = _normal((2, 8, 8, 64), 1.0, torch.float32, 1).requires_grad_()
    leaves = (x,) + tuple(layer.parameters())
    grads = []
    for look in (False, True):
        with torch.autocast("cuda", dtype=torch.bfloat16):
            if look:
                with torch.no_grad():
                    layer(x)
            torch.manual_seed(5)
            y = layer(x)
        grads.append(torch.autograd.grad(y, leaves, torch.ones_like(y)))
    assert all(torch.equal(a, b) for a, b in zip(*grads))
