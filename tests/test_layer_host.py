"""A layer's epilogue without a device: the oracle against known answers, and every refusal of the
C entry points and of the binding."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2309_15275_b200 as lbp
from oracle import layer_oracle as Y
from paper_2309_15275_b200 import binding as B


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2309_15275_b200.build import build_library
    build_library()


# ------------------------------------------------------------------------- oracle ----
@pytest.mark.parametrize("counter,key,want", [
    ((0, 0, 0, 0), (0, 0), (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
    ((0xffffffff,) * 4, (0xffffffff,) * 2, (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
    ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0),
     (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1)),
])
def test_philox_known_answers(counter, key, want):
    assert tuple(int(v) for v in Y.philox4x32(counter, key)) == want


def test_dropped_share_and_mean():
    n = np.arange(1 << 18)
    for p in (0.1, 0.5, 0.9):
        t = Y.threshold(p) / 65536
        # the share of 2^18 draws is within five standard deviations of t
        share = 1 - Y.keep(n, p, 7, 12).mean()
        assert abs(share - t) < 5 * np.sqrt(t * (1 - t) / n.size)
        mean = Y.drop(np.ones(n.size), n, p, 7, 12).mean()
        assert abs(mean - 1) < 5 * np.sqrt(t / (1 - t) / n.size)
    assert Y.threshold(0.0) == 0 and Y.threshold(1.0) == 65536 and Y.threshold(2 ** -18) == 0
    # other offsets, other choices: agreement as of independent draws
    a, b = Y.keep(n, 0.5, 7, 12), Y.keep(n, 0.5, 7, 16)
    assert abs((a == b).mean() - 0.5) < 5 * 0.5 / np.sqrt(n.size)


@pytest.mark.parametrize("a", ["relu", "gelu", "gelu_tanh", "silu"])
def test_slopes_are_the_differences_of_the_activations(a):
    z = np.linspace(-9, 9, 2001) + 1e-3
    h = 1e-5
    # central difference: h^2 / 6 |f'''| (|f'''| < 3) and rounding 2^-52 |f| / h
    assert np.max(np.abs((Y.act(z + h, a) - Y.act(z - h, a)) / (2 * h) - Y.act_slope(z, a))) < 3 * h * h + 9 * 2 ** -51 / h


# ----------------------------------------------------------------------- refusals ----
P = 1 << 20   # never dereferenced: every check is made on the host, before the CUDA runtime is touched


def _ep(**more):
    e = B.Epilogue()
    for k, v in more.items():
        setattr(e, k, v)
    return e


def _linear(rows=4, Cin=64, Cout=32, dtype=lbp.LBP_BF16, x=P, W=2 * P, bias=None, residual=None, y=3 * P, z=None,
            pitch=None, ep=None, ws=5 * P, n=None):
    lib = B._lib()
    if n is None:
        n = max(lib.lbp_linear_workspace_bytes(rows, Cin, Cout, dtype), 1024)
    return lib.lbp_linear(x, W, bias, residual, y, z, rows, Cin, Cout, dtype, pitch, ep, ws, n, None)


NULL, SHAPE, BASIS, DTYPE, ALIGN, WORKSPACE, OVERLAP = 1, 2, 4, 5, 6, 7, 12


@pytest.mark.parametrize("want,more", [
    (NULL, dict(x=None)), (NULL, dict(W=None)), (NULL, dict(y=None)),
    (SHAPE, dict(rows=-1)), (SHAPE, dict(Cin=0)), (SHAPE, dict(Cout=-8)),
    (DTYPE, dict(dtype=2)),
    (ALIGN, dict(Cin=60)), (ALIGN, dict(Cout=36)), (ALIGN, dict(dtype=lbp.LBP_F32, Cin=62)),
    (ALIGN, dict(x=P + 8)), (ALIGN, dict(bias=P + 2)), (ALIGN, dict(residual=4 * P + 4)), (ALIGN, dict(z=4 * P + 8)),
    (WORKSPACE, dict(ws=None)), (WORKSPACE, dict(n=16)),
    (SHAPE, dict(pitch=B.Pitches(x=56))), (ALIGN, dict(pitch=B.Pitches(y=36))), (SHAPE, dict(pitch=B.Pitches(z=-8))),
    (SHAPE, dict(ep=_ep(act=5))), (SHAPE, dict(ep=_ep(act=-1))), (SHAPE, dict(ep=_ep(p=-0.1))),
    (SHAPE, dict(ep=_ep(p=1.5))), (SHAPE, dict(ep=_ep(p=float("nan")))), (SHAPE, dict(ep=_ep(first=-8))),
    (ALIGN, dict(ep=_ep(first=4))), (ALIGN, dict(ep=_ep(number=B.View(0, 0, 12)))), (ALIGN, dict(ep=_ep(seed_dev=P + 4))),
    (OVERLAP, dict(y=P)), (OVERLAP, dict(y=2 * P + 64)), (OVERLAP, dict(z=3 * P)), (OVERLAP, dict(z=P + 128)),
    (OVERLAP, dict(residual=3 * P + 16)), (OVERLAP, dict(residual=3 * P, pitch=B.Pitches(y=64))),
    (OVERLAP, dict(residual=4 * P, z=4 * P)), (OVERLAP, dict(y=5 * P + 16)),
])
def test_linear_refusals(want, more):
    assert _linear(**more) == want


def _pointwise(name, a=P, b=2 * P, out=3 * P, rows=4, Cc=64, dtype=lbp.LBP_BF16, pitch=None, ep=None):
    return getattr(B._lib(), name)(a, b, out, rows, Cc, dtype, pitch, ep, None)


@pytest.mark.parametrize("name", ["lbp_linear_grad", "lbp_dropout"])
@pytest.mark.parametrize("want,more", [
    (NULL, dict(a=None)), (NULL, dict(out=None)), (SHAPE, dict(rows=-2)), (SHAPE, dict(Cc=0)), (DTYPE, dict(dtype=-1)),
    (ALIGN, dict(Cc=4)), (ALIGN, dict(a=P + 2)), (ALIGN, dict(b=2 * P + 8)), (ALIGN, dict(out=3 * P + 8)),
    (SHAPE, dict(ep=_ep(p=2.0))), (SHAPE, dict(ep=_ep(act=9))), (OVERLAP, dict(out=P + 16)), (OVERLAP, dict(out=2 * P + 256)),
    (SHAPE, dict(pitch=B.Pitches(x=32))), (SHAPE, dict(pitch=B.Pitches(y=32))),
])
def test_pointwise_refusals(name, want, more):
    assert _pointwise(name, **more) == want


def test_pointwise_refusals_of_one():
    assert _pointwise("lbp_linear_grad", b=None, ep=_ep(act=2)) == NULL
    assert _pointwise("lbp_dropout", ep=_ep(act=2)) == SHAPE
    # in place with another pitch
    assert _pointwise("lbp_dropout", out=P, pitch=B.Pitches(x=64, y=128)) == OVERLAP
    assert _pointwise("lbp_linear_grad", out=P, pitch=B.Pitches(y=128, x=64)) == OVERLAP


def test_no_rows_is_no_call():
    assert _linear(rows=0) == 0
    assert _pointwise("lbp_dropout", rows=0) == 0
    assert _pointwise("lbp_linear_grad", rows=0, a=None, b=None, out=None) == 0


def _project(gy=P, z=2 * P, out=3 * P, B_=2, H=16, W=16, Cc=64, k=8, r=4, dtype=lbp.LBP_BF16, view=None, ep=None, ws=5 * P,
             n=None, bases=None):
    lib = B._lib()
    if n is None:
        n = max(lib.lbp_project_grad_workspace_bytes(B_, H, W, Cc, k, r, dtype), 1024)
    bases = lbp.lbp_select_bases(8, lbp.SEL_PREFIX, r) if bases is None else bases
    return lib.lbp_project_grad(gy, z, out, B_, H, W, Cc, k, B._bases(bases), len(bases), dtype, view, ep, ws, n, None)


@pytest.mark.parametrize("want,more", [
    (NULL, dict(gy=None)), (NULL, dict(out=None)), (NULL, dict(z=None, ep=_ep(act=1))), (SHAPE, dict(B_=0)),
    (3, dict(k=5)), (BASIS, dict(bases=[(0, 0), (0, 0)])), (BASIS, dict(bases=[(0, 8)])), (ALIGN, dict(Cc=4)),
    (ALIGN, dict(z=2 * P + 8)), (WORKSPACE, dict(ws=None)), (WORKSPACE, dict(n=100)), (SHAPE, dict(ep=_ep(p=7.0))),
    (SHAPE, dict(view=B.View(0, 0, 64))), (SHAPE, dict(view=B.View(4096, 1024, 32))), (ALIGN, dict(view=B.View(16396, 1024, 64))),
    (ALIGN, dict(ep=_ep(first=12))),
])
def test_project_grad_refusals(want, more):
    assert _project(**more) == want


def _backward(ep=None, z=7 * P, n=None, gy=2 * P, ex=None, x=P, x_hat=None, z_extra=None, first_extra=0, number_extra=0,
              lay=None, null_grad=False):
    lib = B._lib()
    lay = lay or B._layer(2, 16, 16, 64, 128, 8, lbp.LBP_BF16, lbp.LBP_F32)
    bases = lbp.lbp_select_bases(8, lbp.SEL_PREFIX, 4)
    g = B.LayerGrad()
    g.epilogue, g.z, g.z_extra, g.first_extra, g.number_extra = ep or B.Epilogue(), z, z_extra, first_extra, number_extra
    if n is None:
        n = max(lib.lbp_workspace_bytes_act(C.byref(lay), 4, ex, 0), 1024)
    return lib.lbp_backward_act(x, x_hat, gy, 3 * P, 4 * P, 5 * P, C.byref(lay), B._bases(bases), 4, ex,
                                None if null_grad else C.byref(g), 16 * P, n, None)


def _extra(n=3, pitch=0):
    ex = B.Extras()
    ex.n_extra, ex.x_extra, ex.gy_extra, ex.gx_extra, ex.gy_extra_pitch = n, 8 * P, 9 * P, 10 * P, pitch
    return C.pointer(ex)


@pytest.mark.parametrize("want,more", [
    (NULL, dict(null_grad=True)), (NULL, dict(gy=None)), (NULL, dict(x=None)), (NULL, dict(x_hat=11 * P)),
    (NULL, dict(ep=_ep(act=2), z=None)), (NULL, dict(ep=_ep(act=2), ex=_extra())), (ALIGN, dict(z=7 * P + 8)),
    (SHAPE, dict(ep=_ep(act=7))), (SHAPE, dict(ep=_ep(p=-1.0))), (SHAPE, dict(first_extra=-8)), (ALIGN, dict(number_extra=12)),
    (WORKSPACE, dict(n=4096)), (ALIGN, dict(ex=_extra(pitch=132), ep=_ep(act=0))),
    (SHAPE, dict(lay=B._layer(2, 0, 16, 64, 128, 8, lbp.LBP_BF16, lbp.LBP_F32))),
])
def test_backward_act_refusals(want, more):
    assert _backward(**more) == want


def test_backward_act_asks_for_the_gradient_it_forms():
    lib = B._lib()
    lay = B._layer(2, 16, 16, 64, 128, 8, lbp.LBP_BF16, lbp.LBP_F32)
    plain = lib.lbp_workspace_bytes_ex(C.byref(lay), 4, None)
    n = lib.lbp_workspace_bytes_act(C.byref(lay), 4, None, 0)
    assert n >= plain
    # one byte less than it asks for is refused
    assert _backward(n=n - 1) == WORKSPACE
    assert lib.lbp_workspace_bytes_act(C.byref(B._layer(2, 16, 16, 60, 128, 8, lbp.LBP_BF16, lbp.LBP_F32)), 4, None, 0) == 0


def test_structs_of_the_epilogue_have_the_librarys_layout():
    lib = B._lib()
    for which, cls in ((4, B.Epilogue), (5, B.Pitches), (6, B.LayerGrad)):
        assert lib.lbp_test_struct_size(which) == C.sizeof(cls), cls.__name__


@pytest.mark.parametrize("want,more", [
    # columns of one wide matrix (pitch 160 elements of 2 bytes): x 0..63, y 64..95, z 96..127
    (None, dict(y=P + 128, z=P + 192, pitch=B.Pitches(x=160, y=160, z=160))),
    # the residual ahead of y in the rows, one row further on
    (None, dict(y=P + 128 + 320, residual=P + 256, pitch=B.Pitches(x=160, y=160, residual=160))),
    (OVERLAP, dict(y=P + 112, pitch=B.Pitches(x=160, y=160))),                      # into x's columns
    (OVERLAP, dict(y=P + 288, pitch=B.Pitches(x=160, y=160))),                      # into the next row's
    (OVERLAP, dict(y=P + 128, z=P + 176, pitch=B.Pitches(x=160, y=160, z=160))),    # into y's
    (OVERLAP, dict(y=P + 128, pitch=B.Pitches(x=160, y=320))),                      # another distance: not looked into
])
def test_columns_of_one_matrix_are_apart(want, more):
    # (accepted: what is left to fail is the machine without a device)
    assert _linear(**more) in ((8, 9) if want is None else (want,))


def test_binding_refuses_on_the_cpu_and_names_the_error():
    x, W = torch.zeros(3, 64), torch.zeros(32, 64)
    with pytest.raises(ValueError, match="CUDA"):
        lbp.lbp_linear(x, W)
    with pytest.raises(ValueError, match="does not match"):
        lbp.lbp_linear(x, W[:, :32])
    with pytest.raises(ValueError, match="activation"):
        lbp.lbp_linear(x, W, activation="tanh")
    with pytest.raises(TypeError):
        lbp.lbp_linear(x.half(), W.half())
    for p in (-0.5, 1.5, float("nan")):
        with pytest.raises(ValueError, match="probability"):
            lbp.lbp_dropout(x, p)
    for seed in (-1, 2 ** 64, 0.5):
        with pytest.raises(ValueError, match="seed"):
            lbp.lbp_dropout(x, 0.5, seed=seed)
    with pytest.raises(ValueError, match="rng"):
        lbp.lbp_dropout(x, 0.5, rng=torch.zeros(3, dtype=torch.int64))
    with pytest.raises(ValueError, match="CUDA"):
        lbp.lbp_linear_grad(x, x, activation="gelu")
    with pytest.raises(ValueError, match="B, H, W, C"):
        lbp.lbp_project_grad(x, None, 8, [(0, 0)])
    for bad in (dict(activation="swish"), dict(dropout=-0.1), dict(dropout=2.0)):
        with pytest.raises(ValueError):
            lbp.LbpLinear(64, 32, 8, [(0, 0)], **bad)
    layer = lbp.LbpLinear(64, 32, 8, [(0, 0)], activation="gelu")
    with pytest.raises(ValueError, match="CUDA"):
        layer(torch.zeros(1, 8, 8, 64))


@pytest.mark.parametrize("more", [dict(seed_dev=8 * P, offset_dev=8 * P + 8, used=8 * P), dict(seed_dev=8 * P + 8, used=8 * P),
                                  dict(offset_dev=8 * P, used=8 * P)])
def test_used_may_not_be_what_is_read(more):
    ep = _ep(p=0.5, **more)
    assert _linear(ep=ep) == _pointwise("lbp_dropout", ep=ep) == _project(ep=ep) == _backward(ep=ep) == OVERLAP


def test_sizes_past_the_kernels_integers_are_refused():
    wide = (1 << 30) + 8
    assert _linear(Cin=wide) == _linear(Cout=wide) == _pointwise("lbp_dropout", Cc=wide) == SHAPE
    assert B._lib().lbp_linear_workspace_bytes(4, wide, 8, lbp.LBP_BF16) == 0
    assert _project(B_=1, H=1 << 16, W=1 << 15, Cc=8) == SHAPE
    lay = B._layer(1, 1 << 16, 1 << 15, 8, 8, 8, lbp.LBP_BF16, lbp.LBP_F32)
    assert B._lib().lbp_workspace_bytes_act(C.byref(lay), 4, None, 0) == 0
    assert _backward(lay=lay, n=1 << 50) == SHAPE


FAR = 1 << 62


@pytest.mark.parametrize("rows,first,step", [
    ((1 << 18) + 1, 0, 1 << 45),                    # 2^63: past the kernels' signed sums
    ((1 << 12) + 2, 0, (1 << 50) - 8), (2, FAR - 64 - 8, 64), (1, FAR - 56, 0), (1 << 40, 0, (1 << 50) - 8),
])
def test_numbers_past_2_62_are_refused(rows, first, step):
    ep = _ep(first=first, number=B.View(0, 0, step))
    assert _linear(rows=rows, Cout=64, ep=ep, n=1 << 60) == SHAPE
    assert _pointwise("lbp_dropout", rows=rows, ep=ep) == _pointwise("lbp_linear_grad", rows=rows, ep=ep) == SHAPE


@pytest.mark.parametrize("which", range(4))
def test_numbers_of_a_grid_past_2_62_are_refused(which):
    # along each of the strides, and of the first number alone
    big = (1 << 50) - 8
    view = [B.View(big, 64, 64), B.View(64, big, 64), B.View(64, 64, big), B.View(64, 64, 64)][which]
    shape = [dict(B_=4100, H=1, W=1), dict(B_=1, H=4100, W=1), dict(B_=1, H=1, W=4100), dict(B_=1, H=1, W=1)][which]
    ep = _ep(first=FAR - 56 if which == 3 else 0, number=view)
    assert _project(ep=ep, **shape) == SHAPE
    lay = B._layer(shape["B_"], shape["H"], shape["W"], 64, 64, 8, lbp.LBP_BF16, lbp.LBP_F32)
    assert _backward(ep=ep, lay=lay) == SHAPE


def test_the_last_number_below_2_62_is_accepted():
    accepted = (8, 9)   # (what is left to fail is the machine without a device)
    ep = _ep(first=FAR - 128, number=B.View(0, 0, 64))
    assert _linear(rows=2, Cout=64, ep=ep) in accepted and _pointwise("lbp_dropout", rows=2, ep=ep) in accepted
    # of extra tokens
    big = (1 << 50) - 8
    assert _backward(ex=_extra(n=4100), number_extra=big) == SHAPE
    assert _backward(ex=_extra(n=3), number_extra=big) in accepted
    assert _backward(ex=_extra(n=1), first_extra=FAR - 120) == SHAPE


@pytest.mark.parametrize("dtype,es", [(lbp.LBP_BF16, 2), (lbp.LBP_F32, 4)])
def test_pitches_past_a_tensor_maps_stride_are_refused(dtype, es):
    """A stride of 2^40 bytes and more is the caller's mistake, not a failed CUDA call."""
    accepted = (8, 9)   # (what is left to fail is the machine without a device)
    for pitch, want in (((1 << 40) // es, (SHAPE,)), ((1 << 40) // es - 16, accepted)):
        for name in ("x", "residual", "y", "z"):
            p = B.Pitches(**{name: pitch})
            assert _linear(rows=1, dtype=dtype, pitch=p) in want
            assert _pointwise("lbp_dropout", rows=1, dtype=dtype, pitch=p) in want
            assert _pointwise("lbp_linear_grad", rows=1, dtype=dtype, pitch=p) in want


def test_tensors_past_2_58_elements_are_refused():
    """Nothing that large exists; rows times channels or a pitch would run over the sums of sizes and places."""
    assert _linear(rows=1 << 40, Cout=1 << 20, n=1 << 60) == _linear(rows=1 << 40, Cin=1 << 20, n=1 << 60) == SHAPE
    assert B._lib().lbp_linear_workspace_bytes(1 << 40, 1 << 20, 64, lbp.LBP_BF16) == 0
    for name in ("lbp_dropout", "lbp_linear_grad"):
        assert _pointwise(name, rows=1 << 40, Cc=1 << 27) == SHAPE
        assert _pointwise(name, rows=1 << 40, Cc=64, pitch=B.Pitches(x=1 << 30)) == SHAPE
    assert _linear(rows=1 << 40, pitch=B.Pitches(x=1 << 30), n=1 << 60) == SHAPE
    assert _project(B_=1 << 29, H=1, W=1, view=B.View(1 << 38, 64, 64), n=1 << 60) == SHAPE


@pytest.mark.parametrize("number", [B.View(4096, 0, 0), B.View(0, 64, 0), B.View(4096, 64, 0)])
def test_a_numbering_without_its_innermost_stride_is_refused(number):
    """All three zero is dense; a zero for the tokens alone read as dense too, whatever the others said."""
    ep = _ep(p=0.5, number=number)
    assert _linear(ep=ep) == _pointwise("lbp_dropout", ep=ep) == _pointwise("lbp_linear_grad", ep=ep) == SHAPE
    assert _project(ep=ep) == _backward(ep=ep) == SHAPE


def test_a_modules_dropout_may_be_set_to_a_whole_number():
    """layer.dropout = 0 switches it off, as it does for torch's own layer."""
    layer = lbp.LbpLinear(64, 32, 8, [(0, 0)], activation="gelu", dropout=0.1)
    for p in (0, 1, np.float32(0.5)):
        layer.dropout = p
        with pytest.raises(ValueError, match="CUDA"):     # (and nothing is said of the arguments' kinds)
            layer(torch.zeros(1, 8, 8, 64))
    layer.dropout = 2
    with pytest.raises(ValueError, match="CUDA|probability"):
        layer(torch.zeros(1, 8, 8, 64))
