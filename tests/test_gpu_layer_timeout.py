"""The exit path of an expired wait with loads and products behind it: the first block of the operands is fetched and
multiplied, the next never comes (include/lbp_test_hooks.h).  Every wait is bounded, so each call ends by itself; it reports
the expiry, settles what it has begun, gives its tensor memory back, and the next call on the same workspace is right."""
import pytest
import torch

import paper_2309_15275_b200 as lbp
from oracle import lbp_oracle as O

pytestmark = pytest.mark.gpu

LBP_ERR_TIMEOUT = 10


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    return torch.device("cuda:0")


def _normal(shape, std, dtype, seed):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * std).to(dtype).cuda()


def _stalled(call, **where):
    lbp.lbp_test_stall_products(True, late=True, **where)
    try:
        call()
    finally:
        lbp.lbp_test_stall_products(False)


# K shared among four and two CTAs of a cluster (several blocks to each), a CTA a tile, CTA pairs
@pytest.mark.parametrize("rows,Cin,Cout", [(100, 1024, 192), (1000, 2304, 768), (100, 128, 192), (1000, 192, 512)])
def test_expired_wait_behind_a_first_block_of_the_layers_product(dev, rows, Cin, Cout):
    x, W = _normal((rows, Cin), 1.0, torch.bfloat16, 1), _normal((Cout, Cin), Cin ** -0.5, torch.bfloat16, 2)
    ws = torch.zeros(lbp.lbp_linear_workspace_bytes(rows, Cin, Cout, lbp.LBP_BF16), dtype=torch.uint8, device=dev)
    want = lbp.lbp_linear(x, W, activation="gelu", p=0.1, seed=1, save_z=True, ws=ws)
    assert lbp.lbp_poll_status(ws) == 0
    for _ in range(2):
        _stalled(lambda: lbp.lbp_linear(x, W, activation="gelu", p=0.1, seed=1, save_z=True, ws=ws), linear=True)
        assert lbp.lbp_poll_status(ws) == LBP_ERR_TIMEOUT
        assert lbp.lbp_poll_status(ws) == 0
        got = lbp.lbp_linear(x, W, activation="gelu", p=0.1, seed=1, save_z=True, ws=ws)
        assert lbp.lbp_poll_status(ws) == 0
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("grad", [False, True])
def test_expired_wait_behind_a_first_block_of_the_projection(dev, grad):
    """Order 16: a block of tokens comes in four parts, the first of which is fetched."""
    g, z = (_normal((2, 32, 32, 256), 1.0, torch.bfloat16, s) for s in (1, 2))
    bases = O.select_bases(16, O.RULE_PREFIX, 6)
    ws = torch.zeros(lbp.lbp_project_grad_workspace_bytes(2, 32, 32, 256, 16, 6, lbp.LBP_BF16), dtype=torch.uint8, device=dev)

    def call():
        if grad:
            return lbp.lbp_project_grad(g, z, 16, bases, activation="gelu", p=0.2, ws=ws)
        return lbp.lbp_project(g, 16, bases, ws=ws)

    want = call()
    assert lbp.lbp_poll_status(ws) == 0
    _stalled(call, projection=True)
    assert lbp.lbp_poll_status(ws) == LBP_ERR_TIMEOUT
    got = call()
    assert lbp.lbp_poll_status(ws) == 0 and torch.equal(got, want)
