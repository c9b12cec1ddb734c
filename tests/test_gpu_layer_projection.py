"""The projection that forms its gradient, on strided tokens with strided numbers, in every order: bit for bit the
projection of the gradient written out, row of tokens by row of tokens, under the same numbers."""
import pytest
import torch

import paper_2309_15275_b200 as lbp
from oracle import lbp_oracle as O
from paper_2309_15275_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    return torch.device("cuda:0")


def _normal(shape, std, dtype, seed):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * std).to(dtype).cuda()


def _written_out(g, z, a, p, first, number):
    """lbp_linear_grad of each row of tokens, whose numbers are an arithmetic series."""
    Bn, H, W, Cc = g.shape
    g, z = g.contiguous(), z.contiguous()
    out = torch.empty_like(g)
    for b in range(Bn):
        for h in range(H):
            e = B._epilogue(a, p, 4, 8, None, g.device)
            e.first, e.number = first + b * number[0] + h * number[1], B.View(0, 0, number[2])
            zz = None if a == "none" else z[b, h].data_ptr()
            assert B._lib().lbp_linear_grad(g[b, h].data_ptr(), zz, out[b, h].data_ptr(), W, Cc, lbp.LBP_BF16, None, e, B._stream()) == 0
    return out


@pytest.mark.parametrize("k,r,H,W", [(4, 3, 9, 22), (4, 13, 14, 14), (8, 8, 14, 14), (8, 40, 9, 17), (16, 6, 14, 14), (16, 40, 20, 33)])
@pytest.mark.parametrize("numbering", ["sequence", "spread", "far"])
@pytest.mark.parametrize("a,p", [("gelu", 0.3), ("none", 0.5), ("silu", 0.7)])
def test_strided_tokens_with_strided_numbers(dev, k, r, H, W, numbering, a, p):
    Bn, Cc, n = 3, 136, 1
    bases = O.select_bases(k, O.RULE_PREFIX, r)
    seq_g, seq_z = (_normal((Bn, n + H * W, Cc), 1.0, torch.bfloat16, s) for s in (1, 2))
    strides = ((n + H * W) * Cc, W * Cc, Cc)
    g, z = (t.as_strided((Bn, H, W, Cc), strides + (1,), n * Cc) for t in (seq_g, seq_z))
    first, number = {"sequence": (n * Cc, strides), "spread": (24, (8 * (H * (W * Cc + 40) + 7), W * Cc + 40, Cc + 8)),
                     "far": (2 ** 36 + 16, (2 ** 37, 2 ** 33 + 64, 2 ** 20 + 8))}[numbering]
    e = B._epilogue(a, p, 4, 8, None, g.device)
    e.first, e.number = first, B.View(*number)
    out = torch.empty((Bn, -(-H // k), -(-W // k), r, Cc), dtype=torch.bfloat16, device=dev)
    ws = torch.zeros(lbp.lbp_project_grad_workspace_bytes(Bn, H, W, Cc, k, r, lbp.LBP_BF16), dtype=torch.uint8, device=dev)
    assert B._lib().lbp_project_grad(g.data_ptr(), None if a == "none" else z.data_ptr(), out.data_ptr(), Bn, H, W, Cc, k,
                                     B._bases(bases), r, lbp.LBP_BF16, B.View(*strides), e, ws.data_ptr(), ws.numel(),
                                     B._stream()) == 0
    assert lbp.lbp_poll_status(ws) == 0
    gz = _written_out(g, z, a, p, first, number)
    assert torch.equal(out, lbp.lbp_project(gz, k, bases))
    assert bool((gz == 0).float().mean() > 0.8 * p)
