"""GPU: the token operators give no gradients, and say so where one would be lost."""
import pytest
import torch

import paper_2604_12841_amd as pdx

pytestmark = pytest.mark.gpu


def zeros(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype, device="cuda")


def calls():
    """(operator, arguments, the names of those that may ask for a gradient)."""
    b = torch.bfloat16
    sites = zeros(6, 4, dtype=torch.int32)
    return [
        (pdx.rms_norm, dict(x=zeros(6, 64), gain=zeros(64), residual=zeros(6, 64), sum_out=zeros(6, 64), out=zeros(6, 64)),
         ("x", "gain", "residual", "sum_out", "out")),
        (pdx.matmul8, dict(a=zeros(6, 64, dtype=torch.int8), a_scales=zeros(6), w=zeros(8, 64, dtype=torch.int8), w_scales=zeros(8), out=zeros(6, 8),
                           bias=zeros(8)), ("a_scales", "w_scales", "out", "bias")),
        (pdx.rope, dict(x=zeros(6, 2, 32), sites=sites, out=zeros(6, 2, 32), sections=(8, 4, 4)), ("x", "out")),
        (pdx.attention, dict(q=zeros(1, 6, 2, 64, dtype=b), k=zeros(1, 6, 2, 64, dtype=b), v=zeros(1, 6, 2, 64, dtype=b),
                             out=zeros(1, 6, 2, 64, dtype=b), q_sites=sites, k_sites=sites, slopes=zeros(2)), ("q", "k", "v", "out", "slopes")),
    ]


@pytest.mark.parametrize("n", range(4))
def test_a_gradient_that_would_be_lost_is_refused(n):
    op, args, names = calls()[n]
    op(**args)
    for name in names:
        asks = args | {name: args[name].clone().requires_grad_()}
        with pytest.raises(ValueError, match="gradient"):
            op(**asks)
        with torch.no_grad():
            op(**asks)
        with torch.inference_mode():
            op(**asks)
        op(**(args | {name: asks[name].detach()}))
    torch.cuda.synchronize()
