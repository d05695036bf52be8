"""GPU: attention over as many keys as 32 bits count."""
import math

import pytest
import torch

import paper_2604_12841_amd as pdx

pytestmark = pytest.mark.gpu


def test_the_last_tile_of_2_to_the_31_keys():
    """n_k = 2^31 - 1: the last tile of 64 keys holds 63, and its end lies past the largest int32."""
    n, D, H = (1 << 31) - 1, 64, 1
    # a key's row is the eight values after the row before it, and 56 of its: 34 GB for all
    buf = torch.zeros(8 * (n - 1) + D, dtype=torch.bfloat16, device="cuda")
    buf[-8:] = 1.0  # seen by the last key alone
    kv = buf.as_strided((1, n, H, D), (0, 8, D, 1))
    q = torch.zeros(1, 1, H, D, dtype=torch.bfloat16, device="cuda")
    q[..., -8:] = 21.5
    out = torch.full_like(q, 9.0)
    pdx.attention(q, kv, kv, out, scale=0.125)
    torch.cuda.synchronize()
    del buf, kv
    torch.cuda.empty_cache()
    # the last key's score is 21.5, the others' 0
    share = math.exp(21.5) / (math.exp(21.5) + n - 1)
    assert torch.all(out[..., :-8] == 0)
    # rounded probabilities (2^-8) and result (2^-8), the score's roundings
    assert torch.all((out[..., -8:].double() - share).abs() <= (2.0 ** -7 + 200 * 2.0 ** -24) * share)
