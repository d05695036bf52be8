"""Host-side checks of sizes whose products leave 64 bits: refused before any device call."""
import pytest

import paper_2604_12841_amd as pdx
from paper_2604_12841_amd import tokens

P = 4096  # an aligned address that no call may touch


def matmul(**kw):
    a = dict(M=4, N=8, K=32, codes_type=2, out_dtype=1, act=0, a=P, a_stride=32, a_scales=P, w=P, w_stride=32, w_scales=P, out=P, out_stride=8) | kw
    return tokens._functions().predecoder_matmul8(None, tokens.Matmul8Args(**a))


@pytest.mark.parametrize("M,N", [((1 << 63) - 1, 8), (1 << 62, (1 << 31) - 1), (1 << 56, 1 << 20), ((1 << 30) + 1, 1), (1 << 29, 256)])
def test_products_of_too_many_tiles(M, N):
    assert matmul(M=M, N=N, out_stride=N) == pdx.PD_ERR_UNSUPPORTED


@pytest.mark.parametrize("rows,width", [((1 << 63) - 1, 64), (1 << 62, 32768), (1 << 50, 32768), ((1 << 40) + 1, 1)])
def test_norms_of_too_many_rows(rows, width):
    a = dict(rows=rows, width=width, dtype=1, codes_type=0, eps=1e-6, x=P, x_stride=width, out=P, out_stride=width)
    assert tokens._functions().predecoder_rms_norm(None, tokens.NormArgs(**a)) == pdx.PD_ERR_UNSUPPORTED
