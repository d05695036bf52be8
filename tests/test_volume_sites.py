"""The sites of a volume's activations, on the CPU."""
import pytest
import torch

import paper_2604_12841_amd as pdx


@pytest.mark.parametrize("layout,H", [("plaquette", 6), ("paper", 5)])
def test_sites_in_memory_order(layout, H):
    s = pdx.volume_sites(5, 3, volume=2, first_round=7, layout=layout, device="cpu")
    assert s.shape == (3 * H * H, 4) and s.dtype == torch.int32 and s.is_contiguous()
    want = [[7 + t, i, j, 2] for t in range(3) for i in range(H) for j in range(H)]
    assert s.tolist() == want


@pytest.mark.parametrize("layout", ["Paper", "", None, 1])
def test_unknown_layouts_are_refused(layout):
    with pytest.raises(ValueError, match="layout"):
        pdx.volume_sites(5, 3, layout=layout, device="cpu")
