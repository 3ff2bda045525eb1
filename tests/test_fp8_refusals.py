"""Refusals of 8-bit products' Python calls, before any device work (no GPU needed)."""
import pytest
import torch


def test_runs_of_columns_need_offsets():
    """Without them the call would be another product: one matrix over all columns."""
    import paper_2106_08846_gb300 as bsr
    a, b = bsr.Fp8Matrix(4, 256, device="cpu"), bsr.Fp8Matrix(8, 256, device="cpu")
    with pytest.raises(ValueError, match="offsets"):
        bsr.bsr_fp8_product(a, b, over="columns")
    with pytest.raises(ValueError, match="offsets"):
        bsr.bsr_fp8_product(a, b, over="columns", Y=torch.zeros(4, 8))
