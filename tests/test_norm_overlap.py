"""Outputs that are the inputs' own memory are refused before anything touches a GPU."""
import pytest
import torch

import paper_2510_00236_b200 as pe


def test_outputs_on_top_of_inputs_are_refused():
    x = torch.zeros(2, 3, 16, dtype=torch.bfloat16)
    r = torch.zeros(2, 3)
    with pytest.raises(ValueError, match="overlap"):
        pe.pe_norm_forward(x, out=x)
    dy = torch.zeros_like(x)
    with pytest.raises(ValueError, match="overlap"):
        pe.pe_norm_backward(x, dy, None, r, r, "square", dx=dy)
