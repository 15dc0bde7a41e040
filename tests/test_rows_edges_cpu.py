"""Refusals of the operators between embedding rows and scores at the ends of what
the library's types hold (CPU only)."""
import pytest
import torch

from paper_2407_15462_amd import mol


@pytest.mark.parametrize("d", [1 << 31, (1 << 32) + 8, (1 << 32) + 16385])
def test_rows_past_int32_are_refused(d):
    """A row's size goes to the library as int32: a larger one is turned down, not cut off to one that it takes."""
    x, ws = torch.empty(0, d), torch.empty(0, dtype=torch.uint8)
    for call in (lambda: mol.layer_norm(x), lambda: mol.layer_norm(x, out=x), lambda: mol.normalize(x), lambda: mol.normalize_grad(x, x),
                 lambda: mol.layer_norm_grad(x, x), lambda: mol.layer_norm_grad(x, x, weights=False), lambda: mol.layer_norm_grad(x, x, ws=ws),
                 lambda: mol.layer_norm_grad_workspace(x), lambda: mol.gated_scan(x, x), lambda: mol.gated_step(x, x, x)):
        with pytest.raises(ValueError, match="2.31"):
            call()
