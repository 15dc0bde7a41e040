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


@pytest.mark.parametrize("d,most", [(1, 1 << 30), (64, 1 << 30), (65, (1 << 30) - 128), (128, (1 << 30) - 128), (129, (1 << 29) - 128),
                                    (512, 268435328), (65536, 128 * ((1 << 14) - 1))])
def test_the_largest_scans_are_those_that_the_header_names(d, most):
    assert mol.mol_gated_scan_workspace(most, d, 1) > 0
    for T in (most + 1, 1 << 31 if most == 1 << 30 else 1 << 30):
        with pytest.raises((mol.MolError, ValueError)):
            mol.mol_gated_scan_workspace(T, d, 1)
