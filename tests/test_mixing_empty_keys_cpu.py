"""Keys without elements are refused in the library's own manner, not by an error of
arithmetic in the binding."""
import pytest
import torch

import paper_2308_15152_amd as pkg


def test_keys_of_size_zero():
    q, v, g = torch.zeros(1, 20, 2, 0), torch.zeros(1, 20, 2, 8), torch.zeros(1, 20, 2)
    for query in (pkg.delta_emu_forward_workspace, pkg.delta_emu_backward_workspace):
        with pytest.raises(pkg.SgemmEmuError) as e:
            query(q, q, v, g, g)
        assert "unsupported" in str(e.value).lower() or "-6" in str(e.value)
