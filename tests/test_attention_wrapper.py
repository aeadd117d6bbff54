"""What the Python binding of the cache and attention checks of its tensors: nothing here touches a device."""
from types import SimpleNamespace

import pytest
import torch

import paper_2602_11688_amd as g
from paper_2602_11688_amd import attention as ga

CACHE = SimpleNamespace(head_dim=64, row_dtype=torch.bfloat16, device=torch.device("cpu"))
BATCH = SimpleNamespace(tokens=5)


def test_tensors_that_wait_for_a_gradient_are_refused():
    """Keys, values, queries and given results all pass here; without gradients, detached or under no_grad, they are taken."""
    leaf = torch.zeros((5, 8, 64), dtype=torch.bfloat16, requires_grad=True)
    for t in (leaf, leaf * 2, leaf[:, :, :]):
        with pytest.raises(g.GorgoError, match="q requires a gradient"):
            ga._rows(t, 8, CACHE, BATCH, "q")
        with torch.no_grad():
            assert ga._rows(t, 8, CACHE, BATCH, "q").data == t.data_ptr()
        assert ga._rows(t.detach(), 8, CACHE, BATCH, "q").token_stride == 512


def test_caches_that_wait_for_a_gradient_are_refused():
    k = torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16)
    for pair in ((k.clone().requires_grad_(), k), (k, k.clone().requires_grad_())):
        with pytest.raises(g.GorgoError, match="requires a gradient"):
            g.KvCache(*pair)


def test_lengths_without_a_dimension_are_refused():
    for lengths in (torch.tensor(3, dtype=torch.int32), torch.zeros((2, 2), dtype=torch.int32)):
        with pytest.raises(g.GorgoError, match="lengths"):
            g.KvBatch(torch.zeros((2, 3), dtype=torch.int32), lengths)
