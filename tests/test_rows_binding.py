"""What the binding makes of a caller's numbers before a call (nothing here reaches a GPU)."""
import numpy as np
import pytest
import torch

from paper_2412_12706_amd import kvqp


@pytest.mark.parametrize("parents", [[-1, 0, 0, 1, 2], [[-1, 0, 1], [-1, -1, 0]]])
def test_parents_may_be_lists_arrays_or_tensors(parents):
    want = kvqp.tree_mask(parents, device="cpu")
    for given in (tuple(parents), np.array(parents), torch.tensor(parents), torch.tensor(parents, dtype=torch.int32)):
        assert torch.equal(kvqp.tree_mask(given, device="cpu"), want)
