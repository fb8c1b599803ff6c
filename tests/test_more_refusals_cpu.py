"""Refusals of the linear operator, the layer norm and the cross entropy that need no device."""
import pytest
import torch

import paper_2504_18454_b200 as P


@pytest.mark.parametrize("out", [(), (None,), (None, None, None)])
def test_cross_entropy_takes_a_pair_of_outputs(out):
    with pytest.raises(P.PalsgdError, match="out must be"):
        P.cross_entropy_forward(torch.zeros(1, 2, 4), torch.zeros(1, 2, dtype=torch.int32), out=out)
