"""Refusals of the operators' Python entry points that come after the tensors have been found to be on the GPU."""
import pytest
import torch

import paper_2111_00705_amd as P

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("k", [-1, 9, 129])
def test_a_number_of_alternatives_that_there_are_not(k):
    z = torch.zeros(2, 8 if k == 9 else 1000, device="cuda")
    with pytest.raises(P.CompAmsError, match="k=") as e:
        P.token_logprobs(z, None, k)
    assert "must be in" in str(e.value)
