"""Calls of the sequence operators that are refused, beyond the ones beside each operator's tests."""
import pytest
import torch

from paper_2309_12252_amd import deer

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def refused(call):
    with pytest.raises(deer.DeerError) as e:
        call()
    assert e.value.status == deer.DEER_ERR_INVALID_ARG


@pytest.mark.parametrize("seed,draw", [(0, 1 << 32), (0, -1), (1 << 64, 0)])
def test_draws_and_seeds(seed, draw):
    x = torch.zeros(2, 8, 4, device=DEV)
    refused(lambda: deer.dropout(x, 0.5, seed, draw))
    refused(lambda: deer.diagrec_solve(x, x, drop=0.5, seed=seed, draw=draw))
    refused(lambda: deer.diagrec_grad(x, x, x, x, drop=0.5, seed=seed, draw=draw))
