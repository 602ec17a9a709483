"""What the Python calls of the operators on a relayed cache refuse, and what they tell of a call that went wrong on the device."""
import pytest
import torch

import paper_2604_13349_b200 as P
from tests.test_attend import _small


@pytest.mark.gpu
@pytest.mark.parametrize("n_q", [1, 40])
def test_a_workspace_that_is_not_memory_of_its_own_is_refused(n_q):
    q, k, v = _small(n_q=n_q)
    need = P.attend_workspace(q, k).numel()
    for ws in (torch.zeros(1, dtype=torch.uint8, device="cuda").expand(need), torch.zeros(2 * need, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(ValueError, match="workspace"):
            P.attend(q, k, v, workspace=ws)
        with pytest.raises(ValueError, match="workspace"):
            P.attend_shared(q, k[0], v[0], k, v, workspace=ws)
