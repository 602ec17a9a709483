"""What the Python calls of the operators on a relayed cache refuse, and what they tell of a call that went wrong on the device."""
import pytest
import torch

import paper_2604_13349_b200 as P
from paper_2604_13349_b200 import binding
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


@pytest.mark.gpu
@pytest.mark.parametrize("n_q", [1, 40])
def test_a_call_s_status_can_be_asked_for(n_q):
    q, k, v = _small(n_q=n_q)
    good, bad = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([600, 1], [601, 1]))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    calls = [P.attend(q, k, v, lens=n, want_status=True, stream=s) for n in (bad, good) for s in (None, side)]
    shared = [P.attend_shared(q, k[0], v[0], k, v, lens=n, want_status=True) for n in (bad, good)]
    torch.cuda.synchronize()
    assert [P.obf_last_device_status(c["workspace"]) for c in calls + shared] == [binding.OBF_DEV_INTERNAL] * 2 + [0] * 2 + [binding.OBF_DEV_INTERNAL, 0]
    assert all(torch.equal(c["out"], calls[0]["out"]) for c in calls)
    assert "workspace" not in P.attend(q, k, v, lens=bad)
    ws = P.attend_workspace(q, k)
    assert P.attend(q, k, v, lens=bad, workspace=ws, want_status=True)["workspace"] is ws


@pytest.mark.gpu
def test_a_wait_that_ran_out_shows_in_the_status():
    q, k, v = _small(B=1, n_q=64)
    got = P.attend(q, k, v, flags=binding.OBF_FLAG_TEST_WAIT_EXPIRES, want_status=True)
    assert P.obf_last_device_status(got["workspace"]) == binding.OBF_DEV_TIMEOUT
