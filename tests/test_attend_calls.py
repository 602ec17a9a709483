"""What the Python calls of the operators on a relayed cache refuse, and what they tell of a call that went wrong on the device."""
import pytest
import torch

import paper_2604_13349_b200 as P
from paper_2604_13349_b200 import binding
from tests.test_attend import _small


def _calls(q, k, v, m):
    return {"q": lambda x: P.attend(x(q), k, v), "k": lambda x: P.attend(q, x(k), v), "v": lambda x: P.attend(q, k, x(v)),
            "mass_in": lambda x: P.attend(q, k, v, mass_in=x(m), mass_out=torch.zeros_like(m)),
            "shared q": lambda x: P.attend_shared(x(q), k[0], v[0], k, v), "k_prefix": lambda x: P.attend_shared(q, x(k[0]), v[0], k, v),
            "v_prefix": lambda x: P.attend_shared(q, k[0], x(v[0]), k, v), "shared k": lambda x: P.attend_shared(q, k[0], v[0], x(k), v),
            "shared v": lambda x: P.attend_shared(q, k[0], v[0], k, x(v)), "evicted k": lambda x: P.evict_by_mass(x(k), v, m, 10),
            "evicted v": lambda x: P.evict_by_mass(k, x(v), m, 10), "mass": lambda x: P.evict_by_mass(k, v, x(m), 10)}


def _leaf(t):
    return t.detach().clone().requires_grad_()


def test_tensors_that_require_a_gradient_are_refused():
    # (before anything else is looked at: nothing reaches a device)
    for name, call in _calls(torch.zeros(1, 4, 1, 64), torch.zeros(1, 2, 30, 64), torch.zeros(1, 2, 30, 64), torch.zeros(1, 2, 30)).items():
        with pytest.raises(ValueError, match="gradient"):
            call(_leaf)
            pytest.fail(name)


@pytest.mark.gpu
def test_without_a_graph_they_are_taken():
    q, k, v = _small(cap=100)
    for call in _calls(q, k, v, torch.rand(2, 2, 100, device="cuda")).values():
        want = call(lambda t: t)
        for mode in (torch.no_grad, torch.inference_mode):
            with mode():
                got = call(_leaf)
            assert all(torch.equal(got[n], want[n]) for n in want)


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
