"""The bounded waits of the tensor-core attention: what never comes ends in a status word, not in a kernel that does not."""
import ctypes

import pytest
import torch

import paper_2604_13349_b200 as P
from paper_2604_13349_b200 import binding
from tests import _attend_ref as ref
from tests.test_attend import BF16, INVALID, _args, _check, _data, _prefix

EXPIRES = binding.OBF_FLAG_TEST_WAIT_EXPIRES
SHAPE = dict(batch=1, kv_heads=2, q_heads=8, n_q=64, capacity=300, flags=EXPIRES)


@pytest.mark.parametrize("kw", [dict(batch=3), dict(n_q=2049), dict(capacity=2049), dict(n_q=4), dict(dtype=P.OBF_F32), dict(flags=EXPIRES | 1),
                                dict(n_q=8, mass_out=0x1000), dict(kv_heads=1, q_heads=130)])
def test_the_hook_is_refused_where_its_kernel_is_not_used_and_in_large_calls(kw):
    assert P.obf_attend_workspace_bytes(_args(**SHAPE)) >= 256
    a = _args(**{**SHAPE, **kw})
    with pytest.raises(P.ObfError) as e:
        P.obf_attend_workspace_bytes(a)
    assert e.value.code == INVALID
    lib = binding.load()
    assert lib.obf_attend(ctypes.byref(a), 0x100, 1 << 50, None) == INVALID
    x = _prefix()
    assert lib.obf_attend_shared(ctypes.byref(_args(**SHAPE)), ctypes.byref(x), 0x100, 1 << 50, None) == INVALID
    assert lib.obf_last_launch_count() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,kv,G,n_q,cap,window,sinks", [
    (1, 1, 4, 64, 64, 0, 0),             # one tile of keys: the softmax waits for the products' end
    (1, 2, 4, 60, 60, 0, 0),             # its last keys are cleared of what lies behind them: waits for the values themselves
    (2, 2, 4, 200, 500, 0, 0),           # several tiles: the next logits do not come
    (2, 1, 2, 600, 900, 100, 4),
    (1, 4, 8, 2048, 2048, 0, 0),         # several items per block
    (1, 1, 4, 40, 2000, 0, 0),           # parts and a join
])
def test_values_that_never_come_are_reported(d, B, kv, G, n_q, cap, window, sinks):
    gen = torch.Generator().manual_seed(n_q)
    q, k, v = (x.cuda() for x in _data(gen, B, kv, G, d, n_q, cap, BF16))
    ws = P.attend_workspace(q, k, window=window, sinks=sinks)
    want = P.attend(q, k, v, window=window, sinks=sinks, want_lse=True, workspace=ws)
    assert P.obf_last_device_status(ws) == 0
    for _ in range(2):
        P.attend(q, k, v, window=window, sinks=sinks, workspace=ws, flags=EXPIRES)
        torch.cuda.synchronize()
        assert P.obf_last_device_status(ws) == binding.OBF_DEV_TIMEOUT
    # the workspace, the streams and the device are as usable as before
    got = P.attend(q, k, v, window=window, sinks=sinks, want_lse=True, workspace=ws)
    torch.cuda.synchronize()
    assert P.obf_last_device_status(ws) == 0
    assert torch.equal(got["out"], want["out"]) and torch.equal(got["lse"], want["lse"])
    if n_q <= 600:
        w = ref.attend(q.cpu(), k.cpu(), v.cpu(), [cap] * B, [n_q] * B, window, sinks)
        _check(got["out"], w[0], w[1], "out")
