"""Calls on a relayed cache held in 8 or 4 bits: what they refuse, captured and concurrent calls over rows read back, limits, precision."""
import ctypes
import math

import pytest
import torch

import paper_2604_13349_b200 as P
from paper_2604_13349_b200 import binding, build
from tests import _quant_ref as qref
from tests import test_quantized

BF16, F32 = torch.bfloat16, torch.float32


def _held(gen, B, kv, cap, d, bits):
    """A cache of any codes and scales of five bits, on the device."""
    cache = P.quantized_cache(B, kv, cap, d, bits)
    for i in range(2):
        c = torch.randint(0, 256, cache[i].shape, generator=gen, dtype=torch.int32).to(torch.uint8)
        cache[i].copy_(c.view(torch.int8) if bits == 8 else c)
        cache[2 + i].copy_(torch.randint(16, 32, cache[2 + i].shape, generator=gen) * (0.0005 if bits == 8 else 0.0078125))
    return cache


def _rows_bytes(attend_bytes, bits, B, kv, cap, d):
    """The workspace of a call that reads rows back: that of `attend` over them, K and V in bf16, in 8 bits two factors of each row of a head."""
    def up(x, n=256):
        return (x + n - 1) // n * n
    return up(attend_bytes) + 2 * up(B * kv * cap * d * 2) + (up((B * kv * up(cap, 4) + 128) * 8) if bits == 8 else 0)


def _reads_back(ws, q, cache, **kw):
    return ws.numel() == _rows_bytes(P.attend_workspace(q, cache.k, **kw).numel(), 8 if cache.k.dtype is torch.int8 else 4, *cache.k.shape[:3], q.shape[3])


# ---- gradients ------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("which", ["k_scale", "v_scale"])
def test_scales_that_require_a_gradient_are_refused(bits, which):
    host = P.quantized_cache(1, 2, 10, 64, bits, device="cpu")
    leaf = host._replace(**{which: getattr(host, which).clone().requires_grad_()})
    x = torch.zeros(1, 2, 3, 64)
    for call in (lambda: P.attend_quantized(x, leaf), lambda: P.read_quantized(leaf), lambda: P.write_quantized(leaf, x, x)):
        with pytest.raises(ValueError, match="gradient"):
            call()
        with torch.no_grad(), pytest.raises(ValueError, match="on a device"):        # the next check: tensors of the host
            call()


# ---- outputs ---------------------------------------------------------------------------------------------------------
@pytest.mark.gpu
def test_outputs_of_another_number_of_dimensions_are_refused():
    cache = P.quantized_cache(1, 2, 10, 64)
    q = torch.zeros(1, 2, 3, 64, dtype=BF16, device="cuda")
    for out in (torch.zeros(2, 3, 64, dtype=BF16, device="cuda"), torch.zeros(64, dtype=BF16, device="cuda"), torch.zeros((), dtype=BF16, device="cuda"),
                torch.zeros(1, 1, 2, 3, 64, dtype=BF16, device="cuda")):
        with pytest.raises(ValueError, match="out"):
            P.attend_quantized(q, cache, out=out)
        with pytest.raises(ValueError, match="k_out"):
            P.read_quantized(cache, k_out=out, v_out=out)
        with pytest.raises(ValueError, match="k_values"):
            P.write_quantized(cache, q, q, k_values=out, v_values=out)
    for name in ("k", "v", "k_scale", "v_scale"):
        with pytest.raises(ValueError, match="cache"):
            P.read_quantized(cache._replace(**{name: getattr(cache, name)[0]}))
        with pytest.raises(ValueError, match="cache"):
            P.read_quantized(cache._replace(**{name: getattr(cache, name).reshape(-1)[0]}))


# ---- calls that read rows back ----------------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d,B,kv,G,n_q,cap,window", [(128, 2, 2, 4, 600, 2200, 600), (64, 3, 1, 2, 1500, 1500, 600), (128, 1, 1, 4, 300, 6000, 0)])
def test_calls_that_read_rows_back_at_the_same_time_and_from_graphs(bits, d, B, kv, G, n_q, cap, window):
    """Two calls on two streams, each with its workspace, and two captured ones that are replayed side by side while lengths and caches change: what each
    gives is what it gives alone."""
    gen = torch.Generator().manual_seed(n_q + bits)
    caches = [_held(gen, B, kv, cap, d, bits) for _ in range(2)]
    q = [torch.randn(B, kv * G, n_q, d, generator=gen).to(BF16).cuda() for _ in range(2)]
    lens = [torch.tensor([cap - 7 * i * (b + 1) for b in range(B)], dtype=torch.int32, device="cuda") for i in range(2)]
    kw = dict(window=window, sinks=3)
    ws = [P.attend_quantized_workspace(q[0], caches[0], **kw) for _ in range(2)]
    assert all(_reads_back(w, q[0], c, **kw) for w, c in zip(ws, caches))
    out = [torch.empty_like(x) for x in q]
    alone = [P.attend_quantized(q[i], caches[i], lens=lens[i], **kw)["out"] for i in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    graphs = []
    for i in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i], stream=streams[i]):
            P.attend_quantized(q[i], caches[i], lens=lens[i], out=out[i], workspace=ws[i], **kw)
    for turn in range(8):
        if turn >= 4:                                                # other lengths and rows
            for i in range(2):
                lens[i] -= 5
                caches[i].k.add_(1 if bits == 8 else 0x10)
                caches[i].v_scale.mul_(-1)
                alone[i] = P.attend_quantized(q[i], caches[i], lens=lens[i], **kw)["out"]
        for x, w in zip(out, ws):
            x.fill_(-77.0)
            w.fill_(0xFF)
        torch.cuda.synchronize()
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                if turn % 2:
                    graphs[i].replay()
                else:
                    P.attend_quantized(q[i], caches[i], lens=lens[i], out=out[i], workspace=ws[i], **kw)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, alone))


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


def _need(lib, bits, B, kv, G, d, n_q, cap, window=0, sinks=0, flags=0):
    """The workspaces of a call and of `attend` over the same rows."""
    a = P.ObfAttend(batch=B, kv_heads=kv, q_heads=kv * G, head_dim=d, n_q=n_q, capacity=cap, window=window, sinks=sinks, dtype=P.OBF_BF16, flags=flags)
    n = ctypes.c_size_t(0)
    assert lib.obf_attend_quantized_workspace_bytes(ctypes.byref(a), ctypes.byref(P.ObfQuantized(bits=bits)), ctypes.byref(n)) == 0
    return n.value, P.obf_attend_workspace_bytes(a)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d,kw", test_quantized.BIG + [(128, dict(B=1, kv=2, G=8, n_q=900, cap=1400, window=301, sinks=3))])
def test_the_large_cases_read_rows_back(lib, bits, d, kw):
    # the cases of test_attention_over_rows_read_back and of test_rows_read_back_hold_nothing_of_what_is_not_seen
    size = {n: kw[n] for n in ("B", "kv", "G", "n_q", "cap", "window", "sinks") if n in kw}
    got, plain = _need(lib, bits, d=d, **size)
    codes, _ = _need(lib, bits, d=d, flags=binding.OBF_FLAG_GENERIC_PATH, **size)
    assert got == _rows_bytes(plain, bits, kw["B"], kw["kv"], kw["cap"], d) != codes


def test_rows_are_read_back_up_to_a_size_of_the_workspace(lib):
    # a window over a cache of a million rows: 4 GB of rows are read back, where they would be more the call stays on codes
    def need(batch, n_q, **kw):
        return _need(lib, 4, batch, 8, 4, 128, n_q, 1 << 20, window=1024, **kw)[0]
    assert need(1, 1024) > 1 << 32 and need(2, 1024) < 1 << 31
    assert need(1, 1024, flags=binding.OBF_FLAG_GENERIC_PATH) < 1 << 31 and need(1, 1) < 1 << 31


@pytest.mark.gpu
def test_a_call_whose_rows_would_take_too_much_stays_on_codes():
    # the same rows at the end of caches of a million rows and in caches of their own
    gen = torch.Generator().manual_seed(2)
    cap, near, kv, d, n_q, window = 1 << 20, 2500, 8, 128, 600, 1024
    small = _held(gen, 2, kv, near, d, 4)
    wide = P.QuantizedCache(*(torch.empty((2, kv, cap, t.shape[-1]), dtype=t.dtype, device="cuda") for t in small))
    for w, t in zip(wide, small):
        w[:, :, :-near].view(torch.uint8).fill_(0xFF)               # scales that are not numbers
        w[:, :, -near:] = t
    q = torch.randn(2, 4 * kv, n_q, d, generator=gen).to(BF16).cuda()
    ws = P.attend_quantized_workspace(q, small, window=window), P.attend_quantized_workspace(q, wide, window=window)
    assert _reads_back(ws[0], q, small, window=window) and not _reads_back(ws[1], q, wide, window=window) and ws[1].numel() < 1 << 31
    got = [P.attend_quantized(q, c, window=window, workspace=w, want_lse=True) for c, w in zip((small, wide), ws)]
    # both within weights and outputs rounded to bf16 of the same numbers: 2^-8 of the values' largest, each, twice
    size = qref.values(P.QuantizedCache(*(t.cpu() for t in small)))[1].abs().max().item()
    assert (got[0]["out"].float() - got[1]["out"].float()).abs().max().item() <= 4 * 2.0 ** -8 * size
    assert (got[0]["lse"] - got[1]["lse"]).abs().max().item() <= 2.0 ** -12


# ---- precision of fp32 calls -------------------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("G,n_q", [(1, 1), (4, 1), (8, 1), (4, 4), (8, 3), (4, 9)])
def test_precision_of_fp32_calls(d, bits, G, n_q):
    """Numbers of one sign, so that nothing cancels and every bound is relative.

    Outputs with equal weights (queries of zero).  A weight times a scale in three bf16 parts: 2^-24.  The product over sixteen keys: seventeen numbers cut
    off at 2^-23 of the power of two below the largest, in all at most 17 / 1024 128 2^-23 = 4.3 2^-24 of the sum (codes of 64 to 127, scales of one to
    two; less for codes of 3 to 7).  Added up by a warp: 1024 / 64 sums, the running one growing by equal steps: 16 / 2 roundings of 2^-24.  Joining
    warps and parts, dividing: six.  Less than 20 * 2^-24 = 1.2e-6.
    Logits (single keys' logarithms).  A query in two parts: 2^-22.  What the second parts add, 64 numbers to each of two sums, is cut off at 2^-23
    of the running sum (the first parts' products are multiples of that), half as much on average: 32 * 2^-23.  Factors: six roundings.  4.5e-6."""
    gen = torch.Generator().manual_seed(bits + d + n_q)
    B, kv, cap = 2, 2, 1024
    cache = P.quantized_cache(B, kv, cap, d, bits)
    for i in range(2):
        if bits == 8:
            cache[i].copy_(torch.randint(64, 128, cache[i].shape, generator=gen))
            cache[2 + i].copy_(torch.rand(cache[2 + i].shape, generator=gen) + 1.0)
        else:
            two = torch.randint(3, 8, (2, *cache[i].shape), generator=gen) + 8
            cache[i].copy_(two[0] | (two[1] << 4))
            cache[2 + i].copy_(torch.randint(16, 32, cache[2 + i].shape, generator=gen) / 16.0)
    k, v = qref.values(cache)
    zero = torch.zeros(B, kv * G, n_q, d, device="cuda")
    got = P.attend_quantized(zero, cache)["out"].double().cpu()
    for i in range(n_q):
        want = v[:, :, : cap - n_q + i + 1].mean(2)[:, :, None]
        assert ((got[:, :, i].reshape(B, kv, G, d) - want).abs() / want).max() <= 2e-6
    q = torch.rand(B, kv * G, n_q, d, generator=gen) + 1.0
    lens = torch.full((B,), 1, dtype=torch.int32, device="cuda")
    first = P.attend_quantized(q[:, :, :1].cuda(), cache, lens=lens, want_lse=True)["lse"].double().cpu()[:, :, 0]
    want = (q[:, :, 0].double().reshape(B, kv, G, d) @ k[:, :, 0, :, None])[..., 0].reshape(B, kv * G) / math.sqrt(d)
    assert ((first - want).abs() / want).max() <= 4.5e-6


# ---- held again ----------------------------------------------------------------------------------------------------------
def _rows(gen, shape, dtype):
    x = torch.randn(shape, generator=gen) * torch.exp2(torch.randint(-100, 100, (*shape[:-1], 1), generator=gen).float())
    x[..., ::7, :] = 0.0
    return x.to(dtype)


@pytest.mark.parametrize("d", [64, 128])
def test_values_in_4_bits_are_held_as_they_are_by_definition(d):
    # the largest code of a group is 7 (max / 7 rounded to five bits is within 1/32 of itself, 7 / (1 -+ 1/32) rounds to 7), so the largest value over 7 is
    # the scale itself
    x = _rows(torch.Generator().manual_seed(d), (5000, d), F32)
    codes, scale = qref.quantize(x.double().numpy(), 4)
    again = qref.quantize(codes * scale[..., qref.group(d)], 4)
    assert (again[0] == codes).all() and (again[1] == scale).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
def test_values_in_4_bits_are_held_as_they_are(d, dtype):
    x = [_rows(torch.Generator().manual_seed(d + i), (2, 3, 501, d), dtype).cuda() for i in range(2)]
    one, two = (P.quantized_cache(2, 3, 501, d, 4) for _ in range(2))
    values = P.write_quantized(one, *x, want_values=True)
    back = P.read_quantized(one, dtype=dtype)
    again = P.write_quantized(two, back["K"], back["V"], want_values=True)
    assert all(torch.equal(a, b) for a, b in zip(one, two))
    assert all(torch.equal(values[n], back[n]) and torch.equal(again[n], back[n]) for n in "KV")
