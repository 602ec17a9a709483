"""A relayed cache held in 8 or 4 bits: rows written, read back, attended over."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2604_13349_b200 as P
from paper_2604_13349_b200 import binding, build
from tests import _attend_ref as ref
from tests import _quant_ref as qref

BF16, F32 = torch.bfloat16, torch.float32
INVALID, UNSUPPORTED, WORKSPACE = binding.OBF_ERR_INVALID_ARG, binding.OBF_ERR_UNSUPPORTED, binding.OBF_ERR_WORKSPACE


# ---- refusals: decided on the host, nothing reaches a device ------------------------------------------------------
@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


def _fill(cls, kw, defaults):
    d = {**defaults, **kw}
    a = cls(**{n: x for n, x in d.items() if not n.endswith("stride")})
    for n, x in d.items():
        if n.endswith("stride"):
            setattr(a, n, (ctypes.c_int64 * 3)(*x))
    return a


def _cache(**kw):
    return _fill(P.ObfQuantized, kw, dict(bits=4, k=0x1000, v=0x1000, k_scale=0x1000, v_scale=0x1000, k_stride=(6400, 3200, 32), v_stride=(6400, 3200, 32),
                                          k_scale_stride=(400, 200, 2), v_scale_stride=(400, 200, 2)))


def _write(**kw):
    return _fill(P.ObfQuantizedWrite, kw, dict(batch=2, kv_heads=2, head_dim=64, capacity=100, rows=3, dtype=P.OBF_BF16, k=0x1000, v=0x1000,
                                               k_stride=(384, 192, 64), v_stride=(384, 192, 64)))


def _read(**kw):
    return _fill(P.ObfQuantizedRead, kw, dict(batch=2, kv_heads=2, head_dim=64, capacity=100, first=10, rows=5, dtype=P.OBF_F32, k_out=0x1000, v_out=0x1000,
                                              k_out_stride=(640, 320, 64), v_out_stride=(640, 320, 64)))


def _attend(**kw):
    return _fill(P.ObfAttend, kw, dict(batch=2, kv_heads=2, q_heads=8, head_dim=64, n_q=3, capacity=100, dtype=P.OBF_BF16, q=0x1000, out=0x1000,
                                       q_stride=(1536, 192, 64), out_stride=(1536, 192, 64)))


BAD_CACHES = [
    (dict(bits=5), UNSUPPORTED), (dict(bits=0), UNSUPPORTED), (dict(k=0), INVALID), (dict(v=0), INVALID), (dict(k_scale=0), INVALID), (dict(v_scale=0), INVALID),
    (dict(k=0x1008), INVALID), (dict(v=0x1001), INVALID), (dict(k_scale=0x1002), INVALID), (dict(v_scale=0x1001), INVALID), (dict(k_stride=(6400, 3200, 31)), INVALID),
    (dict(k_stride=(6400, 3200, 40)), INVALID), (dict(v_stride=(6400, -3200, 32)), INVALID), (dict(v_stride=(1 << 40, 3200, 32)), INVALID),
    (dict(k_scale_stride=(400, 200, 1)), INVALID), (dict(v_scale_stride=(401, 200, 2)), INVALID), (dict(v_scale_stride=(400, 0, 2)), INVALID),
    (dict(k_scale_stride=(1 << 39, 200, 2)), INVALID), (dict(bits=8, k_stride=(6400, 3200, 32)), INVALID),
]


@pytest.mark.parametrize("kw,code", BAD_CACHES)
def test_bad_caches_are_refused(lib, kw, code):
    c = ctypes.byref(_cache(**kw))
    assert lib.obf_quantized_write(ctypes.byref(_write()), c, None) == code
    assert lib.obf_quantized_read(ctypes.byref(_read()), c, None) == code
    assert lib.obf_attend_quantized(ctypes.byref(_attend()), c, 0x100, 1 << 50, None) == code
    assert lib.obf_last_launch_count() == 0


@pytest.mark.parametrize("kw,code", [
    (dict(batch=0), INVALID), (dict(kv_heads=0), INVALID), (dict(capacity=0), INVALID), (dict(capacity=(1 << 20) + 1), INVALID), (dict(rows=0), INVALID),
    (dict(rows=(1 << 20) + 1), INVALID), (dict(head_dim=96), UNSUPPORTED), (dict(dtype=2), UNSUPPORTED), (dict(k=0), INVALID), (dict(v=0x1004), INVALID),
    (dict(k_values=0x1000), INVALID), (dict(k_values=0x1000, v_values=0x1008), INVALID), (dict(k_values=0x1000, v_values=0x1000), INVALID),
    (dict(k_stride=(384, 192, 63)), INVALID), (dict(v_stride=(384, 0, 64)), INVALID), (dict(lens=0x1002), INVALID), (dict(new_lens=0x1001), INVALID),
    (dict(batch=1 << 20, kv_heads=32), UNSUPPORTED), (dict(batch=1 << 14, kv_heads=16, rows=1 << 13), UNSUPPORTED),
])
def test_write_refuses(lib, kw, code):
    assert lib.obf_quantized_write(ctypes.byref(_write(**kw)), ctypes.byref(_cache()), None) == code
    assert lib.obf_quantized_write(None, ctypes.byref(_cache()), None) == INVALID
    assert lib.obf_quantized_write(ctypes.byref(_write()), None, None) == INVALID
    assert lib.obf_last_launch_count() == 0


@pytest.mark.parametrize("kw,code", [
    (dict(batch=0), INVALID), (dict(capacity=0), INVALID), (dict(first=-1), INVALID), (dict(rows=0), INVALID), (dict(first=96), INVALID), (dict(rows=91), INVALID),
    (dict(head_dim=32), UNSUPPORTED), (dict(dtype=7), UNSUPPORTED), (dict(k_out=0), INVALID), (dict(v_out=0x1004), INVALID),
    (dict(k_out_stride=(640, 320, 60)), INVALID), (dict(v_out_stride=(640, 320, 66)), INVALID), (dict(lens=0x1001), INVALID),
])
def test_read_refuses(lib, kw, code):
    assert lib.obf_quantized_read(ctypes.byref(_read(**kw)), ctypes.byref(_cache()), None) == code
    assert lib.obf_quantized_read(None, ctypes.byref(_cache()), None) == INVALID
    assert lib.obf_last_launch_count() == 0


@pytest.mark.parametrize("kw,code", [
    (dict(batch=0), INVALID), (dict(q_heads=7), INVALID), (dict(q_heads=0), INVALID), (dict(kv_heads=0), INVALID), (dict(n_q=0), INVALID), (dict(capacity=0), INVALID),
    (dict(window=-1), INVALID), (dict(sinks=-1), INVALID), (dict(scale=-1.0), INVALID), (dict(scale=math.nan), INVALID), (dict(flags=2), INVALID),
    (dict(flags=binding.OBF_FLAG_TEST_WAIT_EXPIRES), INVALID), (dict(head_dim=80), UNSUPPORTED), (dict(dtype=4), UNSUPPORTED), (dict(mass_out=0x1000), UNSUPPORTED),
    (dict(mass_in=0x1000), UNSUPPORTED), (dict(batch=1 << 20, n_q=1 << 10), UNSUPPORTED), (dict(q=0), INVALID), (dict(out=0x1004), INVALID), (dict(k=0x1000), INVALID),
    (dict(v=0x1000), INVALID), (dict(lens=0x1002), INVALID), (dict(q_lens=0x1001), INVALID), (dict(lse_out=0x1002), INVALID), (dict(q_stride=(1536, 192, 63)), INVALID),
    (dict(out_stride=(1536, 0, 64)), INVALID),
])
def test_attend_refuses(lib, kw, code):
    assert lib.obf_attend_quantized(ctypes.byref(_attend(**kw)), ctypes.byref(_cache()), 0x100, 1 << 50, None) == code
    assert lib.obf_last_launch_count() == 0


def test_attend_refuses_a_small_or_misaligned_workspace(lib):
    a, c, need = _attend(), _cache(), ctypes.c_size_t(0)
    assert lib.obf_attend_quantized_workspace_bytes(ctypes.byref(a), ctypes.byref(c), ctypes.byref(need)) == 0
    need = need.value
    assert need >= 256 and need % 256 == 0
    for ws, n in ((None, need), (0x110, need), (0x100, need - 1)):
        assert lib.obf_attend_quantized(ctypes.byref(a), ctypes.byref(c), ws, n, None) == WORKSPACE
    assert lib.obf_attend_quantized_workspace_bytes(ctypes.byref(a), ctypes.byref(c), None) == INVALID
    assert lib.obf_attend_quantized_workspace_bytes(ctypes.byref(a), None, ctypes.byref(ctypes.c_size_t(0))) == INVALID


def test_struct_sizes_match_the_header():
    assert [ctypes.sizeof(x) for x in (P.ObfQuantized, P.ObfQuantizedWrite, P.ObfQuantizedRead)] == [136, 168, 104]


def test_python_wrappers_refuse():
    host = P.quantized_cache(1, 2, 10, 64, device="cpu")
    x = torch.zeros(1, 2, 3, 64)
    for call in (lambda: P.write_quantized(host, x, x), lambda: P.read_quantized(host), lambda: P.attend_quantized(x, host),
                 lambda: P.quantized_cache(1, 2, 10, 64, bits=2), lambda: P.quantized_cache(1, 2, 10, 96, device="cpu")):
        with pytest.raises(ValueError):
            call()
    leaf = x.clone().requires_grad_()
    for call in (lambda: P.write_quantized(host, leaf, x), lambda: P.write_quantized(host, x, leaf), lambda: P.attend_quantized(leaf, host)):
        with pytest.raises(ValueError, match="gradient"):
            call()


# ---- on the device --------------------------------------------------------------------------------------------------
def _empty(B, kv, cap, d, bits, token_major=False, sentinel=0x5A):
    """A cache whose bytes are all `sentinel`; token_major: rows of a token's heads side by side."""
    order = (0, 2, 1, 3) if token_major else (0, 1, 2, 3)

    def make(shape, dtype):
        n = [shape[i] for i in order[: len(shape)]]
        return torch.full(n, sentinel, dtype=torch.uint8, device="cuda").repeat_interleave(torch.empty(0, dtype=dtype).element_size(), -1).view(dtype).permute(
            [order.index(i) for i in range(len(shape))])
    codes, scales = (B, kv, cap, d if bits == 8 else d // 2), (B, kv, cap) if bits == 8 else (B, kv, cap, d // 32)
    if bits == 8 and token_major:
        s = [make((B, kv, cap, 1), F32)[..., 0] for _ in range(2)]
    else:
        s = [make(scales, F32 if bits == 8 else BF16) for _ in range(2)]
    return P.QuantizedCache(*(make(codes, torch.int8 if bits == 8 else torch.uint8) for _ in range(2)), *s)


def _bytes(t):
    return t.contiguous().view(torch.uint8).cpu().numpy()


def _numbers(gen, shape, dtype):
    """Rows with what is hard to quantise: numbers half, three quarters and a seventh of the largest, rows of one size, large and small rows."""
    x = torch.randn(shape, generator=gen, dtype=F32)
    top = x.abs().amax(-1, keepdim=True)
    pick = torch.randint(0, 12, shape, generator=gen)
    for i, f in enumerate((0.5, 0.75, 1.0 / 7, 1.5 / 7, 0.25)):
        x = torch.where(pick == i, top.to(dtype).float() * f * torch.sign(x), x)
    x = x * torch.exp2(torch.randint(-90, 90, (*shape[:-1], 1), generator=gen).float())
    return x.to(dtype)


def _check_rows(cache, before, x, at, bits, which):
    """Rows x [n, d] (CPU) of one head stand in rows `at` of codes and scales [capacity, ...], everything else is as before."""
    codes, scales = qref.quantize(x.double().numpy(), bits)
    want_c, want_s = before[0].copy(), before[1].copy()
    want_c[at] = qref.pack(codes, bits).view(np.uint8)
    s = torch.from_numpy(scales).to(F32 if bits == 8 else BF16)
    assert bits == 8 or torch.equal(torch.nan_to_num(s.double()), torch.nan_to_num(torch.from_numpy(scales)))
    want_s[at] = s.reshape(len(at), -1).view(torch.uint8).numpy()
    assert np.array_equal(which[0], want_c)
    nan = np.repeat(np.isnan(scales).reshape(len(at), -1), s.element_size(), -1)
    got_s = which[1].copy()
    got_s[at], want_s[at] = np.where(nan, 0, got_s[at]), np.where(nan, 0, want_s[at])
    assert np.array_equal(got_s, want_s)
    return codes, scales


def _values_of(codes, scales, bits, d):
    return codes * (scales[..., None] if bits == 8 else scales[..., qref.group(d)])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,kv,cap,rows,lens,new,token_major", [
    (1, 1, 1, 1, None, None, False), (3, 2, 70, 1, [1, 70, 33], None, True), (4, 3, 40, 9, [9, 40, 7, 0], [9, 0, 5, 7], False),
    (2, 5, 300, 300, [300, 257], [300, 257], True), (2, 2, 50, 60, None, None, False), (3, 1, 20, 8, [25, 4, -3], [8, 8, 9], False),
    (2, 2, 33, 30, None, [0, 29], True),
])
def test_rows_written(dtype, bits, d, B, kv, cap, rows, lens, new, token_major):
    gen = torch.Generator().manual_seed(B * 1000 + cap + bits + d)
    x = [_numbers(gen, (B, rows, kv, d) if token_major else (B, kv, rows, d), dtype) for _ in range(2)]
    x = [t.transpose(1, 2) for t in x] if token_major else x
    dev = [torch.empty_strided(t.size(), t.stride(), dtype=dtype, device="cuda").copy_(t) for t in x]
    cache = _empty(B, kv, cap, d, bits, token_major)
    before = [_bytes(t) for t in cache]
    vals = [torch.full_like(t, -77.0) for t in dev]
    ints = [None if t is None else torch.tensor(t, dtype=torch.int32, device="cuda") for t in (lens, new)]
    got = P.write_quantized(cache, *dev, lens=ints[0], new_lens=ints[1], k_values=vals[0], v_values=vals[1])
    assert got["K"] is vals[0] and got["V"] is vals[1]
    plain = _empty(B, kv, cap, d, bits, token_major)
    assert P.write_quantized(plain, *dev, lens=ints[0], new_lens=ints[1]) == {}
    after = [_bytes(t) for t in cache]
    assert all(np.array_equal(a, _bytes(t)) for a, t in zip(after, plain))
    for b in range(B):
        m = min(max(rows if new is None else new[b], 0), rows)
        n = m if lens is None else lens[b]
        took = [i for i in range(m) if 0 <= n - m + i < cap]
        for h in range(kv):
            for w in range(2):
                if not took:
                    assert all(np.array_equal(before[i][b, h], after[i][b, h]) for i in (w, 2 + w)) and bool((vals[w][b, h] == -77).all())
                    continue
                scales = [t[2 + w].reshape(B, kv, cap, -1) for t in (before, after)]
                codes, s = _check_rows(cache, (before[w][b, h], scales[0][b, h]), x[w][b, h, took], [n - m + i for i in took], bits, (after[w][b, h], scales[1][b, h]))
                want = torch.full((rows, d), -77.0, dtype=dtype)
                want[took] = torch.from_numpy(_values_of(codes, s, bits, d).astype(np.float32)).to(dtype)
                assert torch.equal(vals[w][b, h].cpu(), want)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d", [64, 128])
def test_rows_that_are_not_finite_or_tiny(dtype, bits, d):
    x = torch.ones(1, 1, 9, d)
    x[..., 1, 5], x[..., 2, d - 1], x[..., 3, 0] = math.nan, math.inf, -math.inf
    x[..., 4, :] = 0.0
    x[..., 5, :] = 2.0 ** -111
    x[..., 6, :] = 2.0 ** -110
    x[..., 7, ::2], x[..., 7, 1::2] = 2.0 ** -130, 2.0 ** -105
    x[..., 8, :] = 3.38e38
    x = x.to(dtype)
    cache = _empty(1, 1, 9, d, bits)
    before = [_bytes(t) for t in cache]
    got = P.write_quantized(cache, x.cuda(), x.cuda(), want_values=True)
    after = [_bytes(t) for t in cache]
    codes, scales = _check_rows(cache, (before[0][0, 0], before[2].reshape(9, -1)), x[0, 0], list(range(9)), bits, (after[0][0, 0], after[2].reshape(9, -1)))
    want = torch.from_numpy(_values_of(codes, scales, bits, d).astype(np.float32)).to(dtype)
    assert torch.equal(torch.isnan(got["K"][0, 0].cpu()), torch.isnan(want)) and torch.equal(torch.nan_to_num(got["K"][0, 0].cpu()), torch.nan_to_num(want))
    assert torch.isnan(want).any(-1).tolist() == [False, True, True, True] + [False] * 5
    assert bool((want[4:6] == 0).all()) and bool((want[6] != 0).all())
    assert torch.equal(torch.nan_to_num(P.read_quantized(cache, dtype=dtype)["V"][0, 0].cpu()), torch.nan_to_num(want))


def _held(gen, B, kv, cap, d, bits, token_major=False, fill=None):
    """A cache of any codes (the lowest among them) and scales of all bits, on the device."""
    cache = _empty(B, kv, cap, d, bits, token_major)
    for i in range(2):
        c = torch.randint(0, 256, cache[i].shape, generator=gen, dtype=torch.int32).to(torch.uint8)
        cache[i].copy_(c.view(torch.int8) if bits == 8 else c)
        s = torch.randn(cache[2 + i].shape, generator=gen).mul(0.4).exp() * (0.01 if bits == 8 else 0.2)
        cache[2 + i].copy_(s)
    return cache


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,kv,cap,first,rows,lens,token_major", [
    (1, 1, 1, 0, 1, None, False), (2, 3, 77, 0, 77, [77, 20], True), (3, 2, 130, 31, 65, [130, 40, 31], False), (2, 1, 90, 80, 10, [-5, 95], True),
])
def test_rows_read_back(dtype, bits, d, B, kv, cap, first, rows, lens, token_major):
    cache = _held(torch.Generator().manual_seed(cap + bits), B, kv, cap, d, bits, token_major)
    out = [torch.full((B, rows, kv, d), -77.0, dtype=dtype, device="cuda").transpose(1, 2) for _ in range(2)]
    n = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    got = P.read_quantized(cache, lens=n, first=first, rows=rows, k_out=out[0], v_out=out[1])
    for name, x in zip("KV", qref.values(cache)):
        want = x[:, :, first : first + rows].float().to(dtype)               # 8 and 4 bits times 24 and 8: rounded to fp32 at most once before
        for b in range(B):
            m = max(0, min(cap if lens is None else lens[b], cap) - first)
            want[b, :, m:] = -77.0
        assert torch.equal(got[name].cpu(), want)
    again = P.read_quantized(cache, dtype=dtype, first=first, rows=rows)
    assert again["K"].dtype is dtype and torch.equal(again["V"].float().cpu(), qref.values(cache)[1][:, :, first : first + rows].float().to(dtype).float())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("start,gap", [(1, 0), (0, 1), (1, 1), (1, 2)])
def test_rows_read_back_to_places_of_16_bytes(dtype, bits, d, start, gap):
    """Rows that begin on multiples of 16 bytes that are none of 32; what lies between them stays."""
    cache = _held(torch.Generator().manual_seed(d + bits + start), 2, 2, 37, d, bits)
    e = 16 // dtype.itemsize
    step = d + gap * e
    want = [x.float().to(dtype) for x in qref.values(cache)]
    w = [torch.full((start * e + 2 * 2 * 37 * step,), -77.0, dtype=dtype, device="cuda") for _ in range(2)]
    out = [torch.as_strided(x, (2, 2, 37, d), (2 * 37 * step, 37 * step, step, 1), start * e) for x in w]
    P.read_quantized(cache, k_out=out[0], v_out=out[1])
    for x, got, y in zip(w, out, want):
        assert torch.equal(got.cpu(), y)
        got.fill_(-77.0)
        assert bool((x == -77.0).all())


def _hold(t, want, tol, what):
    off = (t.double().cpu() - want).abs()
    worst = (off / tol.clamp_min(1e-300)).max().item() if off.numel() else 0.0
    assert bool((off <= tol).all()), "%s: %.3g of the bound" % (what, worst)


def _offset_tol(q, k, v_scale, d, L, QL, window=0, sinks=0, scale=0.0):
    """Codes are multiplied with an offset of 8 (128) that a second product takes away again: sixteen keys at a time, numbers of up to 16 (256)
    times weight and scale are added up in fp32, twice, 17 of them with the last bit cut off: 2 * 17 * 2^-24 * 16 < 2^-14.9 of the sum of weights times
    scales (16 times that for 8 bits), whatever the codes are."""
    eight = v_scale.dim() == 3
    s = v_scale.double().abs()
    s = s[..., None].expand(*s.shape, d) if eight else s[..., torch.from_numpy(qref.group(d))]
    return ref.attend(q, k, s, L, QL, window=window, sinks=sinks, scale=scale)[0] * 2.0 ** (-10.9 if eight else -14.9)


def _rounded_tol(q, k, v, L, QL, window, sinks, scale):
    """Scales of more than five bits: a bf16 call of many queries rounds the values to bf16 (half a step, 2^-8 of each) before it multiplies them.
    A logit is then off by 2^-8 sum |q_c k_c| scale: ex; the lse by ex, a weight by 2 ex of itself, a value by 2^-8 of itself.  (lse, out)"""
    B, hq, n_q, d = q.shape
    G, sc = hq // k.shape[1], scale or 1.0 / math.sqrt(d)
    ex = torch.zeros(B, hq, n_q, dtype=torch.float64)
    for b in range(B):
        t, j = torch.arange(QL[b])[:, None] + (L[b] - QL[b]), torch.arange(L[b])[None]
        sees = (j <= t) & ((j > t - window) | (j < sinks) if window else torch.ones(1, 1, dtype=torch.bool))
        for h in range(hq):
            x = 2.0 ** -8 * sc * (q[b, h, : QL[b]].double().abs() @ k[b, h // G, : L[b]].abs().T) * sees
            if x.numel():
                ex[b, h, : QL[b]] = x.amax(1)
    return ex, (2 * ex[..., None] + 2.0 ** -8) * ref.attend(q, k, v.abs(), L, QL, window=window, sinks=sinks, scale=scale)[0]


def _attended(B, kv, G, d, n_q, cap, bits, dtype, lens=None, q_lens=None, window=0, sinks=0, scale=0.0, token_major=False, flags=0, seed=0, spoil=True, size=1.0, five=False):
    gen = torch.Generator().manual_seed(seed)
    cache = _held(gen, B, kv, cap, d, bits, token_major)
    if five and bits == 4:
        for s in cache[2:]:                                          # as the library writes them
            s.copy_(torch.from_numpy(np.ldexp(np.rint(np.frexp(s.double().cpu().numpy())[0] * 32), np.frexp(s.double().cpu().numpy())[1] - 5)))
    q = torch.randn(B, n_q, kv * G, d, generator=gen).mul(size).to(dtype).transpose(1, 2)
    q = q if token_major else q.contiguous()
    L, QL = lens or [cap] * B, q_lens or [n_q] * B
    clean = P.QuantizedCache(*(t.cpu() for t in cache))
    if spoil:
        # what no query sees may hold anything
        for b in range(B):
            for t in cache[2:]:
                t[b, :, max(0, L[b]) :] = math.nan
            if window:
                lo = max(0, L[b] - QL[b] - window + 1)
                for t in cache[2:]:
                    t[b, :, min(sinks, lo) : lo] = math.inf
    dev = torch.empty_strided(q.size(), q.stride(), dtype=dtype, device="cuda").copy_(q)
    out = torch.full_like(dev, -77.0)
    lse = torch.full((B, kv * G, n_q), -77.0, device="cuda")
    ints = [None if t is None else torch.tensor(t, dtype=torch.int32, device="cuda") for t in (lens, q_lens)]
    got = P.attend_quantized(dev, cache, lens=ints[0], q_lens=ints[1], window=window, sinks=sinks, scale=scale, out=out, lse_out=lse, flags=flags, want_status=True)
    assert P.obf_last_device_status(got["workspace"]) == 0
    k, v = qref.values(clean)
    o, o_tol, l, l_tol, _, _ = ref.attend(q, k, v, L, QL, window=window, sinks=sinks, scale=scale)
    o_tol = o_tol + _offset_tol(q, k, clean.v_scale, d, L, QL, window, sinks, scale)
    if bits == 4 and dtype is BF16 and not five and not flags and G * n_q > 16:
        more = _rounded_tol(q, k, v, L, QL, window, sinks, scale)
        l_tol, o_tol = l_tol + more[0], o_tol + more[1]
    for b in range(B):
        assert bool((out[b, :, QL[b] :] == -77).all()) and bool((lse[b, :, QL[b] :] == -77).all())
        out[b, :, QL[b] :], lse[b, :, QL[b] :] = 0, 0
    none = torch.isneginf(l)
    assert torch.equal(torch.isneginf(lse.cpu()), none)
    _hold(torch.where(none.cuda(), 0.0, lse), torch.where(none, 0.0, l), torch.where(none, 0.0, l_tol), "lse")
    _hold(out, o, o_tol, "out")
    return got


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kw", [
    dict(B=1, kv=1, G=1, n_q=1, cap=1),
    dict(B=3, kv=2, G=4, n_q=1, cap=203, lens=[203, 1, 0]),
    dict(B=2, kv=2, G=8, n_q=1, cap=1500, lens=[1500, 700], token_major=True),
    dict(B=2, kv=1, G=7, n_q=2, cap=333, lens=[333, 1], q_lens=[2, 2]),
    dict(B=2, kv=2, G=3, n_q=5, cap=130, lens=[130, 64], q_lens=[5, 3], window=20, sinks=3),
    dict(B=1, kv=2, G=4, n_q=40, cap=300, window=1, sinks=0, token_major=True),
    dict(B=2, kv=1, G=6, n_q=33, cap=200, lens=[200, 16], q_lens=[33, 33], window=50, sinks=130),
    dict(B=1, kv=1, G=33, n_q=1, cap=600, scale=0.3),
    dict(B=2, kv=1, G=2, n_q=150, cap=150, lens=[150, 149], q_lens=[150, 149]),
    dict(B=40, kv=2, G=4, n_q=1, cap=700, lens=[700 - 17 * i for i in range(40)]),
    dict(B=1, kv=1, G=4, n_q=1, cap=9000, window=5000, sinks=4),
    dict(B=1, kv=2, G=5, n_q=1, cap=5001, size=12.0),
    dict(B=3, kv=2, G=2, n_q=2, cap=65, lens=[65, 0, 64], q_lens=[0, 2, 1], window=3),
])
def test_attention(dtype, bits, d, kw):
    _attended(d=d, bits=bits, dtype=dtype, seed=bits + d + kw["cap"], **kw)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kw", [
    dict(B=2, kv=2, G=4, n_q=40, cap=300, lens=[300, 41], q_lens=[40, 17], token_major=True),
    dict(B=1, kv=1, G=1, n_q=1000, cap=1000, window=100, sinks=5),
    dict(B=2, kv=1, G=6, n_q=70, cap=700, lens=[700, 0], q_lens=[70, 3], window=33, sinks=70),
    dict(B=3, kv=2, G=8, n_q=13, cap=515, lens=[515, 7, 13], q_lens=[13, 13, 1], window=200, sinks=1),
    dict(B=1, kv=1, G=128, n_q=3, cap=140, scale=0.3), dict(B=1, kv=1, G=100, n_q=1, cap=4097, window=4000),
    dict(B=1, kv=2, G=3, n_q=301, cap=301, size=15.0), dict(B=1, kv=1, G=129, n_q=1, cap=70),
    dict(B=3, kv=1, G=4, n_q=30, cap=90, lens=[90, 50, 0], q_lens=[0, 30, 0]), dict(B=2, kv=2, G=5, n_q=4, cap=450, lens=[450, 300], token_major=True), dict(B=1, kv=3, G=23, n_q=1, cap=1100, window=700, sinks=2), dict(B=2, kv=1, G=5, n_q=60, cap=2000, window=1, sinks=300),
])
@pytest.mark.parametrize("dtype,flags", [(BF16, 0), (BF16, binding.OBF_FLAG_GENERIC_PATH), (F32, 0)])
def test_attention_of_many_queries(bits, d, kw, dtype, flags):
    _attended(d=d, bits=bits, dtype=dtype, seed=bits + d + kw["cap"], flags=flags, five=True, **kw)


BIG = [
    # (channels, case): calls of enough rows and keys to read rows back first
    (128, dict(B=2, kv=2, G=8, n_q=200, cap=1000, lens=[1000, 333], q_lens=[200, 77], token_major=True)),
    (64, dict(B=1, kv=2, G=4, n_q=1050, cap=1050, window=1000, sinks=5)),
    (128, dict(B=2, kv=1, G=6, n_q=600, cap=1101, lens=[1101, 0], q_lens=[600, 3], window=801, sinks=70)),
    (64, dict(B=3, kv=1, G=8, n_q=300, cap=1115, lens=[1115, 7, 300], q_lens=[300, 13, 1], window=903, sinks=33)),
    (128, dict(B=1, kv=1, G=128, n_q=50, cap=1100, scale=0.3)), (128, dict(B=1, kv=2, G=3, n_q=1301, cap=1301, size=15.0)),
    (64, dict(B=2, kv=1, G=5, n_q=600, cap=1500, window=999, sinks=600)), (128, dict(B=1, kv=1, G=4, n_q=801, cap=4097, window=2050, sinks=17)),
]


@pytest.mark.gpu
@pytest.mark.parametrize("bits,five", [(4, True), (4, False), (8, True)])
@pytest.mark.parametrize("d,kw", BIG)
def test_attention_over_rows_read_back(bits, five, d, kw):
    _attended(d=d, bits=bits, dtype=BF16, seed=bits + d + kw["cap"], five=five, **kw)
    assert P.obf_last_launch_count() >= 2


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [4, 8])
def test_rows_read_back_hold_nothing_of_what_is_not_seen(bits):
    # the workspace is full of what is not a number, and so is the cache behind the window and the last key
    gen = torch.Generator().manual_seed(9)
    cache = _held(gen, 1, 2, 1400, 128, bits)
    q = torch.randn(1, 16, 900, 128, generator=gen).to(BF16).cuda()
    lens = torch.tensor([1303], dtype=torch.int32, device="cuda")
    kw = dict(lens=lens, window=301, sinks=3)
    want = P.attend_quantized(q, cache, **kw)["out"]
    lo = 1303 - 900 - 301 + 1
    for t in cache[2:]:
        t[:, :, 1303:] = math.nan
        t[:, :, 3:lo] = math.inf
    ws = P.attend_quantized_workspace(q, cache, window=301, sinks=3)
    ws.fill_(0xFF)
    assert torch.equal(P.attend_quantized(q, cache, workspace=ws, **kw)["out"], want)
    assert P.obf_last_launch_count() >= 2


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [4, 8])
def test_queries_of_any_size(bits):
    # rows scaled apart by powers of two give results scaled likewise: queries are brought to one size first
    gen = torch.Generator().manual_seed(3)
    cache = _held(gen, 1, 1, 100, 128, bits)
    q = torch.randn(1, 1, 6, 128, generator=gen).to(BF16).cuda()
    for e in (-126, -60, 0, 40, 100):
        s = 2.0 ** e
        for dtype in (BF16, F32):
            got = P.attend_quantized((q.to(dtype) * s), cache, scale=2.0 ** -3 / s if e <= 100 and e > -126 else 2.0 ** 100, want_lse=True)
            if e > -126:
                want = P.attend_quantized(q.to(dtype), cache, scale=2.0 ** -3, want_lse=True)
                assert torch.equal(got["out"], want["out"]) and torch.equal(got["lse"], want["lse"])
            assert bool(torch.isfinite(got["lse"]).all())
    zero = P.attend_quantized(torch.zeros_like(q), cache, want_lse=True)
    seen = torch.arange(95, 101, dtype=torch.float64)
    assert torch.allclose(zero["lse"][0, 0].double().cpu(), seen.log(), rtol=2 ** -20, atol=0)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n_q", [1, 3, 900])
def test_values_of_any_size(bits, dtype, n_q):
    # scales larger and smaller by powers of two give outputs likewise, and another sign of them the other sign
    gen = torch.Generator().manual_seed(4)
    cache = _held(gen, 1, 2, 900, 128, bits)
    q = torch.randn(1, 8, n_q, 128, generator=gen).to(dtype).cuda()
    want = P.attend_quantized(q, cache)["out"]
    for f in (2.0 ** -50, 2.0 ** 40, -1.0):
        got = P.attend_quantized(q, cache._replace(v_scale=cache.v_scale * f))["out"]
        assert torch.equal(got, want * f)


@pytest.mark.gpu
def test_positions_beyond_any_number_are_not_written():
    cache = _empty(4, 1, 20, 64, 4)
    before = [_bytes(t) for t in cache]
    x = torch.ones(4, 1, 700, 64, dtype=BF16, device="cuda")
    n = torch.tensor([-(1 << 31), (1 << 31) - 1, 1 << 20, -1], dtype=torch.int32, device="cuda")
    P.write_quantized(cache, x, x, lens=n)
    assert all(np.array_equal(a, _bytes(t)) for a, t in zip(before, cache))


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("n_q", [1, 12, 50, 800])
def test_scales_that_are_not_numbers_are_seen(bits, n_q):
    gen = torch.Generator().manual_seed(5)
    cap = max(100, n_q)
    cache = _held(gen, 2, 2, cap, 64, bits)
    q = torch.randn(2, 8, n_q, 64, generator=gen).to(BF16).cuda()
    want = P.attend_quantized(q, cache)["out"]
    cache.v_scale[0, 1, cap - n_q // 2 - 1] = math.nan
    got = P.attend_quantized(q, cache)["out"]
    assert bool(torch.isnan(got[0, 4:, n_q - n_q // 2 - 1 :]).any(-1).all()) and torch.equal(got[1], want[1]) and torch.equal(got[0, :4], want[0, :4])


@pytest.mark.gpu
def test_lengths_out_of_range_are_clamped_and_told():
    gen = torch.Generator().manual_seed(6)
    cache = _held(gen, 3, 1, 60, 64, 4)
    q = torch.randn(3, 2, 4, 64, generator=gen).to(BF16).cuda()

    def call(lens, q_lens):
        n, m = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (lens, q_lens))
        return P.attend_quantized(q, cache, lens=n, q_lens=m, want_status=True, want_lse=True)
    bad, good = call([61, -1, 60], [4, 4, 9]), call([60, 0, 60], [4, 4, 4])
    assert P.obf_last_device_status(bad["workspace"]) == binding.OBF_DEV_INTERNAL and P.obf_last_device_status(good["workspace"]) == 0
    assert torch.equal(bad["out"], good["out"]) and torch.equal(bad["lse"], good["lse"])


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [4, 8])
def test_a_cache_beyond_32_bits(bits):
    # heads and sequences 4 GB apart: offsets in bytes pass 2^32
    gen = torch.Generator().manual_seed(7)
    small = _held(gen, 2, 2, 50, 128, bits)
    far = 1 << 32
    wide = torch.zeros(3 * far + (1 << 20), dtype=torch.uint8, device="cuda")
    big = []
    for i, t in enumerate(small):
        w = wide.view(t.dtype) if i < 2 else wide[i << 14 :].view(t.dtype)
        step = far // t.element_size()
        st = (2 * step, step, *t.stride()[2:])
        v = torch.as_strided(w, t.size(), st, storage_offset=(i << 16) // t.element_size())
        v.copy_(t)
        big.append(v)
    big = P.QuantizedCache(*big)
    q = torch.randn(2, 4, 3, 128, generator=gen).to(BF16).cuda()
    assert torch.equal(P.attend_quantized(q, big)["out"], P.attend_quantized(q, small)["out"])
    assert all(torch.equal(P.read_quantized(big)[n], P.read_quantized(small)[n]) for n in "KV")
    x = torch.randn(2, 2, 50, 128, generator=gen).to(BF16).cuda()
    P.write_quantized(big, x, -x)
    P.write_quantized(small, x, -x)
    assert all(torch.equal(a, b) for a, b in zip(big, small))


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [4, 8])
def test_captured_steps_on_another_stream_follow_the_lengths(bits):
    gen = torch.Generator().manual_seed(8)
    B, kv, G, d, cap = 3, 2, 4, 128, 80
    cache = _held(gen, B, kv, cap, d, bits)
    lens = torch.tensor([40, 1, 77], dtype=torch.int32, device="cuda")
    x = [torch.randn(B, kv, 1, d, generator=gen).to(BF16).cuda() for _ in range(2)]
    q = torch.randn(B, kv * G, 1, d, generator=gen).to(BF16).cuda()
    out = torch.zeros_like(q)
    ws = P.attend_quantized_workspace(q, cache)

    def step(c, o, n, stream=None):
        P.write_quantized(c, *x, lens=n, stream=stream)
        return P.attend_quantized(q, c, lens=n, out=o, workspace=ws, stream=stream)["out"]
    warm = P.QuantizedCache(*(t.clone() for t in cache))
    step(warm, torch.zeros_like(q), lens)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(cache, out, lens)
    want = P.QuantizedCache(*(t.clone() for t in cache))
    for _ in range(3):
        lens += 1
        for t in x + [q]:
            t.mul_(-0.75)
        graph.replay()
        plain = step(want, torch.zeros_like(q), lens)
        torch.cuda.synchronize()
        assert torch.equal(out, plain) and all(torch.equal(a, b) for a, b in zip(cache, want))
    # the same on a stream of its own, named by the caller
    side.wait_stream(torch.cuda.current_stream())
    again = step(want, None, lens, stream=side)
    side.synchronize()
    assert torch.equal(again, plain)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d,B,kv,G,n_q,cap", [(128, 2, 2, 4, 257, 1301), (64, 3, 1, 2, 700, 1500), (128, 2, 2, 4, 6, 1301), (64, 5, 4, 4, 1, 4099)])
def test_calls_at_the_same_time_and_from_graphs_keep_apart(bits, d, B, kv, G, n_q, cap):
    """Two calls on two streams, each with its workspace, and two captured ones that are replayed side by side, over rows read back and over codes: what each
    gives is what it gives alone."""
    gen = torch.Generator().manual_seed(n_q + bits)
    caches = [_held(gen, B, kv, cap, d, bits) for _ in range(2)]
    q = [torch.randn(B, kv * G, n_q, d, generator=gen).to(BF16).cuda() for _ in range(2)]
    lens = [torch.tensor([cap - 7 * i * (b + 1) for b in range(B)], dtype=torch.int32, device="cuda") for i in range(2)]
    ws = [P.attend_quantized_workspace(q[0], caches[0], window=600, sinks=3) for _ in range(2)]
    out = [torch.empty_like(x) for x in q]
    alone = [P.attend_quantized(q[i], caches[i], lens=lens[i], window=600, sinks=3)["out"] for i in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    graphs = []
    for i in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i], stream=streams[i]):
            P.attend_quantized(q[i], caches[i], lens=lens[i], window=600, sinks=3, out=out[i], workspace=ws[i])
    for replayed in (False, True):
        for _ in range(5):
            for x in out:
                x.fill_(-77.0)
            torch.cuda.synchronize()
            for i in range(2):
                with torch.cuda.stream(streams[i]):
                    if replayed:
                        graphs[i].replay()
                    else:
                        P.attend_quantized(q[i], caches[i], lens=lens[i], window=600, sinks=3, out=out[i], workspace=ws[i])
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, alone))


@pytest.mark.gpu
def test_from_the_relay_s_int8_copy_to_a_cache_that_goes_on():
    # compress with an int8 copy; the next agent attends over the copy as it is; its rows go on in a cache with room, in 8 and 4 bits, that grows
    # and is read back, evicted from and compressed again
    from paper_2604_13349_b200 import synth
    w = synth.workload("c2")
    a = synth.gen_cache(w, 0)

    def dev(x):
        return torch.from_numpy(x.view(np.int16)).cuda().view(BF16)
    params = P.make_params(w.layers, w.kv_heads, w.q_heads, 128, w.n_obs, 1, P.OBF_BF16)
    relay = P.compress_caches(params, [{"K": dev(a["K"]), "V": dev(a["V"]), "Q": dev(a["Q"]), "budget": 100}], want_int8=True)[0]
    copy = P.QuantizedCache(relay["K_q8"], relay["V_q8"], relay["K_scale"], relay["V_scale"])
    back = P.read_quantized(copy, dtype=F32)
    q = dev(a["Q"])[:, :, :3].contiguous()
    k, v = qref.values(copy)
    got = P.attend_quantized(q, copy, want_lse=True)
    L, QL = [100] * w.layers, [3] * w.layers
    o, o_tol, l, l_tol, _, _ = ref.attend(q.cpu(), k, v, L, QL)
    o_tol = o_tol + _offset_tol(q.cpu(), k, copy.v_scale.cpu(), 128, L, QL)
    _hold(got["out"], o, o_tol, "out")
    _hold(got["lse"], l, l_tol, "lse")
    for bits in (8, 4):
        cache = P.quantized_cache(w.layers, w.kv_heads, 140, 128, bits)
        held = P.write_quantized(cache, relay["K_out"], relay["V_out"], want_values=True)
        if bits == 8:
            assert torch.equal(cache.k[:, :, :100], copy.k) and torch.equal(cache.v_scale[:, :, :100], copy.v_scale)
            assert torch.equal(held["K"].float(), back["K"].to(BF16).float())
        lens = torch.full((w.layers,), 100, dtype=torch.int32, device="cuda")
        for _ in range(5):
            lens += 1
            x = torch.randn(w.layers, w.kv_heads, 1, 128, device="cuda").to(BF16)
            P.write_quantized(cache, x, x, lens=lens)
            step = P.attend_quantized(q[:, :, :1], cache, lens=lens)
        rows = P.read_quantized(cache, lens=lens)
        plain = P.attend(q[:, :, :1], rows["K"], rows["V"], lens=lens)["out"]
        # 4 bits: the same numbers (two calls, each within the bound of 2^-8 weights and outputs); 8 bits: rows rounded to bf16 on their way
        assert (step["out"].float() - plain.float()).abs().max() <= (4 if bits == 4 else 8) * 2.0 ** -8 * rows["V"].abs().max().float()
        kept = P.evict_by_mass(rows["K"], rows["V"], torch.rand(w.layers, w.kv_heads, 140, device="cuda"), 64, lens=lens)
        small = P.quantized_cache(w.layers, w.kv_heads, 64, 128, bits)
        again = P.write_quantized(small, kept["K_out"], kept["V_out"], want_values=True)
        if bits == 4:
            # values of the cache, held again: the largest of a group may come out as another scale, the others within half a step of it
            assert bool(torch.isfinite(again["K"]).all())
        assert P.read_quantized(small)["K"].shape == (w.layers, w.kv_heads, 64, 128)
