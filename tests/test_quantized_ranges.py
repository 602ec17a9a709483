"""A relayed cache held in 8 or 4 bits at the ends of its ranges: sizes of scales and logits, and calls that read rows back."""
import math

import pytest
import torch

import paper_2604_13349_b200 as P
from paper_2604_13349_b200 import binding
from tests import _attend_ref as ref
from tests import _quant_ref as qref

BF16, F32 = torch.bfloat16, torch.float32

# rows of queries per KV head that reach every kernel and tile: (G, n_q)
SHAPES = [(1, 1), (4, 1), (8, 1), (4, 4), (8, 3), (4, 8), (8, 400)]


def _cache(B, kv, cap, d, bits, k_codes, v_codes, k_scale, v_scale):
    """A cache with the given codes [B, kv, cap, d] (whole numbers) and scales, one or one for each row."""
    def pack(c):
        c = c.expand(B, kv, cap, d).contiguous()
        if bits == 8:
            return c.to(torch.int8).cuda()
        u = (c + 8).to(torch.uint8)
        return (u[..., 0::2] | (u[..., 1::2] << 4)).cuda()

    def scale(s):
        s = torch.as_tensor(s, dtype=F32).expand(B, kv, cap)
        return s.contiguous().cuda() if bits == 8 else s[..., None].expand(B, kv, cap, d // 32).to(BF16).contiguous().cuda()
    return P.QuantizedCache(pack(k_codes), pack(v_codes), scale(k_scale), scale(v_scale))


def _top(bits):
    return 127 if bits == 8 else 7


def _hold(got, want, tol):
    off = (got.double().cpu() - want).abs()
    assert bool((off <= tol).all()), "%.3g of the bound" % (off / tol).nan_to_num(math.inf).max().item()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d", [(BF16, 128), (BF16, 64), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("G,n_q", SHAPES)
@pytest.mark.parametrize("same", [True, False])
def test_values_at_the_ends_of_their_range(dtype, d, bits, G, n_q, same):
    # the largest and the smallest scales of values, thousands of keys of equal weight: the largest codes, and any
    gen = torch.Generator().manual_seed(bits + d + n_q)
    cap, t = 3000, _top(bits)
    codes = torch.full((1, 2, cap, d), t) if same else torch.randint(-t, t + 1, (1, 2, cap, d), generator=gen)
    q = torch.zeros(1, 2 * G, n_q, d, dtype=dtype)
    for size in (44 if dtype is BF16 else 100, -60):
        cache = _cache(1, 2, cap, d, bits, codes, codes, 1.0, 2.0 ** size)
        got = P.attend_quantized(q.cuda(), cache, want_lse=True)
        _, v = qref.values(cache)
        out, tol, lse, lse_tol, _, _ = ref.attend(q, torch.zeros_like(v), v, [cap], [n_q])
        _hold(got["out"], out, tol)
        _hold(got["lse"], lse, lse_tol)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype,flags", [(F32, 0), (BF16, 0), (BF16, binding.OBF_FLAG_GENERIC_PATH)])
def test_the_largest_values_of_many_keys_that_barely_leave_their_reference(d, dtype, flags):
    # all keys but the first weigh 2^7.9 times as much, too little for their reference to be raised
    cap, G, n_q, size = 1 << 16, 8, 1 << 13, 2.0 ** (100 if dtype is F32 else 44)
    k = torch.zeros(1, 1, cap, d)
    k[:, :, 128:, 0] = 100
    cache = _cache(1, 1, cap, d, 8, k, torch.full((1, 1, 1, d), 127), 1.0, size)
    q = torch.zeros(1, G, n_q, d, dtype=dtype)
    q[..., 0] = 1.0
    for rows in (n_q, 1):
        out = P.attend_quantized(q[:, :, :rows].contiguous().cuda(), cache, scale=7.9 * math.log(2) / 100, flags=flags)["out"].float()
        # an average of equal numbers: 2^16 sums in fp32, a division; a bf16 weight and output
        assert bool(((out / size - 127).abs() <= 127 * (2.0 ** 16 * 2.0 ** -24 + 2.0 ** -20 + (2 * 2.0 ** -8 if dtype is BF16 else 0.0))).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d", [(BF16, 128), (BF16, 64), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("G,n_q", SHAPES)
@pytest.mark.parametrize("size", [24, 34, 60])
def test_logits_of_any_size(dtype, d, bits, G, n_q, size):
    # keys with a logit of about 2^size among others whose is zero, all of one value: the output is that value, whatever its scale.  (Not an average of several: where
    # keys are cut into parts, those are weighed by their fp32 lse, whose last bit is a power of two in the weights from logits of 2^24 on.)
    gen = torch.Generator().manual_seed(bits + d + n_q + size)
    cap, t = 3000, _top(bits)
    hot = torch.rand(1, 2, cap, generator=gen) < 0.02
    hot[..., cap - n_q] = True                                       # every query sees one
    k = torch.zeros(1, 2, cap, d)
    k[..., 0] = hot * t
    value = torch.randint(-t, t + 1, (1, 2, 1, d), generator=gen)
    v = torch.where(hot[..., None], value, torch.randint(-t, t + 1, (1, 2, cap, d), generator=gen))
    q = torch.zeros(1, 2 * G, n_q, d, dtype=dtype)
    q[..., 0] = 8.0
    for e in (0, -14, -24, -44):
        step = 2.0 ** (size - 3 - t.bit_length())                    # of the keys
        got = P.attend_quantized(q.cuda(), _cache(1, 2, cap, d, bits, k, v, step, 2.0 ** e), scale=1.0, want_lse=True)
        want = value.double().repeat_interleave(G, 1).expand(1, 2 * G, n_q, d) * 2.0 ** e
        # a sum of at most 3000 numbers, a bf16 weight and the output's rounding
        _hold(got["out"], want, (cap * 2.0 ** -24 + 2.0 ** -20 + 2 * ref.STEP[dtype]) * want.abs())
        # the logit: exact products, scaled with three roundings; the number of keys; the sum's rounding
        n = (torch.tril(torch.ones(n_q, cap, dtype=torch.float64), cap - n_q) * hot[0, :, None]).sum(-1)
        x = 8.0 * t * step
        _hold(got["lse"].reshape(2, G, n_q), x + n.log()[:, None], torch.full((2, 1, n_q), 2.0 ** -21 * x))


def _held(gen, kv, cap, d, bits, k_size):
    t = _top(bits)
    codes = [torch.randint(-t, t + 1, (1, kv, cap, d), generator=gen) for _ in range(2)]
    scale = [torch.randint(16, 32, (1, kv, cap), generator=gen) * 2.0 ** -4 * x for x in (k_size, 2.0 ** -4)]
    return _cache(1, kv, cap, d, bits, *codes, *scale)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d", [(BF16, 128), (BF16, 64), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("G,n_q", SHAPES)
def test_queries_of_any_size_over_keys_of_any_size(dtype, d, bits, G, n_q):
    # powers of two moved between the keys' scales and the queries change nothing; and queries of up to 2^112 against 64 bits
    gen = torch.Generator().manual_seed(bits + d + n_q)
    cap = 3000
    cache = _held(gen, 2, cap, d, bits, 2.0 ** -3 / _top(bits))
    q = torch.randn(1, 2 * G, n_q, d, generator=gen).clamp(-4, 4).to(dtype)
    want = P.attend_quantized(q.cuda(), cache, want_lse=True)
    for e in (100, 30, -60, -97):
        got = P.attend_quantized((q * 2.0 ** e).cuda(), cache._replace(k_scale=cache.k_scale * 2.0 ** -e), want_lse=True)
        assert torch.equal(got["out"], want["out"]) and torch.equal(got["lse"], want["lse"])
    k, v = qref.values(cache)
    out, tol, lse, lse_tol, _, _ = ref.attend(q, k, v, [cap], [n_q])
    got = P.attend_quantized((q * 2.0 ** 110).cuda(), cache._replace(k_scale=cache.k_scale * 2.0 ** -110), want_lse=True)
    _hold(got["out"], out, tol)
    _hold(got["lse"], lse, lse_tol)
