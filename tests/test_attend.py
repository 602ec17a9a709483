"""Operators on a relayed cache: attention with a window and sinks, over a shared prefix, masses, eviction by mass."""
import ctypes
import math

import pytest
import torch

import paper_2604_13349_b200 as P
from paper_2604_13349_b200 import binding, build
from tests import _attend_ref as ref

GENERIC = binding.OBF_FLAG_GENERIC_PATH
BF16, F32 = torch.bfloat16, torch.float32


# ---- refusals: decided on the host, nothing reaches a device ------------------------------------------------------
@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


def _args(**kw):
    d = dict(batch=2, kv_heads=2, q_heads=8, head_dim=64, n_q=3, capacity=100, window=0, sinks=0, dtype=P.OBF_BF16, scale=0.0, decay=1.0, flags=0,
             q=0x1000, k=0x1000, v=0x1000, out=0x1000)
    d.update(kw)
    a = P.ObfAttend(**{n: x for n, x in d.items() if not n.endswith("stride")})
    D = a.head_dim
    strides = dict(q_stride=(a.q_heads * a.n_q * D, a.n_q * D, D), out_stride=(a.q_heads * a.n_q * D, a.n_q * D, D),
                   k_stride=(a.kv_heads * a.capacity * D, a.capacity * D, D), v_stride=(a.kv_heads * a.capacity * D, a.capacity * D, D))
    strides.update({n: x for n, x in d.items() if n.endswith("stride")})
    for n, x in strides.items():
        setattr(a, n, (ctypes.c_int64 * 3)(*x))
    return a


def _prefix(rows=50, D=64, k=0x1000, **kw):
    x = P.ObfPrefix(k, 0x1000, (ctypes.c_int64 * 2)(rows * D, D), (ctypes.c_int64 * 2)(rows * D, D), rows)
    for n, y in kw.items():
        setattr(x, n, y)
    return x


INVALID, UNSUPPORTED, WORKSPACE = binding.OBF_ERR_INVALID_ARG, binding.OBF_ERR_UNSUPPORTED, binding.OBF_ERR_WORKSPACE


@pytest.mark.parametrize("kw,code", [
    (dict(batch=0), INVALID), (dict(kv_heads=0), INVALID), (dict(q_heads=7), INVALID), (dict(q_heads=0), INVALID), (dict(n_q=0), INVALID),
    (dict(n_q=(1 << 20) + 1), INVALID), (dict(capacity=0), INVALID), (dict(capacity=(1 << 20) + 1), INVALID), (dict(window=-1), INVALID),
    (dict(sinks=-1), INVALID), (dict(scale=-0.5), INVALID), (dict(scale=math.nan), INVALID), (dict(scale=math.inf), INVALID),
    (dict(decay=-1.0), INVALID), (dict(decay=math.nan), INVALID), (dict(flags=2), INVALID), (dict(head_dim=96), UNSUPPORTED),
    (dict(dtype=5), UNSUPPORTED), (dict(mass_in=0x1000), INVALID), (dict(mass_out=0x1000, n_q=17), UNSUPPORTED),
    (dict(batch=1 << 20, n_q=1 << 10), UNSUPPORTED),
])
def test_attend_refuses_bad_shapes(lib, kw, code):
    with pytest.raises(P.ObfError) as e:
        P.obf_attend_workspace_bytes(_args(**kw))
    assert e.value.code == code
    assert lib.obf_attend(ctypes.byref(_args(**kw)), 0x100, 1 << 50, None) == code
    assert lib.obf_last_launch_count() == 0


@pytest.mark.parametrize("kw", [
    dict(q=0), dict(k=0), dict(v=0), dict(out=0), dict(q=0x1008), dict(k=0x1002), dict(v=0x1004), dict(out=0x1008), dict(lens=0x1002), dict(q_lens=0x1001),
    dict(lse_out=0x1002), dict(mass_out=0x1002), dict(q_stride=(1536, 192, 63)), dict(k_stride=(12800, 6400, 68)), dict(v_stride=(12800, -6400, 64)),
    dict(out_stride=(1536, 0, 64)), dict(k_stride=(1 << 39, 6400, 64)),
])
def test_attend_refuses_bad_pointers_and_strides(lib, kw):
    assert lib.obf_attend(ctypes.byref(_args(**kw)), 0x100, 1 << 50, None) == INVALID
    assert lib.obf_last_launch_count() == 0


def test_a_stride_that_is_never_stepped_over_may_be_anything():
    a = _args(batch=1, n_q=1, q_stride=(0, 64, 3), out_stride=(5, 64, 0))
    need = P.obf_attend_workspace_bytes(a)
    assert binding.load().obf_attend(ctypes.byref(a), 0x100, need - 1, None) == WORKSPACE        # past the checks of strides


def test_attend_refuses_a_small_or_misaligned_workspace(lib):
    a = _args()
    need = P.obf_attend_workspace_bytes(a)
    assert need >= 256 and need % 256 == 0
    for ws, n in ((None, need), (0x110, need), (0x100, need - 1)):
        assert lib.obf_attend(ctypes.byref(a), ws, n, None) == WORKSPACE
    assert P.obf_attend_workspace_bytes(_args(mass_out=0x1000)) > need
    x = _prefix()
    need = P.obf_attend_workspace_bytes(a, x)
    assert lib.obf_attend_shared(ctypes.byref(a), ctypes.byref(x), 0x100, need - 1, None) == WORKSPACE


@pytest.mark.parametrize("kw,px", [
    (dict(window=5), {}), (dict(sinks=1), {}), (dict(mass_out=0x1000), {}), (dict(), dict(rows=0)), (dict(), dict(rows=(1 << 20) + 1)),
    (dict(), dict(k=0)), (dict(), dict(v=0x1008)), (dict(), dict(k_stride=(ctypes.c_int64 * 2)(3200, 60))),
])
def test_attend_shared_refuses(lib, kw, px):
    rows = px.pop("rows", 50)
    a, x = _args(**kw), _prefix(**px)
    x.rows = rows
    assert lib.obf_attend_shared(ctypes.byref(a), ctypes.byref(x), 0x100, 1 << 50, None) == INVALID
    assert lib.obf_attend_shared(ctypes.byref(_args()), None, 0x100, 1 << 50, None) == INVALID


def _evict_args(**kw):
    d = dict(batch=2, kv_heads=2, head_dim=64, capacity=100, dtype=P.OBF_BF16, keep=10, sinks=2, recent=3, k=0x1000, v=0x1000, k_out=0x1000, v_out=0x1000,
             mass=0x1000, idx_out=0x1000, mass_out_rows=10)
    strides = dict(k_stride=(12800, 6400, 64), v_stride=(12800, 6400, 64), k_out_stride=(1280, 640, 64), v_out_stride=(1280, 640, 64))
    for n, x in kw.items():
        (strides if n in strides else d)[n] = x
    a = P.ObfEvict(**d)
    for n, x in strides.items():
        setattr(a, n, (ctypes.c_int64 * 3)(*x))
    return a


@pytest.mark.parametrize("kw,code", [
    (dict(batch=0), INVALID), (dict(kv_heads=0), INVALID), (dict(capacity=0), INVALID), (dict(keep=0), INVALID), (dict(keep=4), INVALID),
    (dict(sinks=-1), INVALID), (dict(recent=-1), INVALID), (dict(sinks=(1 << 31) - 1, recent=(1 << 31) - 1), INVALID), (dict(head_dim=80), UNSUPPORTED),
    (dict(dtype=3), UNSUPPORTED), (dict(k=0), INVALID), (dict(mass=0), INVALID), (dict(v_out=0x1008), INVALID), (dict(lens=0x1001), INVALID),
    (dict(idx_out=0x1002), INVALID), (dict(idx_out=0), INVALID), (dict(mass_out=0x1000, mass_out_rows=9), INVALID), (dict(k_stride=(12800, 6400, 65)), INVALID),
    (dict(v_out_stride=(1280, 0, 64)), INVALID), (dict(batch=1 << 20, kv_heads=32), UNSUPPORTED),
])
def test_evict_by_mass_refuses(lib, kw, code):
    assert lib.obf_evict_by_mass(ctypes.byref(_evict_args(**kw)), None) == code
    assert lib.obf_last_launch_count() == 0
    assert lib.obf_evict_by_mass(None, None) == INVALID


def test_struct_sizes_match_the_header():
    assert (ctypes.sizeof(binding.ObfAttend), ctypes.sizeof(binding.ObfPrefix), ctypes.sizeof(binding.ObfEvict)) == (216, 56, 208)


def test_a_workspace_for_any_window_and_for_no_other_type():
    q, k = torch.zeros(1, 4, 8, 64, dtype=BF16), torch.zeros(1, 2, 100, 64, dtype=BF16)
    assert P.attend_workspace(q, k, window=1 << 40, sinks=1 << 33).numel() >= 256
    with pytest.raises(P.ObfError):
        P.attend_workspace(q.half(), k.half())


def test_python_wrappers_refuse_host_tensors():
    with pytest.raises(ValueError):
        P.attend(torch.zeros(1, 4, 1, 64), torch.zeros(1, 2, 8, 64), torch.zeros(1, 2, 8, 64))
    with pytest.raises(ValueError):
        P.evict_by_mass(torch.zeros(1, 2, 8, 64), torch.zeros(1, 2, 8, 64), torch.zeros(1, 2, 8), 4)


# ---- on the device --------------------------------------------------------------------------------------------------
SENTINEL = -77.0


def _data(gen, B, kv, G, d, n_q, cap, dtype):
    q = torch.randn(B, kv * G, n_q, d, generator=gen).to(dtype)
    k = torch.randn(B, kv, cap, d, generator=gen).to(dtype)
    v = (torch.randn(B, kv, cap, d, generator=gen) + 0.5).to(dtype)
    return q, k, v


def _check(got, want, tol, what):
    got = got.double().cpu()
    assert torch.equal(torch.isinf(got), torch.isinf(want)), what
    fine = ~torch.isinf(want)
    assert torch.equal(got[~fine], want[~fine]), what
    off = torch.where(fine, got - want, 0.0).abs()
    bad = ~(off <= tol)
    assert not bad.any(), "%s: %d values off, worst %.3g against %.3g" % (what, int(bad.sum()), float(off[bad].max()), float(tol[bad][off[bad].argmax()]))


def _spoil_unseen(k, v, lens, q_lens, window, sinks):
    """NaN and infinities wherever no query of the sequence looks."""
    cap = k.shape[2]
    for b, (n, ql) in enumerate(zip(lens, q_lens)):
        j = torch.arange(cap)
        seen = torch.zeros(cap, dtype=torch.bool)
        for i in range(ql):
            t = n - ql + i
            seen |= (j <= t) & (j < n) & ((j > t - window) | (j < sinks) if window else torch.ones(cap, dtype=torch.bool))
        k[b, :, ~seen] = math.nan
        v[b, :, ~seen] = math.inf
        v[b, :, ~seen, 1] = math.nan


def _attend_case(B, kv, G, d, n_q, cap, lens, q_lens, dtype, window=0, sinks=0, scale=0.0, mass=False, decay=1.0, prefix_rows=0, flags=0, seed=0,
                 token_major=False):
    gen = torch.Generator().manual_seed(seed)
    q, k, v = _data(gen, B, kv, G, d, n_q, cap, dtype)
    px = None
    if prefix_rows:
        px = (torch.randn(kv, prefix_rows, d, generator=gen).to(dtype), torch.randn(kv, prefix_rows, d, generator=gen).to(dtype))
    mass_in = torch.rand(B, kv, cap, generator=gen) if mass else None
    want = ref.attend(q, k, v, lens, q_lens, window, sinks, scale, px, mass_in, decay, mass)
    _spoil_unseen(k, v, lens, q_lens, window, sinks)
    dev = lambda x: x.cuda()                                                       # noqa: E731
    for b in range(B):
        q[b, :, q_lens[b]:] = math.nan
    if token_major:
        qd = dev(q.transpose(1, 2).contiguous()).transpose(1, 2)
        out = torch.full((B, n_q, kv * G, d), SENTINEL, dtype=dtype, device="cuda").transpose(1, 2)
    else:
        qd, out = dev(q), torch.full((B, kv * G, n_q, d), SENTINEL, dtype=dtype, device="cuda")
    lse = torch.full((B, kv * G, n_q), SENTINEL, device="cuda")
    ln, ql = torch.tensor(lens, dtype=torch.int32, device="cuda"), torch.tensor(q_lens, dtype=torch.int32, device="cuda")
    ws = P.attend_workspace(qd, dev(k), window=window, sinks=sinks, mass=mass, prefix_rows=prefix_rows, flags=flags)
    if prefix_rows:
        P.attend_shared(qd, dev(px[0]), dev(px[1]), dev(k), dev(v), lens=ln, q_lens=ql, scale=scale, out=out, lse_out=lse, flags=flags, workspace=ws)
    else:
        m_out = torch.full((B, kv, cap), SENTINEL, device="cuda") if mass else None
        P.attend(qd, dev(k), dev(v), lens=ln, q_lens=ql, workspace=ws, window=window, sinks=sinks, scale=scale, out=out, lse_out=lse,
                     mass_in=dev(mass_in) if mass else None, mass_out=m_out, decay=decay, flags=flags)
    assert P.obf_last_device_status(ws) == 0
    for b in range(B):
        assert (out[b, :, q_lens[b]:] == SENTINEL).all() and (lse[b, :, q_lens[b]:] == SENTINEL).all(), "written behind the queries"
        out[b, :, q_lens[b]:] = 0
        lse[b, :, q_lens[b]:] = 0
        if mass:
            assert (m_out[b, :, lens[b]:] == SENTINEL).all(), "masses written behind the keys"
            m_out[b, :, lens[b]:] = 0
    _check(out, want[0], want[1], "out")
    _check(lse, want[2], want[3], "lse")
    if mass:
        _check(m_out, want[4], want[5], "mass")


PATHS = [pytest.param(BF16, 0, id="bf16"), pytest.param(BF16, GENERIC, id="bf16-generic"), pytest.param(F32, 0, id="f32")]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,flags", PATHS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n_q,cap,lens,window,sinks", [
    (1, 1, 1, [1, 0], 0, 0),                  # one key, and none
    (4, 1, 64, [64, 63], 0, 0),
    (4, 1, 700, [700, 513], 0, 0),
    (4, 1, 700, [700, 3], 100, 4),            # decoding with a window; a sequence shorter than its sinks
    (4, 1, 300, [300, 129], 1, 0),            # the query's own key alone
    (3, 1, 1300, [1300, 1025], 1000, 77),
    (8, 2, 257, [257, 255], 50, 51),
    (7, 5, 400, [399, 5], 16, 1),
    (16, 1, 130, [130, 17], 0, 0),
    (40, 1, 130, [130, 17], 90, 2),           # more heads in a group than a tile of 16 rows holds
])
def test_attend_few_queries(dtype, flags, d, G, n_q, cap, lens, window, sinks):
    q_lens = [min(n_q, n) for n in lens]
    _attend_case(2, 2, G, d, n_q, cap, lens, q_lens, dtype, window, sinks, flags=flags, mass=n_q * G <= 64, decay=0.75, seed=cap)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,flags", PATHS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n_q,cap,lens,q_lens,window,sinks", [
    (1, 300, 300, [300, 257], [300, 257], 0, 0),              # whole prompts, ragged
    (4, 200, 200, [200, 1], [200, 1], 0, 0),
    (2, 513, 513, [513, 129], [513, 129], 128, 4),            # window of a tile
    (1, 400, 400, [400, 399], [400, 399], 127, 130),          # more sinks than the window
    (3, 150, 400, [400, 151], [150, 149], 33, 2),             # a chunk of queries at the end of a longer cache; a group that divides no tile
    (5, 64, 1500, [1500, 700], [64, 3], 0, 0),                # few rows over many keys
    (4, 70, 64, [64, 0], [70, 5], 20, 3),                     # more queries than keys: rows that see nothing
    (8, 40, 300, [300, 40], [40, 0], 7, 0),                   # a sequence without queries
    (130, 2, 90, [90, 61], [2, 1], 0, 0),                     # a group larger than a tile of rows
    (1, 129, 385, [385, 384], [129, 128], 256, 17),
])
def test_attend_many_queries(dtype, flags, d, G, n_q, cap, lens, q_lens, window, sinks):
    _attend_case(2, 1 if G > 64 else 2, G, d, n_q, cap, lens, q_lens, dtype, window, sinks, flags=flags, token_major=cap % 2 == 0, seed=cap)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,flags", PATHS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,G,n_q,cap,lens,q_lens,rows", [
    (1, 4, 1, 8, [8], [1], 1),
    (3, 4, 1, 40, [40, 1, 17], [1, 1, 1], 129),
    (5, 2, 1, 70, [70, 0, 64, 65, 1], [1, 1, 1, 0, 1], 1012),    # a sequence without own keys, one without a query
    (33, 4, 1, 16, [16 - i % 16 for i in range(33)], [1] * 33, 300),
    (3, 3, 40, 90, [90, 40, 41], [40, 40, 17], 257),
    (2, 1, 200, 300, [300, 250], [200, 199], 64),
    (4, 8, 9, 20, [20, 9, 10, 3], [9, 9, 2, 9], 700),            # more queries than own keys
    (300, 1, 1, 3, [1 + i % 3 for i in range(300)], [1] * 300, 130),
])
def test_attend_shared(dtype, flags, d, B, G, n_q, cap, lens, q_lens, rows):
    _attend_case(B, 2, G, d, n_q, cap, lens, q_lens, dtype, prefix_rows=rows, flags=flags, token_major=B % 2 == 0, seed=rows)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,flags", PATHS)
def test_attend_scale_and_large_logits(dtype, flags):
    _attend_case(1, 2, 4, 64, 1, 500, [500], [1], dtype, scale=3.0, flags=flags)           # logits of hundreds: one weight near one
    _attend_case(1, 2, 4, 128, 90, 200, [200], [90], dtype, scale=2.5, flags=flags, window=50, sinks=3)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,flags", PATHS)
@pytest.mark.parametrize("n_q", [1, 64])
@pytest.mark.parametrize("low,high", [(-400.0, 400.0), (400.0, -400.0), (-500.0, -480.0), (480.0, 500.0), (-60.0, -40.0)])
def test_attend_logits_that_drift(dtype, flags, n_q, low, high):
    # logits (before the scale, which is one) run from low to high along the cache, far beyond what an exponential in fp32 holds
    gen = torch.Generator().manual_seed(11)
    d, cap, kv, G = 64, 900, 2, 4
    u = torch.full((d,), 0.125)
    ramp = torch.linspace(low, high, cap)
    q = (u + 0.01 * torch.randn(1, kv * G, n_q, d, generator=gen)).to(dtype)
    k = (ramp[:, None] * u + 0.05 * torch.randn(1, kv, cap, d, generator=gen)).to(dtype)
    v = torch.randn(1, kv, cap, d, generator=gen).to(dtype)
    for window, sinks in ((0, 0), (700, 5)):
        want = ref.attend(q, k, v, [cap], [n_q], window, sinks, 1.0)
        got = P.attend(q.cuda(), k.cuda(), v.cuda(), window=window, sinks=sinks, scale=1.0, want_lse=True, flags=flags)
        _check(got["out"], want[0], want[1], "out")
        _check(got["lse"], want[2], want[3], "lse")


@pytest.mark.gpu
@pytest.mark.parametrize("d,dtype", [(64, BF16), (128, BF16), (128, F32)])
@pytest.mark.parametrize("cap,lens,keep,sinks,recent", [
    (1, [1, 0], 1, 0, 0), (64, [64, 10], 16, 4, 4), (300, [300, 299], 299, 0, 0), (1000, [1000, 512], 101, 4, 16), (700, [700, 650], 64, 60, 4),
    (500, [500, 3], 700, 5, 5), (2100, [2100, 2049], 1500, 0, 1), (8193, [8193, 8000], 5000, 1, 8), (16384, [16384, 16383], 2500, 2500, 0),
    (20000, [20000, 17000], 300, 4, 100), (16385, [16385, 2], 16384, 0, 0),
])
def test_evict_by_mass(d, dtype, cap, lens, keep, sinks, recent):
    gen = torch.Generator().manual_seed(cap)
    k, v = (torch.randn(2, 2, cap, d, generator=gen).to(dtype) for _ in range(2))
    mass = torch.exp(3 * torch.randn(2, 2, cap, generator=gen))
    mass[:, :, ::3] = torch.round(mass[:, :, ::3])                                         # many equal ones
    mass[:, 1, 1::11], mass[:, 1, 2::13] = math.nan, math.inf
    mass[0, 0, 5::17], mass[0, 0, 6::17] = 0.0, -0.0
    mass[:, 1, 3::29] = -math.inf
    extra = 3
    k_out, v_out = (torch.full((2, 2, keep + extra, d), SENTINEL, dtype=dtype, device="cuda") for _ in range(2))
    idx = torch.full((2, 2, keep), -1, dtype=torch.int32, device="cuda")
    m_out = torch.full((2, 2, keep + extra), SENTINEL, device="cuda")
    r = P.evict_by_mass(k.cuda(), v.cuda(), mass.cuda(), keep, lens=torch.tensor(lens, dtype=torch.int32, device="cuda"), sinks=sinks, recent=recent,
                        k_out=k_out, v_out=v_out, idx_out=idx, mass_out=m_out)
    want = ref.evict(mass, lens, keep, sinks, recent)
    assert r["lens"].tolist() == [min(n, keep) for n in lens]
    for b in range(2):
        for h in range(2):
            w = want[b][h]
            n = len(w)
            assert idx[b, h, :n].tolist() == w, (b, h)
            assert (idx[b, h, n:] == -1).all() and (m_out[b, h, n:] == SENTINEL).all()
            assert torch.equal(k_out[b, h, :n].cpu(), k[b, h, w]) and torch.equal(v_out[b, h, :n].cpu(), v[b, h, w])
            assert (k_out[b, h, n:] == SENTINEL).all() and (v_out[b, h, n:] == SENTINEL).all()
            assert torch.equal(m_out[b, h, :n].cpu().nan_to_num(nan=-5.0), mass[b, h, w].nan_to_num(nan=-5.0))


# ---- in use -----------------------------------------------------------------------------------------------------------
def _small(dtype=BF16, B=2, kv=2, G=4, d=128, n_q=1, cap=600, seed=1):
    gen = torch.Generator().manual_seed(seed)
    q, k, v = _data(gen, B, kv, G, d, n_q, cap, dtype)
    return q.cuda(), k.cuda(), v.cuda()


@pytest.mark.gpu
@pytest.mark.parametrize("n_q", [1, 50])
def test_the_same_call_gives_the_same_bits_on_any_stream_and_whatever_the_workspace_held(n_q):
    q, k, v = _small(n_q=n_q)
    first = P.attend(q, k, v, window=300, sinks=3, want_lse=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ws = P.attend_workspace(q, k, window=300, sinks=3)
    ws.fill_(0xFF)
    side.wait_stream(torch.cuda.current_stream())
    for stream in (side, side.cuda_stream, None):
        again = P.attend(q, k, v, window=300, sinks=3, want_lse=True, workspace=ws, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(again["out"], first["out"]) and torch.equal(again["lse"], first["lse"])
        assert P.obf_last_device_status(ws) == 0
    with torch.cuda.stream(side):
        again = P.attend(q, k, v, window=300, sinks=3, want_lse=True)              # the current stream, its own workspace
    torch.cuda.synchronize()
    assert torch.equal(again["out"], first["out"])


@pytest.mark.gpu
def test_outputs_made_for_another_stream_are_cleared_on_it():
    q, k, v = _small(n_q=4)
    lens = torch.tensor([600, 500], dtype=torch.int32, device="cuda")
    ql = torch.tensor([4, 2], dtype=torch.int32, device="cuda")
    m = torch.rand(2, 2, 600, device="cuda")
    want = P.attend(q, k, v, lens=lens, q_lens=ql)["out"]
    kept = P.evict_by_mass(k, v, m, 550, lens=lens)
    side, busy = torch.cuda.Stream(), torch.rand(1 << 26, device="cuda")
    torch.cuda.synchronize()
    for _ in range(5):
        for _ in range(20):
            busy.mul_(1.0)                                                         # the current stream is behind
        got, e = P.attend(q, k, v, lens=lens, q_lens=ql, stream=side)["out"], P.evict_by_mass(k, v, m, 550, lens=lens, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(got, want) and (got[1, :, 2:] == 0).all()
        assert all(torch.equal(e[n], kept[n]) for n in kept)


@pytest.mark.gpu
def test_calls_at_once_on_two_streams():
    cases = [_small(seed=s, n_q=n, cap=900) for s, n in ((1, 1), (2, 1), (3, 90), (4, 90))]
    want = [P.attend(*c)["out"] for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    got = [[P.attend(*c, stream=s)["out"] for c, s in zip(cases, streams)] for _ in range(10)]
    torch.cuda.synchronize()
    for r in got:
        assert all(torch.equal(a, b) for a, b in zip(r, want))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n_q", [1, 33])
def test_captured_calls_follow_the_lengths(dtype, n_q):
    q, k, v = _small(dtype, n_q=n_q)
    lens = torch.tensor([100, 40], dtype=torch.int32, device="cuda")
    ws = P.attend_workspace(q, k, window=200, sinks=2)
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:3], device="cuda")
    P.attend(q, k, v, lens=lens, window=200, sinks=2, out=out, lse_out=lse, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.attend(q, k, v, lens=lens, window=200, sinks=2, out=out, lse_out=lse, workspace=ws)
    for pair in ([600, 599], [1, 0], [333, 257]):
        lens.copy_(torch.tensor(pair, dtype=torch.int32))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        want = P.attend(q, k, v, lens=lens, window=200, sinks=2, want_lse=True)
        assert torch.equal(out, want["out"]) and torch.equal(lse, want["lse"])
        w = ref.attend(q.cpu(), k.cpu(), v.cpu(), pair, [n_q, n_q], 200, 2)
        _check(out, w[0], w[1], "out")


@pytest.mark.gpu
def test_a_call_captured_first_leaves_nothing_of_the_graph_behind():
    q, k, v = _small(cap=100)
    want = P.attend(q, k, v)["out"]
    binding._status_words.clear()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = P.attend(q, k, v)["out"]
    assert not binding._status_words
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    del graph, got
    assert torch.equal(P.attend(q, k, v)["out"], want)


@pytest.mark.gpu
def test_refusals_name_the_tensor():
    q, k, v = _small(cap=100)
    for kw, name in ((dict(v=v[:, :, :50]), "v"), (dict(v=v.float()), "v"), (dict(k=k[:, :, :, :64]), "k"), (dict(lens=torch.ones(3, dtype=torch.int32, device="cuda")), "lens"),
                     (dict(lens=torch.ones(2, dtype=torch.int64, device="cuda")), "lens"), (dict(out=q.float()), "out"), (dict(v=v.cpu()), "v"),
                     (dict(mass_out=torch.zeros(2, 2, 99, device="cuda")), "mass_out"), (dict(q=q.transpose(2, 3)), "q")):
        args = dict(q=q, k=k, v=v)
        args.update(kw)
        with pytest.raises(ValueError, match=name):
            P.attend(args.pop("q"), args.pop("k"), args.pop("v"), **args)
    m = torch.rand(2, 2, 100, device="cuda")
    for kw, name in ((dict(v=v[:, :1]), "v"), (dict(mass=m.double()), "mass"), (dict(k_out=k[:, :, :5]), "k_out"), (dict(k_out=k.float()), "k_out")):
        args = dict(k=k, v=v, mass=m)
        args.update(kw)
        with pytest.raises(ValueError, match=name):
            P.evict_by_mass(args.pop("k"), args.pop("v"), args.pop("mass"), 10, **args)


@pytest.mark.gpu
def test_lengths_out_of_range_are_clamped_and_reported():
    for n_q in (1, 40):
        q, k, v = _small(n_q=n_q)
        ws = P.attend_workspace(q, k)
        want = P.attend(q, k, v, lens=torch.tensor([600, 0], dtype=torch.int32, device="cuda"))["out"]
        got = P.attend(q, k, v, lens=torch.tensor([60000, -5], dtype=torch.int32, device="cuda"), workspace=ws)["out"]
        assert P.obf_last_device_status(ws) == binding.OBF_DEV_INTERNAL
        assert torch.equal(got, want)
        P.attend(q, k, v, workspace=ws)
        assert P.obf_last_device_status(ws) == 0                                   # the next call's word is its own


@pytest.mark.gpu
def test_masses_in_place_and_without_a_start():
    q, k, v = _small()
    m = torch.rand(2, 2, 600, device="cuda")
    want = P.attend(q, k, v, mass_in=m.clone(), mass_out=torch.zeros_like(m), decay=0.5)["mass"]
    got = P.attend(q, k, v, mass_in=m, mass_out=m, decay=0.5)["mass"]
    assert got is m and torch.equal(got, want)
    bare = P.attend(q, k, v, mass_out=torch.full_like(m, 3.0))["mass"]
    assert torch.allclose(bare.sum(-1), torch.full((2, 2), 4.0, device="cuda"), atol=1e-3)      # four query rows, each one in all


@pytest.mark.gpu
@pytest.mark.parametrize("n_q", [1, 60])
def test_values_that_are_not_finite_reach_the_queries_that_see_them(n_q):
    q, k, v = _small(n_q=n_q, cap=200)
    k[0, 0, 150, 3] = math.nan
    v[1, 1, 10, 5] = math.inf
    out = P.attend(q, k, v)["out"]
    t = torch.arange(200 - n_q, 200)
    assert out[0, :4, t >= 150].isnan().all() and out[0, 4:].isfinite().all()
    hit = out[1, 4:, :, 5]
    assert not hit.isfinite().any() and out[1, 4:, :, 6].isfinite().all() and out[1, :4].isfinite().all()


@pytest.mark.gpu
@pytest.mark.parametrize("n_q,window", [(4, 0), (50, 0), (50, 70), (300, 0)])
def test_what_lies_behind_a_sequence_s_queries_changes_no_bit(n_q, window):
    gen = torch.Generator().manual_seed(23)
    q, k, v = (x.cuda() for x in _data(gen, 2, 2, 2, 128, n_q, 500, BF16))
    ql = torch.tensor([n_q - 1, n_q // 2], dtype=torch.int32, device="cuda")
    got = []
    for fill in (0.0, 300.0, -300.0, math.inf, math.nan):
        x = q.clone()
        for b in range(2):
            x[b, :, int(ql[b]):] = fill
        got.append(P.attend(x, k, v, q_lens=ql, window=window, sinks=3, want_lse=True))
    for g in got[1:]:
        assert torch.equal(g["out"], got[0]["out"]) and torch.equal(g["lse"], got[0]["lse"])


@pytest.mark.gpu
@pytest.mark.parametrize("n_q", [1, 64])
def test_very_large_values(n_q):
    gen = torch.Generator().manual_seed(21)
    q, k, v = _data(gen, 1, 2, 2, 128, n_q, 300, BF16)
    q, v = (q.float() * 2).to(BF16), (v.float() * 1e27).to(BF16)                     # logits of up to some 20
    w = ref.attend(q, k, v, [300], [n_q])
    _check(P.attend(q.cuda(), k.cuda(), v.cuda())["out"], w[0], w[1], "out")


@pytest.mark.gpu
@pytest.mark.parametrize("n_q", [1, 64])
def test_offsets_beyond_32_bits(n_q):
    # the second sequence's rows lie more than 2^32 bytes (and 2^31 elements) behind the first's
    cap, d = 1100, 128
    big = torch.empty(2, (1 << 31) + 4096, dtype=BF16, device="cuda")
    k = big.as_strided((2, 1, cap, d), (big.stride(0), 0, d, 1))
    v = big.as_strided((2, 1, cap, d), (big.stride(0), 0, d, 1), cap * d)
    gen = torch.Generator().manual_seed(5)
    q, kc, vc = _data(gen, 2, 1, 2, d, n_q, cap, BF16)
    k.copy_(kc)
    v.copy_(vc)
    w = ref.attend(q, kc, vc, [cap, cap - 7], [n_q, n_q], 500, 4)
    out = P.attend(q.cuda(), k, v, lens=torch.tensor([cap, cap - 7], dtype=torch.int32, device="cuda"), window=500, sinks=4)["out"]
    _check(out, w[0], w[1], "out")


@pytest.mark.gpu
@pytest.mark.parametrize("n_q", [1, 40])
def test_strided_caches_and_outputs(n_q):
    gen = torch.Generator().manual_seed(9)
    q, kc, vc = _data(gen, 2, 3, 2, 64, n_q, 150, BF16)
    kv = torch.zeros(2, 150, 3, 2, 64, dtype=BF16)                                   # token-major, keys and values in turn
    kv[:, :, :, 0], kv[:, :, :, 1] = kc.transpose(1, 2), vc.transpose(1, 2)
    kv = kv.cuda()
    out = torch.zeros(2, n_q, 6, 72, dtype=BF16, device="cuda")[..., :64].transpose(1, 2)       # rows 144 bytes apart: no multiple of 32
    P.attend(q.cuda(), kv[:, :, :, 0].transpose(1, 2), kv[:, :, :, 1].transpose(1, 2), window=60, sinks=5, out=out)
    w = ref.attend(q, kc, vc, [150, 150], [n_q, n_q], 60, 5)
    _check(out, w[0], w[1], "out")


@pytest.mark.gpu
def test_chain_relay_attention_masses_and_eviction():
    """A prompt is compressed, the relay is shared by a batch that decodes over it, and a cache that has grown is evicted from by the
    masses that its tokens gathered: every step against the plain form on what the library left of the step before."""
    layers, kv, G, d, T, W = 1, 2, 4, 128, 512, 8
    gen = torch.Generator().manual_seed(3)
    K, V = (torch.randn(layers, kv, T, d, generator=gen).to(BF16) for _ in range(2))
    Q = torch.randn(layers, kv * G, W, d, generator=gen).to(BF16)
    # what an earlier relay's keys take of the observation queries' softmax
    old = torch.randn(1, kv, 70, d, generator=gen).to(BF16)
    extra = P.attend(Q.cuda(), old.cuda(), old.cuda(), want_lse=True)                 # causal: the last of the 70 keys' positions
    full = P.attend_shared(Q.cuda(), old[0].cuda(), old[0].cuda(), old.cuda(), old.cuda(), lens=torch.zeros(1, dtype=torch.int32, device="cuda"), want_lse=True)
    x = torch.einsum("bhtd,bhjd->bhtj", Q.double().reshape(1, kv, G * W, d), old.double()) / math.sqrt(d)
    assert torch.allclose(full["lse"].double().cpu().reshape(1, kv, G * W), torch.logsumexp(x, -1), atol=1e-5)
    assert (extra["lse"] <= full["lse"] + 1e-5).all()
    params = P.make_params(layers, kv, kv * G, d, W, 2, P.OBF_BF16)
    r = P.compress_caches(params, [{"K": K.cuda(), "V": V.cuda(), "Q": Q.cuda(), "budget": 100, "lse_extra": full["lse"].contiguous()}], want_scores=True)[0]
    torch.cuda.synchronize()
    relay_k, relay_v = r["K_out"][0], r["V_out"][0]
    # three agents, one token each, over the shared relay
    q, k, v = _data(gen, 3, kv, G, d, 1, 30, BF16)
    lens = [30, 11, 1]
    got = P.attend_shared(q.cuda(), relay_k, relay_v, k.cuda(), v.cuda(), lens=torch.tensor(lens, dtype=torch.int32, device="cuda"))
    w = ref.attend(q, k, v, lens, [1, 1, 1], prefix=(relay_k.cpu(), relay_v.cpu()))
    _check(got["out"], w[0], w[1], "out")
    # one agent goes on: its cache is the relay and room for more, its masses begin as the selection's
    cap = 140
    ck, cv = (torch.zeros(1, kv, cap, d, dtype=BF16, device="cuda") for _ in range(2))
    ck[0, :, :100], cv[0, :, :100] = relay_k, relay_v
    mass = torch.zeros(1, kv, cap, device="cuda")
    mass[0, :, :100] = torch.gather(r["scores"][0], 1, r["idx"][0].long())
    length = torch.tensor([100], dtype=torch.int32, device="cuda")
    for step in range(20):
        q1, k1, v1 = _data(gen, 1, kv, G, d, 1, 1, BF16)
        ck[0, :, 100 + step], cv[0, :, 100 + step] = k1[0, :, 0].cuda(), v1[0, :, 0].cuda()
        length += 1
        before = mass.cpu()
        got = P.attend(q1.cuda(), ck, cv, lens=length, window=64, sinks=4, mass_in=mass, mass_out=mass, decay=0.9)
        w = ref.attend(q1, ck.cpu(), cv.cpu(), [101 + step], [1], 64, 4, mass_in=before, decay=0.9, want_mass=True)
        _check(got["out"], w[0], w[1], "out")
        _check(mass, w[4], w[5], "mass")
    e = P.evict_by_mass(ck, cv, mass, 48, lens=length, sinks=4, recent=8)
    kept = ref.evict(mass.cpu(), [120], 48, 4, 8)
    assert e["lens"].tolist() == [48]
    for h in range(kv):
        assert e["idx"][0, h].tolist() == kept[0][h]
        assert torch.equal(e["K_out"][0, h], ck[0, h, kept[0][h]]) and torch.equal(e["V_out"][0, h], cv[0, h, kept[0][h]])
