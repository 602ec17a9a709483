"""Forms of the attention over a relayed cache that come with the size of a call: blocks that work through several items, keys in one
part, in more parts than a cluster takes or a warp has lanes, with masses and without; references that have to follow the logits."""
import pytest
import torch

import paper_2604_13349_b200 as P
from tests import _attend_ref as ref
from tests.test_attend import BF16, F32, GENERIC, _attend_case, _check

MULTIPROCESSORS = 148


def _workspace(B, kv, G, d, n_q, cap, dtype, window=0, sinks=0, mass=False, prefix_rows=0):
    q, k = torch.empty(B, kv * G, n_q, d, dtype=dtype, device="meta"), torch.empty(B, kv, cap, d, dtype=dtype, device="meta")
    return P.attend_workspace(q, k, window=window, sinks=sinks, mass=mass, prefix_rows=prefix_rows).numel()


def _parts(B, kv, G, d, n_q, cap, dtype, **kw):
    """All parts of a row of a call whose parts are joined by a kernel of their own; 0: no such join.  (A part leaves d + 1 fp32 words per
    row, a mass call a logit per row and key; sections are aligned to 256 bytes.)"""
    rows = B * kv * G * n_q
    size = _workspace(B, kv, G, d, n_q, cap, dtype, **kw) - 256
    if kw.get("mass"):
        size -= (rows * cap * 4 + 255) // 256 * 256
    return size // (rows * (d + 1) * 4)


# ---- blocks of the tensor-core kernel that work through more than one item ------------------------------------------------------


def _ragged(n_q, cap):
    q_lens = [n_q if b % 4 == 0 else 0 if b % 4 == 1 else (b * 7) % n_q + 1 if b % 4 == 2 else 1 + b // 4 for b in range(24)]
    lens = [cap - 5 * b if b % 3 else max(q_lens[b] - b % 2, 1) for b in range(24)]
    return lens, q_lens


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_q,cap,window,sinks", [
    (130, 200, 0, 0),                # three pairs of tiles per (sequence, head): 576 items for 148 blocks, many of them without queries
    (130, 333, 70, 3),
    (65, 260, 40, 90),               # the second tile of a pair empty or of one query, more sinks than the window
])
def test_blocks_work_through_many_items(d, n_q, cap, window, sinks):
    lens, q_lens = _ragged(n_q, cap)
    _attend_case(24, 8, 4, d, n_q, cap, lens, q_lens, BF16, window, sinks, seed=n_q + cap, token_major=window == 0)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
def test_blocks_work_through_many_items_of_parts(d):
    # two parts of the keys and more; of the short sequences' keys the later parts hold nothing
    B, kv, G, n_q, cap = 18, 5, 4, 40, 4111
    assert _parts(B, kv, G, d, n_q, cap, BF16) >= 2 and B * kv * _parts(B, kv, G, d, n_q, cap, BF16) > MULTIPROCESSORS
    lens = [cap if b % 5 == 0 else 40 + 9 * b if b % 5 < 3 else cap // 2 for b in range(B)]
    _attend_case(B, kv, G, d, n_q, cap, lens, [n_q if b % 3 else b for b in range(B)], BF16, seed=7)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_q,rows", [(130, 200), (9, 900)])
def test_blocks_work_through_many_items_of_a_shared_prefix(d, n_q, rows):
    # 49 pairs of tiles per KV head, and 4 of them in several parts
    lens, q_lens = _ragged(n_q, 150)
    _attend_case(24, 8, 4, d, n_q, 150, lens, q_lens, BF16, prefix_rows=rows, seed=rows)


# ---- few query rows: parts ---------------------------------------------------------------------------------------------------------
TYPES = [pytest.param(BF16, id="bf16"), pytest.param(F32, id="f32")]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,flags", [pytest.param(BF16, 0, id="bf16"), pytest.param(BF16, GENERIC, id="bf16-generic"), pytest.param(F32, 0, id="f32")])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n_q,cap,lens,window,sinks", [
    (1, 1, 1, [1, 0], 0, 0),
    (4, 1, 700, [700, 3], 100, 4),
    (3, 1, 1300, [1300, 1025], 1000, 77),
    (8, 2, 257, [257, 255], 50, 51),
    (7, 2, 400, [399, 1], 16, 1),
    (16, 1, 130, [130, 17], 0, 0),
])
def test_few_queries_without_masses(dtype, flags, d, G, n_q, cap, lens, window, sinks):
    _attend_case(2, 2, G, d, n_q, cap, lens, [min(n_q, n) for n in lens], dtype, window, sinks, flags=flags, seed=cap)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n_q,window,sinks", [(4, 1, 0, 0), (4, 1, 300, 4), (3, 3, 77, 90), (8, 2, 0, 0)])
def test_few_queries_in_one_part(dtype, d, G, n_q, window, sinks):
    B, kv, cap = 80, 8, 500
    assert _workspace(B, kv, G, d, n_q, cap, dtype, window=window, sinks=sinks) == 256                # the blocks store the rows themselves
    _attend_case(B, kv, G, d, n_q, cap, [cap - 6 * b for b in range(B)], [n_q if b % 7 else b % 2 for b in range(B)], dtype, window, sinks, seed=G)


@pytest.mark.gpu
@pytest.mark.parametrize("mass", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,kv,cap,lens,window,sinks,least", [
    (1, 1, 5000, [4999], 0, 0, 9),                                     # more parts than a cluster has
    (3, 1, 5200, [5200, 300, 1], 4700, 4, 9),                          # and most of them empty
    (1, 1, 70001, [70001], 0, 0, 33),                                  # more than a warp's lanes join at once
    (2, 1, 40000, [39000, 20], 30011, 200, 33),
])
def test_few_queries_in_many_parts(mass, dtype, d, B, kv, cap, lens, window, sinks, least):
    assert _parts(B, kv, 4, d, 1, cap, dtype, window=window, sinks=sinks, mass=mass) >= least
    _attend_case(B, kv, 4, d, 1, cap, lens, [1] * B, dtype, window, sinks, mass=mass, decay=0.5, seed=cap)


@pytest.mark.gpu
@pytest.mark.parametrize("mass", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
def test_few_queries_joined_a_warp_per_row(mass, dtype, d):
    # rows enough for a warp each, in two parts and more
    B, kv, G, n_q, cap = 20, 4, 4, 2, 6000
    assert _parts(B, kv, G, d, n_q, cap, dtype, mass=mass) >= 2
    _attend_case(B, kv, G, d, n_q, cap, [cap - 290 * b for b in range(B)], [n_q if b % 6 else 1 for b in range(B)], dtype, mass=mass, decay=0.9, seed=6)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,G,n_q,cap,lens,rows", [
    (3, 4, 1, 40, [40, 0, 17], 5000),                                  # few rows over the prefix, too
    (2, 2, 4, 30, [30, 3], 4100),
    (1, 8, 2, 70, [70], 9001),
    (4, 1, 1, 4500, [4500, 2, 0, 4097], 130),
    (2, 3, 1, 9, [9, 1], 66000),
    (40, 4, 1, 300, [300 - 7 * b for b in range(40)], 2500),           # many over the prefix, few of each sequence
])
def test_few_queries_over_a_long_shared_prefix(dtype, d, B, G, n_q, cap, lens, rows):
    assert _parts(B, 2, G, d, n_q, cap, dtype, prefix_rows=rows) >= 2
    _attend_case(B, 2, G, d, n_q, cap, lens, [n_q] * B, dtype, prefix_rows=rows, seed=rows)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B", [4, 5, 8])
def test_few_queries_on_either_side_of_one_launch(dtype, B):
    # a prefix that each sequence's blocks read by themselves, or that is read once and joined
    _attend_case(B, 8, 4, 128, 1, 40, [40 - 5 * b for b in range(B)], [1] * B, dtype, prefix_rows=1012, seed=B)


# ---- references that follow the logits ---------------------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,sinks", [(0, 0), (4000, 5)])
@pytest.mark.parametrize("logit", [17.9, 19.0, 21.0, 22.5])
@pytest.mark.parametrize("cap,power", [(1400, 89), (9000, 86)])
def test_many_large_weights_behind_small_ones_do_not_overflow(d, window, sinks, logit, cap, power):
    # the first tiles' logits leave every row's reference at zero; of the others, 2^25.8 to 2^32.5 above it, each alone keeps its weight
    # within range, but not all of them together.  Values times keys stay below 2^100.
    gen = torch.Generator().manual_seed(3)
    n_q, kv, G = 74, 4, 128                                                         # 148 pairs of tiles: keys in one part, all rows alike
    assert _workspace(1, kv, G, d, n_q, cap, BF16, window=window, sinks=sinks) == 256
    u = torch.full((d,), 1 / 8 if d == 64 else 1 / 16)
    level = torch.zeros(cap)
    level[300:] = logit * (1 if d == 64 else 2)
    q = u.expand(1, 1, n_q, d).to(BF16)
    k = (level[:, None] * u).expand(1, 1, cap, d).to(BF16)
    v = ((1 + 0.25 * torch.rand(1, 1, cap, d, generator=gen)) * 2.0 ** (power - 1)).to(BF16)
    want = ref.attend(q, k, v, [cap], [n_q], window, sinks, 1.0)
    got = P.attend(q.repeat(1, kv * G, 1, 1).cuda(), k.repeat(1, kv, 1, 1).cuda(), v.repeat(1, kv, 1, 1).cuda(), window=window, sinks=sinks, scale=1.0,
                   want_lse=True)
    for h in (0, 1, kv * G // 2, kv * G - 1):
        _check(got["out"][:, h:h + 1], want[0], want[1], "out")
        _check(got["lse"][:, h:h + 1], want[2], want[3], "lse")
    assert torch.equal(got["out"], got["out"][:, :1].expand_as(got["out"])) and torch.equal(got["lse"], got["lse"][:, :1].expand_as(got["lse"]))


# ---- layouts, and calls captured together ---------------------------------------------------------------------------------------------
def _token_major(t):
    """The same [.., heads, rows, d] values, laid out row by row with a gap of eight channels behind each."""
    x = torch.zeros(*t.shape[:-3], t.shape[-2], t.shape[-3], t.shape[-1] + 8, dtype=t.dtype, device="cuda")[..., : t.shape[-1]].transpose(-3, -2)
    return x.copy_(t)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,flags", [pytest.param(BF16, 0, id="bf16"), pytest.param(BF16, GENERIC, id="bf16-generic"), pytest.param(F32, 0, id="f32")])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,n_q,rows", [(2, 1, 200), (3, 1, 5000), (2, 40, 300), (40, 1, 600)])
def test_strided_caches_prefixes_and_outputs(dtype, flags, d, B, n_q, rows):
    gen = torch.Generator().manual_seed(B + rows)
    kv, G, cap = 3, 2, 150
    q, k, v = torch.randn(B, kv * G, n_q, d, generator=gen).to(dtype), *(torch.randn(B, kv, cap, d, generator=gen).to(dtype) for _ in range(2))
    pk, pv = (torch.randn(kv, rows, d, generator=gen).to(dtype) for _ in range(2))
    lens = [cap - b for b in range(B)]
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    qd, kd, vd, pkd, pvd = (_token_major(x) for x in (q, k, v, pk, pv))
    out = _token_major(torch.zeros_like(q))
    got = P.attend_shared(qd, pkd, pvd, kd, vd, lens=n, out=out, flags=flags)
    w = ref.attend(q, k, v, lens, [n_q] * B, prefix=(pk, pv))
    _check(got["out"], w[0], w[1], "out over a prefix")
    m = torch.rand(B, kv, cap, generator=gen)
    mass = n_q * G <= 64
    out.zero_()
    if mass:
        got = P.attend(qd, kd, vd, lens=n, window=60, sinks=5, out=out, mass_in=m.cuda(), mass_out=torch.zeros(B, kv, cap, device="cuda"), flags=flags)
    else:
        got = P.attend(qd, kd, vd, lens=n, window=60, sinks=5, out=out, flags=flags)
    w = ref.attend(q, k, v, lens, [n_q] * B, 60, 5, mass_in=m if mass else None, want_mass=mass)
    _check(got["out"], w[0], w[1], "out")
    if mass:
        _check(got["mass"], w[4], w[5], "mass")
    kept = P.evict_by_mass(kd, vd, m.cuda(), 40, lens=n, sinks=2, recent=5, k_out=_token_major(torch.zeros(B, kv, 50, d, dtype=dtype)),
                           v_out=_token_major(torch.zeros(B, kv, 45, d, dtype=dtype)))
    want = ref.evict(m, lens, 40, 2, 5)
    for b in range(0, B, 7):
        for h in range(kv):
            assert kept["idx"][b, h].tolist() == want[b][h]
            assert torch.equal(kept["K_out"][b, h, :40].cpu(), k[b, h, want[b][h]]) and torch.equal(kept["V_out"][b, h, :40].cpu(), v[b, h, want[b][h]])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,cap,rows", [(2, 300, 400), (3, 600, 5000), (40, 300, 700), (2, 17000, 300)])
def test_a_captured_chain_follows_the_lengths(dtype, B, cap, rows):
    # over a prefix, with masses, evicted by them, over what was kept; the library's kernels one behind the other, each started early
    gen = torch.Generator().manual_seed(rows)
    kv, G, d, keep = 2, 4, 128, 100
    q, k, v = (torch.randn(B, h, n, d, generator=gen).to(dtype).cuda() for h, n in ((kv * G, 1), (kv, cap), (kv, cap)))
    pk, pv = (torch.randn(kv, rows, d, generator=gen).to(dtype).cuda() for _ in range(2))
    mass = torch.rand(B, kv, cap, generator=gen).cuda()
    lens = torch.full((B,), cap, dtype=torch.int32, device="cuda")

    def chain():
        a = P.attend_shared(q, pk, pv, k, v, lens=lens, want_lse=True)
        b = P.attend(a["out"], k, v, lens=lens, window=cap // 2, sinks=3, mass_in=mass, mass_out=torch.zeros_like(mass), decay=0.5)
        e = P.evict_by_mass(k, v, b["mass"], keep, lens=lens, sinks=3, recent=9)
        c = P.attend(b["out"], e["K_out"], e["V_out"], lens=e["lens"], want_lse=True)
        return [a["out"], a["lse"], b["out"], b["mass"], *(e[n] for n in ("K_out", "V_out", "idx", "mass", "lens")), c["out"], c["lse"]]

    chain()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = chain()
    for shift in (0, 1, cap // 3):
        lens.copy_(torch.tensor([max(cap - shift * (b + 1), b % 3) for b in range(B)], dtype=torch.int32))
        for _ in range(2):
            graph.replay()
        torch.cuda.synchronize()
        want = chain()
        assert all(torch.equal(x, y) for x, y in zip(got, want))
    n = lens.tolist()
    w = ref.attend(q.cpu(), k.cpu(), v.cpu(), n, [1] * B, prefix=(pk.cpu(), pv.cpu()))
    _check(got[0], w[0], w[1], "out over a prefix")
    w = ref.attend(got[0].cpu(), k.cpu(), v.cpu(), n, [1] * B, cap // 2, 3, mass_in=mass.cpu(), decay=0.5, want_mass=True)
    _check(got[2], w[0], w[1], "out")
    _check(got[3], w[4], w[5], "mass")
    kept = ref.evict(got[3].cpu(), n, keep, 3, 9)
    assert all(got[6][b, h, : len(kept[b][h])].tolist() == kept[b][h] for b in range(B) for h in range(kv))


# ---- logits beyond fp32's whole numbers -------------------------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("dtype,flags", [pytest.param(BF16, 0, id="bf16"), pytest.param(BF16, GENERIC, id="bf16-generic"), pytest.param(F32, 0, id="f32")])
@pytest.mark.parametrize("n_q", [1, 64, 300])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("significand", [165 / 128, 219 / 128])
@pytest.mark.parametrize("power", [10, 13, 20, 26, 30, 33, 100])
def test_equal_logits_of_any_size_weigh_the_same(dtype, flags, n_q, sign, power, significand):
    # the largest logit belongs to two keys in different tiles; a short significand, so the products and their sums are exact and the
    # logits equal, though not the products with a constant; the other keys, 2^(power - 1) or more below, weigh nothing
    gen = torch.Generator().manual_seed(power)
    d, cap, first, second = 64, 700, 10, 500
    u = torch.full((d,), 1 / 8)
    top = sign * significand * 2.0 ** power
    level = torch.full((cap,), top * (0.5 if sign > 0 else 2.0))
    level[first] = level[second] = top
    q = u.expand(1, 4, n_q, d).to(dtype)
    k = (level[:, None] * u).expand(1, 2, cap, d).to(dtype)
    v = torch.randn(1, 2, cap, d, generator=gen).to(dtype)
    got = P.attend(q.cuda(), k.cuda(), v.cuda(), scale=1.0, want_lse=True, flags=flags)
    t = torch.arange(cap - n_q, cap)
    both = (t >= second)[None, None, :, None]
    a, b = (v[:, :, j].double().repeat_interleave(2, 1)[:, :, None] for j in (first, second))
    want = torch.where(both, (a + b) / 2, a.expand(1, 4, n_q, d))
    # fp32 sums of one or two weights of one, one division, the output's rounding: 2^-22 of the magnitudes and half a step of the output
    _check(got["out"], want, 2.0 ** -22 * (a.abs() + b.abs()) + ref.STEP[dtype] * want.abs() + 1e-30, "out")
    lse = top + torch.where(both[..., 0], torch.log(torch.tensor(2.0, dtype=torch.float64)), 0.0).expand(1, 4, n_q)
    # the scaling, the logarithm's addition and the way back to natural logarithms round once each, and so do the two constants
    _check(got["lse"], lse, (2.0 ** -21 * lse.abs()), "lse")
