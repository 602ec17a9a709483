"""The operators on a relayed cache that are measured: attention with a sliding window and sinks (with the accumulated mass of
every key, or without), attention of a batch over one shared relay, eviction by accumulated mass.

Each has its plain form in elementary torch operations (`own` false) and the library's call (`own` true), on the same inputs.
Shapes: q [batch, q_heads, n_q, dim], k, v [batch, kv_heads, capacity, dim], q head = kv_head * group + g; the keys of sequence b
are rows 0 .. lens[b] - 1, query i of it (i < q_lens[b]) is the token at position lens[b] - q_lens[b] + i.
"""
import math

import numpy as np
import torch

own = False          # set by whoever runs the cases: False = the plain forms, True = the library's calls

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _case(kind, name=None, **kw):
    base = dict(kind=kind, batch=1, kv_heads=8, group=4, dim=128, dtype="bf16", n_q=1, capacity=1024, shortest=1024,
                token_major=False, window=0, sinks=0, mass=False, decay=1.0, prefix=0, keep=0, recent=0)
    base.update(kw)
    if name is not None:
        base["name"] = name
    return base


def listed():
    return [
        # one agent's next token over a short relay: what counts is latency
        _case("window", "step_one", capacity=1024, shortest=1000, window=256, sinks=4),
        # a served batch of agents at different lengths, window of half the longest prompt
        _case("window", "step_batch", batch=32, capacity=8192, shortest=1024, window=4096, sinks=4),
        # few agents with very long chains of relays, every key visible
        _case("window", "step_long", batch=4, capacity=131072, shortest=100001),
        # a step of agents whose caches will be evicted from: the masses come with the attention
        _case("window", "step_mass", batch=16, capacity=8192, shortest=7000, sinks=4, mass=True),
        # a long prompt through a windowed layer
        _case("window", "prompt_8192", n_q=8192, capacity=8192, shortest=8192, window=1024, sinks=4),
        # prompts of a ragged batch, heads of 64 channels, queries as a model's projection leaves them, an odd window
        _case("window", "prompt_ragged", batch=4, dim=64, group=2, n_q=2048, capacity=2048, shortest=701, token_major=True,
              window=511, sinks=1),
        # the same in fp32, as the small reference configurations run
        _case("window", "prompt_f32", dim=64, dtype="f32", n_q=1024, capacity=1024, shortest=1024, window=300, sinks=4),
        # a handful of agents reading one relay of the paper's length, each with its 40 latent steps
        _case("shared", "shared_few", batch=4, prefix=1012, capacity=40, shortest=17),
        # many branches of one long relay
        _case("shared", "shared_many", batch=64, prefix=16384, capacity=512, shortest=33),
        # 40 new positions of each of eight agents at once
        _case("shared", "shared_chunk", batch=8, n_q=40, prefix=4096, capacity=299, shortest=40),
        # one agent's cache brought down to a tenth
        _case("evict", "evict_one", capacity=1024, shortest=1024, keep=101, sinks=4, recent=16),
        # a batch's caches brought down to a quarter
        _case("evict", "evict_batch", batch=32, capacity=8192, shortest=3001, keep=2048, sinks=4, recent=128),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["step", "mass", "prompt", "shared", "evict"])
    dim = rng.choice([64, 128])
    kv = rng.choice([1, 2, 4, 5, 8])
    g = rng.choice([1, 2, 3, 4, 6, 7, 8])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    window = rng.choice([0, _log(rng, 1, 8192)])
    sinks = rng.choice([0, 1, 4, rng.randint(1, 200)])
    if kind in ("step", "mass"):
        batch = _log(rng, 1, 64)
        most = max(16, min(131072, (1 << 21) // (batch * kv)))
        cap = _log(rng, 16, most)
        n_q = rng.choice([1, 1, 1, 2, 5])
        return _case("window", batch=batch, kv_heads=kv, group=g, dim=dim, dtype=dtype, n_q=n_q, capacity=cap, shortest=rng.randint(max(1, cap // 4), cap),
                     window=window, sinks=sinks, mass=kind == "mass", decay=rng.choice([1.0, 0.5, 0.99]), token_major=rng.random() < 0.5)
    if kind == "prompt":
        batch = _log(rng, 1, 8)
        most = int(math.sqrt((1 << 29) / (batch * kv * g)))
        cap = _log(rng, 16, min(8192 if dtype == "bf16" else 2048, most))
        return _case("window", batch=batch, kv_heads=kv, group=g, dim=dim, dtype=dtype, n_q=cap, capacity=cap, shortest=rng.randint(max(1, cap // 3), cap),
                     window=window, sinks=sinks, token_major=rng.random() < 0.5)
    if kind == "shared":
        batch = _log(rng, 1, 128)
        n_q = rng.choice([1, 1, 1, 4, 40])
        cap = _log(rng, 8, 1024)
        prefix = _log(rng, 16, max(64, min(32768, (1 << 28) // (batch * n_q * kv * g))))
        return _case("shared", batch=batch, kv_heads=kv, group=g, dim=dim, dtype=dtype, n_q=n_q, capacity=cap, shortest=rng.randint(1, cap), prefix=prefix,
                     token_major=rng.random() < 0.5)
    batch = _log(rng, 1, 32)
    cap = _log(rng, 64, min(32768, (1 << 20 if dtype == "bf16" else 1 << 19) // (batch * kv)))
    keep = _log(rng, 16, cap)
    sinks = rng.randint(0, keep // 4)
    return _case("evict", batch=batch, kv_heads=kv, dim=dim, dtype=dtype, capacity=cap, shortest=rng.randint(max(1, cap // 3), cap), keep=keep, sinks=sinks,
                 recent=rng.randint(0, keep // 2))


def _lens(c):
    """Lengths of the sequences, spread from the capacity down to the shortest."""
    span = c["capacity"] - c["shortest"]
    return [c["capacity"] - (span * b // max(1, c["batch"] - 1)) for b in range(c["batch"])]


def prepare(c, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    t, d, kv, g, B = TYPES[c["dtype"]], c["dim"], c["kv_heads"], c["group"], c["batch"]

    def normal(*shape, dtype=t):
        return torch.randn(shape, generator=gen, device="cuda", dtype=dtype)

    s = dict(c=c)
    s["k"], s["v"] = normal(B, kv, c["capacity"], d), normal(B, kv, c["capacity"], d)
    s["k"][..., : d // 32].mul_(4.0)                                        # outlier channels, as caches have them
    lens = _lens(c)
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    if c["kind"] == "evict":
        # heavy-tailed masses with ties, as sums of a few thousand softmax rows have
        s["mass"] = torch.exp(2.0 * normal(B, kv, c["capacity"], dtype=torch.float32))
        s["mass"][..., ::7] = torch.round(s["mass"][..., ::7])
        shape = (B, kv, c["keep"], d)
        s["k_out"], s["v_out"] = torch.zeros(shape, dtype=t, device="cuda"), torch.zeros(shape, dtype=t, device="cuda")
        s["idx_out"] = torch.zeros(shape[:3], dtype=torch.int32, device="cuda")
        s["mass_out"] = torch.zeros(shape[:3], dtype=torch.float32, device="cuda")
        return s
    n_q, hq = c["n_q"], kv * g
    if c["token_major"]:
        s["q"], s["out"] = normal(B, n_q, hq, d).transpose(1, 2), torch.zeros((B, n_q, hq, d), dtype=t, device="cuda").transpose(1, 2)
    else:
        s["q"], s["out"] = normal(B, hq, n_q, d), torch.zeros((B, hq, n_q, d), dtype=t, device="cuda")
    s["lse"] = torch.zeros((B, hq, n_q), dtype=torch.float32, device="cuda")
    s["q_lens"] = torch.tensor([min(n_q, x) for x in lens], dtype=torch.int32, device="cuda")
    if c["mass"]:
        s["mass"] = torch.exp(normal(B, kv, c["capacity"], dtype=torch.float32))
        s["mass_out"] = torch.zeros_like(s["mass"])
    if c["kind"] == "shared":
        s["k_prefix"], s["v_prefix"] = normal(kv, c["prefix"], d), normal(kv, c["prefix"], d)
        s["k_prefix"][..., : d // 32].mul_(4.0)
    return s


def run(s):
    c = s["c"]
    if own:
        import paper_2604_13349_b200 as P
        if c["kind"] == "evict":
            return P.evict_by_mass(s["k"], s["v"], s["mass"], c["keep"], lens=s["lens"], sinks=c["sinks"], recent=c["recent"],
                                   k_out=s["k_out"], v_out=s["v_out"], idx_out=s["idx_out"], mass_out=s["mass_out"])
        if c["kind"] == "shared":
            return P.attend_shared(s["q"], s["k_prefix"], s["v_prefix"], s["k"], s["v"], lens=s["lens"], q_lens=s["q_lens"],
                                   out=s["out"], lse_out=s["lse"])
        return P.attend(s["q"], s["k"], s["v"], lens=s["lens"], q_lens=s["q_lens"], window=c["window"], sinks=c["sinks"], out=s["out"],
                        lse_out=s["lse"], mass_in=s.get("mass"), mass_out=s.get("mass_out"), decay=c["decay"])
    if c["kind"] == "evict":
        return _plain_evict(s, c)
    return _plain_attend(s, c)


def _plain_attend(s, c):
    B, hq, n_q, d = s["q"].shape
    kv, g, T = c["kv_heads"], c["group"], c["capacity"]
    dev = s["q"].device
    lens, q_lens = s["lens"].long(), s["q_lens"].long()
    i, j = torch.arange(n_q, device=dev), torch.arange(T, device=dev)
    pos = (lens - q_lens)[:, None] + i                                      # [B, n_q]
    real = i < q_lens[:, None]
    seen = (j <= pos[..., None]) & (j < lens[:, None, None])                # [B, n_q, T]
    if c["window"]:
        seen &= (j > pos[..., None] - c["window"]) | (j < c["sinks"])
    seen &= real[..., None]
    q = s["q"].float().reshape(B, kv, g * n_q, d)
    x = torch.matmul(q, s["k"].float().transpose(-1, -2)).mul_(1.0 / math.sqrt(d))               # [B, kv, g * n_q, T]
    x.view(B, kv, g, n_q, T).masked_fill_(~seen[:, None, None], -math.inf)
    v = s["v"].float()
    if c["kind"] == "shared":
        kp, vp = s["k_prefix"].float(), s["v_prefix"].float()
        y = torch.matmul(q, kp.transpose(-1, -2)).mul_(1.0 / math.sqrt(d))
        top = torch.maximum(x.amax(-1, keepdim=True), y.amax(-1, keepdim=True))
        ex, ey = torch.exp(x - top), torch.exp(y - top)
        z = ex.sum(-1, keepdim=True) + ey.sum(-1, keepdim=True)
        out = (torch.matmul(ex, v) + torch.matmul(ey, vp)) / z
    else:
        top = x.amax(-1, keepdim=True).clamp_min(-3e38)
        ex = x.sub_(top).exp_()
        z = ex.sum(-1, keepdim=True)
        ex.div_(z.clamp_min(1e-38))
        out = torch.matmul(ex, v)
    lse = (top + torch.log(z)).squeeze(-1).reshape(B, hq, n_q)
    got = {"out": torch.where(real[:, None, :, None], out.reshape(B, hq, n_q, d), 0.0).to(s["q"].dtype),
           "lse": torch.where(real[:, None], lse, 0.0)}
    if c["mass"]:
        got["mass"] = torch.where(j < lens[:, None, None], c["decay"] * s["mass"] + ex.sum(2), 0.0)
    return got


def _plain_evict(s, c):
    T, keep = c["capacity"], c["keep"]
    lens = s["lens"].long()[:, None, None]
    j = torch.arange(T, device=s["k"].device)
    safe = (j < c["sinks"]) | (j >= lens - c["recent"])
    order = torch.where(safe, math.inf, s["mass"]).masked_fill(j >= lens, -math.inf)
    first = torch.sort(order, dim=-1, descending=True, stable=True)[1][..., :keep]
    r = torch.arange(keep, device=j.device)
    there = r[: first.shape[-1]] < torch.minimum(lens, torch.tensor(keep, device=j.device))
    idx = torch.where(there, first, T).sort(-1)[0]
    there = there.expand_as(idx)
    at = torch.where(there, idx, 0)
    rows = at[..., None].expand(*at.shape, c["dim"])
    return {"K_out": torch.where(there[..., None], torch.gather(s["k"], 2, rows), 0.0).to(s["k"].dtype),
            "V_out": torch.where(there[..., None], torch.gather(s["v"], 2, rows), 0.0).to(s["v"].dtype),
            "idx": at.to(torch.int32), "mass": torch.where(there, torch.gather(s["mass"], 2, at), 0.0),
            "lens": torch.clamp(s["lens"], max=keep)}


def _pairs(c):
    """(visible query-key pairs of a query head, keys of a sequence that some query sees, real queries), summed over the batch."""
    pairs = keys = real = 0
    for n in _lens(c):
        ql = min(c["n_q"], n)
        real += ql
        pos = np.arange(n - ql, n, dtype=np.int64)
        lo = np.maximum(0, pos - c["window"] + 1) if c["window"] else np.zeros_like(pos)
        pairs += int((pos - lo + 1 + np.minimum(lo, c["sinks"])).sum())
        keys += n - int(lo[0]) + min(int(lo[0]), c["sinks"])
    return pairs, keys, real


def work(c):
    e, d, kv, hq, B = (2 if c["dtype"] == "bf16" else 4), c["dim"], c["kv_heads"], c["kv_heads"] * c["group"], c["batch"]
    if c["kind"] == "evict":
        kept = sum(min(n, c["keep"]) for n in _lens(c))
        return {"bytes": kv * (4 * sum(_lens(c)) + kept * (4 * d * e + 8)) + 8 * B, "flops": 0}
    pairs, keys, real = _pairs(c)
    n_bytes = 2 * e * d * kv * (keys + c["prefix"]) + hq * real * (2 * d * e + 4) + 8 * B
    if c["mass"]:
        n_bytes += 8 * kv * sum(_lens(c))
    return {"bytes": n_bytes, "flops": 4 * d * hq * (pairs + real * c["prefix"])}


def exact(c, seed):
    """One head at a time, from the definitions, in 64 bits."""
    s = prepare(c, seed)
    lens, d = _lens(c), c["dim"]
    if c["kind"] == "evict":
        k_out, v_out, idx, mass = (torch.zeros_like(s[n], dtype=torch.float64) if n != "idx_out" else torch.zeros_like(s[n])
                                   for n in ("k_out", "v_out", "idx_out", "mass_out"))
        host = s["mass"].cpu().numpy()
        for b, n in enumerate(lens):
            m = min(n, c["keep"])
            for h in range(c["kv_heads"]):
                if m == n:
                    kept = np.arange(n)
                else:
                    mid = np.arange(c["sinks"], n - c["recent"])
                    best = mid[np.lexsort((mid, -host[b, h, mid].astype(np.float64)))][: m - c["sinks"] - c["recent"]]
                    kept = np.concatenate([np.arange(c["sinks"]), np.sort(best), np.arange(n - c["recent"], n)])
                at = torch.from_numpy(kept).to(s["k"].device)
                k_out[b, h, :m], v_out[b, h, :m] = s["k"][b, h, at].double(), s["v"][b, h, at].double()
                idx[b, h, :m], mass[b, h, :m] = at.to(torch.int32), s["mass"][b, h, at].double()
        return {"K_out": k_out, "V_out": v_out, "idx": idx, "mass": mass, "lens": torch.tensor([min(n, c["keep"]) for n in lens], dtype=torch.int32)}
    pairs, _, real = _pairs(c)
    if (pairs + real * c["prefix"]) * c["kv_heads"] * c["group"] > 1 << 34:
        return None
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros_like(s["lse"], dtype=torch.float64)
    mass = torch.zeros_like(s["mass"], dtype=torch.float64) if c["mass"] else None
    for b, n in enumerate(lens):
        ql = min(c["n_q"], n)
        at = torch.arange(n, device="cuda")
        p = torch.arange(n - ql, n, device="cuda")[:, None]
        hidden = at[None] > p
        if c["window"]:
            hidden = hidden | ((at[None] <= p - c["window"]) & (at[None] >= c["sinks"]))
        for h in range(c["kv_heads"]):
            K, V = s["k"][b, h, :n].double(), s["v"][b, h, :n].double()
            if c["kind"] == "shared":
                K, V = torch.cat([s["k_prefix"][h].double(), K]), torch.cat([s["v_prefix"][h].double(), V])
            total = torch.zeros(K.shape[0], dtype=torch.float64, device="cuda")
            for g in range(h * c["group"], (h + 1) * c["group"]):
                logit = s["q"][b, g, :ql].double() @ K.T / math.sqrt(d)
                logit[:, c["prefix"]:].masked_fill_(hidden, -math.inf)
                lse[b, g, :ql] = torch.logsumexp(logit, -1)
                w = torch.softmax(logit, -1)
                out[b, g, :ql] = w @ V
                total += w.sum(0)
            if mass is not None:
                mass[b, h, :n] = c["decay"] * s["mass"][b, h, :n].double() + total
    got = {"out": out, "lse": lse}
    if mass is not None:
        got["mass"] = mass
    return got
