"""The operators on a relayed cache held in 8 or 4 bits that are measured: quantising keys and values as they are written to it, reading
rows back, attention over it.

Each has its plain form in elementary torch operations (`own` false) and the library's call (`own` true), on the same inputs.
Rows are held by symmetric codes with a scale,

    8 bits: int8 codes, one fp32 scale a row:                   scale = max |x| / 127
    4 bits: two codes plus 8 in a byte, the lower channel in the lower half; one bfloat16 scale for the 32 channels c of a row
            that have the same (c / 4) mod (dim / 32):          scale = max |x| / 7, rounded to five significant bits

code = round-half-even(x / scale), value = code * scale.  (Five bits times a code of three: a value is a bfloat16 number itself.)
Shapes: q [batch, q_heads, n_q, dim], codes [batch, kv_heads, capacity, dim or dim / 2], q head = kv_head * group + g; sequence b
holds rows 0 .. lens[b] - 1, the rows written and the queries are the last of them.
"""
import math

import numpy as np
import torch

own = False          # set by whoever runs the cases: False = the plain forms, True = the library's calls

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _case(kind, name=None, **kw):
    base = dict(kind=kind, batch=1, kv_heads=8, group=4, dim=128, dtype="bf16", bits=4, n_new=1, capacity=1024, shortest=1024, token_major=False,
                window=0, sinks=0)
    base.update(kw)
    if name is not None:
        base["name"] = name
    return base


def listed():
    return [
        # the new token of each agent of a batch, appended to caches of different lengths: latency
        _case("write", "write_step", batch=32, capacity=8192, shortest=1024),
        # the relays of all layers of a model handed over in 8 bits, in caches with room for the next agent's latent steps
        _case("write", "write_relay", batch=36, n_new=1012, capacity=1052, shortest=1012, bits=8),
        # the prompts of a batch as they are computed, with the values that their own attention is to see
        _case("write", "write_prompts", batch=8, n_new=8192, capacity=8192, shortest=3001, token_major=True),
        # one short relay read back in full precision
        _case("read", "read_one", capacity=101, shortest=101, bits=8, dtype="f32"),
        # the grown caches of a batch read back to be compressed again
        _case("read", "read_batch", batch=16, capacity=8192, shortest=3001),
        # one agent's next token over a short relay: latency
        _case("attend", "step_one", capacity=1052, shortest=1013, window=256, sinks=4),
        # a served batch of agents at different lengths
        _case("attend", "step_batch", batch=32, capacity=8192, shortest=1024),
        # few agents with very long chains of relays
        _case("attend", "step_long", batch=4, capacity=131072, shortest=100001),
        # a batch over relays in 8 bits, a layer with a window and sinks
        _case("attend", "step_8_bits", batch=16, capacity=8192, shortest=7000, window=4096, sinks=4, bits=8),
        # five new tokens of each agent in full precision, heads of 64
        _case("attend", "step_f32", batch=16, n_new=5, capacity=8192, shortest=7000, dim=64, dtype="f32"),
        # 40 latent steps of each of eight agents at once, over relays in 8 bits
        _case("attend", "chunk_8_bits", batch=8, n_new=40, capacity=4136, shortest=4001, bits=8),
        # a prompt over the cache that it has just been written to
        _case("attend", "prompt", n_new=4096, capacity=4096, shortest=4096),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["write", "read", "step", "step", "chunk", "prompt"])
    kw = dict(dim=rng.choice([64, 128, 128]), kv_heads=rng.choice([1, 2, 4, 5, 8]), group=rng.choice([1, 2, 3, 4, 6, 7, 8]), bits=rng.choice([4, 4, 8]),
              dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]), token_major=rng.random() < 0.5)
    kv, g = kw["kv_heads"], kw["group"]
    if kind in ("write", "read"):
        batch = _log(rng, 1, 36)
        cap = _log(rng, 16, max(64, (1 << 18) // (batch * kv)))
        n_new = rng.choice([1, min(cap, 5), cap, rng.randint(1, cap)])
        return _case(kind, batch=batch, capacity=cap, shortest=rng.randint(max(1, cap // 4), cap), n_new=n_new, **kw)
    kw.update(window=rng.choice([0, _log(rng, 1, 8192)]), sinks=rng.choice([0, 1, 4, rng.randint(1, 200)]))
    if kind == "step":
        batch = _log(rng, 1, 64)
        cap = _log(rng, 16, max(16, min(131072, (1 << 22) // (batch * kv))))
        n_new = rng.choice([1, 1, 1, 2, 5])
    elif kind == "chunk":
        batch, n_new = _log(rng, 1, 16), rng.randint(6, 64)
        cap = _log(rng, 64, max(64, min(32768, (1 << 28) // (batch * n_new * kv * g))))
    else:
        batch = _log(rng, 1, 8)
        cap = n_new = _log(rng, 16, min(4096 if kw["dtype"] == "bf16" else 2048, int(math.sqrt((1 << 28) / (batch * kv * g)))))
    return _case("attend", batch=batch, capacity=cap, shortest=rng.randint(max(1, cap // 3), cap), n_new=n_new, **kw)


def _lens(c):
    """Lengths of the sequences, spread from the capacity down to the shortest."""
    span = c["capacity"] - c["shortest"]
    return [c["capacity"] - (span * b // max(1, c["batch"] - 1)) for b in range(c["batch"])]


def _five_bits(x):
    """Rounded, half to even, to five significant bits (fp32, not negative, no subnormal numbers)."""
    i = x.view(torch.int32)
    return ((i + 0x3FFFF + ((i >> 19) & 1)) & -0x80000).view(torch.float32)


def prepare(c, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    t, d, kv, B, cap, n_new, bits = TYPES[c["dtype"]], c["dim"], c["kv_heads"], c["batch"], c["capacity"], c["n_new"], c["bits"]

    def normal(*shape, dtype=t):
        return torch.randn(shape, generator=gen, device="cuda", dtype=dtype)

    def rows(heads, fill=normal):
        """[batch, heads, n_new, dim], the tokens outermost in memory or the heads."""
        return fill(B, n_new, heads, d).transpose(1, 2) if c["token_major"] else fill(B, heads, n_new, d)

    def zeros(*shape):
        return torch.zeros(shape, dtype=t, device="cuda")

    s = dict(c=c, lens=torch.tensor(_lens(c), dtype=torch.int32, device="cuda"))
    s["new"] = torch.tensor([min(n_new, n) for n in _lens(c)], dtype=torch.int32, device="cuda")
    if c["kind"] == "write":
        s["k"], s["v"] = rows(kv), rows(kv)
        s["k"][..., : d // 32].mul_(4.0)                                    # outlier channels, as caches have them
        s["k_values"], s["v_values"] = rows(kv, zeros), rows(kv, zeros)
        per = (B, kv, cap, d if bits == 8 else d // 2)
        s["codes"] = [torch.zeros(per, dtype=torch.int8 if bits == 8 else torch.uint8, device="cuda") for _ in range(2)]
        s["scales"] = [torch.zeros(per[:3] if bits == 8 else (*per[:3], d // 32), dtype=torch.float32 if bits == 8 else torch.bfloat16, device="cuda")
                       for _ in range(2)]
        return s
    s["codes"], s["scales"] = [], []
    for i in range(2):
        # codes of rows of normal numbers whose sizes vary by a third; a part of the keys' channels is four times as large
        if bits == 8:
            s["codes"].append(normal(B, kv, cap, d, dtype=torch.bfloat16).mul_(42.0).round_().clamp_(-127, 127).to(torch.int8))
            s["scales"].append(torch.exp(0.3 * normal(B, kv, cap, dtype=torch.float32)) * (0.04 if i == 0 else 0.024))
        else:
            code = normal(B, kv, cap, d, dtype=torch.bfloat16).mul_(2.9).round_().clamp_(-7, 7).add_(8).to(torch.uint8)
            s["codes"].append(code[..., ::2] | (code[..., 1::2] << 4))
            size = torch.exp(0.3 * normal(B, kv, cap, d // 32, dtype=torch.float32)) * 0.35
            if i == 0:
                size[..., 0] *= 4.0
            s["scales"].append(_five_bits(size).to(torch.bfloat16))
            del code, size
    if c["kind"] == "read":
        s["k_out"], s["v_out"] = zeros(B, kv, cap, d), zeros(B, kv, cap, d)
        return s
    hq = kv * c["group"]
    s["q"], s["out"] = rows(hq), rows(hq, zeros)
    s["lse"] = torch.zeros((B, hq, n_new), dtype=torch.float32, device="cuda")
    return s


def run(s):
    c = s["c"]
    if own:
        import paper_2604_13349_b200 as P
        cache = P.QuantizedCache(*s["codes"], *s["scales"])
        if c["kind"] == "write":
            P.write_quantized(cache, s["k"], s["v"], lens=s["lens"], new_lens=s["new"], k_values=s["k_values"], v_values=s["v_values"])
            return {"K": s["k_values"], "V": s["v_values"], "K_scale": s["scales"][0], "V_scale": s["scales"][1]}
        if c["kind"] == "read":
            return P.read_quantized(cache, lens=s["lens"], k_out=s["k_out"], v_out=s["v_out"])
        return P.attend_quantized(s["q"], cache, lens=s["lens"], q_lens=s["new"], window=c["window"], sinks=c["sinks"], out=s["out"], lse_out=s["lse"])
    if c["kind"] == "write":
        return _plain_write(s, c)
    if c["kind"] == "read":
        there = torch.arange(c["capacity"], device="cuda") < s["lens"][:, None, None]
        return {n: torch.where(there[..., None], _values(s, i), 0.0).to(TYPES[c["dtype"]]) for i, n in enumerate("KV")}
    return _plain_attend(s, c)


def _plain_write(s, c):
    B, kv, n, d = s["k"].shape
    i = torch.arange(n, device="cuda")
    real = i < s["new"].long()[:, None]                                     # [B, n]
    at = (s["lens"] - s["new"]).long()[:, None] + i
    b, r = torch.nonzero(real, as_tuple=True)                               # the rows that are written, and where to
    to = at[b, r]
    got = {}
    for k, name in enumerate("KV"):
        x = s["kv"[k]].float()
        if c["bits"] == 8:
            scale = x.abs().amax(-1, keepdim=True) / 127.0
            code = torch.round(x / scale)
            value, kept = code * scale, scale.squeeze(-1)
            s["codes"][k][b, :, to] = code.to(torch.int8).transpose(1, 2)[b, r]
        else:
            u = x.reshape(B, kv, n, 8, d // 32, 4)
            scale = _five_bits(u.abs().amax((3, 5), keepdim=True) / 7.0)
            code = torch.round(u / scale)
            value, kept = (code * scale).reshape(x.shape), scale.reshape(B, kv, n, d // 32).to(torch.bfloat16)
            byte = (code + 8.0).to(torch.uint8).reshape(B, kv, n, d)
            s["codes"][k][b, :, to] = (byte[..., ::2] | (byte[..., 1::2] << 4)).transpose(1, 2)[b, r]
        s["scales"][k][b, :, to] = kept.transpose(1, 2)[b, r]
        got[name] = torch.where(real[:, None, :, None], value, 0.0).to(s["k"].dtype)
        got[name + "_scale"] = s["scales"][k]
    return {n: got[n] for n in ("K", "V", "K_scale", "V_scale")}


def _values(s, i):
    """The cache's keys (0) or values (1), fp32."""
    codes, scale = s["codes"][i], s["scales"][i].float()
    if codes.dtype == torch.int8:
        return codes.float() * scale[..., None]
    x = torch.stack([codes & 15, codes >> 4], -1).float() - 8.0             # [B, kv, T, d / 2, 2]
    return (x.reshape(*codes.shape[:3], 8, -1, 4) * scale[..., None, :, None]).reshape(*codes.shape[:3], -1)


def _plain_attend(s, c):
    B, hq, n_q, d = s["q"].shape
    kv, g, T = c["kv_heads"], c["group"], c["capacity"]
    lens, q_lens = s["lens"].long(), s["new"].long()
    i, j = torch.arange(n_q, device="cuda"), torch.arange(T, device="cuda")
    pos = (lens - q_lens)[:, None] + i                                      # [B, n_q]
    real = i < q_lens[:, None]
    seen = (j <= pos[..., None]) & real[..., None]                          # [B, n_q, T]
    if c["window"]:
        seen &= (j > pos[..., None] - c["window"]) | (j < c["sinks"])
    q = s["q"].float().reshape(B, kv, g * n_q, d)
    x = torch.matmul(q, _values(s, 0).transpose(-1, -2)).mul_(1.0 / math.sqrt(d))                # [B, kv, g * n_q, T]
    x.view(B, kv, g, n_q, T).masked_fill_(~seen[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True).clamp_min(-3e38)
    x = x.sub_(top).exp_()
    z = x.sum(-1, keepdim=True)
    out = torch.matmul(x, _values(s, 1)) / z.clamp_min(1e-38)
    lse = (top + torch.log(z)).squeeze(-1).reshape(B, hq, n_q)
    return {"out": torch.where(real[:, None, :, None], out.reshape(B, hq, n_q, d), 0.0).to(s["q"].dtype), "lse": torch.where(real[:, None], lse, 0.0)}


def _pairs(c):
    """(visible query-key pairs of a query head, keys of a sequence that some query sees, real queries), summed over the batch."""
    pairs = keys = real = 0
    for n in _lens(c):
        ql = min(c["n_new"], n)
        real += ql
        pos = np.arange(n - ql, n, dtype=np.int64)
        lo = np.maximum(0, pos - c["window"] + 1) if c["window"] else np.zeros_like(pos)
        pairs += int((pos - lo + 1 + np.minimum(lo, c["sinks"])).sum())
        keys += n - int(lo[0]) + min(int(lo[0]), c["sinks"])
    return pairs, keys, real


def work(c):
    e, d, kv, hq, B = (2 if c["dtype"] == "bf16" else 4), c["dim"], c["kv_heads"], c["kv_heads"] * c["group"], c["batch"]
    row = d + 4 if c["bits"] == 8 else d // 2 + d // 16                     # bytes of a row of the cache
    if c["kind"] == "write":
        return {"bytes": 2 * kv * sum(min(c["n_new"], n) for n in _lens(c)) * (2 * e * d + row) + 8 * B, "flops": 0}
    if c["kind"] == "read":
        return {"bytes": 2 * kv * sum(_lens(c)) * (e * d + row) + 4 * B, "flops": 0}
    pairs, keys, real = _pairs(c)
    return {"bytes": 2 * kv * keys * row + hq * real * (2 * d * e + 4) + 8 * B, "flops": 4 * d * hq * pairs}


def _held(s, i, b, h, n):
    """The first n rows of a head of the cache, from the format's definition, in 64 bits."""
    codes, scale = s["codes"][i][b, h, :n].cpu().numpy(), s["scales"][i][b, h, :n].double().cpu().numpy()
    if codes.dtype == np.int8:
        return torch.from_numpy(codes.astype(np.float64) * scale[:, None]).cuda()
    d = 2 * codes.shape[1]
    x = np.empty((n, d))
    x[:, 0::2], x[:, 1::2] = (codes % 16).astype(np.float64) - 8, (codes // 16).astype(np.float64) - 8
    return torch.from_numpy(x * scale[:, (np.arange(d) // 4) % (d // 32)]).cuda()


def _exact_write(s, c):
    B, kv, n_new, d = s["k"].shape
    out = {n: torch.zeros((B, kv, n_new, d), dtype=torch.float64) for n in "KV"}
    kept = {n: torch.zeros(s["scales"][0].shape, dtype=torch.float64) for n in "KV"}
    group = (np.arange(d) // 4) % (d // 32)
    for b, n in enumerate(_lens(c)):
        m = min(n_new, n)
        for k, name in enumerate("KV"):
            x = s["kv"[k]][b, :, :m].double().cpu().numpy()                 # [kv, m, d]
            if c["bits"] == 8:
                # the scale is the fp32 number nearest to max / 127, the code the whole number nearest to the fp32 quotient
                scale = (np.abs(x).max(-1, keepdims=True) / 127).astype(np.float32)
                code = np.rint(x.astype(np.float32) / scale).astype(np.float64)
                value, held = code * scale, scale[..., 0]
            else:
                held = np.stack([np.abs(x[..., group == j]).max(-1) for j in range(d // 32)], -1) / 7
                mantissa, exponent = np.frexp(held)
                held = np.ldexp(np.rint(mantissa * 32), exponent - 5)
                value = np.rint(x / held[..., group]) * held[..., group]
            out[name][b, :, :m] = torch.from_numpy(value.astype(np.float64))
            kept[name][b, :, n - m : n] = torch.from_numpy(held.astype(np.float64))
    return {"K": out["K"], "V": out["V"], "K_scale": kept["K"], "V_scale": kept["V"]}


def exact(c, seed):
    """One head at a time, from the definitions, in 64 bits."""
    lens, d, kv = _lens(c), c["dim"], c["kv_heads"]
    if c["kind"] != "attend" and kv * d * sum(lens if c["kind"] == "read" else [min(c["n_new"], n) for n in lens]) > 1 << 27:
        return None
    pairs, keys, _ = _pairs(c)
    if c["kind"] == "attend" and (pairs * kv * c["group"] > 1 << 33 or keys * kv * d > 1 << 30):
        return None
    s = prepare(c, seed)
    if c["kind"] == "write":
        return _exact_write(s, c)
    if c["kind"] == "read":
        got = {n: torch.zeros(s["k_out"].shape, dtype=torch.float64) for n in "KV"}
        for b, n in enumerate(lens):
            for h in range(kv):
                got["K"][b, h, :n], got["V"][b, h, :n] = _held(s, 0, b, h, n), _held(s, 1, b, h, n)
        return got
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros_like(s["lse"], dtype=torch.float64)
    for b, n in enumerate(lens):
        ql = min(c["n_new"], n)
        at = torch.arange(n, device="cuda")
        p = torch.arange(n - ql, n, device="cuda")[:, None]
        hidden = at[None] > p
        if c["window"]:
            hidden = hidden | ((at[None] <= p - c["window"]) & (at[None] >= c["sinks"]))
        for h in range(kv):
            K, V = _held(s, 0, b, h, n), _held(s, 1, b, h, n)
            for g in range(h * c["group"], (h + 1) * c["group"]):
                logit = (s["q"][b, g, :ql].double() @ K.T / math.sqrt(d)).masked_fill_(hidden, -math.inf)
                lse[b, g, :ql] = torch.logsumexp(logit, -1)
                out[b, g, :ql] = torch.softmax(logit, -1) @ V
    return {"out": out, "lse": lse}
