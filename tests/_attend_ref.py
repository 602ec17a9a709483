"""Plain 64-bit form of the operators on a relayed cache, with the error bounds that their results are held to.

`attend` computes, beside every result, a bound on how far the library's may be from it:

    logits    products of the inputs are exact in fp32; a sum of d of them in fp32 is off by at most d 2^-23 sum |q_c k_c| (each of the
              d additions rounds or, on the tensor cores, cuts off the last bit), the scaling adds 2^-22 of the logit: ex
    weights   2^x of a logit that is off by ex log2(e) is off by ex, relatively, the reference (lse) likewise: 2 ex; exponentials
              and divisions add a few units of 2^-22; bf16 weights one half step, 2^-8
    sums      n terms in fp32: n 2^-24 of the sum of magnitudes
    out       the weights' error times sum_j p_j |v_j|, and half a step of the output's type
"""
import math

import torch

STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def attend(q, k, v, lens, q_lens, window=0, sinks=0, scale=None, prefix=None, mass_in=None, decay=1.0, want_mass=False, weight_step=None):
    """CPU tensors of the library's types; lens, q_lens lists.  Returns (out, out_tol, lse, lse_tol, mass, mass_tol), float64, zeros
    behind the lengths."""
    B, hq, n_q, d = q.shape
    kv, cap = k.shape[1], k.shape[2]
    G = hq // kv
    scale = 1.0 / math.sqrt(d) if not scale else scale
    ws = STEP[q.dtype] if weight_step is None else weight_step
    out = torch.zeros(B, hq, n_q, d, dtype=torch.float64)
    out_tol = torch.zeros_like(out)
    lse = torch.zeros(B, hq, n_q, dtype=torch.float64)
    lse_tol = torch.zeros_like(lse)
    mass = torch.zeros(B, kv, cap, dtype=torch.float64)
    mass_tol = torch.zeros_like(mass)
    for b in range(B):
        n, ql = lens[b], q_lens[b]
        P = 0 if prefix is None else prefix[0].shape[1]
        t = torch.arange(ql)[:, None] + (n - ql)
        j = torch.arange(n)[None]
        sees = j <= t
        if window:
            sees = sees & ((j > t - window) | (j < sinks))
        sees = torch.cat([torch.ones(ql, P, dtype=torch.bool), sees], 1)
        for h in range(kv):
            K, V = k[b, h, :n].double(), v[b, h, :n].double()
            if P:
                K, V = torch.cat([prefix[0][h].double(), K]), torch.cat([prefix[1][h].double(), V])
            seen = sees.any(0)
            K, V = torch.where(seen[:, None], K, 0.0), torch.where(seen[:, None], V, 0.0)       # what nobody sees may hold anything
            if mass_in is not None:
                mass[b, h, :n] = decay * mass_in[b, h, :n].double()
            for g in range(h * G, (h + 1) * G):
                Q = q[b, g, :ql].double()
                x = (Q @ K.T * scale).masked_fill(~sees, -math.inf)
                ex = (d * 2.0 ** -23 * scale) * (Q.abs() @ K.abs().T) + 2.0 ** -22 * (Q @ K.T * scale).abs()
                ex = (ex * sees).amax(1, keepdim=True) if ex.shape[1] else torch.zeros(ql, 1, dtype=torch.float64)
                l = torch.logsumexp(x, 1, keepdim=True) if x.shape[1] else torch.full((ql, 1), -math.inf, dtype=torch.float64)
                p = torch.where(sees, torch.exp(x - torch.where(l > -math.inf, l, 0.0)), 0.0)
                rel = 2 * ex + (P + n) * 2.0 ** -24 + 2.0 ** -20
                out[b, g, :ql] = p @ V
                out_tol[b, g, :ql] = (rel + ws) * (p @ V.abs()) + STEP[q.dtype] * (p @ V).abs() + 1e-30
                lse[b, g, :ql] = l[:, 0]
                lse_tol[b, g, :ql] = (rel + 2.0 ** -22 * torch.where(l > -math.inf, l, 0.0).abs())[:, 0]
                if want_mass:
                    mass[b, h, :n] += p.sum(0)[P:]
                    mass_tol[b, h, :n] += (p * rel).sum(0)[P:]
            mass_tol[b, h, :n] += 2.0 ** -22 * mass[b, h, :n].abs()
    return out, out_tol, lse, lse_tol, mass, mass_tol


def evict(mass, lens, keep, sinks, recent):
    """Kept positions of every (sequence, head), ascending, by repeated search for the heaviest (CPU tensor of fp32 masses)."""
    got = []
    for b, n in enumerate(lens):
        per = []
        for h in range(mass.shape[1]):
            if n <= keep:
                per.append(list(range(n)))
                continue
            kept = set(range(sinks)) | set(range(n - recent, n))
            rest = sorted((j for j in range(n) if j not in kept),
                          key=lambda j: (not math.isnan(float(mass[b, h, j])), float(mass[b, h, j]) if not math.isnan(float(mass[b, h, j])) else 0.0, -j),
                          reverse=True)
            per.append(sorted(kept | set(rest[: keep - len(kept)])))
        got.append(per)
    return got
