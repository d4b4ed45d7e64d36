"""Plain 64-bit references of packed-prompt attention, its gradients and the paged cache, with the sums of magnitudes that the
tests' tolerances are made of.  Test infrastructure: no code of the library.

Roundings, by the size of the type: bf16 is off by at most 2^-8 of a value, e4m3 by 2^-4 (2^-10 of its scale below 2^-6), fp32 by 2^-24.
"""
import math

import torch

U16, U32 = 2.0 ** -8, 2.0 ** -24


def rows_of(heads, group):
    return [(a, a // group) for a in range(heads)]


def attention(Q, K, V, q_len, k_len, causal=True, q0=0, k0=0):
    """Q [Tq, Hq, D], K, V [Tk, Hkv, D] (any type) -> dict of fp64: O, lse, and per row: A = sum p |v|, and `off`, by how much a
    weight may be off through its score: fp32 accumulation of D products, the scale, the exponential."""
    Hq, D, Hkv = Q.shape[1], Q.shape[2], K.shape[1]
    G = Hq // Hkv
    r = {"O": torch.zeros(Q.shape, dtype=torch.float64, device=Q.device), "A": torch.zeros(Q.shape, dtype=torch.float64, device=Q.device),
         "lse": torch.full(Q.shape[:2], -math.inf, dtype=torch.float64, device=Q.device),
         "off": torch.zeros(Q.shape[:2], dtype=torch.float64, device=Q.device)}
    for n, m in zip(q_len, k_len):
        for a in range(Hq):
            q, k, v = Q[q0:q0 + n, a].double(), K[k0:k0 + m, a // G].double(), V[k0:k0 + m, a // G].double()
            if n and m:
                s = q @ k.T / math.sqrt(D)
                big = q.abs() @ k.abs().T / math.sqrt(D)
                if causal:
                    s = s.masked_fill(torch.arange(m, device=s.device) > (m - n + torch.arange(n, device=s.device))[:, None], -math.inf)
                lse = torch.logsumexp(s, -1)
                p = torch.where(torch.isneginf(lse)[:, None], torch.zeros_like(s), torch.exp(s - lse[:, None]))
                r["O"][q0:q0 + n, a], r["A"][q0:q0 + n, a] = p @ v, p @ v.abs()
                r["lse"][q0:q0 + n, a] = lse
                # D products and sums, the scale, the reference (as large as a score), the exponential (a few units)
                r["off"][q0:q0 + n, a] = U32 * ((D + 4) * big.amax(-1) + 16)
        q0, k0 = q0 + n, k0 + m
    return r


def output_bound(ref):
    """Of O: the weights' rounding to bf16 and their own error, in numerator and sum; the output's rounding."""
    return U16 * ref["O"].abs() + ref["A"] * (U16 + 4 * ref["off"][..., None]) * (1 + U16) + 1e-30


def lse_bound(ref, keys):
    """Of the log-sum-exp: the scores' errors, the sum of `keys` weights in fp32, the logarithm and the last sum."""
    lse = ref["lse"].abs().nan_to_num(posinf=0.0)
    return 2 * ref["off"] + U32 * (keys + 8) + 8 * U32 * (lse + 16)


def gradients(Q, K, V, O, lse, dO, q_len, k_len, causal=True):
    """The formulas of the backward on the O and lse that it is given -> fp64 dQ, dK, dV and their bounds.

    sum_j dS_j = sum_j p_j dP_j - delta is 0 for the delta that belongs to p; with delta from an O rounded to bf16 something is left of it, and the
    library takes that out of dQ along r, the mean of up to 64 keys of the sequence: dQ = c sum_j dS_j (k_j - r).  In rows of up to 64 keys
    delta is that sum."""
    Hq, D, Hkv = Q.shape[1], Q.shape[2], K.shape[1]
    G, c = Hq // Hkv, 1 / math.sqrt(Q.shape[2])
    out = {n: torch.zeros(t.shape, dtype=torch.float64, device=Q.device) for n, t in (("dQ", Q), ("dK", K), ("dV", V))}
    tol = {n: torch.zeros_like(t) for n, t in out.items()}
    q0 = k0 = 0
    for n, m in zip(q_len, k_len):
        for a in range(Hq):
            if not n or not m:
                continue
            at, kt = (slice(q0, q0 + n), a), (slice(k0, k0 + m), a // G)
            q, k, v, o, g = Q[at].double(), K[kt].double(), V[kt].double(), O[at].double(), dO[at].double()
            l = lse[at].double()
            s, big = q @ k.T * c, q.abs() @ k.abs().T * c
            if causal:
                s = s.masked_fill(torch.arange(m, device=s.device) > (m - n + torch.arange(n, device=s.device))[:, None], -math.inf)
            p = torch.where(torch.isneginf(l)[:, None], torch.zeros_like(s), torch.exp(s - l[:, None]))
            dp, delta = g @ v.T, (g * o).sum(-1, keepdim=True)
            off = U32 * ((D + 4) * big + 4 * l.abs().nan_to_num(posinf=0.0)[:, None] + 16)      # of p, relative
            ddp = U32 * (D + 4) * (g.abs() @ v.abs().T + (g * o).abs().sum(-1, keepdim=True))   # of dp - delta
            # rows of up to 64 keys: off by p's and dP's errors, and those of up to 64 products and sums
            few_keys = (torch.ones_like(p).masked_fill(torch.isneginf(s), 0).sum(-1, keepdim=True) <= 64)
            delta = torch.where(few_keys, (p * dp).sum(-1, keepdim=True), delta)
            e_dp = U32 * (D + 4) * (g.abs() @ v.abs().T)
            e_delta = (p * (e_dp + dp.abs() * off)).sum(-1, keepdim=True) + U32 * 72 * (p * dp.abs()).sum(-1, keepdim=True)
            ddp = torch.where(few_keys, e_dp + e_delta + U32 * (dp.abs() + delta.abs()), ddp)
            ds = p * (dp - delta)
            e_ds = ds.abs() * (U16 + off) + p * ddp * (1 + U16)                                 # dS in bf16
            e_p = p * (U16 + off)
            few = min(m, 64)
            r = k[torch.arange(few, device=k.device) * m // few].mean(0)
            out["dQ"][at] += c * (ds @ k - ds.sum(-1, keepdim=True) * r)
            out["dK"][kt] += c * ds.T @ q
            out["dV"][kt] += p.T @ g
            n32 = 2 * U32 * (m + 4), 2 * U32 * (n * G + 4)  # sums in fp32
            tol["dQ"][at] += c * (e_ds + ds.abs() * n32[0]) @ (k.abs() + r.abs())
            tol["dK"][kt] += c * (e_ds + ds.abs() * n32[1]).T @ q.abs()
            tol["dV"][kt] += (e_p + p * n32[1]).T @ g.abs()
        q0, k0 = q0 + n, k0 + m
    return out, {n: (t * (1 + U16) + U16 * out[n].abs() + 1e-30) for n, t in tol.items()}


def e4m3(x):
    """The nearest e4m3 values, ties to even, of fp64 x."""
    e = torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -30))).clamp_min(-6.0)
    step = torch.exp2(e - 3)
    return (torch.round(x / step) * step).clamp(-448, 448)


def starts(lengths, first=0):
    s = [first]
    for n in lengths:
        s.append(s[-1] + n)
    return torch.tensor(s, dtype=torch.int32)
