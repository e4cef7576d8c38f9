"""Plain 64-bit forms of the attention operators (numpy-like torch on the CPU), and how far results in 16 and 32 bits may be from
them.  Written from the formulas in include/tmac_attn.h."""
import math

import torch

UNIT = {t: torch.finfo(t).eps / 2 for t in (torch.float16, torch.bfloat16)}  # half the distance from 1 to the next number


def rows(q, k, v, scale, sees):
    """q [n, D] over k, v [m, D] with the truth values `sees` [n, m]: out, lse, weights [n, m], bound of the result's error,
    bound of the scores' error per row."""
    q, k, v = q.double(), k.double(), v.double()
    s = torch.where(sees, (q @ k.t()) * scale, -math.inf)
    top = s.amax(dim=1, keepdim=True) if s.shape[1] else torch.full((s.shape[0], 1), -math.inf, dtype=torch.float64)
    safe = torch.where(top == -math.inf, 0.0, top)
    e = torch.exp(s - safe)
    total = e.sum(dim=1, keepdim=True)
    p = torch.where(total > 0, e / total, 0.0)
    out = p @ torch.where(sees.any(0)[:, None], v, 0.0) if v.shape[0] else torch.zeros((q.shape[0], v.shape[1]), dtype=torch.float64)
    lse = (total.log() + safe)[:, 0]
    return out, lse, p


def bounds(q, k, v, scale, sees, p, dtype):
    """Largest errors of (out [n, D], lse [n], a weight relative to itself [n]).

    Scores: D products, each sum rounded to 32 bits (u = 2^-24), so |ds| <= (D + 2) u scale sum |q_d k_d|; the exponent's argument
    and the exponential itself add a few u of the argument's size.  out: every exponential and the result are rounded once to
    the type's unit U, the exponentials below the type's normal range by at most 2^-25 of the largest: (2 U + 2 ds) sum p |v| +
    n 2^-25 max |v| 2^8 (the largest may be 2^8 times the one the sums are taken against... in either direction)."""
    u = 2.0 ** -24
    q, k, v = q.double().abs(), k.double().abs(), v.double().abs()
    size = torch.where(sees, (q @ k.t()) * scale, 0.0)
    most = size.amax(dim=1) if size.shape[1] else torch.zeros(q.shape[0], dtype=torch.float64)
    ds = (q.shape[1] + 2) * u * most + 8 * u * (1 + most)
    vmax = v.amax() if v.numel() else 0.0
    unit = UNIT[dtype]
    sub = sees.sum(1).double()[:, None] * (2.0 ** -24 if dtype == torch.float16 else 0.0) * vmax
    out = (2.1 * unit + 4 * ds[:, None]) * (p @ v) + sub + 2.0 ** -24
    return out, ds * 2 + 16 * u * (1 + most) + 2.0 ** -21, 4 * ds + 2.0 ** -18


def prompt(q, k, v, cu_q, cu_k, causal, scale):
    """(out, lse [Hq, Tq], weight [Hkv, Tk], and the bounds of each) of packed sequences on the CPU."""
    (Tq, Hq, D), (Tk, Hkv, _) = q.shape, k.shape
    G = Hq // Hkv
    out, out_b = torch.zeros((Tq, Hq, D), dtype=torch.float64), torch.zeros((Tq, Hq, D), dtype=torch.float64)
    lse, lse_b = torch.zeros((Hq, Tq), dtype=torch.float64), torch.zeros((Hq, Tq), dtype=torch.float64)
    w, w_b = torch.zeros((Hkv, Tk), dtype=torch.float64), torch.zeros((Hkv, Tk), dtype=torch.float64)
    for b in range(len(cu_q) - 1):
        qs, ks = slice(cu_q[b], cu_q[b + 1]), slice(cu_k[b], cu_k[b + 1])
        nq, nk = cu_q[b + 1] - cu_q[b], cu_k[b + 1] - cu_k[b]
        i, j = torch.arange(nq)[:, None], torch.arange(nk)[None]
        sees = j <= i + nk - nq if causal else torch.ones((nq, nk), dtype=torch.bool)
        for h in range(Hq):
            args = q[qs, h], k[ks, h // G], v[ks, h // G], scale, sees
            out[qs, h], lse[h, qs], p = rows(*args)
            out_b[qs, h], lse_b[h, qs], rel = bounds(*args, p, q.dtype)
            w[h // G, ks] += p.sum(0)
            w_b[h // G, ks] += (p * rel[:, None]).sum(0)
    return out, lse, w, out_b, lse_b, w_b + 2.0 ** -18 * w + 1e-30


def decode(q, k0, v0, k, v, lens, scale):
    """(out, lse [B, Hq], weight [B, Hkv, C], and the bounds of each); k0 and v0 may be None."""
    (B, Hq, D), (_, Hkv, C, _) = q.shape, k.shape
    G = Hq // Hkv
    out, out_b = torch.zeros((B, Hq, D), dtype=torch.float64), torch.zeros((B, Hq, D), dtype=torch.float64)
    lse, lse_b = torch.zeros((B, Hq), dtype=torch.float64), torch.zeros((B, Hq), dtype=torch.float64)
    w, w_b = torch.zeros((B, Hkv, C), dtype=torch.float64), torch.zeros((B, Hkv, C), dtype=torch.float64)
    for b in range(B):
        for h in range(Hkv):
            n, hs = int(lens[b, h]), slice(h * G, (h + 1) * G)
            keys, vals = k[b, h, :n], v[b, h, :n]
            if k0 is not None:
                keys, vals = torch.cat([k0[:, h], keys]), torch.cat([v0[:, h], vals])
            args = q[b, hs], keys, vals, scale, torch.ones((G, len(keys)), dtype=torch.bool)
            out[b, hs], lse[b, hs], p = rows(*args)
            out_b[b, hs], lse_b[b, hs], rel = bounds(*args, p, q.dtype)
            w[b, h, :n] = p.sum(0)[len(keys) - n:]
            w_b[b, h, :n] = (p * rel[:, None]).sum(0)[len(keys) - n:]
    return out, lse, w, out_b, lse_b, w_b + 2.0 ** -18 * w + 1e-30


def leaving(weight, pos, seen, recent):
    """Slots in the order in which eviction takes them."""
    def key(i):
        w = float(weight[i])
        return (int(pos[i]) >= seen - recent, -math.inf if math.isnan(w) else w, i)
    return sorted(range(len(weight)), key=key)
