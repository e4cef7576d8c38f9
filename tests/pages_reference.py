"""Plain forms of the paged cache and the rotation, written from include/tmac_pages.h, and how far results may be from them.  On the CPU:
angles, products and attention in 64 bits; codes in the 32 bits that they are defined in."""
import math

import torch

BT = 32
UNIT = {t: torch.finfo(t).eps / 2 for t in (torch.float16, torch.bfloat16)}  # half the distance from 1 to the next number
MOST = {"i8": 127.0, "e4m3": 448.0}


def turned(x, positions, freq, magnitude, interleaved):
    """x [T, H, D] turned, in 64 bits."""
    x, rot = x.double().clone(), 2 * len(freq)
    a = positions.double()[:, None, None] * freq.double()
    c, s = torch.cos(a) * magnitude, torch.sin(a) * magnitude
    at = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    u, v = x[..., at[0]].clone(), x[..., at[1]].clone()
    x[..., at[0]], x[..., at[1]] = u * c - v * s, v * c + u * s
    return x


def turned_bound(x, freq, magnitude, interleaved):
    """How far 32-bit arithmetic may be from it before the last rounding: cosines and sines are rounded once (half a unit 2^-24 of at most the
    magnitude), each of the two products and their sum once (half a unit of the size of what is added); the angle's error in 64 bits, 2^-52 of it or
    2^-30 at angles of 2^22, and the polynomials' are far below: together at most 1.5 * 2^-24 (|u| + |v|) magnitude, of which twice is allowed."""
    x, rot = x.double().abs(), 2 * len(freq)
    at = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    b = torch.zeros_like(x)
    both = (x[..., at[0]] + x[..., at[1]]) * abs(magnitude) * 3 * 2.0 ** -24
    b[..., at[0]], b[..., at[1]] = both, both
    return b


def rounding(ref, dtype):
    """Of a result that is rounded once: half a step, and half the smallest number of fp16."""
    return ref.abs() * UNIT[dtype] * (1 + 2.0 ** -10) + (2.0 ** -25 if dtype == torch.float16 else 2.0 ** -134)


# --- codes ------------------------------------------------------------------------------------------------------------------------------


def scale_for(code, most):
    most = most.float()
    if code == "i8":
        return (most * torch.tensor(1.0 / 127.0)).clamp(min=2.0 ** -60)
    # 448 = 0.875 * 2^9: the least power of two, times which 448 reaches `most`
    out = torch.full_like(most, 2.0 ** -60)
    for i in range(most.numel()):
        m = float(most.view(-1)[i])
        if m > 0:
            f, e = math.frexp(m)
            out.view(-1)[i] = 2.0 ** max(-60, e - 9 + (f > 0.875))
    return out


def rounded(code, y):
    """32-bit numbers at the nearest value that a code stands for; infinities at the largest, NaN at zero."""
    y = torch.where(y.isnan(), 0.0, y)
    if code == "i8":
        return y.round().clamp(-127, 127)
    return y.clamp(-448, 448).to(torch.float8_e4m3fn).float()


class Held:
    """Pages as dictionaries: (page, block of the page, head, 0 keys or 1 values) -> (values of the codes [32, D], scale)."""

    def __init__(self, code, page, pages, D):
        self.code, self.page, self.pages, self.D, self.blocks = code, page, pages, D, {}

    def place(self, row, token):
        at = token // self.page
        if token < 0 or at >= len(row) or not 0 <= int(row[at]) < self.pages:
            return None
        return int(row[at]), token % self.page // BT

    def append(self, k, v, table, lens, cu, most=None):
        """k, v [T, Hkv, D] in 32 bits as they are to be held."""
        for s in range(len(lens)):
            r0, r1, m = int(cu[s]), int(cu[s + 1]), int(lens[s])
            first = m - (r1 - r0)
            tokens = [t for t in range(max(first, 0), m) if self.place(table[s], t)]
            for b in sorted({t // BT for t in tokens}):
                new = [t for t in tokens if t // BT == b]
                rows = [r0 + t - first for t in new]
                for h in range(k.shape[1]):
                    for which, x in ((0, k), (1, v)):
                        key = (*self.place(table[s], b * BT), h, which)
                        x = x[rows, h].float()
                        most = torch.where(x.isfinite(), x.abs(), 0.0).amax()
                        codes, was = torch.zeros(BT, self.D), 0.0
                        if new[0] % BT:
                            codes, was = self.blocks.get(key, (codes, torch.tensor(0.0)))
                        scale = torch.maximum(torch.as_tensor(was, dtype=torch.float32), scale_for(self.code, most))
                        codes = rounded(self.code, codes * (torch.as_tensor(was, dtype=torch.float32) / scale))
                        codes[[t % BT for t in new]] = rounded(self.code, x * (1.0 / scale))
                        self.blocks[key] = codes, scale

    def values(self, table, n, h, which):
        """Tokens 0 .. n - 1 of a sequence: (codes' values [n, D], scales [n], whether there are such)."""
        codes, scales, there = torch.zeros(n, self.D, dtype=torch.float64), torch.ones(n, dtype=torch.float64), torch.zeros(n, dtype=torch.bool)
        for t in range(n):
            at = self.place(table, t)
            if at is not None:
                there[t] = True
                got = self.blocks.get((*at, h, which))
                if got is not None:
                    codes[t], scales[t] = got[0][t % BT].double(), float(got[1])
        return codes, scales, there


def decoded(cache):
    """What the buffers of a PagedCache hold, by the header's description of them, as a Held."""
    code = "i8" if cache.cache.code == 0 else "e4m3"
    pages, Hkv, blocks, _ = cache.codes.shape
    D, c = cache.D, (cache.D + 15) // 16
    held = Held(code, cache.page, pages, D)
    raw, scales = cache.codes.cpu(), cache.scales.cpu()
    d, t = torch.arange(D)[None], torch.arange(BT)[:, None]
    run = torch.where(c * 16 - d // 32 * 32 < 32, 16, 32)
    at = [(d // 16) * 512 + t * 16 + d % 16,
          512 * c + (d // 32) * 1024 + ((t // 4) % 2 * run + d % 32) * 16 + 8 * (t // 8 % 2) + 4 * (t // 16) + t % 4]
    kind = torch.int8 if code == "i8" else torch.float8_e4m3fn
    for p in range(pages):
        for h in range(Hkv):
            for b in range(blocks):
                for which in (0, 1):
                    held.blocks[p, b, h, which] = raw[p, h, b][at[which]].view(kind).float(), scales[p, h, b, which]
    return held


# --- attention --------------------------------------------------------------------------------------------------------------------------


def attend(q, held, table, lens, cu, scale, Hkv):
    """(out, lse [Hq, T], bounds of each) of rows [cu[0], cu[S]) on the CPU, in 64 bits.

    Bounds.  Scores: D products of numbers that are exact, each sum rounded to 32 bits (u = 2^-24): |ds| <= (D + 2) u scale sum |q_d k_d|, the
    exponent's argument and exponential a few u of the argument's size (the values' scale is part of it: log2 of it, up to 60, too).  out:
    products of exponentials and scales are rounded to fp16 (2^-11 relative, below 2^-20 of the row's largest 2^-31 of that) and the
    result once."""
    (T, Hq, D), u = q.shape, 2.0 ** -24
    G, dtype = Hq // Hkv, q.dtype
    out, out_b = torch.zeros((T, Hq, D), dtype=torch.float64), torch.zeros((T, Hq, D), dtype=torch.float64)
    lse, lse_b = torch.full((Hq, T), -math.inf, dtype=torch.float64), torch.zeros((Hq, T), dtype=torch.float64)
    for s in range(len(lens)):
        r0, r1, m = int(cu[s]), int(cu[s + 1]), int(lens[s])
        n = min(m, len(table[s]) * held.page)
        for h in range(Hkv):
            (kc, ks, there), (vc, vs, _) = held.values(table[s], n, h, 0), held.values(table[s], n, h, 1)
            k, v = kc * ks[:, None], vc * vs[:, None]
            sees = (torch.arange(n)[None] <= torch.arange(m - (r1 - r0), m)[:, None]) & there[None]
            for g in range(G):
                x = q[r0:r1, h * G + g].double()
                a = torch.where(sees, (x @ k.t()) * scale, -math.inf)
                size = torch.where(sees, (x.abs() @ k.abs().t()) * scale, 0.0)
                top = a.amax(dim=1, keepdim=True) if n else torch.full((r1 - r0, 1), -math.inf, dtype=torch.float64)
                safe = torch.where(top == -math.inf, 0.0, top)
                e = torch.exp(a - safe)
                total = e.sum(dim=1, keepdim=True)
                p = torch.where(total > 0, e / total, 0.0)
                out[r0:r1, h * G + g] = p @ v
                lse[h * G + g, r0:r1] = (total.log() + safe)[:, 0]
                most = size.amax(dim=1) if n else torch.zeros(r1 - r0, dtype=torch.float64)
                ds = (D + 2) * u * most + 16 * u * (1 + most) + 64 * u
                weight = (p * vs).amax(dim=1) if n else torch.zeros(r1 - r0, dtype=torch.float64)
                tail = sees.sum(1).double() * 2.0 ** -31 * weight * (vc.abs().amax() if n else 0.0)
                b = (1.1 * 2.0 ** -11 + 4 * ds[:, None]) * (p @ v.abs()) + tail[:, None]
                out_b[r0:r1, h * G + g] = b + rounding(out[r0:r1, h * G + g].abs() + b, dtype)
                lse_b[h * G + g, r0:r1] = 2 * ds + 16 * u * (1 + most) + 2.0 ** -21
    return out, lse, out_b, lse_b
