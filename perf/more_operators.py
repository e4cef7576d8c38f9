"""What is measured of the operators around a paged cache of 8 bits: the rotation of queries and keys by their positions, appending
tokens to the cache (keys rotated on the way), and attention over it.

A case is a dict of plain values, `op` says which operator:

  "rotate"  queries and keys of T tokens turned by their positions (Rotary.rotate), which start at `start`
  "append"  new tokens of S sequences into the pages of their caches: queries and keys turned, keys and values held in 8 bits with a
            scale for every block of 32 tokens and key head, a block that was begun before taken up again (PagedCache.append); and the
            values that the blocks then stand for (PagedCache.read)
  "attend"  attention of the last tokens of S sequences over all that is in their pages (PagedCache.attend)

Hq query heads, Hkv key heads of D elements, of which the first `rot` turn, pairs `interleaved` or not, frequencies scaled by `scaling`;
`dtype` "f16" or "bf16", `code` "e4m3" or "i8", pages of `page` tokens.  S sequences: `new` new tokens the longest, the others by `spread`
(1: all alike; 2, 3: down to one token, evenly in the logarithm), after up to `old` tokens, by `old_spread`.
"""
import math
import random

import torch

own = False

_DTYPE = {"f16": torch.float16, "bf16": torch.bfloat16}
BLOCK = 32                             # tokens that share a scale
FLOOR = 2.0 ** -60                     # the smallest scale

MOST_PAIRS = 64 * 1024 * 8192          # padded (head, query, key) triples of one pass: the largest listed case's
MOST_KEYS = 32 * 8 * 16384             # (head, token) pairs in pages: the largest listed case's
MOST_ROWS = 72 * 16384                 # (head, token) rows of new tokens: the largest listed case's


def listed():
    return [
        # one user's decode step on a 7B-sized decoder: launch and latency
        dict(name="rotate_step", op="rotate", dtype="f16", T=1, start=1000, Hq=32, Hkv=32, D=128, rot=128, interleaved=False, scaling="none"),
        # a prompt of odd length on a 3B-sized decoder (3200 / 32 heads: 100 elements), part of the head, pairs side by side
        dict(name="rotate_part", op="rotate", dtype="bf16", T=2003, start=0, Hq=32, Hkv=32, D=100, rot=52, interleaved=True, scaling="linear"),
        # a long document far into a context that is longer than what was trained on
        dict(name="rotate_long", op="rotate", dtype="f16", T=16384, start=100000, Hq=64, Hkv=8, D=128, rot=128, interleaved=False, scaling="ramp"),
        # a batch's decode step: one token for every sequence
        dict(name="append_step", op="append", dtype="bf16", code="e4m3", page=64, S=24, new=1, spread=1, old=4095, old_spread=2, Hq=64, Hkv=8,
             D=128, rot=128, interleaved=False, scaling="bands"),
        # prompts of odd lengths, some after earlier chunks, on a 3B-sized decoder
        dict(name="append_ragged", op="append", dtype="f16", code="i8", page=32, S=7, new=701, spread=2, old=333, old_spread=3, Hq=32, Hkv=32,
             D=100, rot=100, interleaved=True, scaling="none"),
        # a long document
        dict(name="append_long", op="append", dtype="f16", code="e4m3", page=128, S=1, new=16384, spread=1, old=0, old_spread=1, Hq=64, Hkv=8,
             D=128, rot=128, interleaved=False, scaling="none"),
        # one user's decode step on a 7B-sized decoder with a short context
        dict(name="attend_one", op="attend", dtype="f16", code="e4m3", page=64, S=1, new=1, spread=1, old=300, old_spread=1, Hq=32, Hkv=32, D=128),
        # a batch's decode step with grouped heads and contexts from short to long
        dict(name="attend_batch", op="attend", dtype="bf16", code="i8", page=64, S=32, new=1, spread=1, old=16383, old_spread=2, Hq=64, Hkv=8, D=128),
        # a few drafted tokens a sequence, to be checked at once, on a 3B-sized decoder
        dict(name="attend_drafts", op="attend", dtype="f16", code="e4m3", page=32, S=16, new=5, spread=1, old=1999, old_spread=2, Hq=32, Hkv=32, D=100),
        # chunks of prompts beside decode steps, as a server batches them
        dict(name="attend_mixed", op="attend", dtype="bf16", code="e4m3", page=128, S=9, new=509, spread=3, old=2500, old_spread=2, Hq=40, Hkv=8, D=128),
        # the last chunk of a long document on a 70B-sized decoder
        dict(name="attend_chunk", op="attend", dtype="f16", code="i8", page=64, S=1, new=1024, spread=1, old=7168, old_spread=1, Hq=64, Hkv=8, D=128),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rotate", "append", "append", "attend", "attend", "attend"])
    Hkv, G = rng.choice([(32, 1), (40, 1), (8, 4), (8, 8), (8, 5), (4, 7), (1, 16), (2, 3)])
    D = rng.choice([128, 128, 128, 100, 64, 80])
    c = dict(op=op, dtype=rng.choice(["f16", "bf16"]), Hq=Hkv * G, Hkv=Hkv, D=D)
    if op != "attend":
        c.update(rot=rng.choice([D, D, D // 4 * 2]), interleaved=rng.random() < 0.4, scaling=rng.choice(["none", "none", "linear", "base", "ramp", "bands"]))
    if op == "rotate":
        while True:
            c.update(T=_log_int(rng, 1, 16384), start=rng.choice([0, _log_int(rng, 1, 200000)]))
            if c["T"] * (c["Hq"] + Hkv) <= MOST_ROWS:
                return c
    c.update(code=rng.choice(["e4m3", "i8"]), page=rng.choice([32, 64, 128, 256]))
    while True:
        c.update(S=_log_int(rng, 1, 64), new=rng.choice([1, _log_int(rng, 2, 16), _log_int(rng, 2, 16384 if op == "append" else 2048)]),
                 spread=rng.choice([1, 2, 3]), old=rng.choice([0, _log_int(rng, 1, 16384)]), old_spread=rng.choice([1, 2, 3]))
        n, o = _lengths(c)
        if c["S"] * Hkv * (c["new"] + c["old"]) > MOST_KEYS or sum(n) * (c["Hq"] + Hkv) > MOST_ROWS:
            continue
        if op == "append" or c["S"] * c["Hq"] * c["new"] * (c["new"] + c["old"]) <= MOST_PAIRS:
            return c


def _spread(longest, S, spread, salt):
    """The first is the longest, the others fall evenly in the logarithm, in an order of their own."""
    if spread == 1 or longest < 2:
        return [longest] * S
    got = [longest] + [max(1, int(longest ** (1 - (i / S) * (spread - 1) / 2))) for i in range(1, S)]
    random.Random(S * 1000 + longest + salt).shuffle(got)
    return got


def _lengths(case):
    """New tokens of every sequence, and tokens before them."""
    return _spread(case["new"], case["S"], case["spread"], 0), _spread(case["old"], case["S"], case["old_spread"], 1)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _starts(lengths):
    return _ints([sum(lengths[:i]) for i in range(len(lengths) + 1)])


def _heads(gen, dtype, *shape, gain=1.0):
    """Gaussian with a few large channels, the same for every token of a head, as keys and queries have them."""
    x = torch.randn(shape, device="cuda", generator=gen)
    x *= torch.where(torch.rand((1, *shape[1:]), device="cuda", generator=gen) < 0.02, 2.0, 1.0) * gain
    return x.to(dtype)


# --- frequencies -------------------------------------------------------------------------------------------------------------------------------------------

FACTOR, TRAINED = 8.0, 8192.0  # a context eight times as long as the one that was trained on


def _scaling(case):
    """What a user gives Rotary."""
    return {"none": None, "linear": ("linear", FACTOR), "base": ("base", FACTOR), "ramp": ("ramp", FACTOR, TRAINED, 32.0, 1.0),
            "bands": ("bands", FACTOR, TRAINED, 1.0, 4.0)}[case["scaling"]]


def _frequencies(case):
    """Radians a position of every pair, in 64 bits, and what the cosines and sines are multiplied with."""
    rot, base, kind = case["rot"], 10000.0, case["scaling"]
    i = torch.arange(rot // 2, dtype=torch.float64)
    if kind == "base":
        base *= FACTOR ** (rot / (rot - 2))
    f = base ** (-2 * i / rot)
    if kind == "linear":
        f = f / FACTOR
    if kind == "ramp":
        at = lambda turns: rot * math.log(TRAINED / (2 * math.pi * turns)) / (2 * math.log(base))  # noqa: E731
        lo, hi = max(0, math.floor(at(32.0))), min(rot - 1, math.ceil(at(1.0)))
        ramp = ((i - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        return f * (1 - ramp) + f / FACTOR * ramp, 0.1 * math.log(FACTOR) + 1.0
    if kind == "bands":
        turns = TRAINED * f / (2 * math.pi)
        mix = ((turns - 1.0) / (4.0 - 1.0)).clamp(0, 1)
        f = f * (mix + (1 - mix) / FACTOR)
    return f, 1.0


# --- inputs ---------------------------------------------------------------------------------------------------------------------------------------------------


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt, Hq, Hkv, D = _DTYPE[case["dtype"]], case["Hq"], case["Hkv"], case["D"]
    st = dict(case, dt=dt)
    if "rot" in case:
        f, st["magnitude"] = _frequencies(case)
        st["freq"] = f.cuda()
    if case["op"] == "rotate":
        T = case["T"]
        st["q"], st["k"] = _heads(gen, dt, T, Hq, D, gain=1.5), _heads(gen, dt, T, Hkv, D)
        st["positions"] = case["start"] + torch.arange(T, device="cuda")
        return st
    n, old = _lengths(case)
    lens, page = [a + b for a, b in zip(n, old)], case["page"]
    held = [-(-m // page) for m in lens]
    width, pages = max(held) + 2, sum(held) + 5
    order = torch.randperm(pages, device="cuda", generator=gen).to(torch.int32)
    # pages of a sequence in no order; what is behind a sequence's last page has none
    table = torch.full((case["S"], width), -1, dtype=torch.int32, device="cuda")
    for s, (lo, m) in enumerate(zip(_starts(held).tolist(), held)):
        table[s, :m] = order[lo:lo + m]
    st.update(cu=_starts(n), lens=_ints(lens), table=table, pages=pages, most_new=max(n), most=max(lens),
              q=_heads(gen, dt, sum(n), Hq, D, gain=1.5))
    # what is in the pages before the call
    before = old if case["op"] == "append" else lens
    st["before"], st["before_cu"] = _ints(before), _starts(before)
    st["k0"], st["v0"] = _heads(gen, dt, sum(before), Hkv, D), _heads(gen, dt, sum(before), Hkv, D)
    if case["op"] == "append":
        st["k"], st["v"] = _heads(gen, dt, sum(n), Hkv, D), _heads(gen, dt, sum(n), Hkv, D)
        # the blocks that the new tokens touch, from their first token on
        back = [m - o // BLOCK * BLOCK for m, o in zip(lens, old)]
        st.update(back_cu=_starts(back), back=sum(back), most_back=max(back))
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    if own:
        from paper_2407_00088_amd import PagedCache, Rotary
        if "rot" in case:
            st["rotary"] = Rotary(case["D"], rot=case["rot"], interleaved=case["interleaved"], scaling=_scaling(case))
    if case["op"] == "rotate":
        return st
    k0, v0 = st.pop("k0"), st.pop("v0")
    if own:
        cache = PagedCache(st["pages"], case["Hkv"], case["D"], page=case["page"], code=case["code"], dtype=st["dt"], Hq=case["Hq"])
        if k0.shape[0]:
            cache.append(k0, v0, st["table"], st["before"], st["before_cu"])
        cache.rotary = st.get("rotary")
        st["cache"] = cache
        return st
    # one page more takes what is not to be kept
    shape = (st["pages"] + 1, case["page"], case["Hkv"], case["D"])
    st["kind"] = torch.int8 if case["code"] == "i8" else torch.float8_e4m3fn
    st["codes"] = [torch.zeros(shape, dtype=torch.int8, device="cuda") for _ in range(2)]
    st["scales"] = [torch.zeros((shape[0], shape[1] // BLOCK, shape[2]), device="cuda") for _ in range(2)]
    if k0.shape[0]:
        _plain_store(st, (k0.float(), v0.float()), st["before"], st["before_cu"], int(st["before"].max()))
    return st


# --- the plain forms: elementary operations in 32 bits, angles in 64 ------------------------------------------------------------------------------------------


def _plain_rotated(st, x, positions):
    """x [T, H, D] turned, in 32 bits."""
    angle = positions[:, None].double() * st["freq"]
    c, s = ((f(angle) * st["magnitude"]).float()[:, None] for f in (torch.cos, torch.sin))
    x, rot = x.float(), st["rot"]
    if st["interleaved"]:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * c - b * s, a * s + b * c], dim=-1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat([a * c - b * s, a * s + b * c], dim=-1)
    return torch.cat([turned, x[..., rot:]], dim=-1)


def _plain_codes(code, x):
    """Whole numbers or e4m3 values that are nearest, as 32-bit numbers."""
    if code == "i8":
        return x.round().clamp(-127.0, 127.0)
    return x.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).float()


def _plain_scale(code, most):
    """The scale of a block whose largest value is `most`."""
    if code == "i8":
        return (most / 127.0).clamp(min=FLOOR)
    mantissa, exponent = torch.frexp(most)  # 448 is 0.875 * 2^9
    power = (exponent - 9 + (mantissa > 0.875)).clamp(min=-60)
    return torch.where(most > 0, ((power + 127).int() << 23).view(torch.float32), FLOOR)


def _plain_place(st, blocks, there):
    """(page, block of the page) of the blocks [S, n] of the sequences; those that are not there go to the last page."""
    per = st["page"] // BLOCK
    page = torch.gather(st["table"].long(), 1, (blocks // per).clamp(max=st["table"].shape[1] - 1))
    return torch.where(there & (page >= 0), page, st["pages"]), blocks % per


def _plain_store(st, rows, lens, cu, most_new):
    """New tokens [T, Hkv, D] of keys and values in 32 bits: blocks that they touch get the larger of the old scale and what they need."""
    code, lens, cu = st["code"], lens.long(), cu.long()
    start = lens - (cu[1:] - cu[:-1])
    blocks = start[:, None] // BLOCK + torch.arange((most_new + BLOCK - 2) // BLOCK + 1, device="cuda")
    there = blocks * BLOCK < lens[:, None]
    token = blocks[..., None] * BLOCK + torch.arange(BLOCK, device="cuda")
    new = ((token >= start[:, None, None]) & (token < lens[:, None, None]))[..., None, None]
    begun = (blocks * BLOCK < start[:, None])[..., None]
    page, part = _plain_place(st, blocks, there)
    at = (page[..., None], part[..., None] * BLOCK + torch.arange(BLOCK, device="cuda"))
    row = (cu[:-1, None, None] + token - start[:, None, None]).clamp(0, rows[0].shape[0] - 1)
    for x, codes, scales in zip(rows, st["codes"], st["scales"]):
        x = torch.where(new, x[row], 0.0)
        was = torch.where(begun, scales[page, part], 0.0)
        scale = torch.maximum(was, _plain_scale(code, x.abs().amax(dim=(2, 4))))
        stays = torch.where(begun[..., None, :, None], codes[at].view(st["kind"]).float(), 0.0)
        stays = _plain_codes(code, stays * (was / scale)[:, :, None, :, None])
        got = torch.where(new, _plain_codes(code, x * (1.0 / scale)[:, :, None, :, None]), stays)
        codes[at] = got.to(st["kind"]).view(torch.int8)
        scales[page, part] = scale


def _plain_values(st, lens, cu, most):
    """The last cu[s + 1] - cu[s] tokens of every sequence as 32-bit values [S, most, Hkv, D], and which of them there are."""
    lens, cu = lens.long(), cu.long()
    n = cu[1:] - cu[:-1]
    at = torch.arange(most, device="cuda")
    there = at < n[:, None]
    token = torch.where(there, (lens - n)[:, None] + at, 0)
    page, part = _plain_place(st, token // BLOCK, there)
    got = []
    for codes, scales in zip(st["codes"], st["scales"]):
        got.append(codes[page, part * BLOCK + token % BLOCK].view(st["kind"]).float() * scales[page, part][..., None])
    return got, there


def _plain_append(st):
    n = (st["cu"][1:] - st["cu"][:-1]).long()
    first = (st["lens"].long() - n) - st["cu"][:-1].long()
    positions = torch.arange(st["k"].shape[0], device="cuda") + torch.repeat_interleave(first, n, output_size=st["k"].shape[0])
    q, k = _plain_rotated(st, st["q"], positions).to(st["dt"]), _plain_rotated(st, st["k"], positions)
    _plain_store(st, (k, st["v"].float()), st["lens"], st["cu"], st["most_new"])
    (k, v), there = _plain_values(st, st["lens"], st["back_cu"], st["most_back"])
    return q, k[there].to(st["dt"]), v[there].to(st["dt"])


def _plain_attend(st):
    Hq, Hkv, D, lens, cu = st["Hq"], st["Hkv"], st["D"], st["lens"].long(), st["cu"].long()
    S, G, Lq, Lk, n = lens.numel(), Hq // Hkv, st["most_new"], st["most"], cu[1:] - cu[:-1]
    all_cu = torch.cat([lens.new_zeros(1), lens.cumsum(0)])
    (k, v), there_k = _plain_values(st, lens, all_cu, Lk)
    k, v = k.permute(0, 2, 3, 1).contiguous(), v.permute(0, 2, 1, 3).contiguous()
    i, j = torch.arange(Lq, device="cuda"), torch.arange(Lk, device="cuda")
    there_q = i < n[:, None]
    q = st["q"][(cu[:-1, None] + i).clamp(max=st["q"].shape[0] - 1)].float().permute(0, 2, 1, 3).reshape(S, Hkv, G * Lq, D)
    s = torch.matmul(q, k).reshape(S, Hkv, G, Lq, Lk).mul_(1.0 / math.sqrt(D))
    sees = (j <= i[:, None] + (lens - n)[:, None, None]) & there_k[:, None] & there_q[:, :, None]
    s.masked_fill_(~sees[:, None, None], -math.inf)
    top = s.amax(dim=-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = s.sub_(top).exp_()
    total = p.sum(dim=-1, keepdim=True)
    o = torch.matmul(p.reshape(S, Hkv, G * Lq, Lk), v).reshape(S, Hkv, G, Lq, D) / torch.where(total > 0, total, 1.0)
    out = o.reshape(S, Hq, Lq, D).permute(0, 2, 1, 3)[there_q].to(st["dt"])
    return out, (total.log() + top).reshape(S, Hq, Lq).permute(0, 2, 1)[there_q].t().contiguous()


def run(st):
    op = st["op"]
    if not own:
        if op == "rotate":
            return [_plain_rotated(st, st[x], st["positions"]).to(st["dt"]) for x in ("q", "k")]
        return _plain_append(st) if op == "append" else _plain_attend(st)
    if op == "rotate":
        return st["rotary"].rotate(st["positions"], st["q"], st["k"])
    cache = st["cache"]
    if op == "append":
        q = cache.append(st["k"], st["v"], st["table"], st["lens"], st["cu"], q=st["q"], most=st["most_new"])
        return q, *cache.read(st["table"], st["lens"], st["back_cu"], T=st["back"], most=st["most_back"])
    return cache.attend(st["q"], st["table"], st["lens"], st["cu"], most=st["most_new"])


# --- the definitions in 64 bits -------------------------------------------------------------------------------------------------------------------------------


def _turned64(case, x, positions):
    """Pairs of x as complex numbers, times magnitude e^(i angle)."""
    f, magnitude = _frequencies(case)
    rot = case["rot"]
    x = x.double()
    pairs = x[..., :rot].unflatten(-1, (rot // 2, 2)) if case["interleaved"] else x[..., :rot].unflatten(-1, (2, rot // 2)).transpose(-1, -2)
    turn = torch.polar(torch.full_like(f, magnitude).cuda().expand(len(positions), -1), positions.double()[:, None] * f.cuda())
    z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn[:, None])
    z = z if case["interleaved"] else z.transpose(-1, -2)
    return torch.cat([z.flatten(-2), x[..., rot:]], dim=-1)


def _held64(code, x, was=None, begun=0):
    """One sequence's tokens x [n, Hkv, D] as the cache holds them, where the first `begun` are values that it holds already, in blocks with
    the scales `was` [blocks, Hkv]; blocks start at the first token.  Returns the values and the scales."""
    n, H, D = x.shape
    nb = -(-n // BLOCK)
    x = torch.cat([x.double(), x.new_zeros((nb * BLOCK - n, H, D), dtype=torch.float64)]).reshape(nb, BLOCK, H, D)
    fresh = (torch.arange(nb * BLOCK, device=x.device) >= begun).reshape(nb, BLOCK, 1, 1)
    most = torch.where(fresh, x.abs(), 0.0).amax(dim=(1, 3))
    if code == "i8":
        scale = most.float() / 127     # (scales are numbers of 32 bits, and so are the products that are rounded)
    else:
        scale = torch.exp2(torch.ceil(torch.log2(torch.where(most > 0, most, 1e-300) / 448)))
    scale = scale.float().clamp(min=FLOOR)
    if was is not None:
        scale[:len(was)] = torch.maximum(scale[:len(was)], was)
    y = (x.float() * (1 / scale)[:, None, :, None]).double()
    if code == "i8":
        y = y.round().clamp(-127, 127)
    else:
        y = y.clamp(-448, 448)
        step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
        y = (y / step).round() * step
    return (y * scale.double()[:, None, :, None]).reshape(-1, H, D)[:n], scale


def exact(case, seed):
    st = _inputs(case, seed)
    if case["op"] == "rotate":
        return [_turned64(case, st[x], st["positions"]) for x in ("q", "k")]
    code, D, Hq, G = case["code"], case["D"], case["Hq"], case["Hq"] // case["Hkv"]
    cu, lens, before = st["cu"].tolist(), st["lens"].tolist(), st["before_cu"].tolist()
    if case["op"] == "append":
        got = [[], [], []]
        for s, m in enumerate(lens):
            new, old = slice(cu[s], cu[s + 1]), m - (cu[s + 1] - cu[s])
            where = torch.arange(old, m, device="cuda")
            got[0].append(_turned64(case, st["q"][new], where))
            k = _turned64(case, st["k"][new], where)
            for to, x, x0 in ((got[1], k, st["k0"]), (got[2], st["v"][new].double(), st["v0"])):
                # the block that was begun before, as it was held then
                tail, scales = old % BLOCK, None
                first = x[:0]
                if tail:
                    first, scales = _held64(code, x0[before[s] + old - tail:before[s] + old])
                to.append(_held64(code, torch.cat([first, x]), scales, tail)[0])
        return [torch.cat(x) for x in got]
    out = torch.zeros((cu[-1], Hq, D), dtype=torch.float64, device="cuda")
    lse = torch.zeros((Hq, cu[-1]), dtype=torch.float64, device="cuda")
    for s, m in enumerate(lens):
        k, v = (_held64(code, x[before[s]:before[s + 1]])[0] for x in (st["k0"], st["v0"]))
        n = cu[s + 1] - cu[s]
        hidden = torch.arange(m, device="cuda") > torch.arange(m - n, m, device="cuda")[:, None]
        for h in range(Hq):
            a = st["q"][cu[s]:cu[s + 1], h].double() @ k[:, h // G].t() / math.sqrt(D)
            a[hidden] = -math.inf
            lse[h, cu[s]:cu[s + 1]] = torch.logsumexp(a, dim=1)
            out[cu[s]:cu[s + 1], h] = torch.softmax(a, dim=1) @ v[:, h // G]
    return out, lse


def work(case):
    """Inputs and results moved once, in the pages a byte an element and four a scale; two products over the (query, key) pairs that are seen."""
    Hq, Hkv, D, op = case["Hq"], case["Hkv"], case["D"], case["op"]
    if op == "rotate":
        rows = case["T"] * (Hq + Hkv)
        return {"bytes": rows * D * 4 + 8 * case["T"], "flops": 3 * rows * case["rot"]}
    n, old = _lengths(case)
    T, tokens = sum(n), sum(n) + sum(old)
    if op == "append":
        back = sum(a + o % BLOCK for a, o in zip(n, old))  # tokens of the blocks that are touched
        held = 2 * Hkv * (D + 4 / BLOCK)
        return {"bytes": T * D * (4 * Hq + 4 * Hkv) + T * held + back * (held + 4 * D * Hkv), "flops": 3 * T * (Hq + Hkv) * case["rot"] + 4 * T * Hkv * D}
    pairs = Hq * sum(a * o + a * (a + 1) // 2 for a, o in zip(n, old))
    return {"bytes": tokens * 2 * Hkv * (D + 4 / BLOCK) + T * Hq * (4 * D + 4), "flops": 4 * D * pairs}
