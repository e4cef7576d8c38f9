"""Faults of the paged cache that have been mended, and paths that only long or many caches take, on the GPU: each case is one that came out wrong, or
could have, against the forms in 64 bits of tests/pages_reference.py."""
import math

import pytest
import torch

import pages_reference as R
from test_pages_gpu import BF16, F16, P, close, gen, ints, starts

pytestmark = pytest.mark.gpu

# Every way that attention goes: (new tokens of each sequence, Hq of one key head, pages of 32 tokens that the table has room for)
WAYS = {
    "16 rows, whole": ([1, 1], 2, 24),
    "16 rows, shares": ([1, 1], 2, 200),
    "32 rows, whole": ([40, 9], 1, 24),
    "32 rows, shares": ([40, 9], 1, 200),
    "128 rows, whole": ([150], 2, 24),
    "128 rows, shares": ([150], 2, 200),
    "16 and 128 rows, whole": ([2, 150, 1], 2, 24),
    "16 and 128 rows, shares": ([2, 150, 1, 40], 2, 200),
}


def kept(k, v, lens, width, code, Hq):
    """A cache of bf16 keys and values [T, Hkv, D] of sequences one after the other, and its table."""
    held = [-(-n // 32) for n in lens]
    table = torch.full((len(lens), width), -1, dtype=torch.int32)
    for s, n in enumerate(held):
        table[s, :n] = torch.arange(sum(held[:s]), sum(held[:s]) + n)
    cache = P().PagedCache(sum(held), k.shape[1], k.shape[2], page=32, code=code, dtype=k.dtype, Hq=Hq)
    cache.append(k.cuda(), v.cuda(), table.cuda(), ints(lens), starts(lens).cuda())
    return cache, table


def check(cache, table, q, lens, n, held=None):
    out, lse = cache.attend(q.cuda(), table.cuda(), ints(lens), starts(n).cuda(), most=max(n))
    ref = R.attend(q, held or R.decoded(cache), table, lens, starts(n), 1 / math.sqrt(cache.D), cache.Hkv)
    close(out, ref[0], ref[2], "out")
    close(lse, ref[1], ref[3], "lse")
    return out, ref


# --- queries of bf16 far from one ----------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("code", ["i8", "e4m3"])
@pytest.mark.parametrize("way", WAYS)
def test_small_queries_beside_keys_of_zero(way, code):
    """A row's power of two times the scale of a block of zeros is below the smallest number: tokens that are not seen stayed in the row as
    -infinity times zero."""
    n, Hq, width = WAYS[way]
    g, D = gen(21), 16
    lens = [300 + 7 * i for i in range(len(n))]
    k, v = (torch.randn((sum(lens), 1, D), generator=g) for _ in range(2))
    for lo in starts(lens)[1:].tolist():
        k[lo - 90:lo] = 0.0
    k[:lens[0]] = 0.0
    cache, table = kept(k.bfloat16(), v.bfloat16(), lens, width, code, Hq)
    q = torch.randn((sum(n), Hq, D), generator=g) * 2.0 ** -torch.randint(60, 134, (sum(n), 1, 1), generator=g).double()
    out, _ = check(cache, table, q.bfloat16(), lens, n)
    assert out.isfinite().all()


@pytest.mark.parametrize("code", ["i8", "e4m3"])
@pytest.mark.parametrize("way", WAYS)
def test_smallest_queries_beside_large_keys(way, code):
    """Scores of some units from queries down to bf16's smallest and keys up to 2^125: a row's power of two is no factor of its own, which
    would have lost places below 2^-126."""
    n, Hq, width = WAYS[way]
    g, D = gen(22), 16
    lens = [300 + 7 * i for i in range(len(n))]
    k, v = (torch.randn((sum(lens), 1, D), generator=g) for _ in range(2))
    k = (k.clamp(-3.5, 3.5) * 2.0 ** 123).bfloat16()
    cache, table = kept(k, v.bfloat16(), lens, width, code, Hq)
    q = torch.randn((sum(n), Hq, D), generator=g).clamp(-3.5, 3.5).double() * 2.0 ** -torch.randint(121, 127, (sum(n), 1, 1), generator=g).double()
    _, ref = check(cache, table, q.bfloat16(), lens, n)
    assert ref[0].std() > 0.1


# --- values whose scales are far apart ---------------------------------------------------------------------------------------------------------

FAR = {
    "zeros, then large": [None, 115],
    "large, then zeros": [115, None],
    "large at the end": [None] * 8 + [96],
    "large in one of four": [None, None, 73, None],
    "small and large": [-95, 119, -40, 30, None, 80],
}


@pytest.mark.parametrize("code", ["i8", "e4m3"])
@pytest.mark.parametrize("far", FAR)
@pytest.mark.parametrize("way", WAYS)
def test_blocks_of_values_far_apart(way, far, code):
    """Blocks of values of zero or nearly zero beside ones of up to 2^121 (all of bf16's range), in either order: each has the part of the row's sum that its
    scores give it.  The values' scale is in the exponents, and a block's sums were lost where that lay 2^126 or more apart."""
    n, Hq, width = WAYS[way]
    g, D = gen(23), 16
    lens = [290 + 7 * i for i in range(len(n))]
    k, v = (torch.randn((sum(lens), 1, D), generator=g) for _ in range(2))
    v = v.clamp(-3.5, 3.5)
    for s, lo in enumerate(starts(lens)[:-1].tolist()):
        for b in range(-(-lens[s] // 32)):
            e = FAR[far][(b + s) % len(FAR[far])]
            v[lo + 32 * b:min(lo + 32 * b + 32, lo + lens[s])] *= 0.0 if e is None else 2.0 ** e
    cache, table = kept(k.bfloat16(), v.bfloat16(), lens, width, code, Hq)
    q = torch.randn((sum(n), Hq, D), generator=g)
    q[::3] *= 8.0
    out, _ = check(cache, table, q.bfloat16(), lens, n)
    assert out.isfinite().all()


# --- exponentials as two numbers ---------------------------------------------------------------------------------------------------------------


def two_numbers(n, Hq, width, code, dtype, D, before, mean, gain):
    """Sequences of n new tokens after `before` others, of one key head: those with up to 64 rows, the first nine at most, against 64 bits.

    Bound: exponentials 2^-22 of themselves or 2^-31 of the largest (times their scales), scores and sums in 32 bits as in R.attend, the sum of m products m 2^-24 of what is added."""
    g = gen(24)
    lens = [x + before for x in n]
    k, v = (torch.randn((sum(lens), 1, D), generator=g) for _ in range(2))
    cache, table = kept(k.to(dtype), (v + mean).to(dtype), lens, width, code, Hq)
    held = R.decoded(cache)
    q = (torch.randn((sum(n), Hq, D), generator=g) * gain).to(dtype)
    cu = starts(n)
    out, _ = cache.attend(q.cuda(), table.cuda(), ints(lens), cu.cuda(), most=max(n))
    scale, u, seen = 1 / math.sqrt(D), 2.0 ** -24, 0
    for s in range(min(len(n), 9)):
        if n[s] * Hq > 64:
            continue
        rows, m = slice(int(cu[s]), int(cu[s + 1])), lens[s]
        (kc, ks, _), (vc, vs, _) = held.values(table[s], m, 0, 0), held.values(table[s], m, 0, 1)
        hidden = torch.arange(m)[None] > torch.arange(m - n[s], m)[:, None]
        for h in range(Hq):
            x = q[rows, h].double()
            a = x @ (kc * ks[:, None]).t() * scale
            a[hidden] = -math.inf
            size = (x.abs() @ (kc * ks[:, None]).abs().t() * scale).amax(1, keepdim=True)
            p = torch.softmax(a, dim=1)
            ref, most = p @ (vc * vs[:, None]), (p * vs).amax(1, keepdim=True)
            ds = (D + 2) * u * size + 16 * u * (1 + size) + 64 * u
            b = (2.0 ** -22 + m * u + 2 * ds) * (p @ (vc * vs[:, None]).abs()) + m * 2.0 ** -31 * most * vc.abs().amax()
            close(out[rows, h], ref, b + R.rounding(ref.abs() + b, dtype), f"sequence {s}")
            seen += 1
    assert seen


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("code", ["i8", "e4m3"])
@pytest.mark.parametrize("n,Hq,width", [([1, 3], 4, 8), ([1, 3], 4, 200), ([40, 9], 1, 8), ([40, 9], 1, 200), ([7], 9, 8), ([33, 200, 1, 12, 64], 1, 8), ([33, 200, 1, 12], 1, 200),
                                        ([1, 2, 3, 70], 20, 8), ([3, 70], 20, 200), ([16, 50, 90, 1], 4, 200), ([60] * 130, 1, 200)])
def test_exponentials_of_few_rows_are_two_numbers(n, Hq, width, code, dtype):
    """Rows of sequences with up to 64 rows a key head are as exact with others of any kind beside them as alone: off by the result's rounding and what 32 bits
    give.  One fp16 number an exponential would be off by up to 2^-11 more."""
    two_numbers(n, Hq, width, code, dtype, D=4, before=9, mean=1.5, gain=2)


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("code", ["i8", "e4m3"])
@pytest.mark.parametrize("n,Hq,width", [([1, 2, 1, 1, 2], 8, 24), ([1, 2, 1, 1, 2], 8, 200), ([40, 33], 1, 24), ([40, 33], 1, 200), ([40, 33, 300, 2], 1, 24), ([40, 33, 300, 2], 1, 200)])
def test_exponentials_of_values_that_cancel(n, Hq, width, code, dtype):
    """Values around zero: results are small beside what is added, and their rounding hides less.  (Worked through with one number an exponential, 13 to 16 % of the results in fp16
    and 1.5 to 2.6 % in bf16 lie beyond the bound.)"""
    two_numbers(n, Hq, width, code, dtype, D=16, before=40, mean=0.0, gain=0.7)


# --- long caches, many sequences -----------------------------------------------------------------------------------------------------------------


class Gathered(R.Held):
    """What a cache holds, looked up for all tokens at once."""

    def __init__(self, cache):
        held = R.decoded(cache)
        super().__init__(held.code, held.page, held.pages, held.D)
        blocks = held.page // 32
        order = [[(p, b, h, w) for p in range(held.pages) for h in range(cache.Hkv) for b in range(blocks)] for w in (0, 1)]
        self.all = [torch.stack([held.blocks[at][0] for at in keys]).double().view(held.pages, cache.Hkv, blocks, 32, held.D) for keys in order]
        self.scale = [torch.stack([held.blocks[at][1] for at in keys]).double().view(held.pages, cache.Hkv, blocks) for keys in order]

    def values(self, table, n, h, which):
        t = torch.arange(n)
        page, part = table.long()[t // self.page], t % self.page // 32
        return self.all[which][page, h, part, t % 32], self.scale[which][page, h, part], torch.ones(n, dtype=torch.bool)


def plan(cache, n, lens, width, most):
    """How the library deals a call out: (few, many), each None, "whole", or the units of a share (blocks of 32 tokens, stages of 64), held against the workspace it asks for."""
    from paper_2407_00088_amd import pages as G
    S, T, Hkv, group, W = len(n), sum(n), cache.Hkv, cache.Hq // cache.Hkv, (cache.D + 31) // 32 * 32
    rows, blocks = min(most or T, T) * group, width * cache.page // 32
    is_many = rows > 64
    is_few = not is_many or (S > 1 and group <= 16)
    tile = 32 if rows > 16 and not is_many else 16
    tiles = -(-rows // 32) if tile == 32 else 1
    few = many = None
    need = 0
    if is_few:
        few = "whole"
        if is_many or blocks > (48 if S * Hkv * tiles < 256 else 128):
            mine = [(x, m) for x, m in zip(n, lens) if 0 < x * group <= (tile if tile == 16 else 64)]
            few = max(8, -(-sum(Hkv * -(-x * group // tile) * (max(1, -(-m // 32)) + 16) for x, m in mine) // 256))
            need += 256 * (24 + 2 * tile * (W + 2) * 4)
    if is_many:
        least = (T * group - (16 * S if is_few else 0)) // 128 * Hkv
        many = "whole"
        if least < 448 and blocks > 32:
            mine = [(x, m) for x, m in zip(n, lens) if x * group > (16 if is_few else 0)]
            many = max(4, -(-sum(Hkv * -(-x * group // 128) * (max(1, -(-m // 64)) + 2) for x, m in mine) // 512))
            need += 512 * (24 + 2 * 128 * (W + 2) * 4)
    batch = G.tmac_pages_batch(1 << 20, width, 1 << 20, 1 << 20, S, width, T, most or 0)
    assert G.lib.tmac_pages_attend_workspace_bytes(cache.desc, cache.cache, batch) == need
    return few, many


def attended(cache, table, lens, n, q, most=None):
    """Against 64 bits, and the same bits again on workspaces that hold something."""
    cu = starts(n)
    call = lambda: cache.attend(q.cuda(), table.cuda(), ints(lens), cu.cuda(), most=most)  # noqa: E731
    out, lse = call()
    ref = R.attend(q, Gathered(cache), table, lens, cu, 1 / math.sqrt(cache.D), cache.Hkv)
    close(out, ref[0], ref[2], "out")
    close(lse, ref[1], ref[3], "lse")
    cache.attend_ws.fill_(0xFF)
    for a, b in zip((out, lse), call()):
        assert torch.equal(a, b)


def filled(seed, lens, Hkv, D, page, code, dtype, Hq, width):
    g = gen(seed)
    held = [-(-m // page) for m in lens]
    cache = P().PagedCache(sum(held), Hkv, D, page=page, code=code, dtype=dtype, Hq=Hq)
    order, table = torch.randperm(sum(held), generator=g).int(), torch.full((len(lens), width), -1, dtype=torch.int32)
    for s, m in enumerate(held):
        table[s, :m] = order[sum(held[:s]):sum(held[:s]) + m]
    k, v = (torch.randn((sum(lens), Hkv, D), generator=g) for _ in range(2))
    v += torch.randn((1, Hkv, D), generator=g)
    cache.append(k.to(dtype).cuda(), v.to(dtype).cuda(), table.cuda(), ints(lens), starts(lens).cuda())
    return cache, table, g


@pytest.mark.parametrize("code,dtype", [("i8", F16), ("e4m3", BF16)])
@pytest.mark.parametrize("T,Hq,Hkv,length", [(512, 112, 1, 4500), (64, 880, 11, 4096)], ids=["whole tiles", "shares"])
def test_tiles_of_128_rows_over_more_stages_than_they_have_places_of(T, Hq, Hkv, length, code, dtype):
    """Pieces of more than 32 stages of 64 tokens: pages and scales are looked up 32 stages at a time."""
    cache, table, g = filled(31, [length], Hkv, 32, 32, code, dtype, Hq, 150)
    few, many = plan(cache, [T], [length], 150, None)
    assert few is None and (many == "whole" if Hkv == 1 else many > 33)
    attended(cache, table, [length], [T], (torch.randn((T, Hq, 32), generator=g) * 1.5).to(dtype))


@pytest.mark.parametrize("code,dtype", [("i8", BF16), ("e4m3", F16)])
@pytest.mark.parametrize("n,G", [(1, 2), (20, 1)], ids=["16 rows", "32 rows"])
def test_shares_of_more_blocks_than_they_have_places_of(n, G, code, dtype):
    """Pieces of more than 256 blocks, 64 for each of four wavefronts: sequences of 81920 tokens, whose tables name some pages again and again."""
    S, Hkv, width = 4, 8, 20
    cache, table, g = filled(32, [4096 * 3], Hkv, 4, 4096, code, dtype, Hkv * G, 3)
    table = torch.randint(0, 3, (S, width), generator=g).int()
    lens = [4096 * width - 45 * s for s in range(S)]
    few, many = plan(cache, [n] * S, lens, width, n)
    assert many is None and few > 256 + 16
    attended(cache, table, lens, [n] * S, (torch.randn((S * n, Hkv * G, 4), generator=g) * 2).to(dtype), most=n)


@pytest.mark.parametrize("code,dtype", [("i8", F16), ("e4m3", BF16)])
@pytest.mark.parametrize("long", [0, 100], ids=["alone", "beside many rows"])
def test_shares_of_several_short_sequences(long, code, dtype):
    """A share has whole sequences and pieces of others: sums meet in the same memory one after the other."""
    n = [1 + i % 4 if i % 7 else 0 for i in range(600)] + [long] * (long > 0)
    lens = [(i * 37) % 90 + 4 for i in range(600)] + [700] * (long > 0)
    cache, table, g = filled(33, lens, 1, 16, 32, code, dtype, 4, 200)
    few, many = plan(cache, n, lens, 200, max(n))
    assert few >= 35 and (many is None) == (not long)      # (a sequence has 17 to 19 units)
    attended(cache, table, lens, n, (torch.randn((sum(n), 4, 16), generator=g) * 1.5).to(dtype), most=max(n))


@pytest.mark.parametrize("code,dtype", [("i8", BF16), ("e4m3", F16)])
def test_shares_of_several_sequences_of_many_rows(code, dtype):
    """The same for tiles of 128 rows."""
    n = [70 - i % 3 for i in range(350)]
    lens = [x + i % 50 for i, x in enumerate(n)]
    cache, table, g = filled(34, lens, 3, 16, 32, code, dtype, 3, 40)
    few, many = plan(cache, n, lens, 40, None)
    assert few == 8 and many > 2 * 4
    attended(cache, table, lens, n, (torch.randn((sum(n), 3, 16), generator=g) * 1.5).to(dtype))
