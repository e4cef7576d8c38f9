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


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("code", ["i8", "e4m3"])
@pytest.mark.parametrize("n,Hq,width", [([1, 3], 4, 8), ([1, 3], 4, 200), ([40, 9], 1, 8), ([40, 9], 1, 200), ([7], 9, 8), ([33, 200, 1, 12, 64], 1, 8), ([33, 200, 1, 12], 1, 200),
                                        ([1, 2, 3, 70], 20, 8), ([3, 70], 20, 200), ([16, 50, 90, 1], 4, 200), ([60] * 130, 1, 200)])
def test_exponentials_of_few_rows_are_two_numbers(n, Hq, width, code, dtype):
    """Rows of sequences with up to 64 rows a key head are as exact with others of any kind beside them as alone: off by the result's rounding and what 32 bits
    give.  One fp16 number an exponential would be off by up to 2^-11 more, which half of the results' halves of steps do not cover.

    Bound: exponentials 2^-22 of themselves or 2^-31 of the largest (times their scales), scores and sums in 32 bits as in R.attend, the sum of m products m 2^-24 of what is added."""
    g, D = gen(24), 4
    lens = [x + 9 for x in n]
    k, v = (torch.randn((sum(lens), 1, D), generator=g) for _ in range(2))
    cache, table = kept(k.to(dtype), (v + 1.5).to(dtype), lens, width, code, Hq)
    held = R.decoded(cache)
    q = (torch.randn((sum(n), Hq, D), generator=g) * 2).to(dtype)
    cu = starts(n)
    out, lse = cache.attend(q.cuda(), table.cuda(), ints(lens), cu.cuda(), most=max(n))
    seen = 0
    for s in range(len(n)):
        if n[s] * Hq > 64 or s > 8:
            continue
        rows, m, u = slice(int(cu[s]), int(cu[s + 1])), lens[s], 2.0 ** -24
        (kc, ks, _), (vc, vs, _) = held.values(table[s], m, 0, 0), held.values(table[s], m, 0, 1)
        hidden = torch.arange(m)[None] > torch.arange(m - n[s], m)[:, None]
        for h in range(Hq):
            x = q[rows, h].double()
            a = (x @ (kc * ks[:, None]).t()) / 2
            a[hidden] = -math.inf
            size = ((x.abs() @ (kc * ks[:, None]).abs().t()) / 2).amax(1, keepdim=True)
            p = torch.softmax(a, dim=1)
            ref, most = p @ (vc * vs[:, None]), (p * vs).amax(1, keepdim=True)
            ds = (D + 2) * u * size + 16 * u * (1 + size) + 64 * u
            b = (2.0 ** -22 + m * u + 2 * ds) * (p @ (vc * vs[:, None]).abs()) + m * 2.0 ** -31 * most * vc.abs().amax()
            close(out[rows, h], ref, b + R.rounding(ref.abs() + b, dtype), f"sequence {s}")
            seen += 1
    assert seen
