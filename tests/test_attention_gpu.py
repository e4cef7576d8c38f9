"""The attention operators on the GPU against the plain 64-bit forms of attn_reference.py, at the sizes, strides and masks where
they can go wrong."""
import math

import pytest
import torch

import attn_reference as ref

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def A():
    from paper_2407_00088_amd import attention
    return attention


def rand(seed, *shape, dtype=F16, gain=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * gain).to(dtype)


def cu(lengths):
    return [sum(lengths[:i]) for i in range(len(lengths) + 1)]


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def near(got, want, bound, what):
    got = got.double().cpu()
    assert got.shape == want.shape, what
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]), what
    off = (got - want).abs()[~inf] - bound[~inf]
    assert not torch.isnan(off).any() and (off.numel() == 0 or off.max() <= 0), (what, off.max())


PROMPTS = [  # query lengths, key lengths, Hq, Hkv, D, dtype, causal
    ([1], [1], 1, 1, 128, F16, True),
    ([33], [33], 4, 4, 128, F16, True),
    ([0, 5, 0, 1], [0, 5, 0, 1], 6, 2, 64, BF16, True),
    ([31, 32, 33, 129], [31, 32, 33, 129], 8, 2, 128, BF16, True),
    ([64, 1, 128], [64, 65, 300], 4, 1, 100, F16, True),
    ([127, 255], [127, 255], 2, 2, 4, F16, True),
    ([17, 3], [5, 0], 4, 2, 96, F16, True),           # fewer keys than queries: rows that see nothing
    ([65, 130], [200, 3], 10, 2, 80, BF16, False),
    ([9], [0], 2, 1, 128, F16, False),
    ([257], [1000], 5, 1, 128, F16, True),
    ([3, 2], [3001, 2050], 8, 2, 128, BF16, True),    # few queries after long contexts: the keys are split
    ([1] * 70 + [200], [1] * 70 + [231], 2, 1, 64, F16, True),  # more sequences than lanes
    ([300], [300], 71, 1, 32, F16, True),             # a group of 71 heads
    ([1500], [1500], 16, 2, 128, F16, True),
    ([12], [12], 3, 1, 68, BF16, True),
]


@pytest.mark.parametrize("case", PROMPTS, ids=lambda c: f"{c[0][:3]}-{c[1][:3]}-{c[2]}-{c[3]}-{c[4]}-{c[5]}-{c[6]}".replace("torch.", ""))
def test_prompt_and_weights(A, case):
    nq, nk, Hq, Hkv, D, dt, causal = case
    q, k, v = (rand(i, sum(n), H, D, dtype=dt, gain=g) for i, (n, H, g) in enumerate([(nq, Hq, 1.5), (nk, Hkv, 1.0), (nk, Hkv, 1.0)]))
    want = ref.prompt(q, k, v, cu(nq), cu(nk), causal, 1 / math.sqrt(D))
    out, lse = A.attn_prompt(q.cuda(), k.cuda(), v.cuda(), i32(cu(nq)), i32(cu(nk)), causal=causal)
    near(out, want[0], want[3], "out")
    near(lse, want[1], want[4], "lse")
    w = A.attn_weights(q.cuda(), k.cuda(), lse, i32(cu(nq)), i32(cu(nk)), causal=causal)
    near(w, want[2], want[5], "weight")
    again = A.attn_prompt(q.cuda(), k.cuda(), v.cuda(), i32(cu(nq)), i32(cu(nk)), causal=causal)
    assert torch.equal(again[0], out) and torch.equal(again[1], lse)
    assert torch.equal(A.attn_weights(q.cuda(), k.cuda(), lse, i32(cu(nq)), i32(cu(nk)), causal=causal), w)


@pytest.mark.parametrize("D", [128, 64, 100, 40])
@pytest.mark.parametrize("layout", ["heads_first", "gaps", "shifted"])
def test_prompt_strides(A, D, layout):
    """Heads outermost, rows with gaps (in which there is NaN), and data that are only 8-byte aligned."""
    n, Hq, Hkv = 150, 4, 2
    host = [rand(9 + i, n, H, D) for i, H in enumerate((Hq, Hkv, Hkv))]

    def place(x):
        x = x.cuda()
        if layout == "heads_first":
            return x.transpose(0, 1).contiguous().transpose(0, 1)
        room = torch.full((n, x.shape[1], D + 8), math.nan, dtype=x.dtype, device="cuda")
        if layout == "gaps":
            room[..., :D] = x
            return room[..., :D]
        flat = torch.full((n * x.shape[1] * (D + 4) + 4,), math.nan, dtype=x.dtype, device="cuda")
        view = flat[4:].view(n, x.shape[1], D + 4)[..., :D]
        view.copy_(x)
        return view

    q, k, v = (place(x) for x in host)
    out = place(torch.zeros_like(host[0]))
    want = ref.prompt(*host, [0, n], [0, n], True, 0.2)
    got, lse = A.attn_prompt(q, k, v, i32([0, n]), scale=0.2, out=out)
    assert got is out
    near(out, want[0], want[3], "out")
    near(lse, want[1], want[4], "lse")
    near(A.attn_weights(q, k, lse, i32([0, n]), scale=0.2), want[2], want[5], "weight")


@pytest.mark.parametrize("dt", [F16, BF16])
@pytest.mark.parametrize("G", [1, 4])
@pytest.mark.parametrize("n", [40, 300])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_prompt_hidden_values_do_not_show(A, dt, G, n, bad):
    """Whatever stands in later tokens, and in the tokens of other sequences, earlier rows keep their bits; rows that see an
    infinite value get it."""
    D, Hkv, at = 64, 2, n // 2 + 3
    q, k, v = rand(1, 2 * n, Hkv * G, D, dtype=dt), rand(2, 2 * n, Hkv, D, dtype=dt), rand(3, 2 * n, Hkv, D, dtype=dt)
    c = i32([0, n, 2 * n])
    clean, clean_lse = A.attn_prompt(q.cuda(), k.cuda(), v.cuda(), c)
    for which in "kv":
        k2, v2 = k.clone(), v.clone()
        (k2 if which == "k" else v2)[at, :, 5] = bad
        (k2 if which == "k" else v2)[n + n // 2, 0] = bad
        out, lse = A.attn_prompt(q.cuda(), k2.cuda(), v2.cuda(), c)
        assert torch.equal(out[:at], clean[:at]) and torch.equal(lse[:, :at], clean_lse[:, :at])
        assert torch.equal(out[n:n + n // 2], clean[n:n + n // 2])
        if which == "v":
            assert torch.equal(lse, clean_lse)
            other = [d for d in range(D) if d != 5]
            assert torch.equal(out[:n, :, other], clean[:n, :, other])
            col = out[at:n, :, 5]
            assert torch.isnan(col).all() if math.isnan(bad) else torch.equal(col, torch.full_like(col, bad))
        elif math.isnan(bad):
            assert torch.isnan(out[at:n]).all() and torch.isnan(lse[:, at:n]).all()


def test_prompt_both_infinities_make_nan(A):
    v = rand(3, 50, 1, 64)
    v[10, 0, 7], v[20, 0, 7] = math.inf, -math.inf
    out, _ = A.attn_prompt(rand(1, 50, 1, 64).cuda(), rand(2, 50, 1, 64).cuda(), v.cuda(), i32([0, 50]))
    col = out[:, 0, 7]
    assert torch.isfinite(col[:10]).all() and (col[10:20] == math.inf).all() and torch.isnan(col[20:]).all()


def test_rows_whose_scores_are_all_minus_infinity_are_empty(A):
    q = torch.full((3, 1, 64), 3e38, dtype=BF16)
    k = torch.full((3, 1, 64), -3e38, dtype=BF16)
    out, lse = A.attn_prompt(q.cuda(), k.cuda(), torch.ones_like(k).cuda(), i32([0, 3]))
    assert (out == 0).all() and (lse == -math.inf).all()
    assert (A.attn_weights(q.cuda(), k.cuda(), lse, i32([0, 3])) == 0).all()


def test_lowest_values_and_growing_maxima(A):
    """Scores that grow from tile to tile, by more and by less than the threshold of a rescaling, beside the type's lowest values."""
    n, D = 700, 64
    for step in (0.02, 0.2):
        q, k, v = torch.zeros((n, 1, D)), torch.zeros((n, 1, D)), rand(5, n, 1, D).float()
        q[:, 0, 0], k[:, 0, 0] = 8.0, torch.arange(n) * step
        k[::7, 0, 0] = torch.finfo(F16).min
        q, k, v = q.half(), k.half(), v.half()
        want = ref.prompt(q, k, v, [0, n], [0, n], True, 1.0)
        out, lse = A.attn_prompt(q.cuda(), k.cuda(), v.cuda(), i32([0, n]), scale=1.0)
        near(out, want[0], want[3], "out")
        near(lse, want[1], want[4], "lse")


def filled(A, B, Hq, Hkv, D, C, lens, dt, seed=0, recent=0, garbage=math.nan):
    """A cache whose slots beyond `lens` hold garbage, and what it holds on the host."""
    cache = A.KVCache(B, Hkv, D, C, recent=recent, dtype=dt, Hq=Hq)
    k, v = rand(seed, B, Hkv, C, D, dtype=dt), rand(seed + 1, B, Hkv, C, D, dtype=dt)
    for b in range(B):
        for h in range(Hkv):
            k[b, h, lens[b][h]:], v[b, h, lens[b][h]:] = garbage, garbage
    cache.k.copy_(k), cache.v.copy_(v), cache.lens.copy_(torch.tensor(lens, dtype=torch.int32))
    cache.weight.copy_(torch.rand(cache.weight.shape))
    return cache, k, v


DECODES = [  # B, Hq, Hkv, D, C, P, dtype
    (1, 1, 1, 128, 1, 0, F16),
    (1, 32, 32, 128, 300, 0, F16),
    (3, 8, 2, 64, 129, 1, BF16),
    (2, 40, 1, 100, 200, 65, F16),       # more heads in a group than rows of a tile
    (5, 12, 4, 128, 1500, 700, BF16),
    (40, 8, 2, 128, 33, 513, F16),       # rows of the prefix in tiles of 128
    (9, 4, 4, 4, 70, 30, F16),
    (2, 7, 1, 80, 2100, 0, BF16),
]


@pytest.mark.parametrize("case", DECODES, ids=str)
@pytest.mark.parametrize("weigh", [False, True])
def test_decode(A, case, weigh):
    B, Hq, Hkv, D, C, P, dt = case
    gen = torch.Generator().manual_seed(C)
    lens = torch.randint(0, C + 1, (B, Hkv), generator=gen)
    lens[0, 0], lens[-1, -1] = C, 0 if B * Hkv > 1 else C
    cache, k, v = filled(A, B, Hq, Hkv, D, C, lens.tolist(), dt)
    q, k0, v0 = rand(5, B, Hq, D, dtype=dt, gain=1.5), None, None
    if P:
        k0, v0 = rand(6, P, Hkv, D, dtype=dt), rand(7, P, Hkv, D, dtype=dt)
    want = ref.decode(q, k0, v0, k, v, lens, 1 / math.sqrt(D))
    before = cache.weight.clone()
    out, lse = cache.attend(q.cuda(), k0.cuda() if P else None, v0.cuda() if P else None, weigh=weigh)
    near(out, want[0], want[3], "out")
    near(lse, want[1], want[4], "lse")
    if weigh:
        total = want[2] + before.double().cpu()
        near(cache.weight, total, want[5] + 2.0 ** -23 * total, "weight")
    else:
        assert torch.equal(cache.weight, before)
    assert torch.equal(cache.k.cpu().view(torch.int16), k.view(torch.int16))


def test_decode_strides_and_lengths_out_of_range(A):
    """Prefix and query as slices of wider tensors; lengths beyond the capacity count as the capacity, negative ones as none."""
    B, Hq, Hkv, D, C, P = 2, 4, 2, 100, 50, 40
    cache, k, v = filled(A, B, Hq, Hkv, D, C, [[50, 50], [0, 0]], F16)
    cache.lens.copy_(torch.tensor([[50, 2000000000], [-5, 0]]))
    wide = rand(8, P, 2, Hkv, D + 4).cuda()
    qw = rand(9, B, Hq, D + 20).cuda()
    k0, v0, q = wide[:, 0, :, :D], wide[:, 1, :, 4:], qw[..., 16:D + 16]
    want = ref.decode(q.cpu(), k0.cpu(), v0.cpu(), k, v, torch.tensor([[50, 50], [0, 0]]), 0.1)
    cache.desc.scale = 0.1
    out, lse = cache.attend(q, k0, v0, weigh=False)
    near(out, want[0], want[3], "out")
    near(lse, want[1], want[4], "lse")


def test_decode_of_a_prefix_gives_its_weights_through_attn_weights(A):
    """The rows of a batch over one prefix are a sequence without a causal mask."""
    B, Hq, Hkv, D, P = 6, 4, 2, 64, 300
    cache = A.KVCache(B, Hkv, D, 16, Hq=Hq)
    q, k0, v0 = rand(1, B, Hq, D).cuda(), rand(2, P, Hkv, D).cuda(), rand(3, P, Hkv, D).cuda()
    out, lse = cache.attend(q, k0, v0)
    w = A.attn_weights(q, k0, lse.t().contiguous(), i32([0, B]), i32([0, P]), causal=False)
    want = ref.prompt(q.cpu(), k0.cpu(), v0.cpu(), [0, B], [0, P], False, 1 / 8)
    near(out, want[0], want[3], "out")
    near(w, want[2], want[5], "weight")


FILLS = [  # lengths, Hkv, D, capacity, recent
    ([5], 1, 4, 8, 2), ([8, 0, 9, 1], 2, 64, 8, 0), ([300, 64], 3, 100, 64, 64), ([1000, 77, 2049], 2, 128, 129, 50),
    ([5000], 2, 64, 4999, 1), ([40000], 1, 8, 700, 100), ([33], 1, 128, 1, 0)]


def check_filled(cache, b, h, kept, k, v, w, pos, seen):
    n = len(kept)
    assert int(cache.lens[b, h]) == n and int(cache.seen[b, h]) == seen
    assert torch.equal(cache.k[b, h, :n].cpu().view(torch.int16), k[kept].view(torch.int16))
    assert torch.equal(cache.v[b, h, :n].cpu().view(torch.int16), v[kept].view(torch.int16))
    assert torch.equal(cache.weight[b, h, :n].cpu().view(torch.int32), w[kept].view(torch.int32))
    assert cache.pos[b, h, :n].tolist() == [int(pos[i]) for i in kept]


@pytest.mark.parametrize("kind", ["spread", "ties", "odd"])
@pytest.mark.parametrize("case", FILLS, ids=str)
def test_fill(A, case, kind):
    lengths, Hkv, D, C, recent = case
    T, B = sum(lengths), len(lengths)
    gen = torch.Generator().manual_seed(T)
    k, v, w = rand(1, T, Hkv, D), rand(2, T, Hkv, D), torch.rand((Hkv, T), generator=gen)
    if kind == "ties":
        w = (w * 3).floor()
    if kind == "odd":
        w = w - 0.5
        w[:, ::5], w[:, 1::9], w[:, 2::11], w[:, 3::7], w[:, 4::13] = math.nan, math.inf, -math.inf, -0.0, 0.0
    cache = A.KVCache(B, Hkv, D, C, recent=recent)
    cache.k.fill_(7.0), cache.weight.fill_(7.0)
    cache.fill(k.cuda(), v.cuda(), w.cuda(), i32(cu(lengths)))
    at = 0
    for b, n in enumerate(lengths):
        for h in range(Hkv):
            order = ref.leaving(w[h, at:at + n], range(n), n, recent)
            kept = [at + i for i in sorted(order[max(0, n - C):])]
            check_filled(cache, b, h, kept, k[:, h], v[:, h], w[h], torch.arange(T) - at, n)
            assert (cache.k[b, h, len(kept):] == 7).all() and (cache.weight[b, h, len(kept):] == 7).all()
        at += n


def test_fill_from_a_larger_cache(A):
    B, Hkv, D, C = 2, 3, 100, 500
    lens = [[500, 20, 333], [0, 64, 65]]
    src, k, v = filled(A, B, Hkv, Hkv, D, C, lens, BF16, recent=40)
    src.seen.fill_(900)
    src.pos.copy_(torch.stack([torch.randperm(900)[:C] for _ in range(B * Hkv)]).view(B, Hkv, C))
    cache = A.KVCache(B, Hkv, D, 64, recent=40, dtype=BF16)
    cache.fill_from(src)
    w, pos = src.weight.cpu(), src.pos.cpu()
    for b in range(B):
        for h in range(Hkv):
            n = lens[b][h]
            order = ref.leaving(w[b, h, :n], pos[b, h], 900, 40)
            check_filled(cache, b, h, sorted(order[max(0, n - 64):]), k[b, h], v[b, h], w[b, h], pos[b, h], 900)


@pytest.mark.parametrize("C,recent,kind", [(1, 0, "spread"), (5, 2, "ties"), (257, 64, "odd"), (700, 700, "spread"), (64, 0, "ties")])
def test_append_until_long_after_the_cache_is_full(A, C, recent, kind):
    B, Hkv, D, dt = 2, 2, 36, F16
    cache = A.KVCache(B, Hkv, D, C, recent=recent, dtype=dt)
    gen = torch.Generator().manual_seed(C)
    slots = [[[] for _ in range(Hkv)] for _ in range(B)]   # (k, v, weight, position) on the host
    for t in range(C + 40):
        k, v = rand(2 * t, B, Hkv, D), rand(2 * t + 1, B, Hkv, D)
        cache.append(k.cuda(), v.cuda())
        add = torch.rand((B, Hkv, C), generator=gen)
        if kind == "ties":
            add = (add * 2).floor()
        if kind == "odd":
            add[:, :, ::7], add[:, :, 1::7] = math.nan, -math.inf
        for b in range(B):
            for h in range(Hkv):
                s = slots[b][h]
                new = [k[b, h], v[b, h], torch.tensor(0.0), t]
                if len(s) < C:
                    s.append(new)
                else:
                    s[ref.leaving([x[2] for x in s], [x[3] for x in s], t + 1, recent)[0]] = new
                for i, x in enumerate(s):
                    x[2] = x[2] + add[b, h, i]
        cache.weight += add.cuda()
        if t % 13 == 0 or t > C + 36:
            for b in range(B):
                for h in range(Hkv):
                    s = slots[b][h]
                    got = cache.weight[b, h, :len(s)].cpu()
                    want = torch.stack([x[2] for x in s])
                    assert torch.equal(torch.nan_to_num(got, 1e30), torch.nan_to_num(want, 1e30))
                    assert cache.pos[b, h, :len(s)].tolist() == [x[3] for x in s]
                    assert torch.equal(cache.k[b, h, :len(s)].cpu(), torch.stack([x[0] for x in s]))
                    assert torch.equal(cache.v[b, h, :len(s)].cpu(), torch.stack([x[1] for x in s]))
    assert (cache.lens == C).all() and (cache.seen == C + 40).all()


def test_on_another_stream_and_in_a_graph(A):
    """Work goes to the current stream; a captured step gives the eager steps' results on every replay."""
    B, Hq, Hkv, D, C, P = 2, 8, 2, 128, 200, 300
    steps = 5
    def fresh():
        cache, _, _ = filled(A, B, Hq, Hkv, D, C, [[C, C], [C, C]], F16, recent=10, garbage=0.0)
        cache.pos.copy_(torch.arange(C).expand(B, Hkv, C))
        cache.seen.fill_(C)
        cache.weight.copy_(torch.rand((B, Hkv, C), generator=torch.Generator().manual_seed(3)))
        return cache
    q, k1, v1 = (rand(20 + i, steps, B, H, D).cuda() for i, H in enumerate((Hq, Hkv, Hkv)))
    k0, v0 = rand(30, P, Hkv, D).cuda(), rand(31, P, Hkv, D).cuda()
    eager, want = fresh(), []
    for t in range(steps):
        eager.append(k1[t], v1[t])
        want.append([x.clone() for x in eager.attend(q[t], k0, v0)] + [eager.weight.clone(), eager.pos.clone()])
    cache = fresh()
    bufs = [torch.zeros_like(x[0]) for x in (q, k1, v1)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    def step():
        cache.append(bufs[1], bufs[2])
        return cache.attend(bufs[0], k0, v0)
    state = [cache.k, cache.v, cache.weight, cache.pos, cache.seen, cache.lens]
    kept = [x.clone() for x in state]
    with torch.cuda.stream(side):
        step()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out, lse = step()
    torch.cuda.synchronize()
    for x, y in zip(state, kept):
        x.copy_(y)
    for t in range(steps):
        for buf, x in zip(bufs, (q, k1, v1)):
            buf.copy_(x[t])
        graph.replay()
        torch.cuda.synchronize()
        for got, w in zip((out, lse, cache.weight, cache.pos), want[t]):
            assert torch.equal(got, w)


def test_a_long_cache_beyond_32_bit_offsets(A):
    """Slots further than 2^32 bytes from the cache's start (one sequence, one head, 2^24 + 300 slots of 128 elements: 4.3 GB of keys)."""
    C, D = (1 << 24) + 300, 128
    cache = A.KVCache(1, 1, D, C)
    cache.lens.fill_(C)
    # all keys alike but two, the last ones: with q along one axis their scores carry everything
    q = torch.zeros((1, 1, D), dtype=F16, device="cuda")
    q[0, 0, 0] = 64.0
    cache.k[0, 0, -2:, 0] = 8.0
    cache.v[0, 0, -2], cache.v[0, 0, -1] = 1.0, 3.0
    out, lse = cache.attend(q)
    s = 64.0 * 8.0 / math.sqrt(D)
    assert (out == 2.0).all() and abs(float(lse) - (s + math.log(2.0))) < 1e-4
    assert torch.allclose(cache.weight[0, 0, -2:].cpu(), torch.tensor([0.5, 0.5]), atol=1e-5)


LARGE_PROMPTS = [  # enough rows and heads for workgroups of 128 rows, or enough pairs for two blocks of keys a wavefront
    ([700, 3, 128, 129], [700, 3, 128, 129], 32, 32, 128, F16, True),
    ([40] * 9, [40] * 8 + [1040], 32, 32, 100, BF16, True),
    ([33] * 70 + [200], [33] * 70 + [231], 8, 8, 64, BF16, True),    # more sequences than lanes
    ([512], [700], 64, 8, 100, BF16, True),
    ([1000, 333], [1000, 64], 64, 8, 36, F16, True),                 # fewer keys than queries: rows that see nothing
    ([200, 77], [300, 0], 64, 64, 128, F16, False),                  # no keys
    ([200, 77], [2000, 1700], 64, 64, 64, F16, True),                # slices of the keys
    ([1531], [1531], 64, 8, 128, BF16, True),
    ([2100], [1400], 48, 3, 60, F16, False),
]


@pytest.mark.parametrize("case", LARGE_PROMPTS, ids=lambda c: f"{c[0][:3]}-{c[1][:3]}-{c[2]}-{c[3]}-{c[4]}-{c[5]}-{c[6]}".replace("torch.", ""))
def test_large_prompt_and_weights(A, case):
    test_prompt_and_weights(A, case)


@pytest.mark.parametrize("dt", [F16, BF16])
@pytest.mark.parametrize("D", [60, 128])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_large_prompt_hidden_values_do_not_show(A, dt, D, bad):
    """The same as in small calls where four wavefronts share the stages."""
    n, H, at = 200, 128, 103
    q, k, v = rand(1, 2 * n, H, D, dtype=dt).cuda(), rand(2, 2 * n, H, D, dtype=dt).cuda(), rand(3, 2 * n, H, D, dtype=dt).cuda()
    c = i32([0, n, 2 * n])
    clean, clean_lse = A.attn_prompt(q, k, v, c)
    for which in "kv":
        k2, v2 = k.clone(), v.clone()
        (k2 if which == "k" else v2)[at, :, 5] = bad
        (k2 if which == "k" else v2)[n + n // 2, 0] = bad
        out, lse = A.attn_prompt(q, k2, v2, c)
        assert torch.equal(out[:at], clean[:at]) and torch.equal(lse[:, :at], clean_lse[:, :at])
        assert torch.equal(out[n:n + n // 2], clean[n:n + n // 2]) and torch.equal(out[n:, 1:], clean[n:, 1:])
        if which == "v":
            assert torch.equal(lse, clean_lse)
            other = [d for d in range(D) if d != 5]
            assert torch.equal(out[:n, :, other], clean[:n, :, other])
            col = out[at:n, :, 5]
            assert torch.isnan(col).all() if math.isnan(bad) else torch.equal(col, torch.full_like(col, bad))
        elif math.isnan(bad):
            assert torch.isnan(out[at:n]).all() and torch.isnan(lse[:, at:n]).all()


def test_rows_do_not_depend_on_the_sequences_beside_them(A):
    """A sequence's rows keep their bits whatever other sequences a call of the same shape of workgroups holds."""
    H, D = 64, 128
    a, b, c = (rand(40 + i, 300, 3, H, D).cuda() for i in range(3))
    alone = A.attn_prompt(*torch.cat([a, b]).unbind(1), i32([0, 300, 600]))
    other = A.attn_prompt(*torch.cat([c, a, b, c]).unbind(1), i32([0, 300, 600, 900, 1200]))
    assert torch.equal(alone[0], other[0][300:900]) and torch.equal(alone[1], other[1][:, 300:900])


LARGE_DECODES = [  # enough rows over a long prefix for workgroups of 128 rows
    (64, 32, 8, 128, 33, 6200, F16),
    (33, 64, 4, 100, 70, 8001, BF16),
    (130, 16, 16, 64, 5, 6000, F16),     # the last tile has two rows
]


@pytest.mark.parametrize("case", LARGE_DECODES, ids=str)
@pytest.mark.parametrize("weigh", [False, True])
def test_large_decode(A, case, weigh):
    test_decode(A, case, weigh)


SHORT_PREFIXES = [  # prefix and cache by one workgroup, or just not
    (64, 8, 8, 128, 40, 500, F16),
    (64, 8, 8, 128, 40, 513, F16),
    (20, 128, 16, 128, 300, 512, BF16),
    (33, 16, 8, 100, 512, 3, BF16),
    (1, 4, 2, 68, 30, 482, F16),
    (1, 4, 2, 68, 30, 483, F16),
    (3, 66, 2, 36, 9, 100, F16),         # more heads in a group than rows of a tile
]


@pytest.mark.parametrize("case", SHORT_PREFIXES, ids=str)
@pytest.mark.parametrize("weigh", [False, True])
def test_decode_after_a_short_prefix(A, case, weigh):
    test_decode(A, case, weigh)


@pytest.mark.parametrize("P", [40, 600])
def test_decode_strides_of_the_prefix(A, P):
    B, Hq, Hkv, D, C = 2, 4, 2, 100, 50
    cache, k, v = filled(A, B, Hq, Hkv, D, C, [[50, 13], [0, 1]], BF16)
    wide = rand(8, P, 2, Hkv, D + 4, dtype=BF16).cuda()
    qw = rand(9, B, Hq, D + 20, dtype=BF16).cuda()
    k0, v0, q = wide[:, 0, :, :D], wide[:, 1, :, 4:], qw[..., 16:D + 16]
    want = ref.decode(q.cpu(), k0.cpu(), v0.cpu(), k, v, cache.lens.cpu(), 0.1)
    before = cache.weight.double().cpu()
    cache.desc.scale = 0.1
    out, lse = cache.attend(q, k0, v0)
    near(out, want[0], want[3], "out")
    near(lse, want[1], want[4], "lse")
    total = want[2] + before
    near(cache.weight, total, want[5] + 2.0 ** -23 * total, "weight")
