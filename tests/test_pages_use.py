"""Rotation and paged cache as programs use them: a layer of prompts, chunks, drafts and steps, captured steps, other streams, several threads, pools
beyond 4 GB, both ways through the binding."""
import math
import threading

import pytest
import torch

import pages_reference as R

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def T():
    import paper_2407_00088_amd as T
    return T


def rand(seed, *shape, dtype=F16):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def close(got, ref, bound):
    off = (got.double().cpu() - ref).abs() - bound
    off[ref.isinf()] = 0.0
    assert torch.equal(got.double().cpu()[ref.isinf()], ref[ref.isinf()]) and off.max() <= 0, float(off.max())


@pytest.mark.parametrize("code", ["e4m3", "i8"])
def test_a_layer_over_prompts_chunks_drafts_and_steps(T, code):
    """PagedDecoderAttention: the projections' own outputs, turned, held as the pages hold them, attended to by the definition; and the same table
    after drafts were taken back and a sequence has ended."""
    from paper_2407_00088_amd import decoder
    M, Hq, Hkv, D, batch = 256, 8, 2, 64, 3
    layer = decoder.paged(decoder.random_layer(M, Hq, Hkv, D, batch, capacity=8, recent=4, max_N=256), pages=16, width=6, page=32, code=code)
    freq = layer.cache.rotary.freq.cpu()
    for i, counts in enumerate([[70, 9, 33], [1, 1, 1], [4, 0, 40], [3, 5, 2], [1, 1, 1]]):
        if i == 4:
            layer.take_back([2, 4, layer.table.length[2]])
        old = list(layer.table.length)
        held = R.decoded(layer.cache)
        x = rand(i, sum(counts), M).cuda()
        got = layer.forward(x, counts) if i != 1 else layer.step(x)
        q, k, v = (lin.forward_one_call(x, out_t=T.TMAC_OUT_F16).view(x.shape[0], -1, D).cpu() for lin in (layer.q, layer.k, layer.v))
        lens = [a + b for a, b in zip(old, counts)]
        cu = [sum(counts[:s]) for s in range(4)]
        table = layer.table.table.cpu()
        assert lens == layer.table.length == layer.table.lens.tolist()
        # what the pages hold now: within one step of the turned keys and the values (half a step, twice where a block's scale has grown)
        now = R.decoded(layer.cache)
        positions = torch.cat([torch.arange(a, b) for a, b in zip(old, lens)])
        k64 = R.turned(k, positions, freq, 1.0, False)
        for s in range(3):
            for h in range(Hkv):
                for which, new in ((0, k64), (1, v.double())):
                    codes, scales, there = now.values(table[s], lens[s], h, which)
                    assert there.all()
                    rows = new[cu[s]:cu[s + 1], h]
                    scales = scales[old[s]:, None]
                    step = scales if code == "i8" else torch.exp2(torch.floor(torch.log2((rows.abs() / scales).clamp(min=2.0 ** -6))) - 3) * scales
                    assert ((codes[old[s]:] * scales - rows).abs() <= 0.51 * step + 1e-6).all()
                    if old[s]:      # earlier tokens: as before, or rounded once more where their block's scale has grown
                        before, was, _ = held.values(table[s], old[s], h, which)
                        same = was == now.values(table[s], old[s], h, which)[1]
                        assert torch.equal(before[same], codes[:old[s]][same])
        # queries rounded to fp16 as append leaves them: within the rounding of the exact ones
        q16 = layer.cache.rotary.rotate(positions.cuda(), q.cuda())[0].cpu()
        ref = R.attend(q16, now, table, lens, cu, 1 / 8, Hkv)
        want = layer.o.forward_one_call(ref[0].half().cuda().view(x.shape[0], -1), out_t=T.TMAC_OUT_F16)
        assert (got.float() - want.float()).norm() <= 4e-3 * want.float().norm()   # fp16 tables 2e-3 each, and the attention's
    with pytest.raises(ValueError):
        layer.forward(x, [1, 1, 2])


def test_both_ways_through_the_binding_give_the_same(T):
    """The ordinary call, and the same on a stream that is named, which goes through the checks in Python."""
    rotary = T.Rotary(100, rot=52, interleaved=True, scaling=("linear", 2.0))
    q, k, v = (rand(i, 50, h, 100, dtype=BF16).cuda() for i, h in ((1, 6), (2, 3), (3, 3)))
    positions = torch.arange(50).cuda() * 7
    here = torch.cuda.current_stream()
    for a, b in zip(rotary.rotate(positions, q, k), rotary.rotate(positions, q, k, stream=here)):
        assert torch.equal(a, b)
    got = []
    for stream in (None, here):
        cache = T.PagedCache(5, 3, 100, page=32, code="i8", dtype=BF16, rotary=rotary, Hq=6)
        where = (ints([[4, 0], [2, 1]]), ints([40, 10]), ints([0, 40, 50]))
        out = [cache.append(k, v, *where, q=q, stream=stream), cache.append(k, v, *where, q=q, positions=positions, most=40, stream=stream), cache.codes, cache.scales]
        for _ in range(2):
            out += cache.attend(q, *where, stream=stream)
        out += cache.attend(q[:2], ints([[4, 0], [2, 1]]), ints([40, 10]), stream=stream)
        out += cache.read(*where, T=50, stream=stream)
        out += cache.read(*where, stream=stream)
        assert cache.append(k, v, *where, stream=stream) is None
        got.append(out)
    for a, b in zip(*got):
        assert a.dtype == b.dtype and torch.equal(a, b)


def test_bad_calls_are_worded(T):
    rotary = T.Rotary(64)
    cache = T.PagedCache(4, 2, 64, Hq=4, rotary=rotary)
    q, k = rand(1, 3, 4, 64).cuda(), rand(2, 3, 2, 64).cuda()
    table, lens, cu = ints([[0, 1], [2, 3]]), ints([2, 1]), ints([0, 2, 3])
    positions = torch.arange(3).cuda()
    room = torch.zeros(3 * 4 * 64, dtype=F16, device="cuda")
    overlap = room[:256].view(1, 4, 64).expand(3, 4, 64)
    bad = [lambda: cache.append(k, k, table, lens), lambda: cache.append(k, k[:2], table, lens, cu), lambda: cache.append(k.bfloat16(), k, table, lens, cu),
           lambda: cache.append(k, k, table.long(), lens, cu), lambda: cache.append(k, k, table, lens.long(), cu), lambda: cache.append(k, k, table[:1], lens, cu),
           lambda: cache.append(k, k, table, lens, cu[:2]), lambda: cache.append(k, k, table, lens, cu, q=k), lambda: cache.append(k, k, table, lens, cu, positions=positions.int()),
           lambda: cache.append(k, k, table, lens, cu, q=q, q_out=overlap), lambda: cache.append(k, k, table, lens, cu, q_out=q), lambda: cache.append(k, k, table, lens, cu, most=-1),
           lambda: cache.attend(k, table, lens, cu), lambda: cache.attend(q, table, lens, cu, out=overlap), lambda: cache.attend(q, table, lens, cu, lse=room),
           lambda: cache.attend(q.transpose(1, 2).contiguous().transpose(1, 2), table, lens, cu), lambda: cache.read(table, lens, cu, T=3, k=q),
           lambda: cache.attend(q, table[:, :1].expand(2, 2), lens, cu), lambda: rotary.rotate(positions), lambda: rotary.rotate(positions, q, k[:2]),
           lambda: rotary.rotate(positions, q, k.bfloat16()), lambda: rotary.rotate(positions.int(), q), lambda: rotary.rotate(positions, q, out=[overlap]),
           lambda: rotary.rotate(positions, q, out=[q, q]), lambda: rotary.rotate(positions, q.float()), lambda: rotary.rotate(positions.cpu(), q)]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            print("call", i, "was not refused")
    with pytest.raises(T.TmacError):       # in place, but by other strides
        rotary.rotate(positions, room.view(3, 4, 64), out=[room.view(4, 3, 64).transpose(0, 1)])
    plain = T.PagedCache(4, 2, 64, Hq=4)
    with pytest.raises(ValueError, match="without rotary"):
        plain.append(k, k, table, lens, cu, q=q)
    # calls about nothing
    none = torch.zeros((0, 4, 64), dtype=F16, device="cuda")
    out, lse = cache.attend(none, table, lens, ints([0, 0, 0]))
    assert out.shape == (0, 4, 64) and lse.shape == (4, 0)
    assert cache.append(none[:, :2], none[:, :2], table, lens, ints([0, 0, 0]), q=none).shape == (0, 4, 64)
    assert rotary.rotate(positions[:0], none)[0].shape == (0, 4, 64)
    assert torch.equal(cache.codes, torch.zeros_like(cache.codes))


def test_steps_that_are_captured_follow_the_table(T):
    """One graph for append and attend: replayed while the table grows, with work of its own between the replays; every step as the
    eager one on a cache of its own.  An eager, larger call between them takes another workspace."""
    D, Hkv, Hq, S = 64, 2, 8, 3
    rotary = T.Rotary(D)
    caches = [T.PagedCache(40, Hkv, D, page=32, Hq=Hq, rotary=rotary, code="i8") for _ in range(2)]
    tables = [T.PageTable(S, 100, 40, page=32) for _ in range(2)]
    n = [100, 31, 60]
    k0, v0 = rand(1, sum(n), Hkv, D).cuda(), rand(2, sum(n), Hkv, D).cuda()
    for cache, table in zip(caches, tables):
        cu, most = table.extend(n)
        cache.append(k0, v0, table.table, table.lens, cu, most=most)
    q, k, v = torch.zeros((S, Hq, D), dtype=F16, device="cuda"), *(torch.zeros((S, Hkv, D), dtype=F16, device="cuda") for _ in range(2))
    cache, table = caches[0], tables[0]
    for t in tables:
        t.extend([1] * S)

    def step(cache, table):
        turned = cache.append(k, v, table.table, table.lens, q=q)
        return turned, *cache.attend(turned, table.table, table.lens)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(cache, table)          # (workspaces are there before the capture)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = step(cache, table)
    torch.cuda.current_stream().wait_stream(side)
    assert cache.attend_ws.numel() > 16
    for turn in range(6):
        if turn:
            for t in tables:
                t.extend([1] * S)
        q.copy_(rand(10 + turn, S, Hq, D)), k.copy_(rand(20 + turn, S, Hkv, D)), v.copy_(rand(30 + turn, S, Hkv, D))
        want = [x.clone() for x in step(caches[1], tables[1])]
        torch.cuda.synchronize()
        graph.replay()
        others = [torch.full((size,), 7.0, device="cuda") for size in (2000, 300000)]
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b), turn
        assert torch.equal(caches[0].codes, caches[1].codes) and torch.equal(caches[0].scales, caches[1].scales)
        assert all((x == 7.0).all() for x in others)
        if turn == 2:               # many rows: another plan, a larger workspace, of this cache
            big = rand(40, 300, Hq, D).cuda()
            first = cache.attend_ws
            cache.attend(big, table.table, table.lens, ints([0, 100, 100, 300]))
            assert cache.attend_ws is not first and any(x is first for x in cache.outgrown)


def test_other_streams_and_threads(T):
    """Calls on a stream of the caller's see what was enqueued there; calls from several threads, each with sequences and a stream of its own, on caches of
    their own give what they give alone."""
    D, Hq, Hkv = 128, 8, 2
    rotary = T.Rotary(D)

    def work(seed, stream):
        cache = T.PagedCache(60, Hkv, D, page=64, Hq=Hq, rotary=rotary, code="e4m3")
        table = T.PageTable(2, 30, 60, page=64)
        out = []
        for i, counts in enumerate(([900, 40], [1, 1], [5, 3], [300, 0])):
            cu, most = table.extend(counts)
            q, k, v = (rand(seed + 10 * i + j, sum(counts), h, D).cuda() for j, h in enumerate((Hq, Hkv, Hkv)))
            where = dict(table=table.table, lens=table.lens, cu=cu, most=most, stream=stream)
            turned = cache.append(k, v, q=q, **where)
            out += [turned, *cache.attend(turned, **where), *cache.read(T=sum(counts), **where)]
        return out

    want = [work(s, None) for s in (1, 2, 3)]
    got = [None] * 3

    def run(i):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            got[i] = work(i + 1, stream if i else None)
        stream.synchronize()

    threads = [threading.Thread(target=run, args=(i,)) for i in range(3)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for a, b in zip(want, got):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_one_cache_from_several_threads(T):
    """Threads that call one cache: each call whole, one after the other."""
    cache = T.PagedCache(60, 2, 64, page=32, Hq=4)
    lens = [700, 900]
    table = ints([[i for i in range(30)], [i for i in range(30, 60)]])
    k, v = rand(1, 1600, 2, 64).cuda(), rand(2, 1600, 2, 64).cuda()
    cache.append(k, v, table, ints(lens), ints([0, 700, 1600]))
    qs = [rand(3 + i, 2 + 60 * i, 4, 64).cuda() for i in range(3)]
    cus = [ints([0, 1, 2]), ints([0, 30, 62]), ints([0, 100, 122])]
    want = [cache.attend(q, table, ints(lens), cu) for q, cu in zip(qs, cus)]
    torch.cuda.synchronize()
    bad = []

    def run(i):
        for _ in range(20):
            got = cache.attend(qs[i], table, ints(lens), cus[i])
            if not (torch.equal(got[0], want[i][0]) and torch.equal(got[1], want[i][1])):
                bad.append(i)

    threads = [threading.Thread(target=run, args=(i,)) for i in range(3)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad


@pytest.mark.parametrize("code", ["e4m3", "i8"])
def test_a_pool_beyond_4_gb(T, code):
    """Pages whose bytes lie beyond 32-bit offsets, in both signs: 9 GB of codes."""
    D, Hkv, page = 128, 8, 1024
    pages = 4500                       # of 2 MiB
    cache = T.PagedCache(pages, Hkv, D, page=page, code=code, Hq=16)
    assert cache.codes.numel() > 2 * (1 << 32)
    lens = [1500, 40, 2000]
    table = torch.tensor([[4499, 2100, -1], [1024, -1, -1], [4096, 17, -1]], dtype=torch.int32)
    cu = [0, 1500, 1540, 3540]
    k, v = rand(1, 3540, Hkv, D), rand(2, 3540, Hkv, D)
    cache.append(k.cuda(), v.cuda(), table.cuda(), ints(lens), ints(cu))
    small = T.PagedCache(6, Hkv, D, page=page, code=code, Hq=16)
    near = torch.tensor([[0, 1, -1], [2, -1, -1], [3, 4, -1]], dtype=torch.int32)
    small.append(k.cuda(), v.cuda(), near.cuda(), ints(lens), ints(cu))
    for far_page, page_ in zip((4499, 2100, 1024, 4096, 17), range(5)):
        assert torch.equal(cache.codes[far_page], small.codes[page_]) and torch.equal(cache.scales[far_page], small.scales[page_])
    assert int((cache.scales != 0).any(dim=3).any(dim=2).any(dim=1).sum()) == 5
    for n in ([1, 1, 1], [90, 3, 200]):
        q = rand(3, sum(n), 16, D).cuda()
        c = ints([0, n[0], n[0] + n[1], sum(n)])
        for a, b in zip(cache.attend(q, table.cuda(), ints(lens), c), small.attend(q, near.cuda(), ints(lens), c)):
            assert torch.equal(a, b)
    for a, b in zip(cache.read(table.cuda(), ints(lens), ints(cu), T=3540), small.read(near.cuda(), ints(lens), ints(cu), T=3540)):
        assert torch.equal(a, b)


def test_long_positions(T):
    """Angles are taken in 64 bits: positions of some millions, and turning back."""
    rotary = T.Rotary(128)
    x = rand(1, 64, 2, 128)
    positions = torch.randint(0, 1 << 23, (64,), generator=torch.Generator().manual_seed(2))
    y, = rotary.rotate(positions.cuda(), x.cuda())
    ref = R.turned(x, positions, rotary.freq.cpu(), 1.0, False)
    # (the angle itself is off by 2^-29 here: two roundings of 2^-53 relative to 2^23)
    close(y, ref, R.turned_bound(x, rotary.freq.cpu(), 1.0, False) * 2 + R.rounding(ref, F16))
    back, = rotary.rotate(-positions.cuda(), y)
    assert (back.cpu().float() - x.float()).abs().max() <= 2.0 ** -8     # two roundings to fp16 of values up to four


def test_pages_shared_by_sequences(T):
    """Two sequences read the same pages of a common beginning, and go on in their own."""
    cache = T.PagedCache(6, 1, 64, page=32, Hq=2)
    k, v = rand(1, 64, 1, 64).cuda(), rand(2, 64, 1, 64).cuda()
    cache.append(k, v, ints([[3, 1, -1]]), ints([64]), ints([0, 64]))
    table = ints([[3, 1, 0], [3, 1, 5]])
    k2, v2 = rand(3, 12, 1, 64).cuda(), rand(4, 12, 1, 64).cuda()
    lens, cu = ints([69, 71]), ints([0, 5, 12])
    cache.append(k2, v2, table, lens, cu)
    q = rand(5, 12, 2, 64)
    out, lse = cache.attend(q.cuda(), table, lens, cu)
    ref = R.attend(q, R.decoded(cache), table.cpu(), [69, 71], [0, 5, 12], 1 / 8, 1)
    close(out, ref[0], ref[2])
    close(lse, ref[1], ref[3])


@pytest.mark.parametrize("code", ["e4m3", "i8"])
def test_a_padded_batch(T, code):
    """Tensors with more rows than the starts speak of, a table that is part of a wider one, a sequence without a token, queries turned in place: what is
    behind the last sequence stays, and the rest is as without it."""
    D, Hq, Hkv = 80, 6, 3
    rotary = T.Rotary(D, rot=40)
    n, lens = [37, 0, 5], [50, 9, 5]
    rows, room = sum(n), 64
    wide = torch.full((3, 50), 7, dtype=torch.int32, device="cuda")
    table = wide[:, 10:14]
    table.copy_(torch.tensor([[4, 1, -1, -1], [0, -1, -1, -1], [6, -1, -1, -1]], dtype=torch.int32))
    q, k, v = (rand(i, room, h, D).cuda() for i, h in ((1, Hq), (2, Hkv), (3, Hkv)))
    q[rows:], k[rows:], v[rows:] = math.nan, math.inf, math.nan
    cu = ints([0, 37, 37, 42])
    got = []
    for padded in (True, False):
        cache = T.PagedCache(7, Hkv, D, page=32, code=code, Hq=Hq, rotary=rotary)
        m = room if padded else rows
        x = q[:m].clone()
        turned = cache.append(k[:m], v[:m], table, ints(lens), cu, q=x, q_out=x)
        assert turned is x
        out, lse = torch.full((m, Hq, D), 3.0, dtype=F16, device="cuda"), torch.full((Hq, m), 5.0, device="cuda")
        cache.attend(turned, table, ints(lens), cu, out=out, lse=lse)
        kk, vv = torch.full((m, Hkv, D), 3.0, dtype=F16, device="cuda"), torch.full((m, Hkv, D), 3.0, dtype=F16, device="cuda")
        cache.read(table, ints(lens), cu, k=kk, v=vv)
        if padded:
            assert turned[rows:].isnan().all() and (out[rows:] == 3).all() and (lse[:, rows:] == 5).all() and (kk[rows:] == 3).all() and (vv[rows:] == 3).all()
        got.append((cache.codes, cache.scales, turned[:rows], out[:rows], lse[:, :rows], kk[:rows], vv[:rows]))
        assert out[:rows].isfinite().all()
    for a, b in zip(*got):
        assert torch.equal(a, b)
    assert (wide[:, :10] == 7).all() and (wide[:, 14:] == 7).all()


def test_wrong_contents_stay_within_bounds(T):
    """Starts that fall, lengths beyond the table, numbers that are no page, in every kernel: values are wrong, other pages and rows untouched."""
    D, Hq, Hkv = 64, 8, 2
    cache = T.PagedCache(5, Hkv, D, page=32, Hq=Hq, rotary=T.Rotary(D))
    cache.codes.fill_(9), cache.scales.fill_(1.0)
    q, k = rand(1, 300, Hq, D).cuda(), rand(2, 300, Hkv, D).cuda()
    table = ints([[1, -5, 2, 1 << 30], [3, 5, -1, -(1 << 31)]])
    guard = torch.full((302, Hq, D), 3.0, dtype=F16, device="cuda")
    for lens in ([1 << 30, -(1 << 31)], [(1 << 31) - 1, 70], [0, 0], [100, 128], [5, 3]):
        for cu in ([0, 200, 300], [0, 300, 20], [-50, 1 << 30, -(1 << 31)], [250, 100, 310], [0, 0, 0], [5, 5, 300], [40, 60, 300], [96, 100, 90]):
            for table_ in (table, torch.nn.functional.pad(table, (0, 200), value=-1)):
                for most in (None, 1, 3, 40):
                    cache.append(k, k, table_, ints(lens), ints(cu), q=q, q_out=guard[1:301], most=most)
                    cache.attend(q, table_, ints(lens), ints(cu), most=most, out=guard[1:301])
                    cache.read(table_, ints(lens), ints(cu), T=300, most=most)
    torch.cuda.synchronize()
    assert (guard[0] == 3).all() and (guard[301] == 3).all()
    assert all((cache.codes[p] == 9).all() and (cache.scales[p] == 1).all() for p in (0, 4))


def test_a_layer_refuses_and_stays_as_it_was(T):
    """More tokens than the projections or the pages take, rows that are not the counts', a call without tokens: neither table nor pages change."""
    from paper_2407_00088_amd import decoder
    M, batch = 256, 2
    layer = decoder.paged(decoder.random_layer(M, 4, 2, 64, batch, capacity=8, recent=4, max_N=100), pages=3, width=3, page=32)
    layer.forward(rand(1, 40, M).cuda(), [33, 7])
    before = [t.clone() for t in (layer.cache.codes, layer.cache.scales, layer.table.table, layer.table.lens)]
    for rows, counts, error in ((64, [64, 0], ValueError), (57, [31, 26], MemoryError), (101, [1, 100], AssertionError), (3, [1, 1], ValueError), (3, [3], ValueError),
                                (2, [3, -1], ValueError)):
        with pytest.raises(error):
            layer.forward(rand(2, rows, M).cuda(), counts)
    assert layer.forward(rand(3, 0, M).cuda(), [0, 0]).shape == (0, M)
    for a, b in zip(before, (layer.cache.codes, layer.cache.scales, layer.table.table, layer.table.lens)):
        assert torch.equal(a, b)
    assert layer.table.length == [33, 7] and layer.table.free == []
