"""Faults of the attention operators that have been mended, on the GPU: each case is one that came out wrong, or could have."""
import math

import pytest
import torch

import attn_reference as ref
from test_attention_gpu import A, BF16, F16, cu, filled, i32, near, rand  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("G", [1, 4, 5, 32])
@pytest.mark.parametrize("C,P", [(257, 0), (400, 100), (512, 0)])
def test_weights_of_all_wavefronts_slots(A, G, C, P):
    """Slots from the 257th on are weighed by other wavefronts than the one that has the rows' sums: the formula's weights, and the same
    bits every time."""
    B, Hkv, D = 16, 8, 64
    cache, k, v = filled(A, B, Hkv * G, Hkv, D, C, [[C - (b + h) % 3 for h in range(Hkv)] for b in range(B)], F16)
    q, before = rand(5, B, Hkv * G, D).cuda(), cache.weight.clone()
    k0, v0 = (rand(6, P, Hkv, D), rand(7, P, Hkv, D)) if P else (None, None)
    prefix = [x.cuda() for x in (k0, v0)] if P else []
    want = ref.decode(q.cpu(), k0, v0, k, v, cache.lens.cpu(), 1 / 8)
    total = want[2] + before.double().cpu()
    first = None
    for _ in range(20):
        cache.weight.copy_(before)
        cache.attend(q, *prefix)
        first = cache.weight.clone() if first is None else first
        assert torch.equal(cache.weight, first)
    near(first, total, want[5] + 2.0 ** -23 * total, "weight")


@pytest.mark.parametrize("D", [4, 60, 100])
@pytest.mark.parametrize("dt", [F16, BF16])
def test_half_chunks_of_rows_that_end_with_a_stage(A, D, dt):
    """Sequences whose last row is the last of a whole stage: the half chunk at its end is not followed by another row."""
    for nq, H in (([64, 128], 2), ([256, 128], 64)):           # workgroups of 32 and of 128 rows
        q, k, v = (rand(i, sum(nq), H, D, dtype=dt) for i in range(3))
        want = ref.prompt(q, k, v, cu(nq), cu(nq), True, 1 / math.sqrt(D))
        out, lse = A.attn_prompt(q.cuda(), k.cuda(), v.cuda(), i32(cu(nq)))
        near(out, want[0], want[3], "out")
        near(lse, want[1], want[4], "lse")
    cache, k, v = filled(A, 2, 4, 2, D, 256, [[256, 128], [32, 64]], dt)
    q, k0, v0 = rand(5, 2, 4, D, dtype=dt), rand(6, 128, 2, D, dtype=dt), rand(7, 128, 2, D, dtype=dt)
    for prefix in ((), (k0, v0)):
        want = ref.decode(q, *(prefix or (None, None)), k, v, cache.lens.cpu(), 1 / math.sqrt(D))
        out, lse = cache.attend(q.cuda(), *(x.cuda() for x in prefix), weigh=False)
        near(out, want[0], want[3], "out")
        near(lse, want[1], want[4], "lse")


def test_decoder_layer_starts_anew(A):
    """A second prefix and a second prompt, after prompts and steps of another conversation: the results of a fresh layer."""
    from paper_2407_00088_amd import decoder
    B, M = 2, 256
    layers = [decoder.random_layer(M, 4, 2, 64, B, 24, 8, max_N=256) for _ in range(2)]
    first, second, prompts = rand(1, 30, M).cuda(), rand(2, 50, M).cuda(), [rand(3 + i, 19, M).cuda() for i in range(2)]
    c, steps = i32([0, 12, 19]), [rand(10 + i, B, M).cuda() for i in range(4)]
    used, fresh = layers
    used.share(first)
    used.prompt(prompts[0], c)
    for x in steps:
        used.step(x)

    def follow(layer):
        got = [layer.prompt(prompts[1], c)] + [layer.step(x) for x in steps]
        return got + [t.clone() for t in (layer.position, layer.cache.lens, layer.cache.seen, layer.cache.pos[:, :, :7])]

    fresh.share(first)
    for got, want in zip(follow(used), follow(fresh)):        # another prompt
        assert torch.equal(got, want)
    for layer in layers:
        layer.share(second)
    assert used.position.tolist() == [50, 50] and (used.cache.lens == 0).all()
    for got, want in zip([used.step(x) for x in steps], [fresh.step(x) for x in steps]):   # no prompt after another prefix
        assert torch.equal(got, want)
    fresh = decoder.random_layer(M, 4, 2, 64, B, 24, 8, max_N=256)
    fresh.share(second)
    for got, want in zip(follow(used), follow(fresh)):        # another prefix and another prompt
        assert torch.equal(got, want)


@pytest.mark.parametrize("dt", [F16, BF16])
@pytest.mark.parametrize("Tq,H,Tk", [(8192, 8, 1 << 17), (32, 512, 1 << 19)])
def test_a_flat_tail_beside_a_heavy_key(A, dt, Tq, H, Tk):
    """One key 2^25.5 times as heavy as each of the others, which all its row's sums are taken against: the others' exponentials are below
    what 16 bits hold, if taken against that key's, and together 0.3 (1.1) % of the row.  Workgroups of 128 and of 32 rows; all rows and heads are
    alike, the formula's result is computed once.  The bound: rounding of exponentials and result to the type (2.1 U), scores, and for each
    key in fp16 half a unit of the subnormal numbers, 2^-25, against a largest exponential of 2^6 or more."""
    D = 64
    k, v = torch.zeros((Tk, 1, D), dtype=dt), (torch.rand((Tk, 1, D), generator=torch.Generator().manual_seed(1)) + 0.5).to(dt)
    q = torch.zeros((1, 1, D), dtype=dt)
    q[0, 0, 0], k[0, 0, 0] = 4.0, 4.40625
    out, lse = A.attn_prompt(q.cuda().expand(Tq, H, D), k.cuda().expand(Tk, H, D), v.cuda().expand(Tk, H, D), i32([0, Tq]), i32([0, Tk]),
                             causal=False, scale=1.0)
    assert (out == out[0, 0]).all() and (lse == lse[0, 0]).all()
    args = q[:, 0], k[:, 0], v[:, 0], 1.0, torch.ones((1, Tk), dtype=torch.bool)
    want, want_lse, p = ref.rows(*args)
    _, lse_b, _ = ref.bounds(*args, p, dt)
    s = 4.0 * 4.40625
    u, tail = 2.0 ** -24, Tk * 2.0 ** -31 * 1.5 if dt == F16 else 0.0
    bound = (2.1 * ref.UNIT[dt] + 4 * ((D + 2) * u * s + 8 * u * (1 + s))) * (p @ v[:, 0].double()) + tail + u
    near(out[0, :1], want, bound, "out")
    near(lse[0, :1], want_lse, lse_b, "lse")


@pytest.mark.parametrize("kind", ["spread", "odd"])
@pytest.mark.parametrize("n,C", [(90, 40), (5000, 700), (20000, 40)])
@pytest.mark.parametrize("seen", [0, 6])
def test_recent_tokens_leave_by_their_weights_too(A, kind, n, C, seen):
    """Positions ahead of what the cache has seen, and positions that repeat, make more tokens recent than the cache holds."""
    Hkv, D, recent = 2, 8, 30
    src, k, v = filled(A, 1, Hkv, Hkv, D, n, [[n, n]], F16)
    gen = torch.Generator().manual_seed(n)
    w = torch.rand((1, Hkv, n), generator=gen)
    if kind == "odd":
        w[..., ::5], w[..., 1::9], w[..., 2::11] = math.nan, math.inf, -math.inf
    src.weight.copy_(w), src.seen.fill_(n + seen)
    # head 0: all are recent; head 1: all but one in five
    pos = torch.full((1, Hkv, n), n + seen - 1)
    pos[0, 1, ::5] = 3
    src.pos.copy_(pos)
    cache = A.KVCache(1, Hkv, D, C, recent=recent)
    cache.fill_from(src)
    for h in range(Hkv):
        order = ref.leaving(w[0, h], pos[0, h], n + seen, recent)
        kept = sorted(order[n - C:])
        assert torch.equal(cache.k[0, h].cpu(), k[0, h, kept]) and torch.equal(cache.weight[0, h].cpu().view(torch.int32), w[0, h, kept].view(torch.int32))
        assert cache.pos[0, h].tolist() == pos[0, h, kept].tolist() and int(cache.lens[0, h]) == C
    # one more into a cache all of whose tokens are recent, then into the same with fewer
    for turn in range(3):
        weight, at, new = cache.weight.cpu(), cache.pos.cpu(), rand(turn, 1, Hkv, D)
        goes = [ref.leaving(weight[0, h], at[0, h], n + seen + turn + 1, recent)[0] for h in range(Hkv)]
        cache.append(new.cuda(), new.cuda())
        for h in range(Hkv):
            assert torch.equal(cache.k[0, h, goes[h]].cpu(), new[0, h]) and int(cache.pos[0, h, goes[h]]) == n + seen + turn
            assert float(cache.weight[0, h, goes[h]]) == 0.0
