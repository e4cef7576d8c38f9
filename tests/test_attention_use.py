"""The attention operators as a program uses them: both ways through the binding, streams, growing workspaces, and the decoder layer
that runs them together with low-bit projections."""
import math

import pytest
import torch

import attn_reference as ref
from test_attention_gpu import A, BF16, F16, cu, filled, i32, near, rand  # noqa: F401

pytestmark = pytest.mark.gpu


class Nothing:
    """In place of the library: any call is an error."""

    def __getattr__(self, name):
        raise AssertionError(f"{name} was not called through the native side")


def all_calls(A, stream=None):
    """One of every call on inputs of a fixed seed; the results.  (Inputs are made and results copied on the current stream: what lies
    between waits for them and is waited for.)"""
    wait = torch.cuda.synchronize if stream is not None else lambda: None
    nq, Hq, Hkv, D = [70, 33], 4, 2, 100
    q, k, v = (rand(i, sum(nq), H, D).cuda() for i, H in enumerate((Hq, Hkv, Hkv)))
    c = i32(cu(nq))
    kw = dict(stream=stream) if stream is not None else {}
    wait()
    out, lse = A.attn_prompt(q, k, v, c, **kw)
    w = A.attn_weights(q, k, lse, c, **kw)
    cache = A.KVCache(2, Hkv, D, 40, recent=8, Hq=Hq)
    wait()
    got = [out, lse, w]
    for _ in range(2):  # (the second time the workspaces are there)
        cache.fill(k, v, w, c, **kw)
        cache.append(k[:2], v[:2], **kw)
        got += cache.attend(q[:2], k[:50], v[:50], **kw)
        got += cache.attend(q[:2], weigh=False, **kw)
        wait()
        got += [x.clone() for x in (cache.k, cache.v, cache.weight, cache.pos, cache.lens, cache.seen)]
        wait()
    return got


def test_both_ways_through_the_binding_and_a_stream_of_the_callers(A, monkeypatch):
    from paper_2407_00088_amd import binding as B
    want = all_calls(A)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    on_side = all_calls(A, stream=side)
    torch.cuda.synchronize()
    monkeypatch.setattr(A, "calls", B._NoCalls())
    general = all_calls(A)
    for got in (on_side, general):
        assert len(got) == len(want) and all(torch.equal(x, y) for x, y in zip(got, want))


def test_ordinary_calls_take_the_native_side(A, monkeypatch):
    nq = [5, 9]
    q, k, v, c = rand(1, 14, 4, 64).cuda(), rand(2, 14, 2, 64).cuda(), rand(3, 14, 2, 64).cuda(), i32(cu(nq))
    cache = A.KVCache(2, 2, 64, 8, Hq=4)
    _, lse = A.attn_prompt(q, k, v, c)
    w = A.attn_weights(q, k, lse, c)
    cache.fill(k, v, w, c), cache.append(k[:2], v[:2]), cache.attend(q[:2], k, v)   # workspaces are made on first use
    monkeypatch.setattr(A, "lib", Nothing())
    A.attn_prompt(q, k, v, c, c, causal=False, scale=0.5)
    A.attn_weights(q, k, lse, c)
    cache.fill(k, v, w, c), cache.append(k[:2], v[:2]), cache.attend(q[:2]), cache.attend(q[:2], k, v, weigh=False)


def test_refusals_are_worded(A):
    q, k, c = rand(1, 14, 4, 64).cuda(), rand(2, 14, 2, 64).cuda(), i32([0, 5, 14])
    cache = A.KVCache(2, 2, 64, 8, Hq=4)
    for bad in (lambda: A.attn_prompt(q, k, k[:5], c), lambda: A.attn_prompt(q.float(), k, k, c), lambda: A.attn_prompt(q, k.bfloat16(), k, c),
                lambda: A.attn_prompt(q, k, k, c.long()), lambda: A.attn_prompt(q, k, k, c, c[:2]), lambda: A.attn_prompt(q[:, :3], k, k, c),
                lambda: A.attn_prompt(q.transpose(0, 2).contiguous().transpose(0, 2), k, k, c), lambda: A.attn_prompt(q, k, k, c.cpu()),
                lambda: A.attn_weights(q, k, torch.zeros((14, 4), device="cuda"), c), lambda: cache.attend(q), lambda: cache.attend(q[:2], k),
                lambda: cache.attend(q[:2], k, k[:3]), lambda: cache.append(k[:2], k[:1]), lambda: cache.append(k[:2], k[:2].cpu()),
                lambda: cache.fill(k, k, torch.zeros((2, 13), device="cuda"), c), lambda: cache.fill(k, k, torch.zeros((2, 14), device="cuda"), c[:2]),
                lambda: cache.fill_from(cache), lambda: cache.fill_from(A.KVCache(2, 2, 32, 8)),
                lambda: A.attn_prompt(q, k, k, c, out=torch.empty((14, 4, 60), dtype=F16, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    from paper_2407_00088_amd import TmacError
    wide = rand(3, 4, 2, 132).cuda()
    with pytest.raises(TmacError, match="tmac_attn_prompt"):
        A.attn_prompt(wide, wide, wide, i32([0, 4]))
    with pytest.raises(TmacError):
        A.attn_prompt(q, k, k, c, scale=-1.0)
    odd = torch.empty(14 * 4 * 64 + 1, dtype=F16, device="cuda")[1:].view(14, 4, 64)
    with pytest.raises(TmacError):
        A.attn_prompt(odd, k, k, c)


def test_nothing_to_do(A):
    """No queries, no keys, no sequences that have any."""
    q, k = rand(1, 6, 4, 64).cuda(), rand(2, 6, 2, 64).cuda()
    out, lse = A.attn_prompt(q, k[:0], k[:0], i32([0, 2, 6]), i32([0, 0, 0]))
    assert (out == 0).all() and (lse == -math.inf).all()
    assert A.attn_prompt(q[:0], k, k, i32([0, 0]), i32([0, 6]))[0].shape == (0, 4, 64)
    assert (A.attn_weights(q[:0], k, lse[:, :0].contiguous(), i32([0, 0]), i32([0, 6])) == 0).all()
    cache = A.KVCache(1, 2, 64, 8, Hq=4)
    cache.fill(k[:0], k[:0], torch.zeros((2, 0), device="cuda"), i32([0, 0]))
    assert (cache.lens == 0).all()
    out, lse = cache.attend(q[:1])
    assert (out == 0).all() and (lse == -math.inf).all() and (cache.weight == 0).all()


@pytest.mark.parametrize("causal", [False, True])
def test_infinite_keys_that_nobody_attends_to_have_no_weight(A, causal):
    """Keys at which every query's score is -inf: exactly nothing, whatever the kernels put in the place of queries that are not there."""
    n, D = 37, 64
    q, k = rand(1, n, 2, D), rand(2, n, 1, D)
    q[:, :, 7] = q[:, :, 7].abs() + 0.5
    k[[3, 20], :, 7] = -math.inf
    c = i32([0, n])
    out, lse = A.attn_prompt(q.cuda(), k.cuda(), rand(3, n, 1, D).cuda(), c, causal=causal)
    w = A.attn_weights(q.cuda(), k.cuda(), lse, c, causal=causal)
    want = ref.prompt(q, k, rand(3, n, 1, D), [0, n], [0, n], causal, 1 / 8)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    assert (w[0, [3, 20]] == 0).all() and torch.isfinite(w).all()
    assert torch.allclose(w.double().cpu(), want[2], rtol=1e-4)


def test_a_workspace_that_grows_does_not_disturb_an_earlier_call(A):
    """Larger and larger prefixes in a row, without a wait between the calls."""
    cache, k, v = filled(A, 2, 8, 2, 64, 60, [[60, 60], [7, 0]], BF16)
    q = rand(5, 2, 8, 64, dtype=BF16)
    sizes = [10, 700, 3000, 9000]
    k0, v0 = rand(6, sizes[-1], 2, 64, dtype=BF16), rand(7, sizes[-1], 2, 64, dtype=BF16)
    args = q.cuda(), k0.cuda(), v0.cuda()
    got = [cache.attend(args[0], args[1][:n], args[2][:n], weigh=False) for n in sizes]
    for n, (out, lse) in zip(sizes, got):
        want = ref.decode(q, k0[:n], v0[:n], k, v, cache.lens.cpu(), 1 / 8)
        near(out, want[0], want[3], "out")
        near(lse, want[1], want[4], "lse")


def test_decoder_layer(A):
    """Prompt and steps of the layer against the plain forms on the layer's own projections; the output projection is the same call on both sides,
    on inputs that differ by the attention's own error."""
    from paper_2407_00088_amd import decoder
    from paper_2407_00088_amd.binding import TMAC_OUT_F16
    B, M, Hq, Hkv, D, C, recent, P = 3, 256, 4, 2, 64, 24, 8, 50
    layer = decoder.random_layer(M, Hq, Hkv, D, B, C, recent, max_N=256)
    x0, lengths = rand(1, P, M).cuda(), [40, 5, 24]
    c = i32(cu(lengths))
    x = rand(2, sum(lengths), M).cuda()
    layer.share(x0)
    positions = torch.cat([torch.arange(n) for n in lengths]).cuda() + P
    q, k, v = (t.cpu() for t in layer.project(x, positions))
    k0, v0 = (t.cpu() for t in layer.prefix)

    def same(got, attention):
        want = layer.o.forward_one_call(attention.half().cuda().view(got.shape[0], -1), out_t=TMAC_OUT_F16)
        assert (got.float() - want.float()).norm() <= 4e-3 * want.float().norm()   # fp16 tables 2e-3 each, and the attention's

    got = layer.prompt(x, c)
    keys = torch.cat([t for b in range(B) for t in (k0, k[c[b]:c[b + 1]])])
    vals = torch.cat([t for b in range(B) for t in (v0, v[c[b]:c[b + 1]])])
    cu_k = cu([n + P for n in lengths])
    want = ref.prompt(q, keys, vals, cu(lengths), cu_k, True, 1 / 8)
    same(got, want[0])
    # what the cache has kept: the heaviest and the last
    slots, at = [], 0
    for b, n in enumerate(lengths):
        w = want[2][:, cu_k[b] + P:cu_k[b + 1]]
        for h in range(Hkv):
            m = int(layer.cache.lens[b, h])
            pos = layer.cache.pos[b, h, :m].cpu()
            assert m == min(n, C) and set(range(max(0, n - recent), n)) <= set(pos.tolist())
            gone = [i for i in range(n) if i not in set(pos.tolist())]
            kept = [i for i in pos.tolist() if i < n - recent]
            assert not gone or w[h, gone].max() <= w[h, kept].min() * (1 + 1e-4)
            assert torch.equal(layer.cache.k[b, h, :m].cpu(), k[at:at + n, h][pos.long()])
        at += n
    for t in range(12):
        xt = rand(50 + t, B, M).cuda()
        q, k, v = (s.cpu() for s in layer.project(xt, layer.position))
        got = layer.step(xt)
        cache = layer.cache
        want = ref.decode(q, k0, v0, cache.k.cpu(), cache.v.cpu(), cache.lens.cpu(), 1 / 8)
        same(got, want[0])
        for b in range(B):
            for h in range(Hkv):
                slot = (cache.pos[b, h, :int(cache.lens[b, h])] == int(cache.seen[b, h]) - 1).nonzero()
                assert len(slot) == 1 and torch.equal(cache.k[b, h, int(slot)].cpu(), k[b, h])
    assert layer.cache.lens.tolist() == [[24, 24], [17, 17], [24, 24]] and layer.cache.seen[:, 0].tolist() == [n + 12 for n in lengths]


def test_decoder_example_runs(A, capsys):
    from paper_2407_00088_amd import decoder
    decoder.main(steps=2)
    assert "step 1" in capsys.readouterr().out


def test_a_captured_step_outlives_the_growth_of_its_workspace(A):
    """A graph keeps the workspace that it was captured with, whatever later, larger calls and other tensors take."""
    cache, _, _ = filled(A, 2, 8, 2, 64, 60, [[60, 60], [7, 30]], F16, garbage=0.0)
    q, k0, v0 = rand(5, 2, 8, 64).cuda(), rand(6, 9000, 2, 64).cuda(), rand(7, 9000, 2, 64).cuda()
    want = [x.clone() for x in cache.attend(q, k0[:700], v0[:700], weigh=False)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = cache.attend(q, k0[:700], v0[:700], weigh=False)
    first = cache.attend_ws
    cache.attend(q, k0, v0, weigh=False)
    assert cache.attend_ws is not first and any(x is first for x in cache.outgrown)
    del first
    for turn in range(4):
        others = [torch.full((n,), 7.0, device="cuda") for n in (2000, 30000, 300000)]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        assert all((x == 7.0).all() for x in others)


def test_results_whose_rows_overlap_and_sizes_beyond_32_bits_are_refused(A):
    q, k, c = rand(1, 14, 4, 64).cuda(), rand(2, 14, 2, 64).cuda(), i32([0, 5, 14])
    cache = A.KVCache(2, 2, 64, 8, Hq=4)
    room = torch.zeros(14 * 4 * 64, dtype=F16, device="cuda")
    far = k[:1].expand((1 << 31) + 5, 2, 64)
    for bad in (lambda: A.attn_prompt(q, k, k, c, out=room[:256].view(1, 4, 64).expand(14, 4, 64)),
                lambda: A.attn_prompt(q, k, k, c, out=room.as_strided((14, 4, 64), (252, 64, 1))),
                lambda: cache.attend(q[:2], out=room[:64].view(1, 1, 64).expand(2, 4, 64)),
                lambda: A.attn_prompt(q, far, far, c), lambda: cache.attend(q[:2], far, far),
                lambda: cache.fill(far, far, torch.zeros((2, 1), device="cuda").expand(2, far.shape[0]), c)):
        with pytest.raises(ValueError):
            bad()
    for ok in (room.view(4, 14, 64).transpose(0, 1), room.view(14, 4, 64)):
        assert A.attn_prompt(q, k, k, c, out=ok)[0] is ok
