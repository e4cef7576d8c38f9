"""What the attention entry points refuse, and the sizes they ask for: host logic, no GPU needed."""
import ctypes as C
import os
import re

import pytest
import torch

import paper_2407_00088_amd as T
from paper_2407_00088_amd import attention as A

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P16 = 1 << 20  # an address that is aligned and never read


def test_header_and_binding_name_the_same_functions():
    src = open(os.path.join(ROOT, "include", "tmac_attn.h")).read()
    src = re.sub(r"/\*.*?\*/", "", src, flags=re.S)
    names = set(re.findall(r"\b(tmac_\w+)\s*\(", src))
    assert names == set(A.EXPORTS)
    for name in names:
        assert hasattr(T.lib, name)


def desc(**kw):
    d = A.attn_desc(8, 2, 64, torch.float16)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def view(data=P16, seq=0, token=128, head=64):
    return A.tmac_view(data, seq, token, head)


def prompt(d=None, q=None, k=None, v=None, S=1, Tq=10, Tk=10, cu_q=P16, cu_k=P16, out=None, lse=None, ws=P16, ws_bytes=1 << 40):
    return A.lib.tmac_attn_prompt(d or desc(), q or view(), k or view(), v or view(), S, Tq, Tk, cu_q, cu_k, out or view(), lse, ws, ws_bytes,
                                  None)


BAD_DESCS = [dict(Hq=0), dict(Hq=7), dict(Hkv=0), dict(Hkv=-2), dict(D=0), dict(D=6), dict(D=-4), dict(elem=2), dict(elem=-1), dict(scale=0.0),
             dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(causal=2), dict(causal=-1)]
BAD_VIEWS = [view(data=None), view(data=P16 + 2), view(data=P16 + 4), view(token=130), view(head=-64), view(token=-128), view(head=1 << 41)]


@pytest.mark.parametrize("bad", BAD_DESCS, ids=str)
def test_descriptions_that_are_refused(bad):
    d = desc(**bad)
    assert prompt(d) == T.TMAC_EINVAL
    assert A.lib.tmac_attn_weights(d, view(), view(), P16, 1, 10, 10, P16, P16, P16, P16, 1 << 40, None) == T.TMAC_EINVAL
    assert A.lib.tmac_attn_prompt_workspace_bytes(d, 1, 10, 10) == 0
    assert A.lib.tmac_attn_weights_workspace_bytes(d, 1, 10, 10) == 0
    c = cache()
    c.Hkv, c.D, c.elem = d.Hkv, d.D, d.elem
    if "causal" not in bad:
        assert A.lib.tmac_attn_decode_workspace_bytes(d, c, 10, 1) == 0
        assert decode(d, c=c) == T.TMAC_EINVAL
    d = desc()
    d.reserved[1] = 1
    assert prompt(d) == T.TMAC_EINVAL


@pytest.mark.parametrize("which", ["q", "k", "v", "out"])
@pytest.mark.parametrize("bad", BAD_VIEWS, ids=lambda v: f"{v.data}-{v.token}-{v.head}")
def test_prompt_views_that_are_refused(which, bad):
    assert prompt(**{which: bad}) == T.TMAC_EINVAL
    if which in "qk":
        args = dict(q=view(), k=view())
        args[which] = bad
        assert A.lib.tmac_attn_weights(desc(), args["q"], args["k"], P16, 1, 10, 10, P16, P16, P16, P16, 1 << 40, None) == T.TMAC_EINVAL


def test_prompt_refusals():
    assert prompt(S=-1) == prompt(Tq=-1) == prompt(Tk=-1) == T.TMAC_EINVAL
    assert prompt(cu_q=None) == prompt(cu_k=None) == T.TMAC_EINVAL
    assert prompt(desc(D=132)) == T.TMAC_EUNSUPPORTED
    assert prompt(Tq=(1 << 30)) == T.TMAC_EUNSUPPORTED
    assert prompt(k=view(token=1 << 22)) == T.TMAC_EUNSUPPORTED
    assert prompt(S=0) == prompt(Tq=0) == T.TMAC_OK          # nothing to do, nothing enqueued
    need = A.lib.tmac_attn_prompt_workspace_bytes(desc(), 1, 4, 100000)
    assert need > 0
    assert prompt(Tq=4, Tk=100000, ws_bytes=need - 1) == T.TMAC_ESIZE
    assert prompt(Tq=4, Tk=100000, ws=None) == prompt(Tq=4, Tk=100000, ws=P16 + 8) == T.TMAC_EINVAL


def test_weights_refusals():
    def weights(lse=P16, S=1, Tq=10, Tk=10, cu_q=P16, out=P16, ws=P16, n=1 << 40, d=None):
        return A.lib.tmac_attn_weights(d or desc(), view(), view(), lse, S, Tq, Tk, cu_q, P16, out, ws, n, None)
    assert weights(lse=None) == weights(cu_q=None) == weights(out=None) == weights(S=-1) == T.TMAC_EINVAL
    assert weights(d=desc(D=132)) == T.TMAC_EUNSUPPORTED
    assert weights(S=0) == weights(Tk=0) == T.TMAC_OK
    need = A.lib.tmac_attn_weights_workspace_bytes(desc(), 1, 100000, 128)
    assert need > 0 and weights(Tq=100000, Tk=128, n=need - 1) == T.TMAC_ESIZE


def cache(**kw):
    c = A.tmac_cache(view(seq=2560, token=64, head=1280), view(seq=2560, token=64, head=1280), P16, P16, P16, P16, 3, 2, 64, 20, 4,
                     A.TMAC_ELEM_F16)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def decode(d=None, q=None, k0=None, v0=None, P=10, c=None, acc=1, out=None, ws=P16, n=1 << 40):
    return A.lib.tmac_attn_decode(d or desc(), q or view(seq=512), k0 or view(), v0 or view(), P, c or cache(), acc, out or view(seq=512), None,
                                  ws, n, None)


def test_decode_refusals():
    for bad in BAD_VIEWS[:3] + [view(head=-64), view(seq=-512), view(seq=6)]:
        assert decode(q=bad) == decode(out=bad) == T.TMAC_EINVAL
    for bad in BAD_VIEWS:
        assert decode(k0=bad) == decode(v0=bad) == decode(c=cache(k=bad)) == decode(c=cache(v=bad)) == T.TMAC_EINVAL
    for bad in (dict(B=-1), dict(Hkv=4), dict(D=128), dict(elem=1), dict(capacity=-1), dict(lens_dev=None), dict(weight_dev=None)):
        assert decode(c=cache(**bad)) == T.TMAC_EINVAL, bad
    assert decode(acc=2) == decode(P=-1) == decode(ws=None) == decode(ws=P16 + 8) == T.TMAC_EINVAL
    assert decode(k0=view(token=1 << 22)) == T.TMAC_EUNSUPPORTED
    assert decode(c=cache(B=0)) == T.TMAC_OK
    need = A.lib.tmac_attn_decode_workspace_bytes(desc(), cache(), 10, 1)
    assert need > A.lib.tmac_attn_decode_workspace_bytes(desc(), cache(), 10, 0) > 0
    assert decode(n=need - 1) == T.TMAC_ESIZE


def test_cache_refusals():
    def append(c=None, k=None, v=None):
        return A.lib.tmac_cache_append(c or cache(), k or view(seq=128), v or view(seq=128), None)

    def source(**kw):
        s = A.tmac_cache_source(view(), view(), A.tmac_view(P16, 0, 1, 100), A.tmac_view(), P16, None, None, 100)
        for k, v in kw.items():
            setattr(s, k, v)
        return s

    def fill(c=None, s=None, ws=P16, n=1 << 40):
        return A.lib.tmac_cache_fill(c or cache(), s or source(), ws, n, None)

    for bad in (dict(B=-1), dict(Hkv=0), dict(D=0), dict(D=6), dict(elem=5), dict(capacity=0), dict(recent=-1), dict(recent=21),
                dict(weight_dev=None), dict(pos_dev=None), dict(lens_dev=None), dict(seen_dev=None), dict(k=view(data=None)),
                dict(v=view(token=130))):
        assert append(cache(**bad)) == fill(cache(**bad)) == T.TMAC_EINVAL, bad
    assert append(cache(D=132)) == fill(cache(D=132)) == T.TMAC_EUNSUPPORTED
    assert append(cache(B=0)) == fill(cache(B=0)) == T.TMAC_OK
    for bad in (view(data=None), view(data=P16 + 4), view(seq=-4), view(head=2)):
        assert append(k=bad) == append(v=bad) == T.TMAC_EINVAL
    for bad in BAD_VIEWS:
        assert fill(s=source(k=bad)) == fill(s=source(v=bad)) == T.TMAC_EINVAL
    for bad in (dict(cu_dev=None), dict(lens_dev=P16), dict(total=-1), dict(reserved=1), dict(weight=A.tmac_view()),
                dict(weight=A.tmac_view(P16 + 2, 0, 1, 100)), dict(weight=A.tmac_view(P16, 0, -1, 100)), dict(pos=A.tmac_view(P16, 0, 1, -1))):
        assert fill(s=source(**bad)) == T.TMAC_EINVAL, bad
    need = A.lib.tmac_cache_fill_workspace_bytes(cache())
    assert need == 3 * 2 * 20 * 4 and fill(n=need - 1) == T.TMAC_ESIZE and fill(ws=None) == T.TMAC_EINVAL
    assert A.lib.tmac_cache_fill_workspace_bytes(cache(capacity=0)) == 0


def test_binding_checks_what_the_library_takes_on_trust():
    q, k = torch.zeros((4, 8, 64), dtype=torch.float16), torch.zeros((4, 2, 64), dtype=torch.float16)
    c = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="on the GPU"):
        A.attn_prompt(q, k, k, c)
    with pytest.raises(ValueError, match="float16 or bfloat16"):
        A.attn_prompt(q.float(), k.float(), k.float(), c)
    with pytest.raises(ValueError):
        A.attn_prompt(q[0], k, k, c)
    with pytest.raises(ValueError, match="float16 or bfloat16"):
        A.attn_desc(8, 2, 64, torch.float32)
    with pytest.raises(ValueError, match="recent"):
        A.KVCache(1, 1, 64, 8, recent=9, device="cpu")


def test_workspaces_grow_with_what_is_asked():
    d = desc()
    assert A.lib.tmac_attn_prompt_workspace_bytes(d, 1, 8192, 8192) == 0           # the chip is full without splitting the keys
    assert A.lib.tmac_attn_prompt_workspace_bytes(d, 0, 1, 1) == A.lib.tmac_attn_prompt_workspace_bytes(desc(D=256), 1, 1, 1) == 0
    small, large = (A.lib.tmac_attn_decode_workspace_bytes(d, cache(capacity=n), 0, 1) for n in (100, 100000))
    assert 0 < small < large


def test_lengths_that_do_not_fit_a_32_bit_index():
    one = desc(Hq=1, Hkv=1)
    far = (1 << 30) + 1
    for sizes in ((far, 10, 10), (1, far, 10), (1, 10, far)):
        S, Tq, Tk = sizes
        assert prompt(one, S=S, Tq=Tq, Tk=Tk) == T.TMAC_EUNSUPPORTED
        assert A.lib.tmac_attn_weights(one, view(), view(), P16, S, Tq, Tk, P16, P16, P16, P16, 1 << 40, None) == T.TMAC_EUNSUPPORTED
        assert A.lib.tmac_attn_prompt_workspace_bytes(one, S, Tq, Tk) == A.lib.tmac_attn_weights_workspace_bytes(one, S, Tq, Tk) == 0
    large = cache(capacity=far)
    assert decode(c=large) == decode(P=far) == T.TMAC_EUNSUPPORTED
    assert A.lib.tmac_attn_decode_workspace_bytes(desc(), large, 10, 1) == A.lib.tmac_attn_decode_workspace_bytes(desc(), cache(), far, 1) == 0
    row = view(seq=128)
    assert A.lib.tmac_cache_append(large, row, row, None) == T.TMAC_EUNSUPPORTED
    source = A.tmac_cache_source(view(), view(), A.tmac_view(P16, 0, 1, 100), A.tmac_view(), P16, None, None, 100)
    assert A.lib.tmac_cache_fill(large, source, P16, 1 << 50, None) == T.TMAC_EUNSUPPORTED
    source.total = far
    assert A.lib.tmac_cache_fill(cache(), source, P16, 1 << 40, None) == T.TMAC_EUNSUPPORTED
