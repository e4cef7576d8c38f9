"""What the entry points of pages and rotation refuse, where the elements of a block lie, what a wavefront reads of it, frequencies, which pages
belong to whom: host logic, no GPU needed."""
import ctypes as C
import math
import os
import re
import subprocess

import pytest
import torch

import paper_2407_00088_amd as T
from paper_2407_00088_amd import build
from paper_2407_00088_amd import pages as G

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P16 = 1 << 20  # an address that is aligned and never read


def test_header_and_binding_name_the_same_functions():
    src = open(os.path.join(ROOT, "include", "tmac_pages.h")).read()
    src = re.sub(r"/\*.*?\*/", "", src, flags=re.S)
    assert set(re.findall(r"\b(tmac_\w+)\s*\(", src)) == set(G.EXPORTS)
    for name in G.EXPORTS:
        assert hasattr(T.lib, name)


# --- refusals ------------------------------------------------------------------------------------------------------------------------


def changed(x, kw):
    for k, v in kw.items():
        setattr(x, k, v)
    return x


def view(data=P16, token=512, head=64):
    return G.tmac_view(data, 0, token, head)


BAD_VIEWS = [view(data=None), view(data=P16 + 4), view(token=130), view(head=-64), view(token=-128), view(head=1 << 41)]


def rope(**kw):
    return changed(G.tmac_rope(P16, 1.0, 64, 64, 0, 0), kw)


def item(**kw):
    return changed(G.tmac_rope_item(view(), view(data=2 * P16), 8, 0), kw)


def rotate(r=None, items=None, count=None, positions=P16, tokens=10):
    items = [item()] if items is None else items
    return G.lib.tmac_rotate(r or rope(), (G.tmac_rope_item * max(len(items), 1))(*items), len(items) if count is None else count, positions, tokens, None)


BAD_ROPES = [dict(freq_dev=None), dict(freq_dev=P16 + 4), dict(D=0), dict(D=-4), dict(D=66), dict(rot=0), dict(rot=63), dict(rot=66), dict(rot=-2), dict(interleaved=2),
             dict(interleaved=-1), dict(elem=2), dict(elem=-1), dict(magnitude=math.nan), dict(magnitude=math.inf)]


def test_rotate_refusals():
    for bad in BAD_ROPES:
        assert rotate(rope(**bad)) == T.TMAC_EINVAL, bad
        assert append(r=rope(**bad)) == T.TMAC_EINVAL, bad
    r = rope()
    r.reserved[1] = 1
    assert rotate(r) == T.TMAC_EINVAL
    for bad in BAD_VIEWS:
        assert rotate(items=[item(x=bad)]) == rotate(items=[item(), item(out=bad)]) == T.TMAC_EINVAL
    for bad in (dict(H=0), dict(H=-1), dict(reserved=1), dict(out=view(token=1024))):      # (the last: in place, but not by its strides)
        assert rotate(items=[item(**bad)]) == T.TMAC_EINVAL, bad
    assert rotate(count=0) == rotate(count=5, items=[item()] * 5) == rotate(positions=None) == rotate(positions=P16 + 4) == rotate(tokens=-1) == T.TMAC_EINVAL
    assert G.lib.tmac_rotate(None, (G.tmac_rope_item * 1)(item()), 1, P16, 4, None) == G.lib.tmac_rotate(rope(), None, 1, P16, 4, None) == T.TMAC_EINVAL
    assert rotate(rope(D=132, rot=64)) == rotate(tokens=(1 << 30) + 1) == rotate(items=[item(H=(1 << 24) + 1)]) == T.TMAC_EUNSUPPORTED
    assert rotate(tokens=0) == T.TMAC_OK


def pages(**kw):
    return changed(G.tmac_pages(P16, P16, 10, 64, 2, 64, 1), kw)


def batch(**kw):
    return changed(G.tmac_pages_batch(P16, 5, P16, P16, 3, 5, 10, 0), kw)


def append(p=None, b=None, elem=0, k=None, v=None, r=None, positions=None, q=None, q_out=None, Hq=8):
    return G.lib.tmac_pages_append(p or pages(), b or batch(), elem, k or view(), v or view(), r, positions, q, q_out, Hq, None)


def read(p=None, b=None, elem=0, k=None, v=None):
    return G.lib.tmac_pages_read(p or pages(), b or batch(), elem, k or view(), v or view(), None)


def desc(**kw):
    d = T.attention.attn_desc(8, 2, 64, torch.float16)
    return changed(d, kw)


def attend(d=None, p=None, b=None, q=None, out=None, lse=None, ws=P16, n=1 << 40):
    return G.lib.tmac_pages_attend(d or desc(), p or pages(), b or batch(), q or view(), out or view(), lse, ws, n, None)


BAD_PAGES = [dict(pages=-1), dict(page=0), dict(page=16), dict(page=48), dict(page=8192), dict(page=-64), dict(Hkv=0), dict(Hkv=-2), dict(D=0), dict(D=6), dict(D=-4),
             dict(code=2), dict(code=-1)]
UNSET_PAGES = [dict(codes_dev=None), dict(codes_dev=P16 + 8), dict(scales_dev=None), dict(scales_dev=P16 + 4)]
BAD_BATCHES = [dict(S=-1), dict(T=-1), dict(width=-1), dict(most=-1), dict(table_stride=4), dict(table_stride=-5), dict(cu_dev=None), dict(table_dev=None),
               dict(lens_dev=None)]


def test_pages_refusals():
    for bad in BAD_PAGES:
        p = pages(**bad)
        assert append(p) == read(p) == attend(p=p) == T.TMAC_EINVAL, bad
        assert G.lib.tmac_pages_code_bytes(p) == G.lib.tmac_pages_scale_bytes(p) == G.lib.tmac_pages_attend_workspace_bytes(desc(), p, batch()) == 0
    for bad in UNSET_PAGES:
        p = pages(**bad)
        assert append(p) == read(p) == attend(p=p) == T.TMAC_EINVAL, bad
    p = pages()
    p.reserved[2] = 1
    assert append(p) == read(p) == attend(p=p) == T.TMAC_EINVAL
    for bad in BAD_BATCHES:
        b = batch(**bad)
        assert append(b=b) == read(b=b) == attend(b=b) == T.TMAC_EINVAL, bad
    for bad in BAD_VIEWS:
        assert append(k=bad) == append(v=bad) == read(k=bad) == read(v=bad) == attend(q=bad) == attend(out=bad) == T.TMAC_EINVAL
        assert append(r=rope(), q=bad, q_out=view()) == append(r=rope(), q=view(), q_out=bad) == T.TMAC_EINVAL
    assert append(elem=2) == read(elem=-1) == T.TMAC_EINVAL
    # queries and positions only with a rotation, of the same heads and type; a result for queries that are there
    assert append(q=view(), q_out=view()) == append(positions=P16) == append(r=rope(), positions=P16 + 4) == T.TMAC_EINVAL
    assert append(r=rope(), q=view()) == append(r=rope(), q_out=view()) == append(r=rope(), q=view(), q_out=view(data=2 * P16), Hq=0) == T.TMAC_EINVAL
    assert append(r=rope(D=32, rot=32)) == append(r=rope(elem=1)) == T.TMAC_EINVAL
    for bad in (dict(Hq=7), dict(Hq=0), dict(Hkv=4), dict(D=128), dict(elem=2), dict(scale=0.0), dict(scale=math.nan), dict(causal=0)):
        assert attend(desc(**bad)) == T.TMAC_EINVAL, bad
    far = (1 << 30) + 1
    for b in (batch(S=far), batch(T=far), batch(width=1 << 25, table_stride=1 << 25)):
        assert append(b=b) == read(b=b) == attend(b=b) == T.TMAC_EUNSUPPORTED
    p = pages(D=132)
    assert append(p) == read(p) == attend(desc(D=132), p) == T.TMAC_EUNSUPPORTED
    for b in (batch(S=0), batch(T=0)):
        assert append(b=b) == read(b=b) == attend(b=b) == T.TMAC_OK


def test_attend_workspace():
    wide = batch(width=500, table_stride=500)
    need = G.lib.tmac_pages_attend_workspace_bytes(desc(), pages(), wide)
    assert need > 0
    assert attend(b=wide, n=need - 1) == T.TMAC_ESIZE and attend(b=wide, ws=None) == attend(b=wide, ws=P16 + 8) == T.TMAC_EINVAL
    # a few short sequences: every one by a workgroup of its own, nothing to join
    assert G.lib.tmac_pages_attend_workspace_bytes(desc(), pages(), batch(T=3, cu_dev=None)) == 0
    # what is needed does not depend on lengths, and not on how many rows where none has many
    assert G.lib.tmac_pages_attend_workspace_bytes(desc(), pages(), batch(width=500, table_stride=500, T=3, cu_dev=None)) <= need


def test_sizes():
    assert G.lib.tmac_pages_code_bytes(pages()) == 10 * 2 * 2 * 4096 and G.lib.tmac_pages_scale_bytes(pages()) == 10 * 2 * 2 * 8
    assert G.lib.tmac_pages_code_bytes(pages(D=100)) == 10 * 2 * 2 * 7168
    assert G.lib.tmac_pages_code_bytes(pages(pages=1 << 20, page=4096, Hkv=8, D=128)) == (1 << 20) * 8 * 128 * 8192


def test_binding_checks():
    with pytest.raises(ValueError, match="code"):
        T.PagedCache(4, 1, 64, code="e5m2", device="cpu")
    for bad in (dict(page=48), dict(page=16), dict(D=130), dict(D=6), dict(Hkv=0)):
        with pytest.raises(ValueError):
            T.PagedCache(**{**dict(pages=4, Hkv=1, D=64, device="cpu"), **bad})
    with pytest.raises(ValueError, match="elements"):
        T.PagedCache(4, 1, 64, rotary=T.Rotary(32, device="cpu"), device="cpu")
    for bad in (dict(rot=0), dict(rot=3), dict(rot=66)):
        with pytest.raises(ValueError, match="rot"):
            T.Rotary(64, device="cpu", **bad)
    cache = T.PagedCache(4, 1, 64, device="cpu")
    assert cache.codes.shape == (4, 1, 2, 4096) and cache.scales.shape == (4, 1, 2, 2)
    with pytest.raises(AttributeError, match="replaced"):
        cache.scales = torch.zeros(1)
    with pytest.raises(ValueError, match="elements"):
        cache.rotary = T.Rotary(32, device="cpu")
    k = torch.zeros((2, 1, 64), dtype=torch.float16)
    table, lens = torch.zeros((2, 3), dtype=torch.int32), torch.ones(2, dtype=torch.int32)
    for call in (lambda: cache.append(k, k, table, lens), lambda: cache.attend(k, table, lens), lambda: cache.read(table, lens),
                 lambda: T.Rotary(64, device="cpu").rotate(lens.long(), k)):
        with pytest.raises(ValueError, match="GPU"):
            call()
    with pytest.raises(ValueError, match="one to 4"):
        T.Rotary(64, device="cpu").rotate(lens.long())


# --- where things lie ------------------------------------------------------------------------------------------------------------------

CORE = """
#include "tmac_pages_core.h"
using namespace tmac::pages;
extern "C" int key_at_(int t, int d) { return key_at(t, d); }
extern "C" int value_at_(int c, int t, int d) { return value_at(c, t, d); }
extern "C" int value_token_(int h, int j) { return value_token(h, j); }
extern "C" int reads(int rows, int keys, int i, int lane, int last, int odd) {
  const At a = rows == 16 ? (keys ? Reads16::k(i, lane) : Reads16::v(i, lane, last, odd)) : (keys ? Reads32::k(i, lane) : Reads32::v(i, lane, last, odd));
  return a.lane + a.fixed;
}
extern "C" long long unit_of_(int pages, int shift, int Hkv, const int* table, int width, int block, int head) {
  Pages p = {};
  p.pages = pages, p.shift = shift, p.Hkv = Hkv;
  return p.unit_of(table, width, block, head);
}
"""


@pytest.fixture(scope="module")
def core(tmp_path_factory):
    d = tmp_path_factory.mktemp("core")
    (d / "core.hip").write_text(CORE)
    subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "-x", "hip", "--offload-host-only", "-O1", "-std=c++17", "-fPIC", "-shared", "-I" + build.CSRC,
                    "-I" + os.path.join(ROOT, "include"), str(d / "core.hip"), "-o", str(d / "core.so")], stderr=subprocess.DEVNULL, check=True)
    lib = C.CDLL(str(d / "core.so"))
    lib.unit_of_.restype = C.c_longlong
    return lib


@pytest.mark.parametrize("D", [4, 16, 20, 32, 48, 64, 80, 96, 100, 112, 128])
def test_elements_of_a_block(core, D):
    """Every place of a plane has one element, by the header's description; what the wavefronts read of it is what their products take."""
    c = (D + 15) // 16
    where = {}
    for t in range(32):
        for d in range(16 * c):
            run = 16 if c * 16 - d // 32 * 32 < 32 else 32
            assert core.key_at_(t, d) == d // 16 * 512 + t * 16 + d % 16
            at = d // 32 * 1024 + (t // 4 % 2 * run + d % 32) * 16 + 8 * (t // 8 % 2) + 4 * (t // 16) + t % 4
            assert core.value_at_(c, t, d) == at
            where[at] = t, d
    assert sorted(where) == list(range(512 * c))
    for h in (0, 1):
        assert [core.value_token_(h, j) for j in range(16)] == [where[h * (16 if c == 1 else 32) * 16 + j][0] for j in range(16)]
    ni, odd, plane = (D + 31) // 32, c % 2, 512 * c
    for lane in range(64):
        # 32 rows: keys of token lane % 32, elements 32 i + 16 (lane / 32) on; values of element 32 i + lane % 32, a half's tokens
        for i in range(ni):
            at = core.reads(32, 1, i, lane, 0, 0)
            chunk = 2 * i + lane // 32
            assert at == core.key_at_(lane % 32, 16 * chunk) if chunk < c else at >= plane
            at = core.reads(32, 0, i, lane, i == ni - 1, odd)
            d = 32 * i + lane % 32
            assert [where[at + j] for j in range(16)] == [(core.value_token_(lane // 32, j), d) for j in range(16)] if d < 16 * c else at >= plane
        # 16 rows: keys of token lane % 16 (+ 16), elements of chunk 4 (i / 2) + lane / 16; values of element 16 i + lane % 16, tokens 4 q .. and 16 + 4 q ..
        q = lane // 16
        for i in range((ni + 1) // 2 * 2):
            at, chunk = core.reads(16, 1, i, lane, 0, 0), 4 * (i // 2) + q
            assert at == core.key_at_(i % 2 * 16 + lane % 16, 16 * chunk) if chunk < c else at >= plane
        for i in range(2 * ni):
            at, d = core.reads(16, 0, i, lane, i >= 2 * ni - 2, odd), 16 * i + lane % 16
            if d < 16 * c:
                assert [where[at + j] for j in range(8)] == [(16 * (j // 4) + 4 * q + j % 4, d) for j in range(8)]
            else:   # (nobody reads what these give, and an address past the plane gives zeros)
                assert at >= 0


def test_pages_that_are_not_there_have_no_unit(core):
    table = (C.c_int * 4)(3, -1, 7, 1 << 30)
    unit = lambda block, head=1: core.unit_of_(7, 2, 2, table, 4, block, head)  # noqa: E731
    assert unit(0) == (3 * 2 + 1) * 4 and unit(3, 0) == 3 * 2 * 4 + 3
    assert unit(4) == unit(8) == unit(12) == -1      # no page, one past the last, one far off
    assert unit(16) == unit(1 << 25) == -1           # behind the table, which is not read there
    big = (C.c_int * 1)((1 << 31) - 2)
    assert core.unit_of_((1 << 31) - 1, 7, 64, big, 1, 127, 63) == ((((1 << 31) - 2) * 64 + 63) << 7) + 127


# --- frequencies ----------------------------------------------------------------------------------------------------------------------------


def test_frequencies():
    f, m = G.frequencies(8)
    assert m == 1.0 and torch.allclose(f, torch.tensor([1.0, 0.1, 0.01, 0.001], dtype=torch.float64), rtol=1e-15)
    assert torch.equal(G.frequencies(8, scaling=("linear", 4.0))[0], f / 4)
    g = G.frequencies(8, scaling=("base", 4.0))[0]
    assert abs(g[0] - 1) < 1e-15 and abs(g[3] * 4 / f[3] - 1) < 1e-14 and g[1] < f[1]
    f = G.frequencies(128)[0]
    g, m = G.frequencies(128, scaling=("ramp", 8.0, 8192.0, 32.0, 1.0))
    turns = 8192 * f / (2 * math.pi)
    assert torch.equal(g[turns > 40], f[turns > 40]) and torch.allclose(g[turns < 0.8], f[turns < 0.8] / 8, rtol=1e-12) and (g <= f).all() and (g >= f / 8.0001).all()
    assert abs(m - (0.1 * math.log(8) + 1)) < 1e-15
    g, m = G.frequencies(128, scaling=("bands", 8.0, 8192.0, 1.0, 4.0))
    assert m == 1.0 and torch.equal(g[turns >= 4], f[turns >= 4]) and torch.allclose(g[turns <= 1], f[turns <= 1] / 8, rtol=1e-15)
    mid = (turns > 1) & (turns < 4)
    mix = (turns[mid] - 1) / 3
    assert mid.any() and torch.allclose(g[mid], f[mid] * mix + f[mid] / 8 * (1 - mix), rtol=1e-14)


@pytest.mark.parametrize("bad", [("cubic", 2.0), ("linear",), ("linear", 0.0), ("linear", math.nan), ("base", 2.0, 3.0), ("ramp", 2.0, 4096.0, 1.0, 32.0),
                                 ("bands", 2.0, 4096.0, 4.0, 1.0)])
def test_scalings_that_are_refused(bad):
    with pytest.raises(ValueError):
        G.frequencies(64, scaling=bad)


def test_bases_that_are_refused():
    for base in (1.0, 0.0, -2.0, math.inf):
        with pytest.raises(ValueError):
            G.frequencies(64, base=base)
    with pytest.raises(ValueError):
        G.frequencies(2, scaling=("base", 2.0))


# --- which pages belong to whom ---------------------------------------------------------------------------------------------------------------


def test_page_table():
    t = G.PageTable(3, 4, 7, page=32, device="cpu")
    table, lens = t.table, t.lens

    def whole():
        used = [p for own in t.owned for p in own]
        assert len(used) + len(t.free) == 7 and sorted(used + t.free) == list(range(7))
        for s in range(3):
            assert table[s].tolist() == t.owned[s] + [-1] * (4 - len(t.owned[s]))
            assert len(t.owned[s]) == -(-t.length[s] // 32) and lens[s] == t.length[s]

    cu, most = t.extend([33, 0, 32])
    whole()
    assert cu.tolist() == [0, 33, 33, 65] and cu.dtype == torch.int32 and most == 33
    t.extend([31, 1, 1])
    whole()
    before = [list(o) for o in t.owned], list(t.length), list(t.free)
    with pytest.raises(MemoryError):
        t.extend([64, 64, 32])
    with pytest.raises(ValueError, match="at most 4 pages"):
        t.extend([65, 0, 0])
    for bad in ([1, 1], [1, -1, 1]):
        with pytest.raises(ValueError):
            t.extend(bad)
    for bad in ([65, 0, 0], [0, 0, -1], [1]):
        with pytest.raises(ValueError):
            t.take_back(bad)
    assert before == ([list(o) for o in t.owned], list(t.length), list(t.free))
    t.take_back([64, 0, 1])
    whole()
    assert t.length == [0, 1, 32] and t.table is table and t.lens is lens
    t.extend([128, 0, 0])
    whole()
    with pytest.raises(ValueError):
        G.PageTable(0, 1, 1, device="cpu")
