"""Faults of the attention operators that reading or the CPU can show: what a kernel's wavefronts hand to each other, what its loads
reach, what the entry points refuse.  No GPU needed."""
import ctypes
import os
import re
import subprocess
import threading
import time

import pytest
import torch

import test_attention_host as H
from paper_2407_00088_amd import build


def source(name):
    return open(os.path.join(build.CSRC, name)).read()


def body_of(src, head):
    """The text between the braces that open after `head`."""
    at = src.index("{", src.index(head))
    depth = 0
    for i in range(at, len(src)):
        depth += {"{": 1, "}": -1}.get(src[i], 0)
        if depth == 0:
            return src[at:i + 1]
    raise AssertionError(head)


def test_sums_of_rows_are_handed_over_before_the_last_barrier():
    """The decode kernel of whole rows reads row_lse in every wavefront right after `finish`, whose first wavefront writes it."""
    src = source("tmac_attn.hip")
    finish = body_of(src, "void finish(")
    writes = [m.start() for m in re.finditer(r"row_lse\[", finish)]
    assert writes and max(writes) < finish.rindex("__syncthreads()")


CORE = """
#include "tmac_attn_core.h"
using namespace tmac::attn;
// Bytes from the first row to the end of what the loads of a stage read, of `rows` that are there: of 16 bytes a lane, four bytes at a
// time, those whose offset (without what a scalar register adds) is below the descriptor's range.
template <int DP, int ROWS, int WAVES, bool IS_V>
static long long reach(long long stride, int rows, int D) {
  typedef Stage<DP, ROWS, WAVES, IS_V> St;
  long long most = 0;
  for (int wave = 0; wave < WAVES; ++wave)
    for (int lane = 0; lane < 64; ++lane) {
      const St st(stride, D, wave, lane);
      if (!st.wanted) continue;
      const bool unchecked = St::unchecked(rows, D);
      const long long step = WAVES * Layout<DP>::RPI * stride;
      for (int i = 0; i < St::N; ++i) {
        const long long range = unchecked ? St::span(stride, ROWS, D) : St::span(stride, rows < ROWS ? rows : ROWS, D) - i * step;
        for (int b = 0; b < 16; b += 4)
          if ((long long)st.at + b < range) most = st.at + b + 4 + i * step > most ? st.at + b + 4 + i * step : most;
      }
    }
  return most;
}
extern "C" unsigned scores_in_lds() { return Scores{}.lds; }
extern "C" long long reach_of(int kind, long long stride, int rows, int D) {
  switch (kind + (D > 64 ? 8 : 0)) {
    case 0: return reach<64, 64, 4, false>(stride, rows, D);
    case 1: return reach<64, 64, 4, true>(stride, rows, D);
    case 2: return reach<64, 32, 1, false>(stride, rows, D);
    case 3: return reach<64, 32, 1, true>(stride, rows, D);
    case 8: return reach<128, 64, 4, false>(stride, rows, D);
    case 9: return reach<128, 64, 4, true>(stride, rows, D);
    case 10: return reach<128, 32, 1, false>(stride, rows, D);
    default: return reach<128, 32, 1, true>(stride, rows, D);
  }
}
"""


@pytest.fixture(scope="module")
def core(tmp_path_factory):
    out = tmp_path_factory.mktemp("reach") / "reach.so"
    flags = [f for f in build.HIPCC_FLAGS if not f.startswith(("--offload-arch", "-O", "-amdgpu", "-mllvm"))]
    subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), *flags, "-O1", "--offload-host-only", "-no-hip-rt", "-x", "hip", "-",
                    "-o", str(out)], input=CORE.encode(), stderr=subprocess.DEVNULL, check=True)
    lib = ctypes.CDLL(str(out))
    lib.reach_of.restype, lib.reach_of.argtypes = ctypes.c_longlong, [ctypes.c_int, ctypes.c_longlong, ctypes.c_int, ctypes.c_int]
    lib.scores_in_lds.restype = ctypes.c_uint
    return lib


@pytest.mark.parametrize("D", [4, 8, 36, 60, 64, 68, 100, 124, 128])
def test_stages_end_with_their_last_row(core, D):
    """Nothing is read beyond the last element of the last row that is there, where the tensor and its memory may end, and everything
    before it is."""
    for kind in range(4):
        for stride in (2 * D, 2 * D + 8, 64 * D, 0):
            for rows in [*range(1, 70), 1000]:
                there = min(rows, 64 if kind < 2 else 32)
                end = core.reach_of(kind, stride, rows, D)
                assert end <= (rows - 1) * stride + 2 * D, (kind, stride, rows)
                # (K's last half chunk comes another way)
                assert end >= (there - 1) * stride + 2 * (D if kind % 2 else D // 8 * 8) or D < 8, (kind, stride, rows)


def test_scores_that_are_not_in_lds_have_no_place_there(core):
    """Any offset within the 160 KB of LDS, the first too, is one that the compiler may give to the rows of scores."""
    assert core.scores_in_lds() >= 160 * 1024


def test_weights_refuse_rows_that_are_far_apart():
    """Rows of q and of k go through descriptors of 31-bit ranges, as those of the prompts' k and v do."""
    def weights(q=None, k=None):
        return H.A.lib.tmac_attn_weights(H.desc(), q or H.view(), k or H.view(), H.P16, 1, 10, 10, H.P16, H.P16, H.P16, H.P16, 1 << 40, None)
    for token in (1 << 22, 1 << 27, 1 << 39):
        assert weights(q=H.view(token=token)) == weights(k=H.view(token=token)) == H.T.TMAC_EUNSUPPORTED
        assert H.prompt(k=H.view(token=token)) == H.prompt(v=H.view(token=token)) == H.T.TMAC_EUNSUPPORTED
        assert H.decode(k0=H.view(token=token)) == H.decode(c=H.cache(v=H.view(seq=2560, token=token))) == H.T.TMAC_EUNSUPPORTED


@pytest.mark.parametrize("at", [0, 1])
def test_reserved_fields_of_a_cache_are_zero_in_every_call(at):
    c = H.cache()
    c.reserved[at] = 1
    row = H.view(seq=128)
    assert H.A.lib.tmac_cache_append(c, row, row, None) == H.decode(c=c) == H.T.TMAC_EINVAL
    assert H.A.lib.tmac_attn_decode_workspace_bytes(H.desc(), c, 10, 1) == H.A.lib.tmac_cache_fill_workspace_bytes(c) == 0


def test_launches_of_too_many_threads_are_refused_before_anything_is_launched():
    """2^32 threads or more of either launch of a call.  (Without a GPU any launch is an error of another kind.)"""
    one, many = H.desc(Hq=1, Hkv=1), H.desc(Hq=64, Hkv=64)
    A, P16, view, no = H.A, H.P16, H.view, H.T.TMAC_EUNSUPPORTED
    assert H.prompt(one, S=1 << 24, Tq=1 << 24, Tk=1 << 24) == no
    assert A.lib.tmac_attn_weights(one, view(), view(), P16, 1 << 24, 1 << 24, 1 << 24, P16, P16, P16, P16, 1 << 50, None) == no
    none = A.tmac_cache(A.tmac_view(), A.tmac_view(), None, None, None, None, 1 << 20, 64, 64, 0, 0, 0)
    assert H.decode(many, P=1, c=none, acc=0) == no                       # 2^26 rows: the joining launch
    few = [H.cache(Hkv=64, B=b, capacity=c, D=4) for b, c in ((1 << 18, 100), (1 << 12, 1 << 16))]
    for c in few:
        assert H.decode(H.desc(Hq=64, Hkv=64, D=4), c=c) == no
    row = view(seq=128)
    assert A.lib.tmac_cache_append(few[0], row, row, None) == no
    source = A.tmac_cache_source(view(), view(), A.tmac_view(P16, 0, 1, 100), A.tmac_view(), P16, None, None, 100)
    for c in few + [H.cache(Hkv=64, B=1 << 10, capacity=1 << 20, D=4)]:
        assert A.lib.tmac_cache_fill(c, source, P16, 1 << 60, None) == no


class OneAtATime:
    """In place of the library and of the binding's native side: calls that last, which notes whether another began meanwhile."""

    def __init__(self):
        self.running, self.most, self.calls = 0, 0, 0

    def __getattr__(self, name):
        def call(*args):
            if name.endswith("_bytes"):
                return 64
            self.running += 1
            self.calls += 1
            self.most = max(self.most, self.running)
            time.sleep(0.005)
            self.running -= 1
            return 0 if name.startswith("tmac_") else True
        return call


def test_calls_of_one_cache_from_several_threads_follow_each_other(monkeypatch):
    """Two launches of a call hand on a workspace that belongs to the cache: another thread's must not come between them."""
    made = OneAtATime()
    monkeypatch.setattr(H.A, "calls", made)
    monkeypatch.setattr(H.A, "lib", made)
    monkeypatch.setattr(H.A, "_same_device", lambda *tensors: None)
    monkeypatch.setattr(H.A.B, "_stream_ptr", lambda stream: None)
    one, two = (H.A.KVCache(1, 1, 64, 8, device="cpu") for _ in range(2))
    one.attend_ws = one.fill_ws = torch.empty(64, dtype=torch.uint8)
    row = torch.zeros((1, 1, 64), dtype=torch.float16)
    weight, cu = torch.zeros((1, 1)), torch.zeros(2, dtype=torch.int32)
    turns = [lambda: one.attend(row), lambda: one.append(row, row), lambda: one.fill(row, row, weight, cu), lambda: one.fill_from(two),
             lambda: two.fill_from(one)] * 4
    threads = [threading.Thread(target=turn, daemon=True) for turn in turns]
    for t in threads:
        t.start()
    for t in threads:
        t.join(30)
        assert not t.is_alive()
    assert made.calls == len(turns) and made.most == 1


@pytest.mark.parametrize("name", ["k", "v", "weight", "pos", "lens", "seen"])
def test_tensors_of_a_cache_are_not_replaced(name):
    """The library has their addresses: it would go on writing to a tensor that is no longer there."""
    cache = H.A.KVCache(1, 2, 64, 8, device="cpu")
    before = getattr(cache, name)
    with pytest.raises(AttributeError, match=name):
        setattr(cache, name, before * 1)
    before += 1
    exec(f"cache.{name} *= 3", dict(cache=cache))
    assert getattr(cache, name) is before and (before == 3).all()
