"""Faults of the paged cache's host side that have been mended: no GPU needed."""
import pytest
import torch

import paper_2407_00088_amd as T
from paper_2407_00088_amd import pages as G
from test_pages_host import append, attend, batch, desc, pages, read


def test_a_rotation_is_not_taken_apart():
    """Calls go by the address and the sizes that a Rotary had when it was made: other frequencies would be read where the old ones were, after these are gone."""
    rotary = T.Rotary(64, device="cpu")
    for name, value in (("freq", rotary.freq * 2), ("freq", rotary.freq.float()), ("magnitude", 2.0), ("D", 32), ("rot", 32), ("interleaved", True), ("rope", {})):
        with pytest.raises(AttributeError, match="replaced"):
            setattr(rotary, name, value)
    rotary.freq *= 1.0          # (written to, where it is)
    x = torch.zeros((2, 1, 64), dtype=torch.float16)
    rotary.freq.data = rotary.freq.clone()
    for dtype in (torch.float16, torch.bfloat16):
        with pytest.raises(ValueError, match="other memory"):
            rotary.rotate(torch.arange(2), x.to(dtype))


def test_a_cache_is_not_taken_apart():
    """Tensors are checked against the sizes that the object has, kernels go by the ones that it was made with; the same for where codes and scales are."""
    cache = T.PagedCache(4, 2, 64, Hq=4, device="cpu")
    for name, value in (("Hq", 2), ("Hkv", 1), ("D", 32), ("page", 32), ("dtype", torch.bfloat16), ("desc", None), ("cache", None)):
        with pytest.raises(AttributeError, match="replaced"):
            setattr(cache, name, value)
    cache.rotary, cache.rotary = T.Rotary(64, device="cpu"), None
    table, lens = torch.zeros((2, 3), dtype=torch.int32), torch.ones(2, dtype=torch.int32)
    for name in ("codes", "scales"):
        moved = T.PagedCache(4, 2, 64, Hq=4, device="cpu")
        t = getattr(moved, name)
        t.data = t.clone()
        with pytest.raises(ValueError, match="other memory"):
            moved.read(table, lens)
    assert T.PagedCache(0, 2, 64, device="cpu").codes.numel() == 0
    with pytest.raises(ValueError, match="GPU"):        # (pages none, which have no address)
        T.PagedCache(0, 2, 64, device="cpu").read(table, lens)


def test_more_pages_than_can_be_counted_are_refused():
    """pages * key heads * blocks of a page beyond 2^63: the number of units came out small, and so did the bytes that a caller is told to keep."""
    most = (1 << 31) - 1
    for p, d in ((pages(pages=most, Hkv=most, page=4096), desc(Hkv=most, Hq=most)), (pages(pages=1 << 30, Hkv=1 << 27, page=4096), desc(Hkv=1 << 27, Hq=1 << 27)),
                 (pages(pages=1 << 30, Hkv=1 << 10, page=4096), desc(Hkv=1 << 10, Hq=1 << 10))):
        assert G.lib.tmac_pages_code_bytes(p) == G.lib.tmac_pages_scale_bytes(p) == G.lib.tmac_pages_attend_workspace_bytes(d, p, batch()) == 0
        assert append(p) == read(p) == attend(d, p) == T.TMAC_EUNSUPPORTED
    p = pages(pages=1 << 30, Hkv=8, page=4096)
    assert G.lib.tmac_pages_code_bytes(p) == (1 << 40) * 4096 and G.lib.tmac_pages_scale_bytes(p) == (1 << 40) * 8


def test_a_layer_refuses_counts_below_zero_of_a_call_without_rows():
    from paper_2407_00088_amd.decoder import PagedDecoderAttention
    layer = object.__new__(PagedDecoderAttention)      # (refused before anything on the GPU is looked at)
    layer.table = T.PageTable(2, 2, 4, device="cpu")
    with pytest.raises(ValueError, match="rows"):
        layer.forward(torch.zeros((0, 64), dtype=torch.float16), [1, -1])
