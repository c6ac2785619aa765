"""What the Python calls on pages refuse before the library is asked, and what they pass on (no GPU: nothing here is launched)."""
import pytest
import torch

from paper_2501_19392_amd import binding as B


def layer(**kw):
    return B.Layer(2, 128, None, None, None, torch.bfloat16, **{"rtn_bits": 4, **kw})


def refused_append(lay, pages, K, slots, positions, cos, sin, match):
    with pytest.raises(ValueError, match=match):
        B.aquakv_paged_append(lay, pages, K.shape[0], K, K, slots, positions, cos, sin, None, None)


def test_rotary_tables_have_64_angles_a_row():
    lay = layer()
    pages = B.Pages(lay, 3, 8, device="cpu")
    K, slots, pos = torch.zeros(4, 2, 128, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int64), torch.zeros(4, dtype=torch.int32)
    good, wide = torch.zeros(10, 64), torch.zeros(5, 128)
    for cos, sin in ((wide, wide), (good, wide), (wide, good), (good, good[:5]), (good[0], good[0]), (good.view(-1), good.view(-1)),
                     (good[None], good[None]), (1 << 20, good), (good, 1 << 20)):
        refused_append(lay, pages, K, slots, pos, cos, sin, r"\[positions, 64\]")


def test_pages_of_another_layout():
    """Rows of other sizes would be written behind the end of the tensors."""
    grid = lambda n, heads=2: B.Layer(heads, 128, torch.zeros(n, 2), torch.ones(heads * 128), torch.ones(heads * 128), torch.bfloat16)
    layers = [layer(), layer(rtn_bits=2), grid(16), grid(64), grid(256), grid(256, 4)]
    for lay in layers:
        for other in layers:
            pages = B.Pages(other, 3, 8, device="cpu")
            K = torch.zeros(4, lay.kv_heads, 128, dtype=torch.bfloat16)
            q, table, lens = torch.zeros(2, 4, 128, dtype=torch.bfloat16), torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
            if other is lay:
                with pytest.raises(B.AquaKVError):                          # as far as the library, which wants slots
                    B.aquakv_paged_append(lay, pages, 4, K, K, None, None, None, None, None, None)
                continue
            refused_append(lay, pages, K, torch.zeros(4, dtype=torch.int64), None, None, None, "another layout")
            with pytest.raises(ValueError, match="another layout"):
                B.aquakv_paged_attend(lay, pages, 2, 4, table, lens, q, 1, None, 1.0, q.clone(), None)
    # a layer of the same layout may read another one's pages; a class of one's own is looked at as well

    class Mine(B.Pages):
        pass
    refused_append(layers[0], Mine(layers[1], 3, 8, device="cpu"), torch.zeros(4, 2, 128, dtype=torch.bfloat16), None, None, None, None, "another layout")
    with pytest.raises(B.AquaKVError):
        B.aquakv_paged_append(layers[0], B.Pages(layer(), 3, 8, device="cpu"), 4, *[torch.zeros(4, 2, 128, dtype=torch.bfloat16)] * 2, *[None] * 6)


def test_the_layers_tensors_are_on_the_current_device(monkeypatch):
    """... as those of the call are (the current device is named here: pages and tensors as addresses, which nothing is known of)"""
    pool = B.aquakv_pages(3, 8, 1 << 32, 2 << 32, 3 << 32, 4 << 32)
    grid = B.Layer(2, 128, torch.zeros(16, 2), torch.ones(256), torch.ones(256), torch.bfloat16)
    call = lambda lay: B.aquakv_paged_append(lay, pool, 4, 5 << 32, 6 << 32, None, None, None, None, None, None)
    with pytest.raises(B.AquaKVError):                                      # (no slots)
        call(grid)
    monkeypatch.setattr(B, "_here", lambda: 0)
    with pytest.raises(ValueError, match="current device"):
        call(grid)
    with pytest.raises(ValueError, match="current device"):
        B.aquakv_paged_attend(grid, pool, 2, 4, None, None, 5 << 32, 1, None, 1.0, None, None)
    with pytest.raises(B.AquaKVError):                                      # uniform: it has none
        call(layer())


def test_addresses_have_no_shape():
    """Rows of q and pages of a sequence are counted from the tensors, so that an address will not do (for the other arguments it will)."""
    lay = layer()
    pages = B.Pages(lay, 3, 8, device="cpu")
    q, table, lens = torch.zeros(2, 4, 128, dtype=torch.bfloat16), torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    for x, t in ((q.data_ptr(), table), (None, table), (q, table.data_ptr()), (q, None)):
        with pytest.raises(ValueError, match="must be tensors"):
            B.aquakv_paged_attend(lay, pages, 2, 4, t, lens, x, 1, None, 1.0, q.clone(), None)
    with pytest.raises(B.AquaKVError, match="workspace"):
        B.aquakv_paged_attend(lay, pages, 2, 4, table, 1 << 32, q, 1, None, 1.0, 2 << 32, None)


def test_nothing_to_do():
    """A step without tokens or queries: tensors without elements have no address."""
    lay = layer()
    pages = B.Pages(lay, 3, 8, device="cpu")
    K, slots, pos, cos = torch.zeros(0, 2, 128, dtype=torch.bfloat16), torch.zeros(0, dtype=torch.int64), torch.zeros(0, dtype=torch.int32), torch.zeros(9, 64)
    assert K.data_ptr() == 0
    B.aquakv_paged_append(lay, pages, 0, K, K, slots, None, None, None, None, None)
    B.aquakv_paged_append(lay, pages, 0, K, K, slots, pos, cos, cos, K.clone(), K.clone())
    q, table, lens = torch.zeros(0, 4, 128, dtype=torch.bfloat16), torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    start, ws = torch.zeros(3, dtype=torch.int32), torch.zeros(0, dtype=torch.uint8)
    B.aquakv_paged_attend(lay, pages, 2, 4, table, lens, q, 0, None, 1.0, q.clone(), ws)
    B.aquakv_paged_attend(lay, pages, 2, 4, table, lens, q, 5, start, 1.0, q.clone(), ws)
    B.aquakv_paged_attend(lay, pages, 0, 4, table[:0], lens[:0], q, 1, None, 1.0, q.clone(), ws)
    B.aquakv_paged_attend(lay, pages, 0, 4, table[:0], lens[:0], q, 1, start[:1], 1.0, q.clone(), ws)
    with pytest.raises(B.AquaKVError):                                      # sizes are looked at all the same
        B.aquakv_paged_attend(lay, pages, 2, 5, table, lens, torch.zeros(0, 5, 128, dtype=torch.bfloat16), 0, None, 1.0, None, ws)
    # with addresses and a workspace of no bytes
    p = B.aquakv_pages(3, 8, 1 << 32, 2 << 32, 3 << 32, 4 << 32)
    none = [None] * 4
    assert B._lib.aquakv_paged_append(lay.c, p, 0, None, 256, None, 256, *none, 0, None, None, None) == B.AQUAKV_OK
    for batch, rows, most in ((0, 6, 2), (3, 0, 2), (3, 6, 0)):
        start = 8 << 32
        assert B._lib.aquakv_paged_attend(lay.c, p, batch, 4, 5 << 32, 3, 6 << 32, rows, most, start, 7 << 32, 512, 1.0, 9 << 32, None, 0, None) == B.AQUAKV_OK


def test_the_workspace_of_nothing_and_of_something():
    """A call that has nothing to do takes a workspace of no bytes, any other one not (the binding hands over how many there are)."""
    lay = layer()
    pages = B.Pages(lay, 3, 8, device="cpu")
    q, table, lens = torch.zeros(2, 4, 128, dtype=torch.bfloat16), torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    at = 1 << 33
    B.aquakv_paged_attend(lay, pages, 2, 4, table, lens, q, 0, torch.zeros(3, dtype=torch.int32), 1.0, q.clone(), (at, 0))
    need = B.aquakv_paged_workspace_bytes(lay, pages, 2, 4, 3, 2, 1)
    assert need > 0
    for nbytes in (0, need - 1):
        with pytest.raises(B.AquaKVError) as e:
            B.aquakv_paged_attend(lay, pages, 2, 4, table, lens, q, 1, None, 1.0, q.clone(), (at, nbytes))
        assert e.value.status == B.AQUAKV_EWORKSPACE
