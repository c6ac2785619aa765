"""What the Python calls on trees, weights, selection, moves and rotary positions refuse before the library is asked (no GPU: nothing here is launched)."""
import pytest
import torch

from paper_2501_19392_amd import binding as B


def layer():
    return B.Layer(2, 128, None, None, None, torch.bfloat16, rtn_bits=4)


def parts():
    lay = layer()
    return dict(lay=lay, pages=B.Pages(lay, 3, 8, device="cpu"), table=torch.zeros(2, 3, dtype=torch.int32), lens=torch.zeros(2, dtype=torch.int32),
                q=torch.zeros(4, 4, 128, dtype=torch.bfloat16), tree=torch.zeros(4, 1, dtype=torch.int32), mass=torch.zeros(3, 2, 8),
                kept=torch.zeros(2, 5, dtype=torch.int32), ws=torch.zeros(1 << 20, dtype=torch.uint8))


def tree(p, **kw):
    p = {**p, **kw}
    B.aquakv_paged_attend_tree(p["lay"], p["pages"], 2, 4, p["table"], p["lens"], p["q"], 2, None, p["tree"], 1.0, torch.zeros(4, 4, 128, dtype=torch.bfloat16), None)


def weights(p, **kw):
    p = {**p, **kw}
    B.aquakv_paged_weights(p["lay"], p["pages"], 2, 4, p["table"], p["lens"], p["q"], 2, None, 1.0, 1.0, p["mass"], None)


def select(p, **kw):
    p = {**p, **kw}
    B.aquakv_paged_select(p["lay"], p["pages"], 2, p["table"], p["lens"], p["mass"], 5, 1, 1, p["kept"], p["lens"].clone(), None)


def keep(p, **kw):
    p = {"to": None, **p, **kw}
    B.aquakv_paged_keep(p["lay"], p["pages"], 2, p["table"], p["kept"], p["lens"], None, p["to"], p["mass"], None)


BAD = {
    tree: [dict(tree=torch.zeros(4, dtype=torch.int32)), dict(tree=torch.zeros(3, 1, dtype=torch.int32)), dict(tree=torch.zeros(4, 1, dtype=torch.int64)), dict(tree=None),
           dict(tree=1 << 32), dict(tree=torch.zeros(4, 2, dtype=torch.int32)[:, :1]), dict(q=torch.zeros(4, 4, 128)), dict(table=torch.zeros(3, 3, dtype=torch.int32)),
           dict(lens=torch.zeros(3, dtype=torch.int32)), dict(q=None)],
    weights: [dict(mass=torch.zeros(3, 2, 9)), dict(mass=torch.zeros(3, 2, 8).double()), dict(mass=torch.zeros(3, 8, 2).transpose(1, 2)), dict(lens=torch.zeros(2)),
              dict(table=torch.zeros(6, dtype=torch.int32)), dict(q=torch.zeros(4, 4, 64, dtype=torch.bfloat16))],
    select: [dict(mass=torch.zeros(2, 2, 8)), dict(kept=torch.zeros(2, 4, dtype=torch.int32)), dict(kept=torch.zeros(2, 5, dtype=torch.int64)),
             dict(table=torch.zeros(3, 3, dtype=torch.int32)), dict(table=None), dict(lens=torch.zeros(2, 1))],
    keep: [dict(mass=torch.zeros(3, 2, 7)), dict(kept=torch.zeros(3, 5, dtype=torch.int32)), dict(kept=torch.zeros(10, dtype=torch.int32)), dict(kept=None), dict(to=torch.zeros(3, 3, dtype=torch.int32)),
           dict(to=torch.zeros(2, 3)), dict(table=torch.zeros(2, 6, dtype=torch.int32)[:, ::2])]}


@pytest.mark.parametrize("call,i", [(c, i) for c in BAD for i in range(len(BAD[c]))])
def test_tensors_of_other_shapes_and_types(call, i):
    with pytest.raises(ValueError):
        call(parts(), **BAD[call][i])


@pytest.mark.parametrize("call", list(BAD))
def test_pages_of_another_layout_and_device(call, monkeypatch):
    with pytest.raises(ValueError, match="another layout"):
        call(parts(), pages=B.Pages(B.Layer(2, 128, None, None, None, torch.bfloat16, rtn_bits=2), 3, 8, device="cpu"))
    with pytest.raises(B.AquaKVError, match="workspace"):                   # as far as the library, which wants a workspace
        call(parts())
    monkeypatch.setattr(B, "_here", lambda: 0)
    with pytest.raises(ValueError, match="current device"):
        call(parts())


def rotary(**kw):
    a = dict(x=torch.zeros(3, 4, 128, dtype=torch.bfloat16), positions=torch.zeros(3, dtype=torch.int32), cos=torch.zeros(9, 32), sin=torch.zeros(9, 32), dim=64,
             layout="half", out=torch.zeros(3, 4, 128, dtype=torch.bfloat16))
    a.update(kw)
    B.aquakv_rotary(a["x"], a["positions"], a["cos"], a["sin"], a["dim"], a["layout"], a["out"])


@pytest.mark.parametrize("kw", [
    dict(x=torch.zeros(3, 4, 64, dtype=torch.bfloat16)), dict(x=torch.zeros(3, 512, dtype=torch.bfloat16)), dict(out=torch.zeros(3, 4, 128)),
    dict(out=torch.zeros(3, 5, 128, dtype=torch.bfloat16)), dict(positions=torch.zeros(3, dtype=torch.int64)), dict(positions=torch.zeros(4, dtype=torch.int32)),
    dict(cos=torch.zeros(9, 64)), dict(sin=torch.zeros(8, 32)), dict(dim=128), dict(dim=32), dict(cos=torch.zeros(9, 32).double()), dict(layout="interleaved"),
    dict(cos=torch.zeros(9, 64)[:, ::2], sin=torch.zeros(9, 64)[:, ::2]), dict(cos=torch.zeros(288), sin=torch.zeros(288)),
    dict(x=torch.zeros(3, 128, 4, dtype=torch.bfloat16).transpose(1, 2)), dict(x=torch.zeros(3, 4, 128, dtype=torch.float16), out=torch.zeros(3, 4, 128, dtype=torch.float16))])
def test_rotary_refuses(kw):
    with pytest.raises(ValueError):
        rotary(**kw)


def test_rotary_in_place_of_a_slice_and_of_nothing():
    none = torch.zeros(0, 4, 128, dtype=torch.bfloat16)
    rotary(x=none, out=none, positions=torch.zeros(0, dtype=torch.int32))
    wide = torch.zeros(3, 6, 128, dtype=torch.bfloat16)
    with pytest.raises(B.AquaKVError, match="overlaps"):                     # the same rows one head on
        rotary(x=wide[:, :4], out=wide[:, 1:5])


def test_tables_refuse():
    good = torch.zeros(5, 32)
    for cos, sin in ((good[0], good[0]), (good, good[:4]), (good.double(), good.double()), (good[:, ::2], good[:, ::2])):
        with pytest.raises(ValueError):
            B.aquakv_rotary_tables(cos, sin, 1e4)
    with pytest.raises(B.AquaKVError):
        B.aquakv_rotary_tables(good, good.clone(), -1.0)
