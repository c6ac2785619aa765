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
