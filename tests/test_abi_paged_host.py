"""Host-side checks of the calls on pages: every fault in the arguments is refused before anything is launched."""
import pytest
import torch

from paper_2501_19392_amd import binding as B
from tests.test_abi_host import layer

H, QH, PAGES, PAGE, T = 8, 32, 10, 16, 12
D = H * 128


class Buffers:
    """Addresses that are never dereferenced, far apart from each other."""

    def __init__(self, **kw):
        self.layer = layer(**{"d_in_k": 0, "d_in_v": 0, "w_k": None, "w_v": None, "n_codewords": 256, **kw})
        names = ["k_codes", "k_scales", "v_codes", "v_scales", "K", "V", "slots", "positions", "cos", "sin", "Khat", "Vhat", "table", "lens", "start",
                 "q", "out", "ws"]
        self.a = {n: (i + 1) << 32 for i, n in enumerate(names)}
        if self.layer.vq_dim == 2:
            self.layer.codebook, self.layer.signs_k, self.layer.signs_v = (1 << 44), (1 << 44) + 65536, (1 << 44) + 131072
        self.n = dict(n_pages=PAGES, page_tokens=PAGE, tokens=T, k_stride=D, v_stride=D, rope_rows=99, batch=2, q_heads=QH, table_pages=5, q_rows=6,
                      max_queries=3, q_stride=QH * 128, ws=1 << 20)

    def pages(self):
        return B.aquakv_pages(self.n["n_pages"], self.n["page_tokens"], *(self.a[n] for n in ("k_codes", "k_scales", "v_codes", "v_scales")))

    def append(self):
        a, n = self.a, self.n
        return B._lib.aquakv_paged_append(self.layer, self.pages(), n["tokens"], a["K"], n["k_stride"], a["V"], n["v_stride"], a["slots"], a["positions"],
                                          a["cos"], a["sin"], n["rope_rows"], a["Khat"], a["Vhat"], None)

    def attend(self):
        a, n = self.a, self.n
        return B._lib.aquakv_paged_attend(self.layer, self.pages(), n["batch"], n["q_heads"], a["table"], n["table_pages"], a["lens"], n["q_rows"],
                                          n["max_queries"], a["start"], a["q"], n["q_stride"], 0.1, a["out"], a["ws"], n["ws"], None)

    def size(self):
        n = self.n
        return B._lib.aquakv_paged_workspace_bytes(self.layer, self.pages(), n["batch"], n["q_heads"], n["table_pages"], n["q_rows"], n["max_queries"])


@pytest.mark.parametrize("kw,want", [(dict(d_in_k=1024, w_k=65536), B.AQUAKV_EUNSUPPORTED), (dict(d_in_v=2048, w_v=65536), B.AQUAKV_EUNSUPPORTED),
                                     (dict(rht_group=1024), B.AQUAKV_EUNSUPPORTED), (dict(vq_dim=1, n_codewords=16, rht_group=1024), B.AQUAKV_EUNSUPPORTED),
                                     (dict(head_dim=64), B.AQUAKV_EUNSUPPORTED), (dict(dtype=5), B.AQUAKV_EINVAL)])
def test_layers_that_pages_do_not_hold(kw, want):
    c = Buffers(**kw)
    assert c.append() == want and c.attend() == want and c.size() == 0


@pytest.mark.parametrize("kw,want", [(dict(n_pages=0), B.AQUAKV_EINVAL), (dict(page_tokens=4), B.AQUAKV_EINVAL), (dict(page_tokens=0), B.AQUAKV_EINVAL),
                                     (dict(page_tokens=20), B.AQUAKV_EINVAL), (dict(page_tokens=-8), B.AQUAKV_EINVAL),
                                     (dict(n_pages=1 << 30, page_tokens=1024), B.AQUAKV_EUNSUPPORTED)])
def test_sizes_of_a_pool(kw, want):
    c = Buffers()
    c.n.update(kw)
    assert c.append() == want and c.attend() == want and c.size() == 0


@pytest.mark.parametrize("kw,want", [(dict(tokens=-1), B.AQUAKV_EINVAL), (dict(tokens=1 << 30), B.AQUAKV_EUNSUPPORTED), (dict(k_stride=D - 8), B.AQUAKV_EINVAL),
                                     (dict(v_stride=D + 4), B.AQUAKV_EALIGN), (dict(v_stride=-D), B.AQUAKV_EINVAL), (dict(rope_rows=0), B.AQUAKV_EINVAL)])
def test_sizes_of_an_append(kw, want):
    c = Buffers()
    c.n.update(kw)
    assert c.append() == want


@pytest.mark.parametrize("kw,want", [(dict(batch=-1), B.AQUAKV_EINVAL), (dict(batch=70000), B.AQUAKV_EUNSUPPORTED), (dict(q_heads=12), B.AQUAKV_EINVAL),
                                     (dict(q_heads=0), B.AQUAKV_EINVAL), (dict(table_pages=0), B.AQUAKV_EINVAL), (dict(q_rows=-1), B.AQUAKV_EINVAL),
                                     (dict(max_queries=-1), B.AQUAKV_EINVAL), (dict(table_pages=1 << 28), B.AQUAKV_EUNSUPPORTED),
                                     (dict(max_queries=1 << 27), B.AQUAKV_EUNSUPPORTED)])
def test_sizes_of_an_attention(kw, want):
    c = Buffers()
    c.n.update(kw)
    assert c.attend() == want and c.size() == 0


def test_rows_strides_and_workspace_of_an_attention():
    c = Buffers()
    c.n["q_stride"] = QH * 128 - 8
    assert c.attend() == B.AQUAKV_EINVAL
    c.n["q_stride"] = QH * 128 + 4
    assert c.attend() == B.AQUAKV_EALIGN
    c = Buffers()
    c.a["start"], c.n["q_rows"] = None, 7
    assert c.attend() == B.AQUAKV_EINVAL and "without q_start" in B.aquakv_last_error()
    c = Buffers()
    assert c.size() > 0
    c.n["ws"] = c.size() - 1
    assert c.attend() == B.AQUAKV_EWORKSPACE


@pytest.mark.parametrize("name,append,attend", [("k_codes", 1, 1), ("k_scales", 1, 1), ("v_codes", 1, 1), ("v_scales", 1, 1), ("K", 1, 0), ("V", 1, 0),
                                                 ("slots", 1, 0), ("positions", 1, 0), ("cos", 1, 0), ("sin", 1, 0), ("table", 0, 1), ("lens", 0, 1),
                                                 ("q", 0, 1), ("out", 0, 1), ("ws", 0, 1)])
def test_buffers_are_required_and_aligned(name, append, attend):
    for call, used in (("append", append), ("attend", attend)):
        if used:
            c = Buffers()
            c.a[name] += 2
            assert getattr(c, call)() == B.AQUAKV_EALIGN
            c.a[name] = None
            assert getattr(c, call)() == B.AQUAKV_ENULL
    for name in ("Khat", "Vhat"):
        c = Buffers()
        c.a[name] += 8
        assert c.append() == B.AQUAKV_EALIGN
    c = Buffers()
    c.a["start"] += 2
    assert c.attend() == B.AQUAKV_EALIGN


SIZES = dict(k_codes=PAGES * PAGE * H * 64, k_scales=PAGES * PAGE * H * 2, v_codes=PAGES * PAGE * H * 64, v_scales=PAGES * PAGE * H * 2, K=T * D * 2,
             V=T * D * 2, slots=T * 8, positions=T * 4, cos=99 * 256, sin=99 * 256, Khat=T * D * 2, Vhat=T * D * 2, table=40, lens=8, start=12, q=6 * QH * 256,
             out=6 * QH * 256)


@pytest.mark.parametrize("written", ["k_codes", "k_scales", "v_codes", "v_scales", "Khat", "Vhat", "out", "ws"])
def test_what_is_written_overlaps_nothing(written):
    attend = written in ("out", "ws")
    others = ["k_codes", "k_scales", "v_codes", "v_scales"] + (["table", "lens", "start", "q", "out"] if attend else
                                                                ["K", "V", "slots", "positions", "cos", "sin", "Khat", "Vhat"])
    for other in others:
        if other == written:
            continue
        c = Buffers()
        at = 1 << 46
        c.a[written] = at
        c.a[other] = at - (SIZES[other] - 1) // 16 * 16                     # its last bytes
        assert (c.attend() if attend else c.append()) == B.AQUAKV_EINVAL, (written, other)
        assert "overlaps" in B.aquakv_last_error()
    for name, size in dict(codebook=256 * 8, signs_k=D, signs_v=D).items():
        c = Buffers()
        c.a[written] = 1 << 46
        setattr(c.layer, name, (1 << 46) - size + 16)
        assert (c.attend() if attend else c.append()) == B.AQUAKV_EINVAL, (written, name)


def test_nothing_to_do():
    c = Buffers()
    c.n["tokens"] = 0
    assert c.append() == B.AQUAKV_OK
    for name, rows in (("batch", 6), ("q_rows", 0), ("max_queries", 6)):
        c = Buffers()
        c.n[name] = 0
        assert c.attend() == B.AQUAKV_OK
    c.n.update(ws=0)


def test_the_binding_looks_at_its_tensors():
    lay = B.Layer(2, 128, None, None, None, torch.bfloat16, rtn_bits=4)
    pages = B.Pages(lay, 3, 8, device="cpu")
    assert pages.k_codes.shape == (24, 2, 64) and pages.v_scales.shape == (24, 4, 2)
    with pytest.raises(ValueError):
        B.Pages(lay, 3, 8, k_codes=pages.k_codes, k_scales=pages.k_scales, v_codes=pages.v_codes, v_scales=None)
    with pytest.raises(ValueError):
        B.Pages(lay, 2, 8, k_codes=pages.k_codes, k_scales=pages.k_scales, v_codes=pages.v_codes, v_scales=pages.v_scales)
    K = torch.zeros(4, 2, 128, dtype=torch.bfloat16)
    slots = torch.zeros(4, dtype=torch.int64)
    bad = [(K[:3], K, slots), (K.float(), K, slots), (K.transpose(0, 1), K, slots), (K, K[..., ::2], slots), (K, K, slots.int()), (K, K, slots[:3])]
    for k, v, s in bad:
        with pytest.raises(ValueError):
            B.aquakv_paged_append(lay, pages, 4, k, v, s, None, None, None, None, None)
    q, table, lens = torch.zeros(2, 4, 128, dtype=torch.bfloat16), torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    bad = [(table[0], lens, q, q), (table.long(), lens, q, q), (table, lens.long(), q, q), (table, lens[:1], q, q), (table, lens, q.float(), q),
           (table, lens, q, q[:1]), (table, lens, q.transpose(0, 1), q)]
    for t, n, x, o in bad:
        with pytest.raises(ValueError):
            B.aquakv_paged_attend(lay, pages, 2, 4, t, n, x, 1, None, 1.0, o, slots)


@pytest.mark.parametrize("name", ["batch", "q_rows", "max_queries"])
def test_the_size_of_nothing(name):
    c = Buffers()
    c.n[name] = 0
    assert c.size() > 0                                                     # (a call that has nothing to do still wants a workspace)


@pytest.mark.parametrize("kw", [dict(max_queries=1 << 17, q_rows=1 << 17), dict(max_queries=1, q_heads=1 << 22, q_stride=128 << 22),
                                dict(batch=65535, max_queries=1, q_heads=4096, q_stride=128 * 4096, kv_heads=4096)])
def test_more_than_a_launch_holds(kw):
    """Threads of one launch stay below 2^32."""
    c = Buffers(**({"kv_heads": kw["kv_heads"]} if "kv_heads" in kw else {}))
    c.n.update({k: v for k, v in kw.items() if k != "kv_heads"})
    assert c.attend() == B.AQUAKV_EUNSUPPORTED and c.size() == 0
