"""Host-side checks of trees, attention weights, selection, moves and rotary positions: every fault in the arguments is refused before anything is launched."""
import pytest

from paper_2501_19392_amd import binding as B
from tests.test_abi_host import layer

H, QH, PAGES, PAGE = 8, 32, 10, 16
D = H * 128


class Buffers:
    """Addresses that are never dereferenced, far apart from each other."""

    def __init__(self, **kw):
        self.layer = layer(**{"d_in_k": 0, "d_in_v": 0, "w_k": None, "w_v": None, "n_codewords": 256, **kw})
        names = ["k_codes", "k_scales", "v_codes", "v_scales", "table", "lens", "start", "tree", "q", "out", "ws", "mass", "kept", "n_kept", "first", "to",
                 "x", "positions", "cos", "sin"]
        self.a = {n: (i + 1) << 32 for i, n in enumerate(names)}
        if self.layer.vq_dim == 2:
            self.layer.codebook, self.layer.signs_k, self.layer.signs_v = (1 << 44), (1 << 44) + 65536, (1 << 44) + 131072
        self.n = dict(n_pages=PAGES, page_tokens=PAGE, batch=2, q_heads=QH, table_pages=5, q_rows=6, max_queries=3, q_stride=QH * 128, ws=1 << 24, words=1,
                      keep=1.0, budget=9, n_first=2, n_last=3, max_kept=7, to_pages=4, dtype=B.AQUAKV_BF16, tokens=6, heads=QH, x_stride=QH * 128,
                      out_stride=QH * 128, rows=99, dim=64, layout=0)

    def pages(self):
        return B.aquakv_pages(self.n["n_pages"], self.n["page_tokens"], *(self.a[n] for n in ("k_codes", "k_scales", "v_codes", "v_scales")))

    def tree(self):
        a, n = self.a, self.n
        return B._lib.aquakv_paged_attend_tree(self.layer, self.pages(), n["batch"], n["q_heads"], a["table"], n["table_pages"], a["lens"], n["q_rows"],
                                               n["max_queries"], a["start"], a["tree"], n["words"], a["q"], n["q_stride"], 0.1, a["out"], a["ws"], n["ws"], None)

    def weights(self):
        a, n = self.a, self.n
        return B._lib.aquakv_paged_weights(self.layer, self.pages(), n["batch"], n["q_heads"], a["table"], n["table_pages"], a["lens"], n["q_rows"],
                                           n["max_queries"], a["start"], a["q"], n["q_stride"], 0.1, n["keep"], a["mass"], a["ws"], n["ws"], None)

    def select(self):
        a, n = self.a, self.n
        return B._lib.aquakv_paged_select(self.layer, self.pages(), n["batch"], a["table"], n["table_pages"], a["lens"], a["mass"], n["budget"], n["n_first"],
                                          n["n_last"], a["kept"], a["n_kept"], a["ws"], n["ws"], None)

    def keep(self):
        a, n = self.a, self.n
        return B._lib.aquakv_paged_keep(self.layer, self.pages(), n["batch"], a["table"], n["table_pages"], n["max_kept"], a["kept"], a["n_kept"], a["first"],
                                        a["to"], n["to_pages"], a["mass"], a["ws"], n["ws"], None)

    def rotary(self):
        a, n = self.a, self.n
        return B._lib.aquakv_rotary(n["dtype"], n["tokens"], n["heads"], a["x"], n["x_stride"], a["positions"], a["cos"], a["sin"], n["rows"], n["dim"],
                                    n["layout"], 0, a["out"], n["out_stride"], None)

    def size(self, call):
        n, p = self.n, self.pages()
        return {"tree": lambda: B._lib.aquakv_paged_workspace_bytes(self.layer, p, n["batch"], n["q_heads"], n["table_pages"], n["q_rows"], n["max_queries"]),
                "weights": lambda: B._lib.aquakv_paged_weights_workspace_bytes(self.layer, p, n["batch"], n["q_heads"], n["table_pages"], n["q_rows"], n["max_queries"]),
                "select": lambda: B._lib.aquakv_paged_select_workspace_bytes(self.layer, p, n["batch"], n["table_pages"], n["budget"]),
                "keep": lambda: B._lib.aquakv_paged_keep_workspace_bytes(self.layer, p, n["batch"], n["max_kept"], 1)}[call]()


CALLS = ("tree", "weights", "select", "keep")


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("kw,want", [(dict(d_in_k=1024, w_k=65536), B.AQUAKV_EUNSUPPORTED), (dict(rht_group=1024), B.AQUAKV_EUNSUPPORTED),
                                     (dict(vq_dim=1, n_codewords=16, rht_group=1024), B.AQUAKV_EUNSUPPORTED), (dict(head_dim=64), B.AQUAKV_EUNSUPPORTED),
                                     (dict(dtype=5), B.AQUAKV_EINVAL)])
def test_layers_that_pages_do_not_hold(call, kw, want):
    c = Buffers(**kw)
    assert getattr(c, call)() == want and c.size(call) == 0


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("kw,want", [(dict(n_pages=0), B.AQUAKV_EINVAL), (dict(page_tokens=20), B.AQUAKV_EINVAL), (dict(batch=-1), B.AQUAKV_EINVAL),
                                     (dict(batch=70000), B.AQUAKV_EUNSUPPORTED), (dict(n_pages=1 << 30, page_tokens=1024), B.AQUAKV_EUNSUPPORTED)])
def test_sizes_that_all_refuse(call, kw, want):
    c = Buffers()
    c.n.update(kw)
    assert getattr(c, call)() == want and c.size(call) == 0


@pytest.mark.parametrize("call,kw,want", [
    ("tree", dict(words=0), B.AQUAKV_EINVAL), ("tree", dict(words=-1), B.AQUAKV_EINVAL), ("tree", dict(max_queries=33), B.AQUAKV_EINVAL),
    ("tree", dict(words=(1 << 17) + 1), B.AQUAKV_EUNSUPPORTED), ("tree", dict(q_heads=12), B.AQUAKV_EINVAL), ("tree", dict(table_pages=0), B.AQUAKV_EINVAL),
    ("tree", dict(max_queries=1 << 27, words=1 << 22), B.AQUAKV_EUNSUPPORTED),
    ("weights", dict(keep=float("nan")), B.AQUAKV_EINVAL), ("weights", dict(keep=float("inf")), B.AQUAKV_EINVAL), ("weights", dict(q_heads=12), B.AQUAKV_EINVAL),
    ("weights", dict(table_pages=(1 << 25) - 1000, page_tokens=64), B.AQUAKV_EUNSUPPORTED), ("weights", dict(table_pages=1 << 24, page_tokens=16), B.AQUAKV_EUNSUPPORTED), ("weights", dict(max_queries=-1), B.AQUAKV_EINVAL),
    ("select", dict(budget=-1), B.AQUAKV_EINVAL), ("select", dict(n_first=-1), B.AQUAKV_EINVAL), ("select", dict(n_last=-2), B.AQUAKV_EINVAL),
    ("select", dict(budget=4), B.AQUAKV_EINVAL), ("select", dict(n_first=1 << 30, n_last=1 << 30, budget=2147483647), B.AQUAKV_EINVAL),
    ("select", dict(table_pages=0), B.AQUAKV_EINVAL),
    ("keep", dict(max_kept=-1), B.AQUAKV_EINVAL), ("keep", dict(max_kept=1 << 29), B.AQUAKV_EUNSUPPORTED), ("keep", dict(table_pages=0), B.AQUAKV_EINVAL),
    ("keep", dict(to_pages=0), B.AQUAKV_EINVAL), ("keep", dict(to_pages=1 << 28), B.AQUAKV_EUNSUPPORTED),
    ("rotary", dict(dtype=3), B.AQUAKV_EINVAL), ("rotary", dict(tokens=-1), B.AQUAKV_EINVAL), ("rotary", dict(heads=0), B.AQUAKV_EINVAL),
    ("rotary", dict(rows=0), B.AQUAKV_EINVAL), ("rotary", dict(dim=0), B.AQUAKV_EINVAL), ("rotary", dict(dim=130), B.AQUAKV_EINVAL), ("rotary", dict(dim=33), B.AQUAKV_EINVAL),
    ("rotary", dict(dim=40), B.AQUAKV_EUNSUPPORTED), ("rotary", dict(layout=2), B.AQUAKV_EINVAL), ("rotary", dict(tokens=1 << 25), B.AQUAKV_EUNSUPPORTED),
    ("rotary", dict(tokens=1 << 62), B.AQUAKV_EUNSUPPORTED), ("rotary", dict(tokens=1 << 27, heads=1, x_stride=128, out_stride=128), B.AQUAKV_EUNSUPPORTED), ("rotary", dict(x_stride=QH * 128 - 8), B.AQUAKV_EINVAL), ("rotary", dict(out_stride=QH * 128 + 4), B.AQUAKV_EALIGN)])
def test_sizes_of_each(call, kw, want):
    c = Buffers()
    c.n.update(kw)
    assert getattr(c, call)() == want, B.aquakv_last_error()


REQUIRED = {"tree": ("k_codes", "v_scales", "table", "lens", "tree", "q", "out", "ws"), "weights": ("k_codes", "k_scales", "table", "lens", "q", "mass", "ws"),
            "select": ("table", "lens", "mass", "kept", "n_kept", "ws"), "keep": ("k_codes", "v_codes", "table", "kept", "n_kept", "ws"),
            "rotary": ("x", "positions", "cos", "sin", "out")}


@pytest.mark.parametrize("call,name", [(c, n) for c, names in REQUIRED.items() for n in names])
def test_buffers_are_required_and_aligned(call, name):
    c = Buffers()
    c.a[name] += 2
    assert getattr(c, call)() == B.AQUAKV_EALIGN
    c.a[name] = None
    assert getattr(c, call)() == B.AQUAKV_ENULL


@pytest.mark.parametrize("call,name", [("tree", "start"), ("weights", "start"), ("keep", "first"), ("keep", "to"), ("keep", "mass")])
def test_buffers_that_may_be_absent_are_aligned(call, name):
    c = Buffers()
    c.a[name] += 2
    assert getattr(c, call)() == B.AQUAKV_EALIGN


@pytest.mark.parametrize("call", CALLS)
def test_workspaces(call):
    c = Buffers()
    assert c.size(call) > 0
    c.n["ws"] = c.size(call) - 1
    assert getattr(c, call)() == B.AQUAKV_EWORKSPACE


WRITTEN = {"tree": ("out", "ws"), "weights": ("mass", "ws"), "select": ("kept", "n_kept", "ws"), "keep": ("k_codes", "k_scales", "v_codes", "v_scales", "mass", "ws"),
           "rotary": ("out",)}
READ = {"tree": ("k_codes", "v_scales", "table", "lens", "start", "tree", "q"), "weights": ("k_codes", "k_scales", "v_codes", "table", "lens", "start", "q"),
        "select": ("table", "lens", "mass"), "keep": ("table", "kept", "n_kept", "first", "to"), "rotary": ("positions", "cos", "sin")}


@pytest.mark.parametrize("call,out,name", [(c, o, n) for c in WRITTEN for o in WRITTEN[c] for n in (*READ[c], *WRITTEN[c]) if n != o])
def test_what_is_written_overlaps_nothing(call, out, name):
    c = Buffers()
    c.a[out] = c.a[name]
    assert getattr(c, call)() == B.AQUAKV_EINVAL and "overlaps" in B.aquakv_last_error()


def test_rotary_in_place_and_nearly():
    c = Buffers()
    c.a["out"] = c.a["x"]
    c.n["out_stride"] += 128
    assert c.rotary() == B.AQUAKV_EINVAL and "overlaps" in B.aquakv_last_error()      # (the same rows, other strides)
    c.n["out_stride"] -= 128
    c.a["out"] += 256
    assert c.rotary() == B.AQUAKV_EINVAL and "overlaps" in B.aquakv_last_error()


def test_queries_without_starts():
    for call in ("tree", "weights"):
        c = Buffers()
        c.a["start"], c.n["q_rows"] = None, 7
        assert getattr(c, call)() == B.AQUAKV_EINVAL and "without q_start" in B.aquakv_last_error()


def test_nothing_to_do_is_answered():
    """Without sequences, queries, entries or tokens nothing is looked at but sizes."""
    for call, kw in (("tree", dict(batch=0)), ("tree", dict(q_rows=0)), ("tree", dict(max_queries=0, words=0)), ("weights", dict(batch=0)), ("weights", dict(q_rows=0)),
                     ("weights", dict(max_queries=0)), ("select", dict(batch=0)), ("keep", dict(batch=0)), ("keep", dict(max_kept=0)), ("rotary", dict(tokens=0))):
        c = Buffers()
        c.n.update(kw)
        for name in ("table", "lens", "tree", "q", "out", "ws", "mass", "kept", "n_kept", "first", "to", "x", "positions", "cos", "sin"):
            c.a[name] = None
        if call in ("tree", "weights") and "q_rows" not in kw:
            c.n["q_rows"] = 0
        if call == "keep":
            c.a["to"] = None
        assert getattr(c, call)() == B.AQUAKV_OK, (call, kw, B.aquakv_last_error())


def tables(rows=10, first=0, dim=64, base=1e4, factor=1.0, original=0.0, low=0.0, high=0.0, magnitude=1.0, cos=1 << 32, sin=2 << 32):
    return B._lib.aquakv_rotary_tables(rows, first, dim, base, factor, original, low, high, magnitude, cos, sin, None)


@pytest.mark.parametrize("kw,want", [
    (dict(rows=-1), B.AQUAKV_EINVAL), (dict(first=-1), B.AQUAKV_EINVAL), (dict(rows=1 << 31), B.AQUAKV_EINVAL), (dict(first=(1 << 31) - 10), B.AQUAKV_EINVAL),
    (dict(dim=0), B.AQUAKV_EINVAL), (dict(dim=7), B.AQUAKV_EINVAL), (dict(dim=136), B.AQUAKV_EINVAL), (dict(dim=24), B.AQUAKV_EUNSUPPORTED), (dict(base=0.0), B.AQUAKV_EINVAL),
    (dict(base=float("inf")), B.AQUAKV_EINVAL), (dict(base=float("nan")), B.AQUAKV_EINVAL), (dict(factor=0.0), B.AQUAKV_EINVAL), (dict(factor=float("nan")), B.AQUAKV_EINVAL),
    (dict(original=-1.0), B.AQUAKV_EINVAL), (dict(original=float("inf")), B.AQUAKV_EINVAL), (dict(original=8192.0), B.AQUAKV_EINVAL),
    (dict(original=8192.0, low=4.0, high=1.0), B.AQUAKV_EINVAL), (dict(original=8192.0, low=-1.0, high=1.0), B.AQUAKV_EINVAL),
    (dict(original=8192.0, low=1.0, high=float("inf")), B.AQUAKV_EINVAL), (dict(magnitude=float("nan")), B.AQUAKV_EINVAL), (dict(cos=None), B.AQUAKV_ENULL),
    (dict(sin=None), B.AQUAKV_ENULL), (dict(sin=(2 << 32) + 4), B.AQUAKV_EALIGN), (dict(sin=1 << 32), B.AQUAKV_EINVAL), (dict(sin=(1 << 32) + 1264), B.AQUAKV_EINVAL),
    (dict(rows=1 << 29, dim=128), B.AQUAKV_EUNSUPPORTED), (dict(factor=1e-300), B.AQUAKV_EINVAL), (dict(base=1e-300), B.AQUAKV_EINVAL),
    (dict(rows=0, cos=None, sin=None), B.AQUAKV_OK)])
def test_tables(kw, want):
    assert tables(**kw) == want, B.aquakv_last_error()


@pytest.mark.parametrize("batch,queries", [(32, 2048), (1, 2048), (64, 256), (1, 8192)])
def test_chunks_need_no_results_of_pieces(batch, queries):
    """Chunks of prompts, whose rows fill the chip by themselves: the one size for calls with and without a tree stays small."""
    c = Buffers()
    c.n.update(n_pages=100000, page_tokens=64, batch=batch, table_pages=256, q_rows=batch * queries, max_queries=queries)
    assert 0 < c.size("tree") < 1 << 20


@pytest.mark.parametrize("batch,most", [(1, 32768), (3, 65536), (2, 7)])
def test_rows_to_other_pages_need_no_room_for_them(batch, most):
    """Only moves in place of few sequences go through the workspace."""
    c = Buffers()
    c.n.update(n_pages=100000, page_tokens=64, batch=batch, table_pages=2000, to_pages=1200, max_kept=most)
    c.n["ws"] = 255
    assert c.keep() == B.AQUAKV_EWORKSPACE
    c.n["ws"], c.a["mass"] = 256, c.a["kept"]                 # (what is looked at behind the workspace: nothing is launched)
    assert c.keep() == B.AQUAKV_EINVAL and "overlaps" in B.aquakv_last_error()
    c.a["to"] = None
    if most > 1024:
        assert c.size("keep") > most * 1024 and c.keep() == B.AQUAKV_EWORKSPACE
    else:
        assert c.keep() == B.AQUAKV_EINVAL and "overlaps" in B.aquakv_last_error()


@pytest.mark.parametrize("batch,queries,room,small", [
    (128, 64, 4096, True), (128, 64, 4160, False), (128, 64, 131072, False), (256, 64, 16384, True), (256, 64, 16448, False), (2000, 64, 131072, False), (64, 144, 2048, True),
    (64, 144, 32768, False), (32, 2048, 131072, True)])      # (2048: a sequence's blocks of rows fill the chip)
def test_sequences_are_whole_where_none_can_be_long(batch, queries, room, small):
    """Trees in blocks of 256 rows: with room for long sequences there are results of pieces, of as many as fill the chip, however many sequences there are."""
    c = Buffers()
    c.n.update(n_pages=1000000, page_tokens=64, batch=batch, table_pages=room // 64, q_rows=batch * queries, max_queries=queries)
    size = B._lib.aquakv_paged_attend_workspace_bytes(c.layer, c.pages(), batch, QH, room // 64, batch * queries, queries, 1)
    assert size == 256 if small else 1 << 20 < size < 40 << 20


@pytest.mark.parametrize("call,kw,refused", [
    ("weights", dict(kv=1024, q_heads=16384, table_pages=(1 << 18) - 1, page_tokens=8, max_queries=1), True),       # 2^14 workgroups of 128 tokens, 1024 heads, 256 threads each
    ("weights", dict(kv=1024, q_heads=16384, table_pages=(1 << 18) - 17, page_tokens=8, max_queries=1), False),     # one workgroup less
    ("weights", dict(kv=1024, q_heads=8192, table_pages=(1 << 18) - 1, page_tokens=8, max_queries=1), False),       # few rows: in other workgroups
    ("keep", dict(max_kept=(1 << 29) - 31), True), ("keep", dict(max_kept=(1 << 29) - 32), False),                  # workgroups of 32 entries
    ("keep", dict(max_kept=(1 << 29) - 1, to=None, batch=1), True), ("keep", dict(max_kept=(1 << 29) - 1, to=None, batch=64), False),      # in place, by columns
    ("rotary", dict(tokens=(1 << 27) - 7, heads=1, dtype=B.AQUAKV_FP32, layout=1, x_stride=128, out_stride=128), True),      # 32 threads for a token
    ("rotary", dict(tokens=(1 << 27) - 8, heads=1, dtype=B.AQUAKV_FP32, layout=1, x_stride=128, out_stride=128), False),
    ("rotary", dict(tokens=(1 << 27) - 1, heads=1, layout=1, x_stride=128, out_stride=128), False)])
def test_launches_in_whole_workgroups_stay_below_2_32_threads(call, kw, refused):
    """(Calls that are not refused get as far as buffers that overlap.)"""
    c = Buffers(**({"kv_heads": kw["kv"]} if "kv" in kw else {}))
    c.a = {k: v << 8 for k, v in c.a.items()}                # (as far apart as the buffers are large)
    c.n.update({k: v for k, v in kw.items() if k not in ("kv", "to")}, ws=1 << 62)
    if "kv" in kw:
        c.n.update(q_stride=kw["q_heads"] * 128, q_rows=2)
    if "to" in kw:
        c.a["to"] = None
    c.a[{"weights": "mass", "keep": "mass", "rotary": "out"}[call]] = c.a[{"weights": "lens", "keep": "n_kept", "rotary": "cos"}[call]]
    assert getattr(c, call)() == (B.AQUAKV_EUNSUPPORTED if refused else B.AQUAKV_EINVAL), B.aquakv_last_error()
    assert refused or "overlaps" in B.aquakv_last_error()
