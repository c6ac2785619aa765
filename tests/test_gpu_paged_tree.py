"""aquakv_paged_attend_tree against plain attention in 64 bits, where every draft sees what is cached before the drafts and the drafts of its bits."""
import pytest
import torch

from tests import paged_utils as P
from tests import tree_utils as T

pytestmark = pytest.mark.gpu
SCALE = 128 ** -0.5


def attend(lg, pages, table, lens, q, counts, trees, words=None, max_queries=None, ragged=True, out=None, stream=None):
    from paper_2501_19392_amd import binding as B
    most = max(max(counts), 1) if max_queries is None else max_queries
    words = -(-most // 32) if words is None else words
    tree = torch.cat([T.words_of(t, words) for t in trees]).cuda()
    QH, rows = q.shape[1], q.shape[0]
    start = None
    if ragged:
        start = torch.tensor([sum(counts[:b]) for b in range(len(counts) + 1)], dtype=torch.int32).cuda()
    size = B.aquakv_paged_workspace_bytes(lg, pages, len(counts), QH, table.shape[1], rows, most)
    assert size > 0
    ws = torch.full((size,), 0xff, dtype=torch.uint8, device="cuda")
    out = torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda") if out is None else out
    B.aquakv_paged_attend_tree(lg, pages, len(counts), QH, table.cuda(), lens.cuda(), q, most, start, tree, SCALE, out, ws, stream=stream)
    return out


def queries(gen, rows, QH, dtype):
    return (1.5 * torch.randn(rows, QH, 128, generator=gen)).to(P.storage(dtype)).cuda()


@pytest.mark.parametrize("dtype,fmt,H,QH,lengths,page,counts", [
    ("bf16", "grid256", 8, 32, [700], 64, [26]),                            # waves of 32 rows
    ("bf16", "grid256", 8, 32, [1, 2, 9, 40], 8, [1, 2, 9, 7]),             # no cached tokens but drafts, and hardly any
    ("bf16", "grid64", 2, 2, [300, 77, 32], 24, [5, 8, 1]),                 # one query head: waves of 16 rows
    ("bf16", "grid16", 1, 8, [1000, 999], 40, [16, 3]),                     # exactly 128 rows
    ("bf16", "grid256", 3, 12, [517, 100, 64], 16, [64, 33, 64]),           # blocks of 256 rows; a sequence of drafts alone
    ("bf16", "grid64", 2, 16, [2500, 70], 128, [65, 70]),                   # three words a row
    ("bf16", "grid16", 1, 4, [333], 8, [100]),
    ("bf16", "rtn4", 8, 24, [450, 31, 64], 32, [12, 31, 5]), ("bf16", "rtn2", 2, 14, [129, 1025], 16, [31, 32]),
    ("bf16", "rtn4", 2, 16, [777, 64], 24, [40, 64]), ("bf16", "rtn2", 1, 16, [200], 8, [33]),
    ("fp32", "grid256", 2, 8, [150, 33], 16, [20, 33]), ("fp32", "grid16", 1, 1, [65], 8, [35]), ("fp32", "rtn4", 3, 6, [90, 40, 8], 40, [3, 40, 8]),
    ("fp32", "rtn2", 1, 4, [70], 16, [9]), ("fp32", "grid64", 1, 5, [300], 64, [64])])
def test_drafts_see_their_ancestors(dtype, fmt, H, QH, lengths, page, counts):
    print(f"case tree {dtype} {fmt} H={H} QH={QH} lengths={lengths} counts={counts}", flush=True)
    lo, lg, pages, table, lens, gen = T.cache(dtype, fmt, H, lengths, page)
    trees = [T.random_tree(n, gen) for n in counts]
    q = queries(gen, sum(counts), QH, dtype)
    got = attend(lg, pages, table, lens, q, counts, trees)
    torch.cuda.synchronize()
    P.check(got, *T.reference(lo, pages, table, lens, q, counts, trees, SCALE, dtype), "tree")


@pytest.mark.parametrize("fmt,H,QH,counts,room", [
    ("grid256", 8, 32, [12, 9], 40000), ("grid64", 8, 64, [17, 18], 40000), ("grid16", 4, 24, [8, 1], 70000),      # three columns of rows: 1 and 3 tiles of 48, 1
    ("grid256", 8, 32, [20, 3], 2000), ("rtn4", 8, 24, [27, 30], 2000), ("grid64", 8, 64, [23, 9], 300), ("grid16", 1, 8, [50], 1000),      # 3, 3, 6, 13 tiles of 32
    ("grid256", 8, 32, [64, 50], 40000), ("rtn2", 8, 32, [40, 33], 40000), ("grid16", 2, 32, [40], 600), ("grid256", 1, 16, [130], 500)])      # blocks of 256 rows
def test_row_tiles(fmt, H, QH, counts, room):
    """The ways that rows are shared out go by the sizes a call has room for: wide page tables, of which little is used."""
    page, lengths = 16, [390, 77][:len(counts)]
    lengths[0] = max(lengths[0], counts[0])
    print(f"case row tiles {fmt} H={H} QH={QH} {counts} room={room}", flush=True)
    lo, lg, pages, table, lens, gen = T.cache("bf16", fmt, H, lengths, page, seed=7)
    table = torch.cat([table, torch.full((len(counts), max(room // page - table.shape[1], 0)), -1, dtype=torch.int32)], 1).contiguous()
    trees = [T.random_tree(n, gen) for n in counts]
    q = queries(gen, sum(counts), QH, "bf16")
    got = attend(lg, pages, table, lens, q, counts, trees)
    torch.cuda.synchronize()
    P.check(got, *T.reference(lo, pages, table, lens, q, counts, trees, SCALE, "bf16"), "row tiles")


@pytest.mark.parametrize("fmt,n,QH", [("grid256", 12, 32), ("grid64", 20, 32), ("rtn4", 26, 32)])
def test_long_sequences_in_many_pieces(fmt, n, QH):
    """Several pieces of each row tile, joined."""
    lo, lg, pages, table, lens, gen = T.cache("bf16", fmt, 8, [9000, 5001, n], 64, seed=8)
    trees = [T.random_tree(n, gen) for _ in range(3)]
    q = queries(gen, 3 * n, QH, "bf16")
    got = attend(lg, pages, table, lens, q, [n] * 3, trees, ragged=False)
    torch.cuda.synchronize()
    P.check(got, *T.reference(lo, pages, table, lens, q, [n] * 3, trees, SCALE, "bf16"), "pieces")


@pytest.mark.parametrize("fmt,QH,n", [("grid256", 4, 6), ("grid256", 16, 40), ("rtn4", 4, 6), ("rtn4", 16, 40), ("grid64", 1, 3)])
def test_any_mask_of_the_last_tokens(fmt, QH, n):
    """Bits as they come: rows that see nothing, not even themselves; the future; words behind those that are needed."""
    H, lengths, page = 1, [n, 200, n + 1, 0, n - 2], 16
    lo, lg, pages, table, lens, gen = T.cache("bf16", fmt, H, lengths, page, seed=1)
    trees = [torch.rand(n, n, generator=gen) < 0.4 for _ in lengths]
    trees[0][0] = trees[0][n - 1] = False                                   # nothing cached, nothing seen: 0
    q = queries(gen, n * len(lengths), QH, "bf16")
    got = attend(lg, pages, table, lens, q, [n] * len(lengths), trees, words=5, ragged=False)
    torch.cuda.synchronize()
    want, bound = T.reference(lo, pages, table, lens, q, [n] * len(lengths), trees, SCALE, "bf16")
    assert (want[0] == 0).all() and (want[3 * n:4 * n] == 0).all()
    P.check(got, want, bound, "mask")


@pytest.mark.parametrize("fmt,QH,n", [("grid256", 4, 12), ("grid256", 16, 20), ("rtn2", 4, 12), ("rtn2", 16, 20)])
def test_what_a_draft_does_not_see_has_no_effect(fmt, QH, n):
    """Scales that are not finite in drafts that the others do not see, and pages that are not in the pool."""
    H, page = 1, 8
    lo, lg, pages, table, lens, gen = T.cache("bf16", fmt, H, [90], page, seed=2)
    tree = T.random_tree(n, gen)
    tree[:, 5] = False                                                      # nobody sees draft 5, not even itself
    tree[5] = False
    tree[5, 0] = True
    row = int(table[0, (90 - n + 5) // page]) * page + (90 - n + 5) % page
    for t in (pages.k_scales, pages.v_scales):
        t[row] = 0x7e01 if lo.rtn_bits is None else torch.tensor([0x7c00, -1], dtype=torch.int16, device="cuda")
    table[0, 2], table[0, 4] = -1, pages.n_pages
    q = queries(gen, n, QH, "bf16")
    got = attend(lg, pages, table, lens, q, [n], [tree])
    torch.cuda.synchronize()
    P.check(got, *T.reference(lo, pages, table, lens, q, [n], [tree], SCALE, "bf16"), "unseen")


@pytest.mark.parametrize("QH,n,max_queries", [(4, 7, 4), (16, 40, 33)])
def test_more_rows_than_are_answered(QH, n, max_queries):
    """A sequence of more rows than max_queries: its first ones are answered, rows of no sequence are left; the last drafts have no bits here."""
    lo, lg, pages, table, lens, gen = T.cache("bf16", "grid256", 1, [150], 16, seed=3)
    tree = T.random_tree(n, gen)
    words = -(-max_queries // 32)
    q = queries(gen, n + 3, QH, "bf16")
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    from paper_2501_19392_amd import binding as B
    ws = torch.empty(B.aquakv_paged_workspace_bytes(lg, pages, 1, QH, table.shape[1], n + 3, max_queries), dtype=torch.uint8, device="cuda")
    bits = torch.cat([T.words_of(tree, words), torch.full((3, words), -1, dtype=torch.int32)]).cuda()
    B.aquakv_paged_attend_tree(lg, pages, 1, QH, table.cuda(), lens.cuda(), q, max_queries, torch.tensor([0, n], dtype=torch.int32).cuda(), bits, SCALE, out, ws)
    torch.cuda.synchronize()
    tree[:, 32 * words:] = False
    want, bound = T.reference(lo, pages, table, lens, q[:n], [n], [tree], SCALE, "bf16")
    P.check(out[:max_queries], want[:max_queries], bound[:max_queries], "answered")
    assert (out[max_queries:] == 7.0).all()


def test_a_chain_is_attention_with_a_limit():
    """A tree of one branch: aquakv_paged_attend's result, for few and for many rows."""
    from paper_2501_19392_amd import binding as B
    for QH, n in ((4, 9), (16, 50)):
        lo, lg, pages, table, lens, gen = T.cache("bf16", "grid256", 2, [611, 95], 32, seed=4)
        q = queries(gen, 2 * n, 2 * QH, "bf16")
        got = attend(lg, pages, table, lens, q, [n, n], [torch.ones(n, n, dtype=torch.bool).tril()] * 2, ragged=False)
        want = torch.empty_like(q)
        ws = torch.empty(B.aquakv_paged_workspace_bytes(lg, pages, 2, 2 * QH, table.shape[1], 2 * n, n), dtype=torch.uint8, device="cuda")
        B.aquakv_paged_attend(lg, pages, 2, 2 * QH, table.cuda(), lens.cuda(), q, n, None, SCALE, want, ws)
        torch.cuda.synchronize()
        exact, bound = T.reference(lo, pages, table, lens, q, [n, n], [torch.ones(n, n, dtype=torch.bool).tril()] * 2, SCALE, "bf16")
        P.check(got, exact, bound, "chain")
        P.check(want, exact, bound, "limit")


def test_captured_calls_follow_lengths_and_trees():
    """A graph on a stream of its own, replayed with other lengths, trees and queries; two graphs at once with workspaces of their own."""
    from paper_2501_19392_amd import binding as B
    n, QH, page = 10, 8, 16
    lo, lg, pages, table, lens, gen = T.cache("bf16", "grid256", 2, [420, 310, 64], page, seed=5)
    rows = 3 * n
    size = B.aquakv_paged_workspace_bytes(lg, pages, 3, QH, table.shape[1], rows, n)
    d = dict(table=table.cuda(), lens=lens.cuda(), q=torch.zeros(rows, QH, 128, dtype=torch.bfloat16, device="cuda"),
             tree=torch.zeros(rows, 1, dtype=torch.int32, device="cuda"))
    outs, graphs = [torch.empty_like(d["q"]) for _ in range(2)], []
    spaces = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(2)]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for out, ws in zip(outs, spaces):
            B.aquakv_paged_attend_tree(lg, pages, 3, QH, d["table"], d["lens"], d["q"], n, None, d["tree"], SCALE, out, ws)
    torch.cuda.synchronize()
    for out, ws in zip(outs, spaces):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            B.aquakv_paged_attend_tree(lg, pages, 3, QH, d["table"], d["lens"], d["q"], n, None, d["tree"], SCALE, out, ws)
        graphs.append(g)
    for k, lengths in enumerate(([420, 310, 64], [17, 300, 10], [0, 9, 33])):
        trees = [T.random_tree(n, gen) for _ in range(3)]
        q = queries(gen, rows, QH, "bf16")
        d["q"].copy_(q)
        d["lens"].copy_(torch.tensor(lengths, dtype=torch.int32))
        d["tree"].copy_(torch.cat([T.words_of(t, 1) for t in trees]))
        for out in outs:
            out.fill_(float("nan"))
        torch.cuda.synchronize()
        other = torch.cuda.Stream()
        with torch.cuda.stream(other):
            graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        want = T.reference(lo, pages, table, lengths, q, [n] * 3, trees, SCALE, "bf16")
        for out in outs:
            P.check(out, *want, f"replay {k}")


def test_a_pool_of_more_than_4_gib():
    """Offsets of codes pass 32 bits."""
    page = 64
    rows = (1 << 32) // (8 * 64) + 5 * page
    from paper_2501_19392_amd import binding as B
    from tests import parity_utils as U
    lo, lg = U.make_layers(8, "bf16", 256)
    n_pages = rows // page
    pages = B.Pages(lg, n_pages, page)
    gen = torch.Generator().manual_seed(6)
    lengths, n, QH = [150, 130], 6, 16
    table = torch.tensor([[n_pages - 1, 0, n_pages - 3], [n_pages - 2, n_pages - 4, 1]], dtype=torch.int32)
    used = (table.view(-1, 1).long() * page + torch.arange(page)).view(-1)
    small = B.Pages(lg, 6, page)                                            # the same rows in a pool that the oracle reads
    P.fill(lo, small, gen)
    for name in ("k_codes", "k_scales", "v_codes", "v_scales"):
        getattr(pages, name)[used.cuda()] = getattr(small, name)
    trees = [T.random_tree(n, gen) for _ in lengths]
    q = queries(gen, 2 * n, QH, "bf16")
    lens = torch.tensor(lengths, dtype=torch.int32)
    got = attend(lg, pages, table, lens, q, [n, n], trees)
    wide = queries(gen, 2 * 40, 32, "bf16")                                 # blocks of rows
    wide_trees = [T.random_tree(40, gen) for _ in lengths]
    got_wide = attend(lg, pages, table, lens, wide, [40, 40], wide_trees)
    torch.cuda.synchronize()
    at = torch.arange(6, dtype=torch.int32).view(2, 3)
    P.check(got, *T.reference(lo, small, at, lens, q, [n, n], trees, SCALE, "bf16"), "far")
    P.check(got_wide, *T.reference(lo, small, at, lens, wide, [40, 40], wide_trees, SCALE, "bf16"), "far, blocks of rows")


@pytest.mark.parametrize("fmt", ["grid64", "rtn4"])
def test_many_sequences_in_blocks_of_rows(fmt):
    """So many that each is taken whole: uneven lengths, sequences without rows or tokens, rows that are not answered."""
    H, QH, page, most = 8, 128, 16, 17
    gen = torch.Generator().manual_seed(77)
    lengths = [320, 0, 1, 17, 64, 65] + torch.randint(17, 320, (58,), generator=gen).tolist()
    counts = [17, 0, 1, 17, 17, 0] + torch.randint(0, 18, (58,), generator=gen).tolist()
    lo, lg, pages, table, lens, gen = T.cache("bf16", fmt, H, lengths, page, seed=8)
    trees = [T.random_tree(n, gen) for n in counts]
    q = queries(gen, sum(counts), QH, "bf16")
    got = attend(lg, pages, table, lens, q, counts, trees, max_queries=most)
    P.check(got, *T.reference(lo, pages, table, lens, q, counts, trees, SCALE, "bf16"), fmt)


@pytest.mark.parametrize("fmt,QH,n", [("grid256", 4, 3), ("grid256", 16, 12), ("rtn4", 16, 9), ("grid64", 64, 30), ("rtn2", 64, 20)])
def test_query_without_numbers(fmt, QH, n):
    """Rows of one that has none are NaN (whatever bits it has), all others what they are."""
    H, page, lengths = 1, 16, [700, 90]
    lo, lg, pages, table, lens, gen = T.cache("bf16", fmt, H, lengths, page, seed=9)
    trees = [T.random_tree(n, gen) for _ in lengths]
    q = queries(gen, 2 * n, QH, "bf16")
    want, bound = T.reference(lo, pages, table, lens, q, [n, n], trees, SCALE, "bf16")
    bad = torch.zeros(2 * n, QH, dtype=torch.bool)
    bad[n // 2, QH - 1] = bad[n + 1, 0] = True
    q[bad.cuda()] = float("nan")
    got = attend(lg, pages, table, lens, q, [n, n], trees)
    assert got.cpu()[bad].isnan().all()
    P.check(got.cpu()[~bad], want[~bad], bound[~bad], fmt)


@pytest.mark.parametrize("fmt,batch,long", [("grid64", 70, {3: 5000, 66: 3001}), ("rtn4", 64, {63: 4000}), ("grid256", 130, {0: 2500, 64: 700, 129: 6000}), ("grid16", 66, {})])
def test_long_sequences_among_many_in_blocks_of_rows(fmt, batch, long):
    """With room for long sequences they are cut, and only those: beside sequences in one piece, without rows or tokens, in batches of more than a wave's lanes."""
    from paper_2501_19392_amd import binding as B
    H, QH, page, most = 8, 128, 16, 17
    print(f"case long among many {fmt} {batch} {long}", flush=True)
    gen = torch.Generator().manual_seed(78)
    lengths, counts = torch.randint(17, 320, (batch,), generator=gen).tolist(), torch.randint(0, 18, (batch,), generator=gen).tolist()
    lengths[1], lengths[2], counts[1] = 0, 1, 0
    for b, n in long.items():
        lengths[b], counts[b] = n, 17 - b % 5
    counts[2] = min(counts[2], 1)
    lo, lg, pages, table, lens, gen = T.cache("bf16", fmt, H, lengths, page, seed=12)
    table = torch.cat([table, torch.full((batch, 1100 - table.shape[1]), -1, dtype=torch.int32)], 1).contiguous()
    trees = [T.random_tree(n, gen) for n in counts]
    q = queries(gen, sum(counts), QH, "bf16")
    start = torch.tensor([sum(counts[:b]) for b in range(batch + 1)], dtype=torch.int32).cuda()
    size = B.aquakv_paged_attend_workspace_bytes(lg, pages, batch, QH, 1100, q.shape[0], most, True)
    assert size > 1 << 20
    ws, out = torch.full((size + 4096,), 0xff, dtype=torch.uint8, device="cuda"), torch.full_like(q, float("nan"))
    bits = torch.cat([T.words_of(t, 1) for t in trees]).cuda()
    B.aquakv_paged_attend_tree(lg, pages, batch, QH, table.cuda(), lens.cuda(), q, most, start, bits, SCALE, out, ws[:size])
    torch.cuda.synchronize()
    assert (ws[size:] == 0xff).all()
    P.check(out, *T.reference(lo, pages, table, lens, q, counts, trees, SCALE, "bf16"), fmt)


@pytest.mark.parametrize("dtype,fmt,QH", [("bf16", "grid256", 8), ("bf16", "rtn4", 16), ("bf16", "grid64", 2), ("fp32", "grid16", 4)])
def test_more_sequences_than_a_wave_has_lanes(dtype, fmt, QH):
    """Waves of few rows: pieces are shared out by other code from 65 sequences on."""
    batch, H, page, most = 101, 2, 16, 6
    gen = torch.Generator().manual_seed(79)
    lengths, counts = torch.randint(6, 300, (batch,), generator=gen).tolist(), torch.randint(0, most + 1, (batch,), generator=gen).tolist()
    lengths[3], lengths[70], lengths[80], counts[70] = 2500, 3100, 0, most
    lo, lg, pages, table, lens, gen = T.cache(dtype, fmt, H, lengths, page, seed=13)
    trees = [T.random_tree(n, gen) for n in counts]
    q = queries(gen, sum(counts), QH, dtype)
    got = attend(lg, pages, table, lens, q, counts, trees, max_queries=most)
    torch.cuda.synchronize()
    P.check(got, *T.reference(lo, pages, table, lens, q, counts, trees, SCALE, dtype), fmt)
