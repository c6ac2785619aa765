"""aquakv_paged_select against a sort of the sums in their order, aquakv_paged_keep against rows copied one by one."""
import numpy as np
import pytest
import torch

from tests import paged_utils as P
from tests import tree_utils as T

pytestmark = pytest.mark.gpu
POOL = ("k_codes", "k_scales", "v_codes", "v_scales")


# ------------------------------------------------------------------------------------------------ select
def masses(kind, n_pages, H, page, gen):
    m = (2.0 * torch.randn(n_pages, H, page, generator=gen)).exp()
    if kind == "ties":                                                      # few different sums, -0 and 0 among them
        m = torch.randint(-1, 3, m.shape, generator=gen).float()
        m[torch.rand(m.shape, generator=gen) < 0.2] = -0.0
    elif kind == "equal":
        m = torch.zeros_like(m)
    elif kind == "odd":                                                     # not finite, subnormal, negative
        bad = torch.tensor([float("nan"), float("inf"), -float("inf"), 1e-42, -1e-42, -3.0, 3e38])
        pick = torch.rand(m.shape, generator=gen) < 0.1
        m[pick] = bad[torch.randint(0, len(bad), (int(pick.sum()),), generator=gen)]
    return m


def wanted(mass, table, length, n_pages, page, budget, n_first, n_last):
    room = table.shape[0] * page
    n = min(max(length, 0), room)
    t = np.arange(n)
    pages = table.numpy()[t // page]
    there = (pages >= 0) & (pages < n_pages)
    total = np.zeros(n, dtype=np.float32)
    with np.errstate(all="ignore"):
        for h in range(mass.shape[1]):
            head = mass[np.where(there, pages, 0), h, t % page]
            total = head.copy() if h == 0 else total + head
    always = (t < n_first) | (t >= n - n_last)
    order = np.where(np.isnan(total), 1, 2)                                 # what is no number comes behind every number,
    order = np.where(there, np.where(always, 3, order), 0)                  # what is not there behind that
    by = np.where(order == 2, np.where(np.isnan(total), 0, total), 0)
    first = np.lexsort((t, -by, -order))[:budget]
    return np.sort(first)


def select(lg, pages, table, lens, mass, budget, n_first, n_last):
    from paper_2501_19392_amd import binding as B
    b = table.shape[0]
    kept = torch.full((b, budget), 12345, dtype=torch.int32, device="cuda")
    n_kept = torch.full((b,), 12345, dtype=torch.int32, device="cuda")
    size = B.aquakv_paged_select_workspace_bytes(lg, pages, b, table.shape[1], budget)
    ws = torch.full((size,), 0xff, dtype=torch.uint8, device="cuda")
    B.aquakv_paged_select(lg, pages, b, table.cuda(), lens.cuda(), mass.cuda(), budget, n_first, n_last, kept, n_kept, ws)
    torch.cuda.synchronize()
    return kept.cpu().numpy(), n_kept.cpu().numpy()


@pytest.mark.parametrize("kind", ["plain", "ties", "equal", "odd"])
@pytest.mark.parametrize("H,lengths,page,budget,n_first,n_last", [
    (8, [700, 0, 1, 90, 100, 101], 24, 100, 4, 32), (1, [64, 65, 63, 5000], 64, 64, 0, 0), (3, [37, 8, 9], 8, 7, 3, 4), (2, [200], 16, 1, 0, 0),
    (5, [4097, 1025], 128, 1024, 1000, 24), (8, [50], 40, 1, 1, 0), (2, [129, 2], 8, 3, 0, 3)])
def test_the_largest_masses_are_selected(kind, H, lengths, page, budget, n_first, n_last):
    print(f"case select {kind} H={H} {lengths} budget={budget}", flush=True)
    lo, lg, pages, table, lens, gen = T.cache("bf16", "grid16", H, lengths, page)
    mass = masses(kind, pages.n_pages, H, page, gen)
    if kind == "odd" and table.shape[1] > 3:
        table[0, 1], table[0, 3] = -1, pages.n_pages + 3
    lens = torch.cat([lens[:-1], lens[-1:]])
    kept, n_kept = select(lg, pages, table, lens, mass, budget, n_first, n_last)
    for b, n in enumerate(lengths):
        want = wanted(mass.numpy(), table[b], n, pages.n_pages, page, budget, n_first, n_last)
        assert n_kept[b] == len(want) == min(n, budget)
        assert (kept[b, :len(want)] == want).all(), (b, kept[b], want)
        assert (kept[b, len(want):] == -1).all()


@pytest.mark.parametrize("kind", ["plain", "ties", "equal"])
@pytest.mark.parametrize("n,budget", [(70001, 20000), (300000, 299999), (16384, 5), (16385, 16000), (32769, 1)])
def test_selecting_from_a_long_sequence(kind, n, budget):
    lo, lg, pages, table, lens, gen = T.cache("bf16", "grid16", 1, [n, 3], 128)
    mass = masses(kind, pages.n_pages, 1, 128, gen)
    last = 1 if budget < 5 else 3
    kept, n_kept = select(lg, pages, table, lens, mass, budget, 0, last)
    for b, m in enumerate((n, 3)):
        want = wanted(mass.numpy(), table[b], m, pages.n_pages, 128, budget, 0, last)
        assert n_kept[b] == len(want) and (kept[b, :len(want)] == want).all() and (kept[b, len(want):] == -1).all()


def test_lengths_outside_the_table_and_an_empty_budget():
    lo, lg, pages, table, lens, gen = T.cache("bf16", "grid16", 2, [40, 40], 8)
    mass = masses("plain", pages.n_pages, 2, 8, gen)
    kept, n_kept = select(lg, pages, table, torch.tensor([1 << 30, -5], dtype=torch.int32), mass, 10, 2, 2)
    assert (kept[0] == wanted(mass.numpy(), table[0], 40, pages.n_pages, 8, 10, 2, 2)).all() and list(n_kept) == [10, 0] and (kept[1] == -1).all()
    kept, n_kept = select(lg, pages, table, lens, mass, 0, 0, 0)
    assert list(n_kept) == [0, 0]


# ------------------------------------------------------------------------------------------------ keep
def kept_by_hand(pool, mass, page, n_pages, table, kept, n_kept, first, to_table):
    """The arrays after the moves, from their rows before."""
    def row(tab, t):
        if t < 0 or t >= len(tab) * page or not 0 <= tab[t // page] < n_pages:
            return -1
        return int(tab[t // page]) * page + t % page
    after = {k: v.clone() for k, v in pool.items()}
    new_mass = None if mass is None else mass.clone()
    for b in range(len(kept)):
        for i in range(min(int(n_kept[b]), kept.shape[1])):
            f = 0 if first is None else int(first[b])
            src, dst = row(table[b], int(kept[b, i])), row((table if to_table is None else to_table)[b], f + i)
            if src < 0 or dst < 0 or f < 0:
                continue
            for k in pool:
                after[k][dst] = pool[k][src]
            if mass is not None:
                new_mass[dst // page, :, dst % page] = mass[src // page, :, src % page]
    return after, new_mass


@pytest.mark.parametrize("fmt,H,page,lengths,most,way,with_first,with_mass", [
    ("grid256", 8, 64, [300, 77], 60, "ascending", False, True), ("grid64", 3, 24, [500, 40, 9], 33, "gaps", True, False),
    ("grid16", 1, 8, [1500], 1024, "ascending", False, True), ("grid256", 1, 16, [1500, 3], 1025, "gaps", False, True),
    ("rtn4", 8, 32, [2600], 2500, "gaps", True, True), ("rtn2", 5, 16, [5100, 900], 5000, "ascending", False, False),
    ("grid256", 2, 128, [8300], 8192, "gaps", False, True), ("grid64", 1, 40, [9100, 50], 9000, "ascending", False, True),
    ("rtn4", 3, 8, [9500], 9001, "gaps", True, True), ("grid16", 7, 16, [64], 1, "gaps", True, True),
    ("grid256", 33, 8, [1400, 900], 1200, "ascending", True, True), ("rtn4", 33, 16, [4500], 4300, "gaps", False, True),      # columns of more entries than a round
    ("grid64", 32, 8, [9000], 8700, "ascending", False, True), ("grid16", 64, 24, [1300], 1025, "gaps", False, False),         # ... than a chunk
    ("grid256", 12, 8, [200, 100], 90, "across", False, True), ("rtn2", 2, 24, [700, 60], 600, "across", True, False), ("grid64", 8, 16, [400], 128, "across", True, True),
    ("grid16", 1, 16, [400, 7], 300, "across", False, True), ("rtn4", 5, 32, [90], 33, "across", True, True)])
def test_rows_that_are_kept(fmt, H, page, lengths, most, way, with_first, with_mass):
    from paper_2501_19392_amd import binding as B
    print(f"case keep {fmt} H={H} page={page} {lengths} most={most} {way}", flush=True)
    to_pages = -(-(most + 7) // page)
    extra = len(lengths) * to_pages if way == "across" else 0
    lo, lg, pages, table, lens, gen = T.cache("bf16", fmt, H, lengths, page, room=3 + extra)
    b = len(lengths)
    kept = torch.full((b, most), -1, dtype=torch.int32)
    n_kept, first = torch.zeros(b, dtype=torch.int32), torch.zeros(b, dtype=torch.int32)
    for i, n in enumerate(lengths):
        m = min(most, n)
        first[i] = 5 if with_first and n > 64 and m + 5 <= n else 0
        if way == "across":                                                 # any order, some twice
            kept[i, :m] = torch.randint(0, n, (m,), generator=gen).to(torch.int32)
        else:
            kept[i, :m] = int(first[i]) + torch.randperm(n - int(first[i]), generator=gen)[:m].sort().values.to(torch.int32)
        if way != "ascending" and m > 4:                                    # some that are not there
            kept[i, 2], kept[i, 3], kept[i, 4] = -1, 1 << 30, -(1 << 31)
        n_kept[i] = m if i == 0 else m - m // 3
    if way == "gaps" and table.shape[1] > 4:
        table[0, 3] = -1
    to = None
    if way == "across":
        used = set(table.view(-1).tolist())
        free = [p for p in range(pages.n_pages) if p not in used]
        to = torch.tensor(free[:b * to_pages], dtype=torch.int32).view(b, to_pages)
        to[0, 0] = -1 if b == 1 else to[0, 0]
    mass = torch.rand(pages.n_pages, H, page, generator=gen) if with_mass else None
    pool = {k: getattr(pages, k).cpu() for k in POOL}
    f = first if with_first else None
    want, want_mass = kept_by_hand(pool, mass, page, pages.n_pages, table.tolist(), kept, n_kept, f, None if to is None else to.tolist())
    on = lambda t: None if t is None else t.cuda()  # noqa: E731
    got_mass = on(mass)
    ws = torch.full((B.aquakv_paged_keep_workspace_bytes(lg, pages, b, most, with_mass),), 0xff, dtype=torch.uint8, device="cuda")
    B.aquakv_paged_keep(lg, pages, b, table.cuda(), kept.cuda(), n_kept.cuda(), on(f), on(to), got_mass, ws)
    torch.cuda.synchronize()
    for k in POOL:
        assert torch.equal(getattr(pages, k).cpu(), want[k]), k
    if with_mass:
        assert torch.equal(got_mass.cpu(), want_mass)


def test_counts_beyond_the_list_and_below_zero():
    from paper_2501_19392_amd import binding as B
    lo, lg, pages, table, lens, gen = T.cache("bf16", "grid256", 2, [50, 50, 50], 8)
    kept = torch.tensor([[10, 20, 30]] * 3, dtype=torch.int32)
    n_kept, first = torch.tensor([1 << 30, -3, 2], dtype=torch.int32), torch.tensor([0, 0, -1], dtype=torch.int32)
    pool = {k: getattr(pages, k).cpu() for k in POOL}
    want, _ = kept_by_hand(pool, None, 8, pages.n_pages, table.tolist(), kept, n_kept, first, None)
    ws = torch.empty(B.aquakv_paged_keep_workspace_bytes(lg, pages, 3, 3, False), dtype=torch.uint8, device="cuda")
    B.aquakv_paged_keep(lg, pages, 3, table.cuda(), kept.cuda(), n_kept.cuda(), first.cuda(), None, None, ws)
    torch.cuda.synchronize()
    for k in POOL:
        assert torch.equal(getattr(pages, k).cpu(), want[k]), k


@pytest.mark.parametrize("way", ["in place", "staged", "across"])
def test_rows_behind_4_gib(way):
    """Offsets of codes pass 32 bits."""
    from paper_2501_19392_amd import binding as B
    from tests import parity_utils as U
    page = 64
    n_pages = ((1 << 32) // (8 * 64)) // page + 300
    lo, lg = U.make_layers(8, "bf16", 256)
    pages = B.Pages(lg, n_pages, page)
    table = torch.tensor([[n_pages - 1 - i for i in range(150)]], dtype=torch.int32)
    to = torch.tensor([[n_pages - 160 - i for i in range(140)]], dtype=torch.int32) if way == "across" else None
    rows = (table[0].long()[:, None] * page + torch.arange(page)).view(-1)
    gen = torch.Generator().manual_seed(1)
    src = {}
    for k in POOL:
        x = getattr(pages, k)
        part = torch.randint(0, 256, (len(rows), *x.shape[1:], x.element_size()), generator=gen, dtype=torch.int32).to(torch.uint8).contiguous().view(x.dtype)
        src[k] = part.view(len(rows), *x.shape[1:])
        x[rows.cuda()] = src[k].cuda()
    m = 4000 if way == "staged" else 1000 if way == "in place" else 4000
    kept = torch.randperm(len(rows), generator=gen)[:m].sort().values.to(torch.int32)[None]
    ws = torch.empty(B.aquakv_paged_keep_workspace_bytes(lg, pages, 1, m, False), dtype=torch.uint8, device="cuda")
    B.aquakv_paged_keep(lg, pages, 1, table.cuda(), kept.cuda(), torch.tensor([m], dtype=torch.int32).cuda(), None, None if to is None else to.cuda(), None, ws)
    torch.cuda.synchronize()
    target = rows[:m] if to is None else (to[0].long()[:, None] * page + torch.arange(page)).view(-1)[:m]
    for k in POOL:
        assert torch.equal(getattr(pages, k)[target.cuda()].cpu(), src[k][kept[0].long()]), k


def test_many_rows_to_other_pages_without_room_for_them():
    """One sequence of more entries than go by columns, in a workspace of 256 bytes of which nothing is touched."""
    from paper_2501_19392_amd import binding as B
    most, page, H = 3000, 16, 3
    to_pages = -(-most // page)
    lo, lg, pages, table, lens, gen = T.cache("bf16", "grid64", H, [3500], page, room=3 + to_pages)
    used = set(table.view(-1).tolist())
    to = torch.tensor([p for p in range(pages.n_pages) if p not in used][:to_pages], dtype=torch.int32)[None]
    kept = torch.randperm(3500, generator=gen)[:most].to(torch.int32)[None]
    n_kept = torch.tensor([most], dtype=torch.int32)
    mass = torch.rand(pages.n_pages, H, page, generator=gen)
    assert B.aquakv_paged_keep_workspace_bytes(lg, pages, 1, most, True) > 256
    pool = {k: getattr(pages, k).cpu() for k in POOL}
    want, want_mass = kept_by_hand(pool, mass, page, pages.n_pages, table.tolist(), kept, n_kept, None, to.tolist())
    ws, got = torch.full((4096,), 0xff, dtype=torch.uint8, device="cuda"), mass.cuda()
    B.aquakv_paged_keep(lg, pages, 1, table.cuda(), kept.cuda(), n_kept.cuda(), None, to.cuda(), got, ws[:256])
    torch.cuda.synchronize()
    for k in POOL:
        assert torch.equal(getattr(pages, k).cpu(), want[k]), k
    assert torch.equal(got.cpu(), want_mass) and (ws == 0xff).all()


@pytest.mark.parametrize("kind", ["plain", "ties", "odd"])
@pytest.mark.parametrize("H,lengths,page,budget,n_first,n_last", [
    (8, [40000, 17001, 9000, 30001, 0, 1, 36864], 128, 12000, 100, 1000), (5, [20000, 19999, 16385, 12288], 64, 8193, 4096, 4097), (3, [70000, 50000], 256, 49999, 5, 0),
    (2, [18000, 17000, 300], 40, 0, 0, 0)])
def test_selecting_from_many_long_sequences(kind, H, lengths, page, budget, n_first, n_last):
    """Slabs of several sequences, each with its own: some end inside a slab, one is below the budget, pages are missing, masses are no numbers."""
    print(f"case select long {kind} H={H} {lengths} budget={budget}", flush=True)
    lo, lg, pages, table, lens, gen = T.cache("bf16", "grid16", H, lengths, page)
    mass = masses(kind, pages.n_pages, H, page, gen)
    if kind == "odd":
        for b in range(len(lengths)):
            table[b, 1], table[b, 50 + b], table[b, 1 + b] = -1, pages.n_pages + b, -5
    kept, n_kept = select(lg, pages, table, lens, mass, budget, n_first, n_last)
    for b, n in enumerate(lengths):
        want = wanted(mass.numpy(), table[b], n, pages.n_pages, page, budget, n_first, n_last)
        assert n_kept[b] == len(want) == min(n, budget), b
        assert (kept[b, :len(want)] == want).all(), b
        assert (kept[b, len(want):] == -1).all(), b


@pytest.mark.parametrize("room", [0, 20000])
def test_selecting_from_more_sequences_than_a_wave_has_lanes(room):
    """With page tables as wide as the longest one, and wider: by a workgroup each, and by slabs, most of which have nothing."""
    H, page, batch, budget = 2, 16, 133, 150
    gen = torch.Generator().manual_seed(21)
    lengths = torch.randint(0, 400, (batch,), generator=gen).tolist()
    lo, lg, pages, table, lens, gen = T.cache("bf16", "grid16", H, lengths, page)
    table = torch.cat([table, torch.full((batch, max(room // page - table.shape[1], 0)), -1, dtype=torch.int32)], 1).contiguous()
    mass = masses("ties", pages.n_pages, H, page, gen)
    kept, n_kept = select(lg, pages, table, lens, mass, budget, 3, 20)
    for b, n in enumerate(lengths):
        want = wanted(mass.numpy(), table[b], n, pages.n_pages, page, budget, 3, 20)
        assert n_kept[b] == len(want) and (kept[b, :len(want)] == want).all() and (kept[b, len(want):] == -1).all(), b
