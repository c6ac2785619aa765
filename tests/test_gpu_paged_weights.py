"""aquakv_paged_weights against soft-max weights in 64 bits, added up per token and kv head."""
import pytest
import torch

from tests import paged_utils as P
from tests import tree_utils as T

pytestmark = pytest.mark.gpu
SCALE = 128 ** -0.5


def wanted(lo, pages, table, lens, q, counts, max_queries, keep, mass, scale=SCALE):
    """-> (mass [n_pages, H, page] in fp64, bound on the error of each value, which were written).

    A score is off by at most d = scale * sum |q_i k_i| (2 u + 128 s) (operands to 22 bits, u = 2^-21; sums in fp32, s = 2^-24; Cauchy: at most |q| |k|)
    and by the exponent's argument, |score| 2^-22; a weight by the factor e^(2 d) for its own score, and as much for the largest of them, on which
    numerator and denominator depend; the exponential and the sums over n tokens and the rows: (n + rows + 8) s.  Then the product with keep and the sum."""
    K = P.held(lo, pages.k_codes, pages.k_scales, lo.signs_k)
    QH, H, page = q.shape[1], lo.kv_heads, pages.page_tokens
    rep, u, s = QH // H, 2.0 ** -21, 2.0 ** -24
    out, bound, written = mass.double().clone(), torch.zeros(mass.shape, dtype=torch.float64), torch.zeros(mass.shape, dtype=torch.bool)
    room, at = table.shape[1] * page, 0
    for b, n in enumerate(counts):
        length = min(max(int(lens[b]), 0), room)
        rows = P.sequence_rows(pages, table[b], length)
        t = torch.arange(length)[rows >= 0]
        rows = rows[rows >= 0]
        m = min(n, max_queries)
        if n and len(rows):
            seen = t[None] <= length - n + torch.arange(m)[:, None]
            for h in range(H):
                k = K[rows, h].clone()
                k[~seen.any(0)] = 0
                total, off = (torch.zeros(len(rows), dtype=torch.float64) for _ in range(2))
                for r in range(h * rep, (h + 1) * rep):
                    x = q[at:at + m, r].double().cpu()
                    score = (x @ k.T * scale).masked_fill(~seen, -torch.inf)
                    p = torch.where(seen.any(-1, keepdim=True), torch.softmax(score, -1), 0)
                    d = abs(scale) * x.norm(dim=-1, keepdim=True) * k.norm(dim=-1)[None] * (2 * u + 128 * s) + torch.where(seen, score, 0).abs() * 2.0 ** -22
                    top = torch.where(seen, d, 0).amax(-1, keepdim=True)
                    total += p.sum(0)
                    off += (p * (2 * d + 2 * top + (length + m * rep + 8) * s)).sum(0)
                page_of, place = rows // page, rows % page
                old = torch.where(t < length - n, keep * out[page_of, h, place], 0.0) if keep else torch.zeros(len(rows), dtype=torch.float64)
                out[page_of, h, place] = old + total
                bound[page_of, h, place] = off + 2 * s * (old.abs() + total)
                written[page_of, h, place] = True
        at += n
    return out, bound, written


def weights(lg, pages, table, lens, q, counts, keep, mass, max_queries=None, ragged=True):
    from paper_2501_19392_amd import binding as B
    most = max(max(counts), 1) if max_queries is None else max_queries
    start = torch.tensor([sum(counts[:b]) for b in range(len(counts) + 1)], dtype=torch.int32).cuda() if ragged else None
    size = B.aquakv_paged_weights_workspace_bytes(lg, pages, len(counts), q.shape[1], table.shape[1], q.shape[0], most)
    assert size > 0
    ws = torch.full((size,), 0xff, dtype=torch.uint8, device="cuda")
    got = mass.cuda()
    B.aquakv_paged_weights(lg, pages, len(counts), q.shape[1], table.cuda(), lens.cuda(), q, most, start, SCALE, keep, got, ws)
    torch.cuda.synchronize()
    return got.cpu()


def check(got, mass, want, bound, written, what=""):
    assert torch.equal(got[~written].view(torch.int32), mass[~written].view(torch.int32)), what
    off = (got.double() - want).abs()[written]
    assert torch.isfinite(got[written]).all(), what
    assert (off <= bound[written]).all(), f"{what}: {(off / (bound[written] + 1e-300)).max():.3g} of the bound"


def some_mass(pages, H, gen, old=None):
    """What mass holds: sums so far, anything where no token is yet."""
    return torch.rand(pages.n_pages, H, pages.page_tokens, generator=gen)


def clear_new(mass, pages, table, lens, counts):
    """NaN for the queries' own tokens: it is not read."""
    for b, n in enumerate(counts):
        rows = P.sequence_rows(pages, table[b], int(lens[b]))[max(int(lens[b]) - n, 0):]
        rows = rows[rows >= 0]
        mass[rows // pages.page_tokens, :, rows % pages.page_tokens] = float("nan")


@pytest.mark.parametrize("dtype,fmt,H,QH,lengths,page,counts,keep", [
    ("bf16", "grid256", 8, 32, [700, 3, 1, 64], 64, [1, 1, 1, 1], 1.0),     # a generated token each: scores are kept
    ("bf16", "grid64", 3, 24, [333, 1040], 24, [1, 1], 0.5), ("bf16", "grid16", 1, 2, [2100, 40], 8, [4, 3], 1.0),
    ("bf16", "grid256", 2, 2, [9, 8, 300], 16, [8, 8, 5], 0.0), ("bf16", "rtn4", 8, 24, [500, 31], 32, [1, 1], 1.0), ("bf16", "rtn2", 2, 8, [129, 70], 40, [2, 1], 0.875),
    ("bf16", "grid256", 8, 32, [400, 90], 64, [3, 2], 1.0),                 # more rows: scores are taken twice
    ("bf16", "grid256", 2, 8, [517, 64, 33], 16, [64, 64, 7], 1.0), ("bf16", "grid64", 1, 5, [300], 8, [41], 0.0), ("bf16", "grid16", 3, 12, [160, 1], 128, [20, 1], 0.25),
    ("bf16", "rtn4", 2, 16, [140, 77], 24, [30, 77], 1.0), ("bf16", "rtn2", 1, 16, [260], 16, [9], 1.0),
    ("fp32", "grid256", 2, 8, [222, 17], 16, [1, 1], 1.0), ("fp32", "grid64", 1, 3, [100], 8, [12], 1.0), ("fp32", "grid16", 1, 1, [65], 16, [20], 0.0),
    ("fp32", "rtn4", 3, 6, [90, 40], 40, [3, 4], 1.0), ("fp32", "rtn2", 1, 8, [130], 24, [10], 0.5)])
def test_weights_are_added_up(dtype, fmt, H, QH, lengths, page, counts, keep):
    print(f"case weights {dtype} {fmt} H={H} QH={QH} {lengths} {counts} keep={keep}", flush=True)
    lo, lg, pages, table, lens, gen = T.cache(dtype, fmt, H, lengths, page)
    q = (1.5 * torch.randn(sum(counts), QH, 128, generator=gen)).to(P.storage(dtype)).cuda()
    mass = some_mass(pages, H, gen)
    if keep == 0.0:
        mass.fill_(float("nan"))
    else:
        clear_new(mass, pages, table, lens, counts)
    got = weights(lg, pages, table, lens, q, counts, keep, mass)
    want = wanted(lo, pages, table, lens, q, counts, max(counts), keep, mass)
    check(got, mass, *want)
    # every row's weights are 1 together
    if keep == 0.0:
        for b, n in enumerate(counts):
            rows = P.sequence_rows(pages, table[b], lengths[b])
            total = got[rows // page, :, rows % page].double().sum(0)
            assert (total - n * (QH // H)).abs().max() <= n * (QH // H) * 1e-4
    assert torch.equal(weights(lg, pages, table, lens, q, counts, keep, mass).view(torch.int32), got.view(torch.int32))      # the same bits each time


@pytest.mark.parametrize("QH,counts,max_queries", [(4, [2, 0, 1, 3], 2), (16, [12, 0, 3, 30], 11), (16, [90, 0, 1, 240], 3)])
def test_ragged_and_empty_sequences(QH, counts, max_queries):
    """No queries: left as it was; more rows than are answered; no tokens; pages that are not in the pool."""
    H, page, lengths = 2, 16, [100, 50, 0, 240]
    lo, lg, pages, table, lens, gen = T.cache("bf16", "grid256", H, lengths, page, seed=1)
    table[0, 1], table[3, 4], table[3, 14] = -1, pages.n_pages, -7
    q = (1.5 * torch.randn(sum(counts), QH, 128, generator=gen)).bfloat16().cuda()
    mass = some_mass(pages, H, gen)
    got = weights(lg, pages, table, lens, q, counts, 0.75, mass, max_queries=max_queries)
    check(got, mass, *wanted(lo, pages, table, lens, q, counts, max_queries, 0.75, mass))


@pytest.mark.parametrize("QH,n", [(4, 1), (16, 5)])
def test_what_is_not_seen_and_lengths_outside_the_table(QH, n):
    """Rows ahead of the first token (more queries than tokens), lengths beyond the table and below zero, and in one call with them."""
    H, page, lengths = 1, 8, [40, 2, 24]
    lo, lg, pages, table, _, gen = T.cache("bf16", "grid64", H, lengths, page, seed=2)
    lens = torch.tensor([1 << 30, 2, -4], dtype=torch.int32)
    q = (1.5 * torch.randn(3 * n, QH, 128, generator=gen)).bfloat16().cuda()
    mass = some_mass(pages, H, gen)
    got = weights(lg, pages, table, lens, q, [n] * 3, 1.0, mass, ragged=False)
    check(got, mass, *wanted(lo, pages, table, lens, q, [n] * 3, n, 1.0, mass))


@pytest.mark.parametrize("fmt,n", [("grid256", 1), ("rtn4", 1), ("grid256", 10)])
def test_long_sequences_in_many_pieces(fmt, n):
    H, page, lengths = 2, 128, [20000, 11, 6001]
    lo, lg, pages, table, lens, gen = T.cache("bf16", fmt, H, lengths, page, seed=3)
    q = (1.5 * torch.randn(3 * n, 2 * H, 128, generator=gen)).bfloat16().cuda()
    mass = some_mass(pages, H, gen)
    got = weights(lg, pages, table, lens, q, [n] * 3, 1.0, mass, ragged=False)
    check(got, mass, *wanted(lo, pages, table, lens, q, [n] * 3, n, 1.0, mass))


@pytest.mark.parametrize("n", [1, 6])
def test_far_scores(n):
    """Scores of hundreds: one token has nearly all the weight, most have none."""
    lo, lg, pages, table, lens, gen = T.cache("bf16", "grid256", 1, [300, 64], 16, seed=4, spread=2.0)
    q = (60.0 * torch.randn(2 * n, 4, 128, generator=gen)).bfloat16().cuda()
    mass = some_mass(pages, 1, gen)
    got = weights(lg, pages, table, lens, q, [n] * 2, 1.0, mass, ragged=False)
    check(got, mass, *wanted(lo, pages, table, lens, q, [n] * 2, n, 1.0, mass))


@pytest.mark.parametrize("n", [1, 10])
def test_captured_calls_accumulate(n):
    """A graph that adds the weights of a token after token: replays against eager calls, with other lengths and queries."""
    from paper_2501_19392_amd import binding as B
    H, QH, page = 2, 8, 16
    lo, lg, pages, table, lens, gen = T.cache("bf16", "grid256", H, [400, 300], page, seed=5)
    mass = some_mass(pages, H, gen)
    held, got = mass.cuda(), mass.cuda()
    q, on, tab = torch.zeros(2 * n, QH, 128, dtype=torch.bfloat16, device="cuda"), lens.cuda(), table.cuda()
    size = B.aquakv_paged_weights_workspace_bytes(lg, pages, 2, QH, table.shape[1], 2 * n, n)
    ws = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(2)]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.aquakv_paged_weights(lg, pages, 2, QH, tab, on, q, n, None, SCALE, 1.0, held, ws[0])
    held.copy_(mass)
    for lengths in ([100, 299], [110, 40], [400, 300], [3, 0]):
        on.copy_(torch.tensor(lengths, dtype=torch.int32))
        q.copy_(1.5 * torch.randn(q.shape, generator=gen))
        g.replay()
        B.aquakv_paged_weights(lg, pages, 2, QH, tab, on, q, n, None, SCALE, 1.0, got, ws[1])
        torch.cuda.synchronize()
        assert torch.equal(held.view(torch.int32), got.view(torch.int32))


@pytest.mark.parametrize("n", [1, 9])
def test_a_pool_of_more_than_4_gib(n):
    """Offsets of codes pass 32 bits."""
    from paper_2501_19392_amd import binding as B
    from tests import parity_utils as U
    page, H, QH = 64, 8, 16
    n_pages = ((1 << 32) // (H * 64)) // page + 10
    lo, lg = U.make_layers(H, "bf16", 256)
    pages, small = B.Pages(lg, n_pages, page), B.Pages(lg, 6, page)
    gen = torch.Generator().manual_seed(6)
    P.fill(lo, small, gen)
    table = torch.tensor([[n_pages - 1, 0, n_pages - 3], [n_pages - 2, n_pages - 4, 1]], dtype=torch.int32)
    used = (table.view(-1, 1).long() * page + torch.arange(page)).view(-1).cuda()
    for name in ("k_codes", "k_scales", "v_codes", "v_scales"):
        getattr(pages, name)[used] = getattr(small, name)
    lens, q = torch.tensor([150, 130], dtype=torch.int32), (1.5 * torch.randn(2 * n, QH, 128, generator=gen)).bfloat16().cuda()
    mass = some_mass(small, H, gen)
    big = torch.zeros(n_pages, H, page, device="cuda")
    big[table.view(-1).long().cuda()] = mass.cuda()
    ws = torch.empty(B.aquakv_paged_weights_workspace_bytes(lg, pages, 2, QH, 3, 2 * n, n), dtype=torch.uint8, device="cuda")
    B.aquakv_paged_weights(lg, pages, 2, QH, table.cuda(), lens.cuda(), q, n, None, SCALE, 1.0, big, ws)
    torch.cuda.synchronize()
    at = torch.arange(6, dtype=torch.int32).view(2, 3)
    check(big[table.view(-1).long().cuda()].cpu(), mass, *wanted(lo, small, at, lens, q, [n, n], n, 1.0, mass))


@pytest.mark.parametrize("backbone", ["grid256", "rtn4"])
@pytest.mark.parametrize("n,bad", [(2, 0), (20, 3), (20, 18)])
def test_query_without_numbers(backbone, n, bad):
    """It reaches the tokens that it sees and no others: those get what they get from the later queries."""
    QH, page, length = 4, 16, 150
    lo, lg, pages = P.make(1, "bf16", backbone, 12, page)
    gen = torch.Generator().manual_seed(n + bad)
    P.fill(lo, pages, gen)
    table, lens = torch.arange(12, dtype=torch.int32)[None], torch.tensor([length], dtype=torch.int32)
    q = torch.randn(n, QH, 128, generator=gen).bfloat16().cuda()
    mass = some_mass(pages, 1, gen)
    seen = length - n + bad + 1                             # tokens that the bad query sees
    want, bound, written = wanted(lo, pages, table, lens, q, [n], n, 1.0, mass)
    q[bad, 1, 5] = torch.nan
    got = weights(lg, pages, table, lens, q, [n], 1.0, mass).flatten()
    assert got[:seen].isnan().all()
    off = (got.double() - want.flatten())[seen:length].abs()
    assert (off <= bound.flatten()[seen:length]).all()
    assert torch.equal(got[length:], mass.flatten()[length:])


@pytest.mark.parametrize("fmt,QH,most,batch,room", [("grid256", 8, 1, 70, 0), ("rtn4", 8, 2, 131, 0), ("grid64", 8, 2, 65, 30000), ("grid256", 8, 11, 70, 0), ("rtn2", 16, 5, 129, 9000)])
def test_more_sequences_than_a_wave_has_lanes(fmt, QH, most, batch, room):
    """Pieces are shared out by other code from 65 sequences on; with page tables as wide as the longest one, and much wider."""
    H, page = 2, 16
    print(f"case weights of many {fmt} {batch} sequences of {most}, room {room}", flush=True)
    gen = torch.Generator().manual_seed(31)
    lengths, counts = torch.randint(0, 400, (batch,), generator=gen).tolist(), torch.randint(0, most + 1, (batch,), generator=gen).tolist()
    lengths[5], lengths[64], counts[64] = 3000, 2111, most
    lo, lg, pages, table, lens, gen = T.cache("bf16", fmt, H, lengths, page, seed=7)
    table = torch.cat([table, torch.full((batch, max(room // page - table.shape[1], 0)), -1, dtype=torch.int32)], 1).contiguous()
    q = (1.5 * torch.randn(sum(counts), QH, 128, generator=gen)).bfloat16().cuda()
    mass = some_mass(pages, H, gen)
    got = weights(lg, pages, table, lens, q, counts, 0.75, mass, max_queries=most)
    check(got, mass, *wanted(lo, pages, table, lens, q, counts, most, 0.75, mass))
