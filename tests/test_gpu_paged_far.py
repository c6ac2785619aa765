"""Sequences of almost 2^31 tokens, whose table names few pages over and over: weights, selection and moves at token numbers that leave no room in 32 bits."""
import numpy as np
import pytest
import torch

from tests import paged_utils as P
from tests import test_gpu_paged_weights as W

pytestmark = pytest.mark.gpu
PAGE, PAGES = 128, (1 << 31) // 128 - 33
SCALE = 128 ** -0.5


def make(seed, n_pages=4):
    """Pages 0 ... n_pages - 2 in turn over the whole table, the last one only at its end."""
    lo, lg, pages = P.make(1, "bf16", "grid16", n_pages, PAGE)
    gen = torch.Generator().manual_seed(seed)
    P.fill(lo, pages, gen)
    table = (torch.arange(PAGES, device="cuda", dtype=torch.int32) % (n_pages - 1))[None].contiguous()
    table[0, -1] = n_pages - 1
    return lo, lg, pages, table, gen


def test_weights_of_the_last_page():
    """Every page but the last is there many times: its tokens' weights are those of one page, as often divided."""
    from paper_2501_19392_amd import binding as B
    lo, lg, pages, table, gen = make(1)
    length = PAGES * PAGE - 5
    q = (1.5 * torch.randn(1, 1, 128, generator=gen)).bfloat16().cuda()
    mass = torch.zeros(4, 1, PAGE, device="cuda")
    ws = torch.empty(B.aquakv_paged_weights_workspace_bytes(lg, pages, 1, 1, PAGES, 1, 1), dtype=torch.uint8, device="cuda")
    B.aquakv_paged_weights(lg, pages, 1, 1, table, torch.tensor([length], dtype=torch.int32).cuda(), q, 1, None, SCALE, 0.0, mass, ws)
    torch.cuda.synchronize()
    got = mass[3, 0].cpu().double()
    K = P.held(lo, pages.k_codes, pages.k_scales, lo.signs_k)[:, 0]
    score = (q[0].double().cpu() @ K.T * SCALE)[0].view(4, PAGE)
    e = score.exp()
    times = torch.tensor([len(range(i, PAGES - 1, 3)) for i in range(3)], dtype=torch.float64)
    total = (e[:3].sum(1) * times).sum() + e[3, :PAGE - 5].sum()
    # as for other lengths, but that a lane's sum of its tiles has as many additions as it has tiles: pieces of 2^31 / 32 / 4096 tiles, then their join
    d = SCALE * q[0].double().cpu().norm() * K.norm(dim=-1).max() * (2 * 2.0 ** -21 + 128 * 2.0 ** -24) + score.abs().max() * 2.0 ** -22
    bound = e[3] / total * (4 * d + (2 ** 14 + 4096 + 64) * 2.0 ** -24)
    assert ((got - e[3] / total).abs() <= bound)[:PAGE - 5].all()
    assert (got[PAGE - 5:] == 0).all()


def test_selection_from_almost_2_31_tokens():
    from paper_2501_19392_amd import binding as B
    lo, lg, pages, table, gen = make(2)
    length, budget = PAGES * PAGE - 5, 50
    mass = torch.rand(4, 1, PAGE, generator=gen)
    mass[2, 0, 77] = 5.0                                                    # there every third page: the first ones are kept,
    mass[3, 0, 100] = 7.0                                                   # and the largest, at the end
    ws = torch.empty(B.aquakv_paged_select_workspace_bytes(lg, pages, 1, PAGES, budget), dtype=torch.uint8, device="cuda")
    kept, n = torch.zeros(1, budget, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    B.aquakv_paged_select(lg, pages, 1, table, torch.tensor([length], dtype=torch.int32).cuda(), mass.cuda(), budget, 1, 2, kept, n, ws)
    torch.cuda.synchronize()
    last = (PAGES - 1) * PAGE
    want = [0] + [(3 * i + 2) * PAGE + 77 for i in range(budget - 4)] + [last + 100, length - 2, length - 1]
    assert int(n) == budget and kept[0].cpu().tolist() == want


@pytest.mark.parametrize("across", [False, True])
def test_moves_of_the_last_tokens(across):
    """The last tokens of the sequence become its first ones behind `first`, in pages of their own."""
    from paper_2501_19392_amd import binding as B
    lo, lg, pages, table, gen = make(3, n_pages=7)
    table[:] = -1                                                           # (no page twice where rows move in place)
    table[0, -3:], table[0, :3] = torch.tensor([4, 5, 6], dtype=torch.int32), torch.tensor([0, 1, 2], dtype=torch.int32)
    first = 37
    kept = ((PAGES - 3) * PAGE + torch.arange(0, 3 * PAGE, 2)).to(torch.int32)[None]
    before = {k: getattr(pages, k).cpu().clone() for k in ("k_codes", "k_scales", "v_codes", "v_scales")}
    ws = torch.empty(B.aquakv_paged_keep_workspace_bytes(lg, pages, 1, kept.shape[1], False), dtype=torch.uint8, device="cuda")
    to = torch.tensor([[3, 1, 0]], dtype=torch.int32).cuda() if across else None
    B.aquakv_paged_keep(lg, pages, 1, table, kept.cuda(), torch.tensor([kept.shape[1]], dtype=torch.int32).cuda(), torch.tensor([first], dtype=torch.int32).cuda(),
                        to, None, ws)
    torch.cuda.synchronize()
    source = 4 * PAGE + np.arange(0, 3 * PAGE, 2)
    at = first + np.arange(kept.shape[1])
    target = np.array([3, 1, 0] if across else [0, 1, 2])[at // PAGE] * PAGE + at % PAGE
    for k, x in before.items():
        want = x.clone()
        want[target] = x[source]
        assert torch.equal(getattr(pages, k).cpu(), want), k


def test_drafts_behind_almost_2_31_tokens():
    """A tree at the end of the longest sequence: what is cached counts by its pages, drafts by their bits."""
    from paper_2501_19392_amd import binding as B
    from tests import tree_utils as T
    lo, lg, pages, table, gen = make(4)
    n, length = 6, PAGES * PAGE - 40
    tree = T.random_tree(n, gen)
    q = (0.5 * torch.randn(n, 1, 128, generator=gen)).bfloat16().cuda()
    out = torch.empty_like(q)
    ws = torch.empty(B.aquakv_paged_workspace_bytes(lg, pages, 1, 1, PAGES, n, n), dtype=torch.uint8, device="cuda")
    # drafts that nearly all of the weight goes to: their keys a thousandfold
    lens = torch.tensor([length], dtype=torch.int32)
    drafts = PAGE - 40 - n + torch.arange(n) + 3 * PAGE
    big = pages.k_scales.view(torch.float16)
    big[drafts.cuda()] *= 400.0
    B.aquakv_paged_attend_tree(lg, pages, 1, 1, table, lens.cuda(), q, n, None, T.words_of(tree, 1).cuda(), SCALE, out, ws)
    torch.cuda.synchronize()
    K, V = (P.held(lo, c, s, g)[:, 0] for c, s, g in ((pages.k_codes, pages.k_scales, lo.signs_k), (pages.v_codes, pages.v_scales, lo.signs_v)))
    # all tokens of a page at once: how often it is there
    times = torch.tensor([len(range(i, PAGES - 1, 3)) for i in range(3)] + [1.0], dtype=torch.float64).repeat_interleave(PAGE)
    t = torch.arange(4 * PAGE)
    seen = torch.ones(n, 4 * PAGE, dtype=torch.bool)
    seen[:, t >= drafts[0]] = False
    seen[:, drafts] = tree
    x = (q[:, 0].double().cpu() @ K.T * SCALE + times.log()).masked_fill(~seen, -torch.inf)
    p = torch.softmax(x, -1)
    want = p @ V
    # as for other lengths, with as many additions as a lane of a piece has tiles, and a weight's fp16 for each of them
    u, s = 2.0 ** -11, 2.0 ** -24
    d = SCALE * q[:, 0].double().cpu().norm(dim=-1, keepdim=True) * K.norm(dim=-1)[None] * (2 * u + 128 * s) + torch.where(seen, x, 0).abs() * 2.0 ** -22
    top = torch.where(seen, d, 0).amax(-1, keepdim=True)
    bound = (p * V.norm(dim=-1)[None] * (2 * d + 2 * top + 2 * u + 2 * (2 ** 15) * s)).sum(-1) + 2.0 ** -8 * want.norm(dim=-1)
    assert torch.isfinite(out).all()
    assert ((out[:, 0].double().cpu() - want).norm(dim=-1) <= bound).all()


@pytest.mark.parametrize("backbone,n", [("grid256", 1), ("grid256", 6), ("rtn4", 5), ("grid256", 40)])
def test_pages_beyond_2_32_bytes(backbone, n):
    """The same rows at the start of a pool and beyond 2^32 bytes of codes: the same bits from all calls."""
    from paper_2501_19392_amd import binding as B
    from tests import tree_utils as T
    H, QH, page, m = 8, 32, 256, 40                          # m pages of two sequences
    n_pages = (1 << 32) // (H * 64) // page + m + 8
    lo, lg, pages = P.make(H, "bf16", backbone, n_pages, page)
    assert pages.k_codes.numel() > 1 << 32
    gen = torch.Generator().manual_seed(n)
    few = B.Pages(lg, m, page)
    P.fill(lo, few, gen)
    near, far = torch.arange(m, dtype=torch.int32).view(2, m // 2), n_pages - 1 - torch.arange(m, dtype=torch.int32).view(2, m // 2)
    lens = torch.tensor([m // 2 * page - 3, 1111], dtype=torch.int32).cuda()
    q = torch.randn(2 * n, QH, 128, generator=gen).bfloat16().cuda()
    tree = torch.cat([T.words_of(T.random_tree(n, gen), 2) for _ in range(2)]).cuda()
    first_mass = torch.rand(m, H, page, generator=gen).cuda()
    results = []
    for table in (near, far):
        at = table.flatten().long()
        rows = (at[:, None] * page + torch.arange(page)).flatten().cuda()
        for k in ("k_codes", "k_scales", "v_codes", "v_scales"):
            getattr(pages, k)[rows] = getattr(few, k)
        mass = torch.zeros(n_pages, H, page, device="cuda")
        mass[at.cuda()] = first_mass
        table = table.cuda()
        ws = torch.empty(B.aquakv_paged_workspace_bytes(lg, pages, 2, QH, m // 2, 2 * n, n), dtype=torch.uint8, device="cuda")
        out = torch.empty_like(q)
        B.aquakv_paged_attend_tree(lg, pages, 2, QH, table, lens, q, n, None, tree, SCALE, out, ws)
        ws = torch.empty(B.aquakv_paged_weights_workspace_bytes(lg, pages, 2, QH, m // 2, 2 * n, n), dtype=torch.uint8, device="cuda")
        B.aquakv_paged_weights(lg, pages, 2, QH, table, lens, q, n, None, SCALE, 0.5, mass, ws)
        found = [out.clone(), mass[at.cuda()]]
        kept, n_kept = torch.zeros(2, 700, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
        ws = torch.empty(B.aquakv_paged_select_workspace_bytes(lg, pages, 2, m // 2, 700) + 256, dtype=torch.uint8, device="cuda")
        B.aquakv_paged_select(lg, pages, 2, table, lens, mass, 700, 3, 9, kept, n_kept, ws)
        ws = torch.empty(B.aquakv_paged_keep_workspace_bytes(lg, pages, 2, 700, True) + 256, dtype=torch.uint8, device="cuda")
        B.aquakv_paged_keep(lg, pages, 2, table, kept, n_kept, None, None, mass, ws)
        found += [kept, n_kept, mass[at.cuda()]] + [getattr(pages, k)[rows] for k in ("k_codes", "k_scales", "v_codes", "v_scales")]
        results.append([x.cpu() for x in found])
    for i, (a, b) in enumerate(zip(*results)):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), i
    assert torch.isfinite(results[0][0]).all()


@pytest.mark.parametrize("room,length,batch", [(PAGE, 100, 1), (130 * PAGE, 17, 2), (PAGES * PAGE, PAGES * PAGE - 5, 1)])
def test_a_budget_of_almost_2_31_tokens(room, length, batch):
    """The list's end is reached and not passed: by one workgroup, by all slabs', and where almost as many tokens are kept."""
    from paper_2501_19392_amd import binding as B
    budget, beside = (1 << 31) - 1, 1 << 16
    print(f"case budget room={room} length={length} batch={batch}", flush=True)
    lo, lg, pages, table, gen = make(5)
    table = table[:, :room // PAGE].repeat(batch, 1).contiguous()
    mass = torch.rand(4, 1, PAGE, generator=gen).cuda()
    lens = torch.full((batch,), length, dtype=torch.int32, device="cuda")
    ws = torch.empty(B.aquakv_paged_select_workspace_bytes(lg, pages, batch, room // PAGE, budget), dtype=torch.uint8, device="cuda")
    wide, n = torch.full((beside + batch * budget + beside,), 7, dtype=torch.int32, device="cuda"), torch.zeros(batch, dtype=torch.int32, device="cuda")
    kept = wide[beside:beside + batch * budget].view(batch, budget)
    B.aquakv_paged_select(lg, pages, batch, table, lens, mass, budget, 3, 4, kept, n, ws)
    torch.cuda.synchronize()
    assert n.tolist() == [length] * batch
    part = 1 << 28
    for row in kept:
        for i in range(0, budget, part):
            want = torch.arange(i, min(i + part, budget), device="cuda", dtype=torch.int32)
            want[max(length - i, 0):] = -1
            assert torch.equal(row[i:i + part], want), i
    assert (wide[:beside] == 7).all() and (wide[beside + batch * budget:] == 7).all()
