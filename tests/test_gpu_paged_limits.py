"""Attention over pages at the limits of what its calls admit: the longest sequences, scales of very different sizes, rows that some queries do not see."""
import pytest
import torch

from tests import paged_utils as P
from tests.test_gpu_paged import SCALE, attend, need_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt,QH,queries", [("grid256", 4, 1), ("rtn4", 4, 1), ("grid16", 1, 20), ("rtn2", 1, 130)])
def test_a_sequence_of_almost_2_31_tokens(fmt, QH, queries):
    """2048 pages of 2^20 - 8 tokens, of which the first and the last are in the pool (the same page).  All scores are 0, so a row is the mean over the tokens
    it sees: twice a page, less the last ones that it does not see.  Values are not 0 in two places of the page only, the first 64 tokens and the last 1000 but for as many."""
    need_gpu()
    page, n_pages = 2 ** 20 - 8, 2048
    lo, lg, pages = P.make(1, "bf16", fmt, 1, page)
    gen = torch.Generator().manual_seed(8)
    rows = torch.cat([torch.arange(64), torch.arange(page - 2000, page - 1000)])
    for t in (pages.k_codes, pages.k_scales, pages.v_codes, pages.v_scales):
        t.zero_()
    some = P.make(1, "bf16", fmt, 8, 136)[2]
    P.fill(lo, some, gen)
    pages.v_codes[rows.cuda()], pages.v_scales[rows.cuda()] = some.v_codes[:len(rows)], some.v_scales[:len(rows)]
    table = torch.full((1, n_pages), -1, dtype=torch.int32)
    table[0, 0] = table[0, -1] = 0
    q = torch.randn(queries, QH, 128, generator=gen).bfloat16().cuda()
    print(f"case almost 2^31 tokens {fmt} queries={queries}", flush=True)
    out = attend(lg, pages, table, torch.tensor([page * n_pages], dtype=torch.int32), q, [queries])
    total = P.held(lo, pages.v_codes[rows.cuda()], pages.v_scales[rows.cuda()], lo.signs_v)[:, 0].sum(0)
    seen = 2 * page - (queries - 1 - torch.arange(queries)).double()                     # (tokens that a query does not see have no value)
    want = (2 * total[None] / seen[:, None])[:, None].expand(queries, QH, 128)
    # Weights and grid points are rounded to fp16 (2^-11 each), 2128 values are added in fp32.  A lane adds the weights of a tile, and
    # the sums of a page's tiles, 2^15 of them, one after the other in fp32, each by a rounding of at most 2^-24 of the sum: 2^-9.  At the end one rounding to bf16.
    size = 2 * P.held(lo, pages.v_codes[rows.cuda()], pages.v_scales[rows.cuda()], lo.signs_v)[:, 0].norm(dim=-1).sum() / seen
    bound = (size * (2 * 2.0 ** -11 + 2 * 2128 * 2.0 ** -24) + (2.0 ** -9 + 2.0 ** -8) * want[:, 0].norm(dim=-1))[:, None].expand(queries, QH)
    P.check(out, want, bound, fmt)
    assert (bound < 0.5 * want.norm(dim=-1)).all()                          # (a lost half of them would show)


@pytest.mark.parametrize("fmt", ["rtn4", "rtn2"])
@pytest.mark.parametrize("dtype,QH", [("bf16", 8), ("bf16", 20), ("bf16", 160), ("fp32", 8)])
def test_uniform_steps_of_a_heads_halves_far_apart(dtype, fmt, QH):
    """Each half of a head keeps its own bits, however much larger the other one's step is: keys whose halves are 2^20 apart under queries the other way round, so
    that both count, and values whose halves are 2^22 apart, looked at one by one.  16 sequences of two tokens, the second with a score of 0 and no value: a row is
    sigmoid(score) v.

    A score is off by A (u + 64 s + t), A = scale * sum |q_i| step (code + zero) over the products as they are taken: queries are rounded to u (bf16 layers: fp16,
    2^-11; fp32 layers: two fp16 numbers, 2^-22), codes and zero points are not, sums have 64 roundings of s = 2^-24 on a product's way, and the matrix
    instructions keep codes that are subnormal numbers to t = 2^-17 (bf16 layers).  Besides, fp16 ends at 2^-24: a row's query is held with its largest coordinate at
    2^13 or above, divided by up to 2^bits or 2^(3 * 2) where codes are masked in place (4, 2 bits), so that any coordinate is off by half of 2^-24 * that, which is
    2^-38 * that of the largest one: a 2^-12 of a coordinate that is 2^22 times smaller, as some here are.  (This term was added when fp32 layers had come out at 1.6
    times the bound without it.)  A weight then, relative: (1 - p) of that, 2^-22 |score| of the exponent's argument, and its rounding u (with the step in it).  Weights
    with their steps are fp16 numbers (one, or two) too, and the largest of a row is 2^8 or above, so that each is off by half of 2^-24, 2^-33 of the largest:
    relative to one of a half whose step is r times smaller, of a token that is not the likelier one, 2^-33 r max(1, e^-score).  (Added when that half of fp32
    layers had come out at 2^-11, as it says.)  The rest is below 2^-20, at the end one rounding."""
    need_gpu()
    u, t, last = (2.0 ** -11, 2.0 ** -17, 2.0 ** -8) if dtype == "bf16" else (2.0 ** -22, 0.0, 2.0 ** -24)
    batch, scale = 16, 0.02
    lo, lg, pages = P.make(1, dtype, fmt, batch, 8)
    gen = torch.Generator().manual_seed(QH)
    P.fill(lo, pages, gen, 0.3)
    first = 8 * torch.arange(batch)
    step = lambda x: torch.as_tensor(x).half().view(torch.int16).cuda()
    unit = 2.0 / (2 ** lo.rtn_bits - 1)
    for scales, halves in ((pages.k_scales, (2.0 ** 12, 2.0 ** -8)), (pages.v_scales, (2.0 ** 10, 2.0 ** -12))):
        for i, size in enumerate(halves):
            scales[first.cuda(), i, 0] = step(size * unit * (1 + torch.rand(batch, generator=gen)))
        scales[first.cuda() + 1, :, 0] = 0
    q = 1.5 * torch.randn(batch, QH, 128, generator=gen)
    q[..., :64] *= 2.0 ** -12
    q[..., 64:] *= 2.0 ** 8
    q = q.to(P.storage(dtype)).cuda()
    table, lens = torch.arange(batch, dtype=torch.int32)[:, None], torch.full((batch,), 2, dtype=torch.int32)
    out = attend(lg, pages, table, lens, q, [1] * batch, scale).double().cpu()
    k, v = (P.held(lo, c, s, None)[first, 0] for c, s in ((pages.k_codes, pages.k_scales), (pages.v_codes, pages.v_scales)))
    x = q.double().cpu()
    steps, zeros = (pages.k_scales[first.cuda(), :, i].cpu().contiguous() for i in (0, 1))
    offset = (steps.view(torch.float16).double() * zeros.double()).repeat_interleave(64, 1)
    A = scale * (x.abs() @ (k.abs() + 2 * offset)[:, :, None])[..., 0]
    end = scale * x.abs().amax(-1) * 2.0 ** -38 * (16 if lo.rtn_bits == 4 else 64) * (k.abs() + 2 * offset).sum(-1)[:, None]
    score = scale * (x @ k[:, :, None])[..., 0]
    p = torch.sigmoid(score)
    bound = (1 - p) * (A * (u + 64 * 2.0 ** -24 + t) + end) + score.abs() * 2.0 ** -22 + u + 2.0 ** -20 + last
    assert (A.mean() < 40) and (bound.mean() < 0.05)                        # (else nothing would show)
    v_steps = pages.v_scales[first.cuda(), :, 0].cpu().contiguous().view(torch.float16).double()
    for i, half in enumerate((slice(0, 64), slice(64, 128))):
        bound_half = bound + 2.0 ** -33 * (v_steps.amax(1) / v_steps[:, i])[:, None] * torch.exp(-score).clamp(min=1)
        want = p[..., None] * v[:, None, half]
        off = (out[..., half] - want).norm(dim=-1) / want.norm(dim=-1)
        print(f"  {dtype} {fmt} {QH} {half.start}: worst {(off / bound_half).max().item():.3g} of the bound, {off.max().item():.3g}; A {A.mean().item():.3g}", flush=True)
        assert (off <= bound_half).all()


@pytest.mark.parametrize("dtype,fmt,QH,queries", [("bf16", "grid256", 2, 3), ("bf16", "rtn4", 2, 3), ("bf16", "grid64", 4, 20), ("bf16", "rtn2", 4, 20),
                                                  ("bf16", "grid16", 4, 70), ("bf16", "rtn4", 4, 70), ("fp32", "grid256", 4, 20), ("fp32", "rtn2", 4, 20)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("which", ["keys", "values", "both"])
def test_what_a_query_does_not_see_is_no_matter(dtype, fmt, QH, queries, bad, which):
    """Rows that are not finite, among the last tokens: the queries before them are as if they were not there, those behind them are not finite."""
    need_gpu()
    from tests.test_gpu_paged import build
    lo, lg, pages, table, lens, q, counts = build(dtype, fmt, 1, QH, [150, 97], 16, queries)
    want, bound = P.reference(lo, pages, table, lens, q, counts, SCALE, dtype)            # (finite: what the queries before them see stays the same)
    bad_from = queries // 3
    for b in range(2):
        row = int(P.sequence_rows(pages, table[b], int(lens[b]))[int(lens[b]) - queries + bad_from])
        for name, t in (("keys", pages.k_scales), ("values", pages.v_scales)):
            if which in (name, "both"):
                (t[..., 0] if lo.rtn_bits is not None else t)[row] = int(torch.tensor(bad).half().view(torch.int16))
    out = attend(lg, pages, table, lens, q, counts)
    for b in range(2):
        own = slice(b * queries, b * queries + bad_from)
        P.check(out[own], want[own], bound[own], f"{fmt} {b}")
        if bad != bad or which != "keys":                                   # (an infinite key has a score of -inf, and so no weight, with half of all queries)
            assert (~torch.isfinite(out[b * queries + bad_from:(b + 1) * queries].double())).any(-1).all()


@pytest.mark.parametrize("batch,queries", [(256, 130), (256, 1), (200, 20)])
@pytest.mark.parametrize("step", [0.55, 0.7, 0.95])
def test_equal_weights_of_two_million_tokens(batch, queries, step):
    """Sequences of 2^21 tokens (the same page over and over) with scores of 0, so that a row is the mean of the page.  So many sequences that one workgroup, or a
    few waves, take a whole one each: a lane adds up the weights of 2^19 to 2^20 tokens, all alike.

    Codes, steps and weights with their steps are exact here (2^8), so are sums of values but for 2^-24 of them for each addition; the weights of a tile are added
    first and then to the sum: 2^16 additions, 2^-24 of it each, 2^-8 in all, where one after the other would be 2^20 of them.  One rounding to bf16, 2^-8 of a
    coordinate at most.  Values: additions of 32 products a tile, 2^16 of those or half as many, 2^-8."""
    need_gpu()
    page, pages_each = 2048, 1024
    lo, lg, pages = P.make(1, "bf16", "rtn4", 1, page)
    gen = torch.Generator().manual_seed(3)
    P.fill(lo, pages, gen)
    for t in (pages.k_scales, pages.v_scales):
        t[..., 0] = int(torch.tensor(step).half().view(torch.int16))
        t[..., 1] = 0
    q = torch.zeros(batch * queries, 1, 128, dtype=torch.bfloat16, device="cuda")
    table, lens = torch.zeros(batch, pages_each, dtype=torch.int32), torch.full((batch,), page * pages_each, dtype=torch.int32)
    print(f"case two million tokens batch={batch} queries={queries}", flush=True)
    out = attend(lg, pages, table, lens, q, [queries] * batch).double().cpu()[:, 0]
    want = P.held(lo, pages.v_codes, pages.v_scales, None)[:, 0].mean(0)
    off = ((out - want).norm(dim=-1) / want.norm()).max().item()
    print(f"  off by {off:.3g}", flush=True)
    # (a query sees up to 130 tokens less of 2^21, 2^-14 of them)
    assert off <= 3 * 2.0 ** -8 + 2.0 ** -13


@pytest.mark.parametrize("fmt,QH,counts,tree", [("grid256", 32, [33] * 32, False), ("grid256", 32, [33] * 32, True), ("grid64", 8, [1] * 5, False), ("grid64", 8, [1] * 5, True),
                                                ("rtn4", 32, [64] * 3, False), ("rtn4", 32, [64] * 3, True)])
def test_each_call_with_its_own_workspace(fmt, QH, counts, tree):
    """What its size says and no byte of what lies behind."""
    need_gpu()
    from paper_2501_19392_amd import binding as B
    from tests import tree_utils as T
    print(f"case own workspace {fmt} QH={QH} {counts[0]} of {len(counts)} tree={tree}", flush=True)
    n, batch = counts[0], len(counts)
    lengths = [n + (61 * b) % 240 for b in range(batch)]
    lo, lg, pages, table, lens, gen = T.cache("bf16", fmt, 8, lengths, 16, seed=11)
    trees = [T.random_tree(n, gen) if tree else torch.ones(n, n, dtype=torch.bool).tril() for _ in counts]
    q = (1.5 * torch.randn(n * batch, QH, 128, generator=gen)).bfloat16().cuda()
    size = B.aquakv_paged_attend_workspace_bytes(lg, pages, batch, QH, table.shape[1], n * batch, n, tree)
    if len(counts) == 32:
        assert (size == 256) != tree                       # (sequences fill the chip: whole ones, and trees of few rows in pieces)
    ws, out = torch.full((size + 4096,), 0xFF, dtype=torch.uint8, device="cuda"), torch.full_like(q, float("nan"))
    if tree:
        bits = torch.cat([T.words_of(t, -(-n // 32)) for t in trees]).cuda()
        B.aquakv_paged_attend_tree(lg, pages, batch, QH, table.cuda(), lens.cuda(), q, n, None, bits, SCALE, out, ws[:size])
    else:
        B.aquakv_paged_attend(lg, pages, batch, QH, table.cuda(), lens.cuda(), q, n, None, SCALE, out, ws[:size])
    torch.cuda.synchronize()
    assert (ws[size:] == 0xFF).all()
    P.check(out, *T.reference(lo, pages, table, lens, q, counts, trees, SCALE, "bf16"), fmt)
