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
    # Weights and grid points are rounded to fp16 (2^-11 each), 2128 values are added in fp32.  A lane adds the weights of half a page, 2^19 of them, one after
    # the other in fp32, each by a rounding of at most 2^-24 of the sum: 2^-5.  At the end one rounding to bf16.
    size = 2 * P.held(lo, pages.v_codes[rows.cuda()], pages.v_scales[rows.cuda()], lo.signs_v)[:, 0].norm(dim=-1).sum() / seen
    bound = (size * (2 * 2.0 ** -11 + 2 * 2128 * 2.0 ** -24) + (2.0 ** -5 + 2.0 ** -8) * want[:, 0].norm(dim=-1))[:, None].expand(queries, QH)
    P.check(out, want, bound, fmt)
    assert (bound < 0.5 * want.norm(dim=-1)).all()                          # (a lost half of them would show)
