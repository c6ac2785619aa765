"""The cache in pages of codes: aquakv_paged_append against the oracle's quantizer (and, without rotation, the bits of aquakv_quantize),
aquakv_paged_attend against plain attention in 64 bits over the rows that the oracle reads from the same codes."""
import numpy as np
import pytest
import torch

from tests import paged_utils as P
from tests import parity_utils as U

pytestmark = pytest.mark.gpu
SCALE = 128 ** -0.5


def need_gpu():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible: the gpu-marked tests must run on an MI355X")


def angles(rows, seed=3):
    gen = torch.Generator().manual_seed(seed)
    a = torch.rand(rows, 64, generator=gen, dtype=torch.float64) * 6.28
    return a.cos().float().cuda(), a.sin().float().cuda()


def bits_of(t):
    return t.view(torch.int16 if t.element_size() == 2 else torch.int32 if t.element_size() == 4 else torch.uint8)


# ------------------------------------------------------------------------------------------------ append
@pytest.mark.parametrize("dtype,fmt,H,tokens,page,rope,apart,hats", [
    ("bf16", "grid256", 8, 1, 16, True, True, False), ("bf16", "grid256", 8, 333, 64, True, True, True),
    ("bf16", "grid64", 3, 77, 24, True, False, True), ("bf16", "grid16", 1, 1030, 8, False, True, True),
    ("bf16", "rtn4", 8, 130, 32, True, True, True), ("bf16", "rtn2", 5, 61, 16, False, False, False),
    ("fp32", "grid256", 2, 45, 16, True, True, True), ("fp32", "grid16", 7, 19, 40, False, True, True),
    ("fp32", "rtn4", 1, 257, 128, True, False, True), ("bf16", "grid256", 8, 5000, 128, True, True, True)])
def test_rows_go_to_their_slots(dtype, fmt, H, tokens, page, rope, apart, hats):
    need_gpu()
    from paper_2501_19392_amd import binding as B
    print(f"case append {dtype} {fmt} H={H} tokens={tokens} page={page} rope={rope}", flush=True)
    n_pages = -(-tokens // page) + 2
    lo, lg, pages = P.make(H, dtype, fmt, n_pages, page)
    D, sd, gen = H * 128, P.storage(dtype), torch.Generator().manual_seed(tokens)
    joint = torch.randn(tokens, (3 if apart else 2) * D, generator=gen) * torch.randn(3 * D if apart else 2 * D, generator=gen).exp()
    joint = joint.to(sd).cuda()
    K, V = (joint[:, -2 * D + i * D:joint.shape[1] - D + i * D].view(tokens, H, 128) for i in (0, 1))
    if not apart:
        K, V = K.contiguous(), V.contiguous()
    rows = n_pages * page
    slots = torch.randperm(rows, generator=gen)[:tokens]
    positions = torch.randint(0, 500, (tokens,), generator=gen).to(torch.int32)
    out = torch.zeros(tokens, dtype=torch.bool)                            # tokens that are left out
    for i, bad in enumerate((-1, rows, 1 << 40, -(1 << 62))):
        if tokens > 10:
            slots[2 * i + 1] = bad
            out[2 * i + 1] = True
    if rope and tokens > 10:
        positions[0], positions[10] = -1, 500
        out[0] = out[10] = True
    cos, sin = angles(500) if rope else (None, None)
    for t in (pages.k_codes, pages.v_codes, pages.k_scales, pages.v_scales):
        t.view(torch.uint8).fill_(0xA5)
    Kh, Vh = (torch.full((tokens, H, 128), 7.0, dtype=sd, device="cuda") for _ in range(2)) if hats else (None, None)
    B.aquakv_paged_append(lg, pages, tokens, K, V, slots.cuda(), positions.cuda() if rope else None, cos, sin, Kh, Vh)
    torch.cuda.synchronize()
    used = slots[~out]
    rest = torch.ones(rows, dtype=torch.bool)
    rest[used] = False
    for t in (pages.k_codes, pages.v_codes, pages.k_scales, pages.v_scales):
        assert (t.view(torch.uint8).reshape(rows, -1).cpu()[rest] == 0xA5).all()
    for which, X, codes, scales, signs, hat in (("k", K, pages.k_codes, pages.k_scales, lo.signs_k, Kh), ("v", V, pages.v_codes, pages.v_scales, lo.signs_v, Vh)):
        x = X.cpu()[~out]
        c, s = codes.cpu()[used], scales.cpu()[used]
        if which == "k" and rope:
            a = [t.cpu()[positions.long().clamp(0, 499)][~out] for t in (cos, sin)]
            x64, x32 = P.rotated(x.double(), *a), P.rotated(x.float(), *a).double()
        else:
            x64 = x32 = x.double()
            q = [torch.empty_like(t) for t in lg.alloc_codes(int(x.shape[0]))]
            B.aquakv_quantize(lg, B.AQUAKV_KEY if which == "k" else B.AQUAKV_VALUE, x.shape[0], X[(~out).cuda()].contiguous(), None, *q, None)
            torch.cuda.synchronize()
            assert torch.equal(q[0].cpu(), c) and torch.equal(q[1].cpu(), s)
        if lo.rtn_bits is not None:
            rep = U.compare_rtn_outputs(x64.reshape(len(x), -1).numpy(), c.numpy(), s.numpy(), lo.rtn_bits)
        else:
            rep = U.classify_free_run(x64.numpy(), np.zeros(x64.shape), (x64 - x32).numpy(), signs, lo.codebook, c.numpy(), s.numpy(), lo.n_codewords)
        assert rep.other == 0, f"{which}: {rep}"
        if hat is not None:
            want = P.held(lo, c, s, signs).numpy()
            got = hat.double().cpu().numpy()
            U.assert_close_storage(hat[(~out).cuda()], want, dtype, which)
            assert (got[out.numpy()] == 7.0).all()


@pytest.mark.parametrize("fmt", ["grid16", "grid64", "grid256"])
@pytest.mark.parametrize("hat", ["K", "V"])
def test_without_a_search_table_the_codes_are_the_same(fmt, hat):
    need_gpu()
    from paper_2501_19392_amd import binding as B
    lo, lg, pages = P.make(3, "bf16", fmt, 9, 8)
    other = B.Layer(3, 128, lg.codebook, lg.signs_k, lg.signs_v, torch.bfloat16)
    pools = [pages, B.Pages(other, 9, 8)]
    gen = torch.Generator().manual_seed(3)
    K, V = ((torch.randn(67, 3, 128, generator=gen) * torch.randn(3, 128, generator=gen).exp()).bfloat16().cuda() for _ in range(2))
    slots, hats = torch.randperm(72, generator=gen)[:67].cuda(), []
    for layer, p in zip((lg, other), pools):
        for t in (p.k_codes, p.v_codes, p.k_scales, p.v_scales):
            t.zero_()
        hats.append(torch.empty_like(K))
        B.aquakv_paged_append(layer, p, 67, K, V, slots, None, None, None, hats[-1] if hat == "K" else None, hats[-1] if hat == "V" else None)
    torch.cuda.synchronize()
    for name in ("k_codes", "k_scales", "v_codes", "v_scales"):
        assert torch.equal(getattr(pools[0], name), getattr(pools[1], name)), name
    assert torch.equal(*hats)


def test_zero_rows_and_no_tokens():
    need_gpu()
    from paper_2501_19392_amd import binding as B
    for fmt in P.FORMATS:
        lo, lg, pages = P.make(2, "bf16", fmt, 2, 8)
        Z = torch.zeros(3, 2, 128, dtype=torch.bfloat16, device="cuda")
        Kh, Vh = torch.ones_like(Z), torch.ones_like(Z)
        B.aquakv_paged_append(lg, pages, 3, Z, Z, torch.tensor([3, 15, 0], device="cuda"), None, None, None, Kh, Vh)
        torch.cuda.synchronize()
        assert (Kh == 0).all() and (Vh == 0).all()


# ------------------------------------------------------------------------------------------------ attend
def build(dtype, fmt, H, QH, lengths, page, queries, seed=0, spread=0.5, ragged=None, gap=False):
    """A filled cache and queries; pages in any order, three more than are used."""
    gen = torch.Generator().manual_seed(1000 * seed + 7 * len(lengths) + max(lengths))
    need = [-(-max(n, 0) // page) for n in lengths]
    n_pages = sum(need) + 3
    lo, lg, pages = P.make(H, dtype, fmt, n_pages, page)
    P.fill(lo, pages, gen, spread)
    table = torch.full((len(lengths), max(max(need), 1)), -1, dtype=torch.int32)
    order, at = torch.randperm(n_pages, generator=gen).to(torch.int32), 0
    for b, m in enumerate(need):
        table[b, :m] = order[at:at + m]
        at += m
    # what lies behind the last token must not matter: NaN scales (and any zero points)
    for b, n in enumerate(lengths):
        if n % page and n > 0:
            rows = int(table[b, need[b] - 1]) * page + torch.arange(n % page, page)
            for t in (pages.k_scales, pages.v_scales):
                t[rows.cuda()] = 0x7e01 if lo.rtn_bits is None else torch.tensor([0x7e01, -1], dtype=torch.int16, device="cuda")
    counts = [queries] * len(lengths) if ragged is None else list(ragged)
    q = (1.5 * torch.randn(sum(counts), QH, 128, generator=gen)).to(P.storage(dtype)).cuda()
    return lo, lg, pages, table, torch.tensor(lengths, dtype=torch.int32), q, counts


def attend(lg, pages, table, lens, q, counts, scale=SCALE, q_start=None, max_queries=None, out=None):
    from paper_2501_19392_amd import binding as B
    batch, QH = len(counts), q.shape[1]
    most = max(counts) if max_queries is None else max_queries
    out = torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda") if out is None else out
    size = B.aquakv_paged_workspace_bytes(lg, pages, batch, QH, table.shape[1], q.shape[0], most)
    assert size > 0
    ws = torch.full((size + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    B.aquakv_paged_attend(lg, pages, batch, QH, table.cuda(), lens.cuda(), q, most, q_start, scale, out, ws[:size])
    torch.cuda.synchronize()
    assert (ws[size:] == 0xFF).all()
    return out


@pytest.mark.parametrize("fmt", list(P.FORMATS))
@pytest.mark.parametrize("dtype,H,QH,lengths,page,queries", [
    ("bf16", 8, 32, [1], 16, 1), ("bf16", 2, 8, [31, 32, 33, 64, 65, 127], 8, 1), ("bf16", 1, 1, [700], 64, 1),
    ("bf16", 8, 64, [300, 1500, 5], 24, 1), ("bf16", 3, 15, [200, 90], 40, 1), ("bf16", 4, 16, [100, 17, 258], 16, 4),
    ("bf16", 2, 6, [130, 67], 8, 7), ("bf16", 1, 8, [530], 128, 40), ("bf16", 2, 8, [513, 300], 32, 97),
    ("bf16", 1, 24, [60, 90], 16, 2), ("bf16", 2, 8, [1300, 25, 411], 8, 25), ("bf16", 8, 32, [640], 64, 80), ("bf16", 1, 4, [260], 24, 260), ("fp32", 2, 8, [1, 33, 150, 700], 16, 1), ("fp32", 3, 9, [260], 24, 5), ("fp32", 1, 4, [300], 32, 70)])
def test_attention_over_pages(fmt, dtype, H, QH, lengths, page, queries):
    need_gpu()
    print(f"case attend {fmt} {dtype} H={H} QH={QH} lengths={lengths} page={page} queries={queries}", flush=True)
    lo, lg, pages, table, lens, q, counts = build(dtype, fmt, H, QH, lengths, page, queries)
    out = attend(lg, pages, table, lens, q, counts)
    want, bound = P.reference(lo, pages, table, lens, q, counts, SCALE, dtype)
    print(f"  worst {P.check(out, want, bound, fmt):.3g} of the bound", flush=True)


@pytest.mark.parametrize("queries", [1, 3, 40])
@pytest.mark.parametrize("dtype,fmt", [("bf16", "grid256"), ("bf16", "rtn4"), ("bf16", "grid16"), ("fp32", "grid256")])
def test_rows_without_tokens_and_pages_outside_the_pool(dtype, fmt, queries):
    """Empty and too short sequences (queries that see nothing: 0), lengths over the table's room or below zero, pages that are not
    there in the middle and at the end."""
    need_gpu()
    page, lengths = 8, [0, 2, 100, 40, 64]
    lo, lg, pages, table, lens, q, counts = build(dtype, fmt, 2, 8, lengths, page, queries)
    table[2, 3], table[2, 12] = -1, pages.n_pages
    table[3, :] = torch.tensor([1 << 30] * table.shape[1])                 # nothing of this sequence is there
    lens = torch.tensor([0, 2, 100, 40, 10 ** 9], dtype=torch.int32)       # ... the last: as much as the table has room for
    table[4, 8:] = -1
    out = attend(lg, pages, table, lens, q, counts)
    want, bound = P.reference(lo, pages, table, lens, q, counts, SCALE, dtype)
    P.check(out, want, bound, fmt)
    n = queries
    assert (out[:n] == 0).all() and (out[n:n + max(n - 2, 0)] == 0).all() and (out[3 * n:4 * n] == 0).all()
    lens[1] = -5
    out = attend(lg, pages, table, lens, q, counts)
    assert (out[:2 * n] == 0).all()


@pytest.mark.parametrize("dtype,fmt,ragged,most", [("bf16", "grid256", [1, 0, 5, 2], 5), ("bf16", "rtn4", [40, 3, 0, 1], 40), ("bf16", "grid256", [15, 1, 14, 0], 15),
                                                    ("bf16", "grid64", [0, 70, 9, 1], 70), ("fp32", "grid16", [3, 0, 33, 1], 33)])
def test_ragged_queries_leave_other_rows_alone(dtype, fmt, ragged, most):
    need_gpu()
    lengths = [90, 33, 120, 77]
    lo, lg, pages, table, lens, q, counts = build(dtype, fmt, 2, 10, lengths, 16, 0, ragged=ragged)
    want, bound = P.reference(lo, pages, table, lens, q, counts, SCALE, dtype)
    joint = torch.zeros(len(q) + 6, 14, 128, dtype=q.dtype, device="cuda")  # rows apart, three before and after the sequences'
    joint[3:-3, 4:] = q
    start = torch.tensor([3, *(3 + np.cumsum(ragged))], dtype=torch.int32, device="cuda")
    out = torch.full((len(q) + 6, 10, 128), 5.0, dtype=q.dtype, device="cuda")
    attend(lg, pages, table, lens, joint[:, 4:], counts, q_start=start, max_queries=most, out=out)
    P.check(out[3:-3], want, bound, fmt)
    assert (out[:3] == 5).all() and (out[-3:] == 5).all()
    # fewer than a sequence has: the others are left as they were
    fewer = max(most // 2, 1)
    out.fill_(5.0)
    attend(lg, pages, table, lens, joint[:, 4:], counts, q_start=start, max_queries=fewer, out=out)
    at = 3
    for n in ragged:
        P.check(out[at:at + min(n, fewer)], want[at - 3:at - 3 + min(n, fewer)], bound[at - 3:at - 3 + min(n, fewer)], fmt)
        assert (out[at + min(n, fewer):at + n] == 5).all()
        at += n
    # row numbers outside q are cut off
    wild = start.clone()
    wild[0], wild[-1] = -4, 10 ** 9
    attend(lg, pages, table, lens, joint[:, 4:], counts, q_start=wild, max_queries=1, out=out)


@pytest.mark.parametrize("dtype,fmt,queries", [("bf16", "grid256", 2), ("bf16", "rtn4", 2), ("bf16", "rtn2", 2), ("fp32", "grid256", 2), ("fp32", "rtn4", 2),
                                               ("bf16", "grid256", 5), ("bf16", "rtn4", 5), ("bf16", "grid256", 40), ("bf16", "rtn4", 40)])
@pytest.mark.parametrize("kind", ["sink", "rising", "huge", "tiny", "zero", "outlier", "negative", "flat"])
def test_scores_and_scales_of_any_size(dtype, fmt, queries, kind):
    """One token that outweighs all others, a maximum that grows to the end, scales at both ends of fp16, zero rows, one value row a
    thousand times the others', a score scale that is negative, or 0."""
    need_gpu()
    lo, lg, pages, table, lens, q, counts = build(dtype, fmt, 1, 4, [600], 16, queries)
    rows = P.sequence_rows(pages, table[0], 600)
    ks, vs = (t[..., 0] if lo.rtn_bits is not None else t for t in (pages.k_scales, pages.v_scales))
    set_to = lambda t, r, x: t.__setitem__(r.cuda(), torch.as_tensor(x).half().view(torch.int16).cuda().view(-1, *[1] * (t.dim() - 1)))
    scale = SCALE
    if kind == "sink":
        set_to(ks, rows[5:6], [6.0]); set_to(ks, rows[6:], [0.1] * 594); scale = 0.5
    elif kind == "rising":
        set_to(ks, rows, torch.linspace(0.0, 8.0, 600)); scale = 0.3
    elif kind == "huge":
        set_to(vs, rows, [60000.0 if lo.rtn_bits is None else 4000.0] * 600)
    elif kind == "tiny":
        set_to(vs, rows, [6e-8] * 600); set_to(ks, rows, [6e-8] * 600)
    elif kind == "zero":
        set_to(ks, rows[::2], [0.0] * 300); set_to(vs, rows[::3], [0.0] * 200); set_to(vs, rows[:64], [0.0] * 64)
    elif kind == "outlier":
        set_to(vs, rows[300:301], [1000.0]); set_to(vs, rows[:64], [1e-6] * 64)
    else:
        scale = -SCALE if kind == "negative" else 0.0
    out = attend(lg, pages, table, lens, q, counts, scale)
    want, bound = P.reference(lo, pages, table, lens, q, counts, scale, dtype)
    print(f"  {fmt} {kind}: worst {P.check(out, want, bound, kind):.3g} of the bound", flush=True)


@pytest.mark.parametrize("H,queries", [(2, 3), (1, 3), (1, 40)])
def test_queries_of_any_size_and_not_finite_ones_stay_among_themselves(H, queries):
    """A query's size is no matter of the others': rows of 1e30, 1e-30 and zeros, and a row that is not finite gives such a row and no other."""
    need_gpu()
    for fmt in ("grid256", "rtn4"):
        lo, lg, pages, table, lens, q, counts = build("bf16", fmt, H, 4, [300], 16, queries)
        q[0, 0] = 0
        q[1, 1] *= 1e-30
        want, bound = P.reference(lo, pages, table, lens, q, counts, SCALE, "bf16")
        q[2, 3, 17] = float("inf")
        q[2, 2, 5] = float("nan")
        out = attend(lg, pages, table, lens, q, counts)
        assert not torch.isfinite(out[2, 2].float()).any() and not torch.isfinite(out[2, 3].float()).all()
        out[2, 2:] = want[2, 2:].to(out)
        P.check(out, want, bound, fmt)
        q[:, :] = 0
        q[0, 0], q[1, 1] = 1e30, -1e30                                     # scores of 1e30: the largest takes all
        out = attend(lg, pages, table, lens, q, counts)
        want, _ = P.reference(lo, pages, table, lens, q, counts, SCALE, "bf16")
        P.check(out, want, 2.0 ** -8 * want.norm(dim=-1) + 2.0 ** -10 * want.norm(dim=-1) + 1e-6, fmt)


@pytest.mark.parametrize("fmt", ["grid256", "rtn4"])
@pytest.mark.parametrize("rows", [8, 9, 16, 17, 32, 33, 64, 65, 128, 129, 256, 257])
def test_rows_of_a_kv_head(fmt, rows):
    """As many rows as waves and workgroups hold, and one more; sequences that are cut into several pieces, end with them, have one, or none."""
    need_gpu()
    lo, lg, pages, table, lens, q, counts = build("bf16", fmt, 2, 2, [650, 64, 1, 0, 33, 2048], 64, rows)
    P.check(attend(lg, pages, table, lens, q, counts), *P.reference(lo, pages, table, lens, q, counts, SCALE, "bf16"), f"{fmt} {rows}")


@pytest.mark.parametrize("dtype,fmt,batch,QH,ragged", [("bf16", "grid256", 64, 4, False), ("bf16", "grid256", 65, 4, True), ("bf16", "rtn4", 130, 24, True),
                                                       ("bf16", "grid16", 130, 24, False), ("fp32", "grid64", 70, 2, True), ("bf16", "rtn2", 70, 280, False)])
def test_many_sequences_that_share_pages(dtype, fmt, batch, QH, ragged):
    """More sequences than a wave has lanes, of any lengths, some without tokens or queries; all of them begin with the first one's pages."""
    need_gpu()
    gen = torch.Generator().manual_seed(batch + QH)
    lengths = (torch.rand(batch, generator=gen) ** 3 * 300).long().tolist()
    lengths[0], lengths[5], lengths[-1] = 333, 0, 1
    most = 2 if ragged else 1
    counts = torch.randint(0, most + 1, (batch,), generator=gen).tolist() if ragged else [1] * batch
    lo, lg, pages, table, lens, q, counts = build(dtype, fmt, 2, QH, lengths, 32, 1, 3, ragged=counts)
    for b in range(1, batch):
        if lengths[b] >= 64:
            table[b, :2] = table[0, :2]
    start = torch.tensor([0, *np.cumsum(counts)], dtype=torch.int32, device="cuda") if ragged else None
    out = attend(lg, pages, table, lens, q, counts, q_start=start, max_queries=most)
    P.check(out, *P.reference(lo, pages, table, lens, q, counts, SCALE, dtype), f"{fmt} {batch}")


@pytest.mark.parametrize("dtype,fmt,batch,H,QH", [("bf16", "grid64", 130, 8, 8), ("fp32", "rtn4", 70, 8, 24), ("bf16", "rtn2", 100, 16, 16), ("fp32", "grid16", 70, 8, 8)])
def test_many_rows_of_few_pieces(dtype, fmt, batch, H, QH):
    need_gpu()
    gen = torch.Generator().manual_seed(batch)
    lengths = (torch.rand(batch, generator=gen) ** 4 * 700).long().tolist()
    lengths[3], lengths[7], lengths[8] = 700, 0, 31
    lo, lg, pages, table, lens, q, counts = build(dtype, fmt, H, QH, lengths, 64, 1, 4)
    P.check(attend(lg, pages, table, lens, q, counts), *P.reference(lo, pages, table, lens, q, counts, SCALE, dtype), fmt)


@pytest.mark.parametrize("fmt,lengths,queries", [("grid256", [5000], 150), ("rtn4", [20000], 140), ("grid16", [1100, 200, 0], 300)])
def test_many_queries_over_tokens_in_pieces(fmt, lengths, queries):
    need_gpu()
    lo, lg, pages, table, lens, q, counts = build("bf16", fmt, 1, 1, lengths, 128, queries)
    P.check(attend(lg, pages, table, lens, q, counts), *P.reference(lo, pages, table, lens, q, counts, SCALE, "bf16"), fmt)


@pytest.mark.parametrize("fmt,QH", [("grid256", 1), ("rtn4", 3), ("grid64", 10)])
def test_a_long_sequence(fmt, QH):
    need_gpu()
    lo, lg, pages, table, lens, q, counts = build("bf16", fmt, 1, QH, [70001, 3], 256, 1)
    P.check(attend(lg, pages, table, lens, q, counts), *P.reference(lo, pages, table, lens, q, counts, SCALE, "bf16"), fmt)


@pytest.mark.parametrize("fmt", ["grid256", "grid64", "grid16", "rtn4", "rtn2"])
def test_scores_of_fp32_layers(fmt):
    """4096 rows over two tokens, of which the second has a score of 0 and no value, so that a row gives sigmoid(score) v: what a score is off by shows.

    Off by at most A (3 * 2^-22 + 44 * 2^-24), A = scale * sum |q_i| |k_i| (uniform: |q_i| step (code + zero)) over the products as they are taken: query and grid
    point are two fp16 numbers each (2^-22 of either), the product of the two second ones is left out (2^-22), and 12 instructions add 32 products each
    (44 roundings on a product's way).  Behind it, relative to the result: the exponent's argument, 2^-22 |score|, and all else, 2^-20."""
    need_gpu()
    lo, lg, pages, table, lens, q, counts = build("fp32", fmt, 1, 64, [2], 8, 1)
    rtn = lo.rtn_bits is not None
    first = int(table[0, 0]) * 8
    for t in (pages.k_scales, pages.v_scales):
        (t[..., 0] if rtn else t)[first + 1] = 0
    gen = torch.Generator().manual_seed(21)
    batch = 64
    q = (1.5 * torch.randn(batch, 64, 128, generator=gen)).cuda()
    out = attend(lg, pages, table.repeat(batch, 1), lens.repeat(batch), q, [1] * batch).double().cpu()
    k, v = (P.held(lo, c[first:first + 1], s[first:first + 1], sg)[0, 0] for c, s, sg in
            ((pages.k_codes, pages.k_scales, lo.signs_k), (pages.v_codes, pages.v_scales, lo.signs_v)))
    x = q.double().cpu()
    score = SCALE * (x @ k)
    if rtn:
        step, zero = (pages.k_scales[first, :, i].cpu() for i in (0, 1))
        offset = (step.view(torch.float16).double() * zero.double()).repeat_interleave(64)
        A = SCALE * (x.abs() @ (k.abs() + 2 * offset))
    else:
        d = torch.arange(128)
        odd = sum((d[:, None] & d) >> i & 1 for i in range(7)) % 2
        rot = (1.0 - 2.0 * odd.double()) / 128 ** 0.5 * torch.as_tensor(lo.signs_k).double().view(1, 128)
        A = SCALE * ((x @ rot.T).abs() @ (rot @ k).abs())
    p = torch.sigmoid(score)
    off = (out - p[..., None] * v).norm(dim=-1) / (p * v.norm())
    bound = (1 - p) * A * (3 * 2.0 ** -22 + 44 * 2.0 ** -24) + score.abs() * 2.0 ** -22 + 2.0 ** -20
    print(f"  {fmt}: worst {(off / bound).max().item():.3g} of the bound, {off.max().item():.3g}", flush=True)
    assert (off <= bound).all()


@pytest.mark.parametrize("fmt", ["grid256", "grid16", "rtn4", "rtn2"])
def test_fp32_layers_beside_plain_fp32(fmt):
    """Errors like those of the same attention in plain fp32: what is rounded to 22 bits instead of 24 is off by four times as much, three such factors (query,
    key, weight and value) by 4 sqrt(3) < 8, in the root mean square over 512 rows of 700 tokens."""
    need_gpu()
    lo, lg, pages, table, lens, q, counts = build("fp32", fmt, 1, 64, [700] * 8, 32, 1, spread=0.3)
    out = attend(lg, pages, table, lens, q, counts).double().cpu()
    want, _ = P.reference(lo, pages, table, lens, q, counts, SCALE, "fp32")
    K, V = (P.held(lo, c, s, sg)[:, 0].float() for c, s, sg in ((pages.k_codes, pages.k_scales, lo.signs_k), (pages.v_codes, pages.v_scales, lo.signs_v)))
    plain = torch.empty_like(want)
    for b in range(8):
        rows = P.sequence_rows(pages, table[b], 700)
        plain[b] = (torch.softmax((q[b].cpu() @ K[rows].T) * SCALE, -1) @ V[rows]).double()
    rms = [((x - want).norm(dim=-1) / want.norm(dim=-1)).square().mean().sqrt().item() for x in (out, plain)]
    print(f"  {fmt}: {rms[0]:.3g}, plain {rms[1]:.3g}", flush=True)
    assert rms[0] <= 8 * rms[1]


def test_tensors_that_are_not_on_the_device():
    need_gpu()
    from paper_2501_19392_amd import binding as B
    lo, lg, pages, table, lens, q, counts = build("bf16", "grid256", 2, 4, [50, 20], 16, 1)
    ws = torch.empty(B.aquakv_paged_workspace_bytes(lg, pages, 2, 4, table.shape[1], 2, 1), dtype=torch.uint8, device="cuda")
    good = dict(page_table=table.cuda(), seq_lens=lens.cuda(), q=q, q_start=None, out=torch.empty_like(q), workspace=ws)
    for name, at in dict(page_table=table, seq_lens=lens, q=q.cpu(), q_start=torch.tensor([0, 1, 2], dtype=torch.int32), out=q.cpu(), workspace=ws.cpu()).items():
        k = {**good, name: at}
        with pytest.raises(ValueError, match="device"):
            B.aquakv_paged_attend(lg, pages, 2, 4, k["page_table"], k["seq_lens"], k["q"], 1, k["q_start"], SCALE, k["out"], k["workspace"])
    K = torch.zeros(2, 2, 128, dtype=torch.bfloat16, device="cuda")
    cos, sin = angles(9)
    good = dict(K=K, V=K, slots=torch.tensor([1, 2], device="cuda"), positions=torch.zeros(2, dtype=torch.int32, device="cuda"), cos=cos, sin=sin, Khat=None)
    for name, t in dict(K=K.cpu(), V=K.cpu(), slots=torch.tensor([1, 2]), positions=torch.zeros(2, dtype=torch.int32), cos=cos.cpu(), sin=sin.cpu(), Khat=K.cpu()).items():
        k = {**good, name: t}
        with pytest.raises(ValueError, match="device"):
            B.aquakv_paged_append(lg, pages, 2, k["K"], k["V"], k["slots"], k["positions"], k["cos"], k["sin"], k["Khat"], None)
    with pytest.raises(ValueError, match="device"):
        B.Pages(lg, pages.n_pages, 16, k_codes=pages.k_codes, k_scales=pages.k_scales, v_codes=pages.v_codes.cpu(), v_scales=pages.v_scales)


def test_a_pool_beyond_32_bits():
    """Rows whose bytes start behind 4 GiB."""
    need_gpu()
    from paper_2501_19392_amd import binding as B
    n_pages, page, H = 70000, 128, 8                                       # 8.96 M rows of 512 bytes
    lo, lg, pages = P.make(H, "bf16", "grid256", n_pages, page)
    gen = torch.Generator().manual_seed(4)
    far = [69999, 65536, 0, 32768]
    T = 4 * page - 3
    K, V = (torch.randn(T, H, 128, generator=gen).bfloat16().cuda() for _ in range(2))
    t = torch.arange(T)
    slots = torch.tensor(far)[t // page] * page + t % page
    Kh, Vh = torch.empty_like(K), torch.empty_like(V)
    B.aquakv_paged_append(lg, pages, T, K, V, slots.cuda(), None, None, None, Kh, Vh)
    table, lens = torch.tensor([far], dtype=torch.int32), torch.tensor([T], dtype=torch.int32)
    rows = slots.cuda()
    k, v = (P.held(lo, c[rows], s[rows], sg) for c, s, sg in ((pages.k_codes, pages.k_scales, lo.signs_k), (pages.v_codes, pages.v_scales, lo.signs_v)))
    for n in (1, 8, 80):                                                   # 2, 16 and 160 rows of a kv head
        q = (1.5 * torch.randn(n, 16, 128, generator=gen)).bfloat16().cuda()
        out = attend(lg, pages, table, lens, q, [n])
        seen = torch.arange(T)[None] <= T - n + torch.arange(n)[:, None]
        for h in range(16):
            want, bound = P.attention(q[:, h].double().cpu(), k[:, h // 2], v[:, h // 2], SCALE, seen, "bf16")
            P.check(out[:, h], want, bound, f"{n} queries, head {h}")
    U.assert_close_storage(Kh, k.numpy(), "bf16", "keys")


# ------------------------------------------------------------------------------------------------ together
@pytest.mark.parametrize("dtype,fmt,H,QH", [("bf16", "grid256", 2, 8), ("bf16", "rtn4", 2, 4), ("bf16", "grid64", 1, 8), ("fp32", "grid256", 1, 2)])
def test_a_prompt_and_generated_tokens(dtype, fmt, H, QH):
    """As a program uses them: prompts of two sequences in chunks (appended, then attended to), then tokens one by one for both, pages handed out
    as they are needed; every attention against plain attention over the oracle's reading of everything appended so far."""
    need_gpu()
    from paper_2501_19392_amd import binding as B
    page, n_pages = 16, 40
    lo, lg, pages = P.make(H, dtype, fmt, n_pages, page)
    gen = torch.Generator().manual_seed(11)
    sd, cos_sin = P.storage(dtype), angles(400)
    free = torch.randperm(n_pages, generator=gen).tolist()
    table, lens = torch.full((2, 20), -1, dtype=torch.int32), [0, 0]
    steps = [(70, 33), (45, 1)] + [(1, 1)] * 20 + [(3, 5)]
    for counts in steps:
        slots, positions = [], []
        for b, n in enumerate(counts):
            for t in range(lens[b], lens[b] + n):
                if t % page == 0:
                    table[b, t // page] = free.pop()
                slots.append(int(table[b, t // page]) * page + t % page)
                positions.append(t)
            lens[b] += n
        T = sum(counts)
        qkv = torch.randn(T, QH + 2 * H, 128, generator=gen).to(sd).cuda()
        B.aquakv_paged_append(lg, pages, T, qkv[:, QH:QH + H], qkv[:, QH + H:], torch.tensor(slots).cuda(),
                              torch.tensor(positions, dtype=torch.int32).cuda(), *cos_sin, None, None)
        start = torch.tensor([0, counts[0], T], dtype=torch.int32).cuda()
        q = qkv[:, :QH]
        out = torch.full((T, QH, 128), float("nan"), dtype=sd, device="cuda")
        attend(lg, pages, table, torch.tensor(lens, dtype=torch.int32), q, list(counts), q_start=start, out=out)
        want, bound = P.reference(lo, pages, table, lens, q, counts, SCALE, dtype)
        P.check(out, want, bound, f"lengths {lens}")


@pytest.mark.parametrize("dtype,fmt,queries", [("bf16", "grid256", 1), ("bf16", "rtn4", 3), ("bf16", "grid256", 50), ("fp32", "grid16", 1)])
def test_replays_of_a_captured_step_follow_the_counts(dtype, fmt, queries):
    """Append and attend captured once; every replay sees new tokens, slots, positions and lengths in the same buffers, with eager work on the
    same stream in between, and gives the bits of the eager calls."""
    need_gpu()
    from paper_2501_19392_amd import binding as B
    H, QH, page, batch, n_pages = 2, 8, 16, 3, 64
    lo, lg, pages = P.make(H, dtype, fmt, n_pages, page)
    gen = torch.Generator().manual_seed(5)
    P.fill(lo, pages, gen)
    sd, (cos, sin) = P.storage(dtype), angles(400)
    T = batch * queries
    table = torch.randperm(n_pages, generator=gen)[:60].view(batch, 20).to(torch.int32).cuda()
    bufs = dict(qkv=torch.zeros(T, QH + 2 * H, 128, dtype=sd), slots=torch.full((T,), -1, dtype=torch.int64), positions=torch.zeros(T, dtype=torch.int32),
                lens=torch.zeros(batch, dtype=torch.int32))
    bufs = {k: v.cuda() for k, v in bufs.items()}
    out = torch.zeros(T, QH, 128, dtype=sd, device="cuda")
    ws = torch.empty(B.aquakv_paged_workspace_bytes(lg, pages, batch, QH, 20, T, queries), dtype=torch.uint8, device="cuda")

    def step(pages, out, ws):
        x = bufs["qkv"]
        B.aquakv_paged_append(lg, pages, T, x[:, QH:QH + H], x[:, QH + H:], bufs["slots"], bufs["positions"], cos, sin, None, None)
        B.aquakv_paged_attend(lg, pages, batch, QH, table, bufs["lens"], x[:, :QH], queries, None, SCALE, out, ws)

    step(pages, out, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(pages, out, ws)
    copies = [t.clone() for t in (pages.k_codes, pages.k_scales, pages.v_codes, pages.v_scales)]
    other = B.Pages(lg, n_pages, page, k_codes=copies[0], k_scales=copies[1], v_codes=copies[2], v_scales=copies[3])
    for i in range(5):
        lens = [60 * i + 3, 0 if i == 1 else 100 + i, 317 - 50 * i]
        pos = torch.tensor([[max(n - queries + k, 0) for k in range(queries)] for n in lens])
        slots = torch.gather(table.cpu().long(), 1, pos // page) * page + pos % page
        for b, n in enumerate(lens):
            slots[b, :max(queries - n, 0)] = -1
        bufs["qkv"].copy_(torch.randn(T, QH + 2 * H, 128, generator=gen).to(sd))
        bufs["slots"].copy_(slots.reshape(-1)); bufs["positions"].copy_(pos.reshape(-1)); bufs["lens"].copy_(torch.tensor(lens))
        graph.replay()
        want = torch.empty_like(out)
        step(other, want, torch.empty_like(ws))
        torch.cuda.synchronize()
        assert torch.equal(bits_of(out), bits_of(want)), i
        for a, b in ((pages.k_codes, other.k_codes), (pages.k_scales, other.k_scales), (pages.v_codes, other.v_codes), (pages.v_scales, other.v_scales)):
            assert torch.equal(a, b)
        ref, bound = P.reference(lo, pages, table, lens, bufs["qkv"][:, :QH], [queries] * batch, SCALE, dtype)
        P.check(out, ref, bound, f"replay {i}")


def test_two_calls_at_once_on_two_streams():
    need_gpu()
    from paper_2501_19392_amd import binding as B
    jobs = []
    for seed in (1, 2):
        lo, lg, pages, table, lens, q, counts = build("bf16", "grid256", 8, 32, [3000, 2000 + seed], 32, 1, seed=seed)
        size = B.aquakv_paged_workspace_bytes(lg, pages, 2, 32, table.shape[1], 2, 1)
        jobs.append((lo, lg, pages, table, lens, q, torch.empty(size, dtype=torch.uint8, device="cuda"), torch.cuda.Stream(), torch.zeros_like(q),
                     table.cuda(), lens.cuda()))
    torch.cuda.synchronize()
    for _ in range(8):
        for lo, lg, pages, table, lens, q, ws, stream, out, td, ld in jobs:
            B.aquakv_paged_attend(lg, pages, 2, 32, td, ld, q, 1, None, SCALE, out, ws, stream=stream)
    torch.cuda.synchronize()
    for lo, lg, pages, table, lens, q, ws, stream, out, td, ld in jobs:
        want, bound = P.reference(lo, pages, table, lens, q, [1, 1], SCALE, "bf16")
        P.check(out, want, bound, "streams")


def test_the_same_call_gives_the_same_bits():
    need_gpu()
    lo, lg, pages, table, lens, q, counts = build("bf16", "grid256", 8, 32, [5000, 37], 16, 2)
    first = attend(lg, pages, table, lens, q, counts)
    for _ in range(4):
        assert torch.equal(bits_of(attend(lg, pages, table, lens, q, counts)), bits_of(first))
