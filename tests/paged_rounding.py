"""What attention over pages in bf16 layers comes to with the roundings that the library states, and no others: what a kernel's errors are measured by.

Stated: the (rotated) query, grid points and weights times scale are rounded to fp16 behind powers of two, uniform codes are exact, sums are fp32 or better, the
result is rounded to bf16.  Such errors are some 2^-9 of a row whatever its length; a token too many or too few among n is n^-1/2 of it where weights are
about equal, so that a lost tile, a shifted mask or a piece that is joined twice is far outside."""
import math

import torch

from tests import paged_utils as P

SCALE = 128 ** -0.5
# Errors are compared by their root mean square over all rows, and row by row.  2: the rounding of a number to 11 bits is off by 2^-12 to 2^-11 at most, as its first
# bits have it, and these differ by the powers of two that a kernel puts before them.  8: a row's error is the 2-norm of 128 coordinates, which keeps near its
# mean; rows differ by the few tokens that most of a row comes from, whose roundings are 0 to 2^-11, and by the weights that are smaller than a tile's largest.
OF_ALL, OF_ONE = 2.0, 8.0

# kv heads, query heads, lengths, page, queries of a sequence (or of each), score scale
SHAPES = [(1, 4, [2000], 16, 1, 1.0), (2, 16, [700, 65, 1, 0, 33, 1300], 24, 1, 1 / 16), (8, 64, [3000, 2001], 32, 1, 1 / 16), (1, 4, [2048], 16, 5, 1 / 16),
          (2, 2, [650, 64, 1, 0, 33, 2048], 64, 32, 1.0), (2, 2, [650, 64, 1, 0, 33, 2048], 64, 33, 1 / 16), (1, 4, [530], 128, 40, 1 / 16),
          (2, 8, [1300, 411], 8, 97, 1 / 16), (2, 8, [900, 300], 8, 80, 1.0), (1, 1, [2500], 128, 300, 1 / 16)]
CASES = [(fmt, *s) for s in SHAPES for fmt in P.FORMATS] + [
    ("grid256", 1, 1, [70001, 3], 256, 1, 1 / 64), ("rtn4", 1, 3, [70001, 3], 256, 1, 1 / 64), ("grid64", 1, 10, [40001, 3], 256, 1, 1 / 64),
    ("rtn4", 1, 1, [20000], 128, 140, 1 / 64), ("grid256", 1, 1, [9000], 128, 140, 1 / 16), ("rtn2", 1, 1, [9000], 128, 20, 1 / 16),
    ("grid256", 2, 8, [5000, 37], 16, 3, 1 / 16), ("grid256", 1, 8, [1500, 1200, 600, 2000], 32, [1, 0, 5, 2], 1 / 16), ("rtn4", 1, 8, [1500, 1200, 600, 2000], 32, [40, 3, 0, 1], 1 / 16),
    ("grid64", 2, 10, [400, 333, 1200, 77], 16, [0, 70, 9, 1], 1 / 16), ("grid256", 4, 4, [200 + 7 * i for i in range(70)], 64, 1, 1 / 16),
    ("rtn4", 16, 16, [700] * 9, 8, 1, 1 / 16), ("grid16", 3, 3, [300 + 5 * i for i in range(33)], 40, 7, 1 / 16)]


def name(case):
    fmt, H, QH, lengths, page, queries, scale = case
    n = lengths if len(lengths) < 7 else f"{len(lengths)} of {min(lengths)} to {max(lengths)}"
    return f"{fmt} H={H} QH={QH} lengths={n} page={page} queries={queries} scale={scale}".replace(" ", "-")


def build(case, device):
    """(oracle layer, layer, pages, table, lens, q, counts, score scale)"""
    fmt, H, QH, lengths, page, queries, scale = case
    gen = torch.Generator().manual_seed(sum(map(ord, name(case))))
    need = [-(-n // page) for n in lengths]
    lo, lg, pages = P.make(H, "bf16", fmt, sum(need) + 2, page, device) if device == "cuda" else make_on_cpu(H, fmt, sum(need) + 2, page)
    P.fill(lo, pages, gen)
    if lo.rtn_bits is None:                                                # (with any codes the mean of the grid's points would outweigh what a few tokens add)
        for t in (pages.k_codes, pages.v_codes):
            t.copy_(gaussian_codes(lo, t.shape, gen))
    table, at = torch.full((len(lengths), max(need)), -1, dtype=torch.int32), 0
    order = torch.randperm(sum(need) + 2, generator=gen).to(torch.int32)
    for b, m in enumerate(need):
        table[b, :m] = order[at:at + m]
        at += m
    counts = [queries] * len(lengths) if isinstance(queries, int) else queries
    q = (1.5 * torch.randn(sum(counts), QH, 128, generator=gen)).bfloat16().to(device)
    return lo, lg, pages, table, torch.tensor(lengths, dtype=torch.int32), q, counts, SCALE * scale


def gaussian_codes(lo, shape, gen):
    """Codes of rows [.., heads, bytes] as those of Gaussian values are distributed, packed from the lowest bit on."""
    points = torch.as_tensor(lo.codebook).double()
    x = torch.randn(1 << 14, 2, generator=gen, dtype=torch.float64)
    near = (x @ points.T - 0.5 * points.square().sum(-1)).argmax(-1)
    codes = near[torch.randint(0, 1 << 14, (*shape[:2], 64), generator=gen)]
    if len(points) == 256:
        return codes.to(torch.uint8)
    if len(points) == 16:
        return (codes[..., 0::2] | codes[..., 1::2] << 4).to(torch.uint8)
    word = codes[..., 0::4] | codes[..., 1::4] << 6 | codes[..., 2::4] << 12 | codes[..., 3::4] << 18
    return torch.stack([word & 255, word >> 8 & 255, word >> 16], -1).view(shape).to(torch.uint8)


def make_on_cpu(H, fmt, n_pages, page):
    """(as P.make, without a search table, which is made on the GPU)"""
    from paper_2501_19392_amd import binding as B
    from tests import parity_utils as U
    n, rtn = P.FORMATS[fmt]
    lo, lg = U.make_layers(H, "bf16", n, rtn_bits=rtn, device="cpu", table=False)
    return lo, lg, B.Pages(lg, n_pages, page, "cpu")


def to_fp16(x, top):
    """x behind a power of two with which the largest of its last axis is in [2^(top - 1), 2^top): as fp16 holds that, and the power"""
    e = torch.frexp(x.abs().amax(-1, keepdim=True)).exponent
    power = torch.exp2((top - e).double())
    return (x * power).half().double(), power


def rotation(lo, signs, h):
    d = torch.arange(128)
    odd = sum((d[:, None] & d) >> i & 1 for i in range(7)) % 2
    return (1.0 - 2.0 * odd.double()) / 128 ** 0.5 * torch.as_tensor(signs).double().view(lo.kv_heads, 128)[h]


def attention(lo, h, q, k, v, k_scale, v_scale, visible, scale, rounded, weight=1.0):
    """q [R, 128]; k, v [n, 128] as the rows stand for; scales [n] or [n, 2] (uniform).  rounded: as stated above, otherwise exact.  weight: of each token (1)."""
    if not rounded:
        x = (q @ k.T * scale).masked_fill(~visible, -math.inf)
        p = torch.exp(x - x.amax(-1, keepdim=True)) * weight
        return p @ v / p.sum(-1, keepdim=True)
    if lo.rtn_bits is None:
        q, k, v = q @ rotation(lo, lo.signs_k, h).T, k @ rotation(lo, lo.signs_k, h).T / k_scale[:, None], v @ rotation(lo, lo.signs_v, h).T / v_scale[:, None]
        k, v = ((x.half().double()) for x in (k, v))                       # (grid points are of the order of 1)
        k_scale, v_scale = k_scale[:, None], v_scale[:, None]
    else:
        k, v = ((x.view(-1, 2, 64) / s[..., None]).view(-1, 128) for x, s in ((k, k_scale), (v, v_scale)))
    width = 128 // k_scale.shape[1]                                         # (a scale for the head, or one for each half)
    held, power = to_fp16(q, 14)
    x = sum(held[:, i * width:(i + 1) * width] @ k[:, i * width:(i + 1) * width].T * k_scale[:, i] for i in range(k_scale.shape[1])) / power * scale
    x = x.masked_fill(~visible, -math.inf)
    p = torch.exp(x - x.amax(-1, keepdim=True))
    out = []
    for i in range(v_scale.shape[1]):
        held, power = to_fp16(p * v_scale[:, i], 8)
        out.append(held @ v[:, i * width:(i + 1) * width] / power)
    out = torch.cat(out, -1) / p.sum(-1, keepdim=True)
    if lo.rtn_bits is None:
        out = out @ rotation(lo, lo.signs_v, h)
    return out.bfloat16().double()


def results(built, rounded=False, hidden=None, doubled=None, later=0, mixed=False):
    """[rows, QH, 128].  hidden, doubled: the tokens first ... last of the longest sequence are not seen, count twice; later: rows see so many tokens more or fewer;
    mixed: keys belong to their neighbours."""
    lo, lg, pages, table, lens, q, counts, scale = built
    out, at = torch.zeros(q.shape, dtype=torch.float64), 0
    longest = int(torch.where(torch.tensor(counts) > 0, lens, -1).argmax())
    held = [[x.cpu() for x in t] for t in ((pages.k_codes, pages.k_scales), (pages.v_codes, pages.v_scales))]
    for b, n in enumerate(counts):
        length = int(lens[b])
        if length == 0:
            at += n
            continue
        rows = P.sequence_rows(pages, table[b], length)
        K, V = (P.held(lo, c[rows], s[rows], sg) for (c, s), sg in zip(held, (lo.signs_k, lo.signs_v)))
        step = lambda s: (s[rows] if lo.rtn_bits is None else s[rows][..., 0].reshape(length, lo.kv_heads, 2)).contiguous().view(torch.float16).double()
        ks, vs = (step(s) for _, s in held)
        if mixed:
            K, ks = K.roll(1, 0), ks.roll(1, 0)
        seen = torch.arange(length)[None] <= length - n + later + torch.arange(n)[:, None]
        weight = torch.ones(length, dtype=torch.float64)
        if b == longest and hidden:
            seen[:, hidden[0]:hidden[1]] = False
        if b == longest and doubled:
            weight[doubled[0]:doubled[1]] = 2.0
        there = seen.any(-1)
        for qh in range(q.shape[1]):
            h = qh // (q.shape[1] // lo.kv_heads)
            if there.any():
                out[at:at + n, qh][there] = attention(lo, h, q[at:at + n, qh].double().cpu()[there], K[:, h], V[:, h], ks[:, h], vs[:, h], seen[there], scale, rounded, weight)
        at += n
    return out


def errors(got, want):
    """Of each row that sees something, relative to it; the others have to be 0."""
    size = want.norm(dim=-1)
    assert (got.norm(dim=-1)[size == 0] == 0).all()
    return ((got - want).norm(dim=-1) / size)[size > 0]


def outside(got, want, stated):
    """'' or why errors are not those of the stated roundings"""
    e, s = errors(got, want), errors(stated, want).square().mean().sqrt()
    if not torch.isfinite(e).all():
        return "not finite"
    rms, worst = e.square().mean().sqrt() / s, e.max() / s
    text = f"{rms:.3g} (one row {worst:.3g}) times the stated roundings' {s:.3g}"
    return text if rms > OF_ALL or worst > OF_ONE else ""
