"""A paged cache for the tests and its definition in 64 bits: the rows that codes and scales stand for (by the oracle), plain soft-max
attention over them, and how far a kernel may be off."""
import math

import numpy as np
import torch

from oracle import aquakv_oracle as O
from paper_2501_19392_amd import synth
from tests import parity_utils as U

FORMATS = {"grid16": (16, None), "grid64": (64, None), "grid256": (256, None), "rtn2": (16, 2), "rtn4": (16, 4)}


def make(kv_heads, dtype, fmt, n_pages, page_tokens, device="cuda"):
    """(oracle layer, layer, pages)"""
    from paper_2501_19392_amd import binding as B
    n, rtn = FORMATS[fmt]
    lo, lg = U.make_layers(kv_heads, dtype, n, rtn_bits=rtn, device=device)
    return lo, lg, B.Pages(lg, n_pages, page_tokens, device)


def fill(lo, pages, gen, spread=0.5):
    """Any codes, log-normal scales, zero points inside the range."""
    for t in (pages.k_codes, pages.v_codes):
        t.copy_(torch.randint(0, 256, t.shape, generator=gen, dtype=torch.int32).to(torch.uint8))
    for t in (pages.k_scales, pages.v_scales):
        if lo.rtn_bits is None:
            t.copy_((spread * torch.randn(t.shape, generator=gen)).exp().half().view(torch.int16))
        else:
            top = 2 ** lo.rtn_bits - 1
            t[..., 0].copy_((spread * torch.randn(t.shape[:-1], generator=gen)).exp().mul(2 / top).half().view(torch.int16))
            t[..., 1].copy_(torch.randint(0, top + 1, t.shape[:-1], generator=gen).to(torch.int16))


def held(lo, codes, scales, signs):
    """[rows, H, 128] in fp64"""
    rows = codes.shape[0]
    s = np.ascontiguousarray(scales.cpu().numpy())
    s = s.view(np.uint16) if lo.rtn_bits is not None else s.view(np.float16)
    with np.errstate(all="ignore"):
        x = O._dequantize_stored(lo, codes.cpu().numpy(), s, O._group_signs(signs, lo), rows)
    return torch.from_numpy(x.reshape(rows, lo.kv_heads, 128))


def sequence_rows(pages, table_row, length):
    """Rows of the tokens of a sequence, -1 where the page is not in the pool."""
    t = torch.arange(length)
    page = table_row.cpu().long()[t // pages.page_tokens]
    row = page * pages.page_tokens + t % pages.page_tokens
    return torch.where((page >= 0) & (page < pages.n_pages), row, -1)


# What a kernel may be off by.  u: how exact queries, grid points and weights are held (bf16 layers: fp16, 2^-11 each; fp32 layers: two
# fp16 numbers each, 2^-21); s: fp32 sums, half a step of 2^-24 per addition of n.
UNIT = {"bf16": 2.0 ** -11, "fp32": 2.0 ** -21}
ROUND = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}


def attention(q, K, V, scale, visible, dtype):
    """q [R, 128], K, V [n, 128] in fp64, visible [R, n] -> (out [R, 128], bound [R] on the 2-norm of its error).

    A score is off by at most d = scale * sum |q_i k_i| (2 u + 128 s), in the basis in which the products are taken (Cauchy: at most
    |q| |k|), and by the exponent's argument, |score| 2^-22.  A weight is then off by the factor e^(2 d), and rounded by u; a value by
    u and the sums' n s.  Numerator and denominator: sum_t p_t |v_t| (2 * 2 d + 2 u + 2 n s) in all.  At the end one rounding."""
    if K.shape[0] == 0:
        return torch.zeros_like(q), torch.zeros(q.shape[0], dtype=torch.float64)
    u, s = UNIT[dtype], 2.0 ** -24
    x = (q @ K.T * scale).masked_fill(~visible, -math.inf)
    p = torch.softmax(x, -1)
    p = torch.where(visible.any(-1, keepdim=True), p, 0)
    out = p @ V
    d = abs(scale) * q.norm(dim=-1, keepdim=True) * K.norm(dim=-1)[None] * (2 * u + 128 * s) + torch.where(visible, x, 0).abs() * 2.0 ** -22
    top = torch.where(visible, d, 0).amax(-1, keepdim=True)                # (the maximum that all weights refer to cancels; their own d does not)
    bound = (p * V.norm(dim=-1)[None] * (2 * d + 2 * top + 2 * u + 2 * K.shape[0] * s)).sum(-1)
    return out, bound + ROUND[dtype] * out.norm(dim=-1)


def reference(lo, pages, table, lens, q, counts, scale, dtype):
    """counts[b] queries of sequence b, rows of q one after the other -> (out [rows, QH, 128], bound [rows, QH])"""
    K, V = held(lo, pages.k_codes, pages.k_scales, lo.signs_k), held(lo, pages.v_codes, pages.v_scales, lo.signs_v)
    QH, H = q.shape[1], lo.kv_heads
    out, bound = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape[:2], dtype=torch.float64)
    room, at = table.shape[1] * pages.page_tokens, 0
    for b, n in enumerate(counts):
        length = min(max(int(lens[b]), 0), room)
        rows = sequence_rows(pages, table[b], length)
        seen = (torch.arange(length)[None] <= length - n + torch.arange(n)[:, None]) & (rows >= 0)[None]
        kept = rows >= 0                                                    # (what a page outside the pool holds is not looked at)
        seen, rows = seen[:, kept], rows[kept]
        for h in range(QH):
            k, v = (x[rows, h // (QH // H)] for x in (K, V))
            out[at:at + n, h], bound[at:at + n, h] = attention(q[at:at + n, h].double().cpu(), k, v, scale, seen, dtype)
        at += n
    return out, bound


def check(got, want, bound, what):
    off = (got.double().cpu() - want).norm(dim=-1)
    assert torch.isfinite(got.double()).all(), what
    worst = (off / (bound + 1e-30)).max().item() if off.numel() else 0.0
    assert (off <= bound + 1e-30).all(), f"{what}: {worst:.3g} of the bound"
    return worst


def rotated(x, cos, sin):
    """rope of x [T, H, 128] by angles [T, 64], in x's type"""
    lo, hi = x[..., :64], x[..., 64:]
    c, s = cos[:, None].to(x.dtype), sin[:, None].to(x.dtype)
    return torch.cat([lo * c - hi * s, hi * c + lo * s], -1)


def storage(dtype):
    return synth.torch_dtype(dtype)
