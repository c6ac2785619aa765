"""Trees of drafted tokens over a paged cache for the tests: caches, masks as bits, and attention by its definition in 64 bits."""
import torch

from tests import paged_utils as P


def cache(dtype, fmt, H, lengths, page, seed=0, spread=0.5, room=3, device="cuda"):
    """A filled cache, pages in any order, behind the last tokens anything -> (oracle layer, layer, pages, page table, lengths, generator)"""
    gen = torch.Generator().manual_seed(1000 * seed + 7 * len(lengths) + max(lengths))
    need = [-(-max(n, 0) // page) for n in lengths]
    n_pages = sum(need) + room
    lo, lg, pages = P.make(H, dtype, fmt, n_pages, page, device)
    P.fill(lo, pages, gen, spread)
    table = torch.full((len(lengths), max(max(need), 1)), -1, dtype=torch.int32)
    order, at = torch.randperm(n_pages, generator=gen).to(torch.int32), 0
    for b, m in enumerate(need):
        table[b, :m] = order[at:at + m]
        at += m
    for b, n in enumerate(lengths):
        if n % page and n > 0:
            rows = (int(table[b, need[b] - 1]) * page + torch.arange(n % page, page)).to(device)
            for t in (pages.k_scales, pages.v_scales):
                t[rows] = 0x7e01 if lo.rtn_bits is None else torch.tensor([0x7e01, -1], dtype=torch.int16, device=device)
    return lo, lg, pages, table, torch.tensor(lengths, dtype=torch.int32), gen


def random_tree(n, gen):
    """[n, n]: every draft sees itself and its ancestors, of which the last is one of the drafts before it, or none."""
    sees = torch.eye(n, dtype=torch.bool)
    for i in range(1, n):
        parent = int(torch.randint(-1, i, (1,), generator=gen))
        if parent >= 0:
            sees[i] |= sees[parent]
    return sees


def words_of(sees, words):
    """[rows, n] of truth values -> int32 [rows, words]"""
    bits = torch.zeros(sees.shape[0], 32 * words, dtype=torch.int64)
    bits[:, :min(sees.shape[1], 32 * words)] = sees[:, :32 * words]
    word = (bits.view(-1, words, 32) << torch.arange(32)).sum(-1)
    return torch.where(word >= 2 ** 31, word - 2 ** 32, word).to(torch.int32).contiguous()


def reference(lo, pages, table, lens, q, counts, trees, scale, dtype):
    """trees[b]: [counts[b], counts[b]] -> (out [rows, QH, 128], bound [rows, QH])"""
    K, V = P.held(lo, pages.k_codes, pages.k_scales, lo.signs_k), P.held(lo, pages.v_codes, pages.v_scales, lo.signs_v)
    QH, H = q.shape[1], lo.kv_heads
    out, bound = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape[:2], dtype=torch.float64)
    room, at = table.shape[1] * pages.page_tokens, 0
    for b, n in enumerate(counts):
        length = min(max(int(lens[b]), 0), room)
        rows = P.sequence_rows(pages, table[b], length)
        draft = torch.arange(length) - (length - n)                         # which of the drafts a token is, below 0: none
        seen = torch.where(draft[None] < 0, True, trees[b][:, draft.clamp(min=0)]) if n else torch.zeros(0, length, dtype=torch.bool)
        kept = rows >= 0
        seen, rows = seen[:, kept], rows[kept]
        for h in range(QH):
            k, v = (x[rows, h // (QH // H)].clone() for x in (K, V))
            never = ~seen.any(0)                                            # (what nobody sees may be anything)
            k[never], v[never] = 0, 0
            out[at:at + n, h], bound[at:at + n, h] = P.attention(q[at:at + n, h].double().cpu(), k, v, scale, seen, dtype)
        at += n
    return out, bound
