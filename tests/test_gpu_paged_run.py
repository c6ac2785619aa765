"""The calls on pages together, as a serving program makes them: drafts are rotated, appended and attended to as a tree, the accepted branch is kept, its weights are added
up, tokens with little weight are evicted, and a plain query reads what is left.  Each call is held to its definition on what the pool held before it."""
import pytest
import torch

from tests import paged_utils as P
from tests import test_gpu_paged_weights as W
from tests import test_gpu_paged_evict as E
from tests import tree_utils as T

pytestmark = pytest.mark.gpu
SCALE = 128 ** -0.5
H, QH, PAGE, N = 2, 8, 16, 7
BUDGET, FIRST, LAST = 80, 4, 16


class Program:
    """Two sequences, buffers that a captured program would keep."""

    def __init__(self, dtype, fmt):
        from paper_2501_19392_amd import binding as B
        self.B, self.dtype, self.sd = B, dtype, P.storage(dtype)
        self.lo, self.lg, self.pages = P.make(H, dtype, fmt, 20, PAGE)
        self.gen = torch.Generator().manual_seed(17)
        P.fill(self.lo, self.pages, self.gen)
        self.table = torch.randperm(20, generator=self.gen)[:16].to(torch.int32).view(2, 8)
        self.lens = torch.tensor([70, 61], dtype=torch.int32)
        self.next_position = self.lens.clone()                              # (positions go on where tokens are evicted)
        self.mass = torch.rand(20, H, PAGE, generator=self.gen).cuda()
        self.cos, self.sin = (torch.empty(400, 64, device="cuda") for _ in range(2))
        B.aquakv_rotary_tables(self.cos, self.sin, 10000.0, factor=4.0, original_len=100.0, low_turns=1.0, high_turns=4.0)
        size = max(B.aquakv_paged_workspace_bytes(self.lg, self.pages, 2, QH, 8, 2 * N, N),
                   B.aquakv_paged_weights_workspace_bytes(self.lg, self.pages, 2, QH, 8, 2 * N, N),
                   B.aquakv_paged_select_workspace_bytes(self.lg, self.pages, 2, 8, BUDGET), B.aquakv_paged_keep_workspace_bytes(self.lg, self.pages, 2, BUDGET, True))
        self.ws = torch.empty(size, dtype=torch.uint8, device="cuda")

    def pool(self):
        return {k: getattr(self.pages, k).cpu().clone() for k in E.POOL}

    def rows(self, b, tokens):
        return self.table[b].long()[tokens // PAGE] * PAGE + tokens % PAGE

    def step(self):
        B, gen = self.B, self.gen
        trees = [T.random_tree(N, gen) for _ in range(2)]
        depth = torch.cat([t.sum(1) - 1 for t in trees]).to(torch.int32)
        past = self.lens.clone()
        positions = (self.next_position.repeat_interleave(N) + depth).to(torch.int32)
        # queries and keys side by side in the joint product, rotated by one call, in place
        joint = torch.randn(2 * N, (QH + 2 * H) * 128, generator=gen).to(self.sd)
        on = joint.cuda()
        both = on[:, :(QH + H) * 128].view(2 * N, QH + H, 128)
        B.aquakv_rotary(both, positions.cuda(), self.cos, self.sin, 128, "half", both)
        torch.cuda.synchronize()
        cos, sin = (t.cpu()[positions.long()] for t in (self.cos, self.sin))
        turned = P.rotated(joint[:, :(QH + H) * 128].view(2 * N, QH + H, 128).double(), cos, sin)
        assert ((both.cpu().double() - turned).abs() <= P.ROUND[self.dtype] * turned.abs() + 1e-5).all()
        q, K, V = both[:, :QH], both[:, QH:], on[:, -H * 128:].view(2 * N, H, 128)
        # ... appended: no rotation is left to be made
        self.lens = past + N
        slots = torch.cat([self.rows(b, past[b] + torch.arange(N)) for b in range(2)])
        B.aquakv_paged_append(self.lg, self.pages, 2 * N, K, V, slots.cuda(), None, None, None, None, None)
        out = torch.empty(2 * N, QH, 128, dtype=self.sd, device="cuda")
        bits = torch.cat([T.words_of(t, 1) for t in trees]).cuda()
        table, lens = self.table.cuda(), self.lens.cuda()
        B.aquakv_paged_attend_tree(self.lg, self.pages, 2, QH, table, lens, q, N, None, bits, SCALE, out, self.ws)
        torch.cuda.synchronize()
        P.check(out, *T.reference(self.lo, self.pages, self.table, self.lens, q.contiguous(), [N, N], trees, SCALE, self.dtype), "tree")
        # the branch of the deepest draft is accepted: its nodes, in order
        leaves = [int(t.sum(1).argmax()) for t in trees]
        paths = [t[leaf].nonzero().view(-1) for t, leaf in zip(trees, leaves)]
        kept = torch.full((2, N), -1, dtype=torch.int32)
        for b, path in enumerate(paths):
            kept[b, :len(path)] = past[b] + path.to(torch.int32)
        counts = torch.tensor([len(p) for p in paths], dtype=torch.int32)
        before = self.pool()
        want, _ = E.kept_by_hand(before, None, PAGE, 20, self.table.tolist(), kept, counts, past, None)
        B.aquakv_paged_keep(self.lg, self.pages, 2, table, kept.cuda(), counts.cuda(), past.cuda(), None, None, self.ws)
        torch.cuda.synchronize()
        for k in E.POOL:
            assert torch.equal(getattr(self.pages, k).cpu(), want[k]), k
        self.lens = past + counts
        self.next_position = self.next_position + counts
        # the accepted queries' weights
        picked = torch.cat([q[b * N + p.cuda()] for b, p in enumerate(paths)]).contiguous()
        start = torch.tensor([0, len(paths[0]), len(paths[0]) + len(paths[1])], dtype=torch.int32).cuda()
        old = self.mass.cpu()
        B.aquakv_paged_weights(self.lg, self.pages, 2, QH, table, self.lens.cuda(), picked, N, start, SCALE, 1.0, self.mass, self.ws)
        torch.cuda.synchronize()
        W.check(self.mass.cpu(), old, *W.wanted(self.lo, self.pages, self.table, self.lens, picked, counts.tolist(), N, 1.0, old))
        # back to the budget
        kept, n_kept = torch.empty(2, BUDGET, dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda")
        B.aquakv_paged_select(self.lg, self.pages, 2, table, self.lens.cuda(), self.mass, BUDGET, FIRST, LAST, kept, n_kept, self.ws)
        before, old = self.pool(), self.mass.cpu().clone()
        B.aquakv_paged_keep(self.lg, self.pages, 2, table, kept, n_kept, None, None, self.mass, self.ws)
        torch.cuda.synchronize()
        for b in range(2):
            chosen = E.wanted(old.numpy(), self.table[b], int(self.lens[b]), 20, PAGE, BUDGET, FIRST, LAST)
            assert kept[b].cpu().tolist() == list(chosen) + [-1] * (BUDGET - len(chosen))
        want, want_mass = E.kept_by_hand(before, old, PAGE, 20, self.table.tolist(), kept.cpu(), n_kept.cpu(), None, None)
        for k in E.POOL:
            assert torch.equal(getattr(self.pages, k).cpu(), want[k]), k
        assert torch.equal(self.mass.cpu(), want_mass)
        self.lens = n_kept.cpu()
        # a plain query over what is left
        last = (1.5 * torch.randn(2, QH, 128, generator=gen)).to(self.sd).cuda()
        out = torch.empty_like(last)
        B.aquakv_paged_attend(self.lg, self.pages, 2, QH, table, n_kept, last, 1, None, SCALE, out, self.ws)
        torch.cuda.synchronize()
        P.check(out, *P.reference(self.lo, self.pages, self.table, self.lens, last, [1, 1], SCALE, self.dtype), "plain")


@pytest.mark.parametrize("dtype,fmt", [("bf16", "grid256"), ("bf16", "grid64"), ("bf16", "rtn4"), ("fp32", "grid16"), ("fp32", "rtn2")])
def test_a_program_of_drafts_and_evictions(dtype, fmt):
    print(f"case run {dtype} {fmt}", flush=True)
    program = Program(dtype, fmt)
    for _ in range(4):
        program.step()
    assert program.lens[0] == BUDGET < program.next_position[0]             # (something was evicted)


def test_select_and_keep_in_a_graph():
    """An eviction captured once, replayed as lengths and masses change: kept tokens and counts go from one call to the next on the device."""
    from paper_2501_19392_amd import binding as B
    for page, room, budget in ((16, 8, 50), (128, 300, 9000)):              # keys in LDS; slabs, and rows by way of the workspace
        lo, lg, pages, table, lens, gen = T.cache("bf16", "grid16", 1, [page * room - 3], page)
        table = table.cuda()
        kept, n_kept = torch.zeros(1, budget, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        mass, on = torch.zeros(pages.n_pages, 1, page, device="cuda"), lens.cuda()
        ws = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in (B.aquakv_paged_select_workspace_bytes(lg, pages, 1, table.shape[1], budget),
                                                                          B.aquakv_paged_keep_workspace_bytes(lg, pages, 1, budget, True))]
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            B.aquakv_paged_select(lg, pages, 1, table, on, mass, budget, 2, 3, kept, n_kept, ws[0])
            B.aquakv_paged_keep(lg, pages, 1, table, kept, n_kept, None, None, mass, ws[1])
        for n in (page * room - 3, budget - 1, budget + 7, 0):
            on.fill_(n)
            mass.copy_(E.masses("plain", pages.n_pages, 1, page, gen))
            old, pool = mass.cpu().clone(), {k: getattr(pages, k).cpu().clone() for k in E.POOL}
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            want = E.wanted(old.numpy(), table.cpu()[0], n, pages.n_pages, page, budget, 2, 3)
            assert kept[0].cpu().tolist() == list(want) + [-1] * (budget - len(want)) and int(n_kept) == len(want)
            after, after_mass = E.kept_by_hand(pool, old, page, pages.n_pages, table.tolist(), kept.cpu(), n_kept.cpu(), None, None)
            for k in E.POOL:
                assert torch.equal(getattr(pages, k).cpu(), after[k]), k
            assert torch.equal(mass.cpu(), after_mass)
