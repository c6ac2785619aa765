"""What surrounds attention over the paged cache of codes, as it is measured: drafted trees, eviction, rotary positions.

Each in its plain form (elementary torch operations in 32 or 64 bits) and as the library offers it:

  rotary   queries and keys of the joint product are rotated to their positions.
  tables   the angles that takes: cos, sin of position x frequency, frequencies scaled for long contexts.
  tree     the last tokens of every sequence are drafts that form a tree: each sees what is cached and its own ancestors.
  weights  the attention weight that each cached token gets from the last queries, added to what it has had so far.
  evict    the tokens with the largest weight are selected, beside the first and the last ones, and go to pages of their own.
  keep     given tokens of a sequence become consecutive, in the pages they are in: the accepted branch of a drafted tree, or what
           an eviction leaves.

Shapes are those of this repository: 8 kv heads x 128, 24 to 64 query heads, grids of 16 / 64 / 256 points or the uniform
backbone, contexts from a few tokens to 131072.
"""
import functools
import math

import torch

own = False

H, G = 8, 128
D = H * G
SCALE = G ** -0.5
CODE_BITS = {("grid", 2): 4, ("grid", 3): 6, ("grid", 4): 8, ("rtn", 2): 4, ("rtn", 4): 8}     # bits per pair of values
ROPE_ROWS = 131072
N_FIRST, N_LAST = 4, 32                                        # tokens that an eviction never takes


# ---------------------------------------------------------------------------------------------------- the cases
def listed():
    def rotary(name, tokens, q_heads=32, layout="half", dim=G, in_place=False, transposed=False, padded=False):
        return dict(name=name, kind="rotary", tokens=tokens, q_heads=q_heads, layout=layout, dim=dim, in_place=in_place,
                    transposed=transposed, padded=padded, dtype="bf16")

    def tables(name, rows, dim=G, base=500000.0, first=0, scaling="none", factor=8.0, magnitude=1.0):
        return dict(name=name, kind="tables", rows=rows, dim=dim, base=base, first=first, scaling=scaling, factor=factor,
                    magnitude=magnitude)

    def cached(name, kind, batch, context, q_heads=32, bits=4, backbone="grid", page=64, dtype="bf16", **more):
        return dict(name=name, kind=kind, batch=batch, context=context, q_heads=q_heads, bits=bits, backbone=backbone, page=page,
                    dtype=dtype, **more)

    return [
        # the newest token of one sequence, once per layer and generated token: latency
        rotary("rotary-1", 1),
        # a long prompt, half of each head, pairs of neighbouring coordinates
        rotary("rotary-8192-pairs-64", 8192, layout="pairs", dim=64),
        # tables of a short context
        tables("tables-4096", 4096),
        # tables of the longest context: slow frequencies are stretched, fast ones left as they are
        tables("tables-131072-parts", 131072, scaling="parts"),
        # a tree of drafts of one chat: latency
        cached("tree-1x26x2000", "tree", 1, 2000, nodes=26, ragged=False),
        # trees of different sizes over a batch, uniform backbone
        cached("tree-32x12x8000-rtn", "tree", 32, 8000, nodes=12, backbone="rtn", page=16, ragged=True),
        # large trees over long sequences, 3 bits
        cached("tree-4x64x16384-3bit", "tree", 4, 16384, nodes=64, bits=3, page=128, ragged=False),
        # one generated token per sequence adds its weights
        cached("weights-32x16384", "weights", 32, 16384, queries=1, keep=1.0),
        # the last 64 queries of a prompt say which of its tokens count
        cached("weights-1x64x12288", "weights", 1, 12288, queries=64, keep=0.0),
        # a batch goes back to its budget
        cached("evict-32x4160", "evict", 32, 4160, budget=4096),
        # a long prompt is cut to a quarter
        cached("evict-1x131072", "evict", 1, 131072, budget=32768, page=128),
        # the accepted branches of a batch of drafted trees
        cached("keep-32x6of26", "keep", 32, 3000, window=26, kept=6, page=24),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["rotary", "tables", "tree", "tree", "weights", "weights", "evict", "keep"])
    if kind == "rotary":
        return dict(kind=kind, tokens=log_int(1, 8192), q_heads=rng.choice([24, 32, 40]), layout=rng.choice(["half", "pairs"]),
                    dim=rng.choice([32, 48, 64, 96, 128, 128]), in_place=rng.random() < 0.5, transposed=rng.random() < 0.3,
                    padded=rng.random() < 0.4, dtype=rng.choice(["bf16", "bf16", "fp32"]))
    if kind == "tables":
        return dict(kind=kind, rows=log_int(512, 131072), dim=rng.choice([32, 48, 64, 96, 128, 128]), base=rng.choice([10000.0, 500000.0, 1e6]),
                    first=rng.choice([0, 0, 12345]), scaling=rng.choice(["none", "linear", "parts", "parts"]),
                    factor=rng.choice([2.0, 4.0, 8.0, 32.0]), magnitude=rng.choice([1.0, 1.0, 1.2079441541679836]))
    backbone, bits = rng.choice([("grid", 4)] * 4 + [("rtn", 4)] * 2 + [("grid", 3), ("grid", 2), ("rtn", 2)])
    c = dict(kind=kind, q_heads=rng.choice([24, 32, 32, 40, 64]), page=rng.choice([8, 16, 24, 32, 64, 128, 256]), bits=bits, backbone=backbone,
             dtype="bf16")
    if kind == "tree":
        batch, nodes = log_int(1, 32), log_int(2, 64)
        if rng.random() < 0.15:
            batch, nodes, c["dtype"] = log_int(1, 4), log_int(2, 16), "fp32"
        rows = c["q_heads"] * nodes * batch
        return dict(c, batch=batch, context=log_int(nodes, min(65536, 262144 // batch, 1500 * 65536 // rows)), nodes=nodes, ragged=rng.random() < 0.5)
    if kind == "weights":
        batch, queries = log_int(1, 32), rng.choice([1, 1, 1, 2, 5])
        if rng.random() < 0.35:                                # a prompt's last queries
            batch, queries = rng.choice([1, 1, 2]), log_int(8, 64)
        if rng.random() < 0.15:
            batch, c["dtype"] = min(batch, 4), "fp32"
        limit = min(131072, 262144 // batch, 1800 * 12288 // (c["q_heads"] * queries * batch) if queries > 5 else 1 << 30)
        return dict(c, batch=batch, context=log_int(queries, limit), queries=queries, keep=rng.choice([1.0, 1.0, 0.0, 0.875]))
    if kind == "evict":
        batch = log_int(1, 32)
        context = log_int(64, min(131072, 131072 // batch))
        return dict(c, batch=batch, context=context, budget=max(N_FIRST + N_LAST, int(context * rng.choice([0.25, 0.5, 0.9, 0.97]))))
    batch = log_int(1, 32)
    context = log_int(16, 131072 // batch)
    window = min(context, log_int(2, 64)) if rng.random() < 0.6 else context
    return dict(c, batch=batch, context=context, window=window, kept=max(1, int(window * rng.uniform(0.1, 0.9))))


def lengths(case):
    """From the longest context down to less than half of it."""
    n, b = case["context"], case["batch"]
    least = case.get("nodes") or case.get("queries") or case.get("window") or 1
    return [max(min(least, n), n - (37 * i * n) // (64 * b)) for i in range(b)]


def node_counts(case):
    """Drafts of each sequence: all trees alike, or from the largest down to half of it."""
    b, n = case["batch"], case["nodes"]
    return [n - (n * i) // (2 * b) if case["ragged"] else n for i in range(b)]


# ---------------------------------------------------------------------------------------------------- inputs
@functools.lru_cache(maxsize=None)
def grid(bits):
    """A Gaussian-optimal grid of 4**bits points in the plane (Lloyd iterations; sums in integers, so the same on every
    run), and the points nearest to 65536 Gaussian samples: codes as they are distributed in a cache."""
    n = 4 ** bits
    gen = torch.Generator(device="cuda").manual_seed(20250131)
    x = torch.randn(1 << 16, 2, generator=gen, device="cuda", dtype=torch.float64)
    fixed = (x * 2.0 ** 32).round().to(torch.int64)

    def nearest(c):
        return torch.cat([((p[:, None, :] - c[None]) ** 2).sum(-1).argmin(1) for p in x.split(1 << 14)])

    c = x[:n].clone()
    for _ in range(50):
        near = nearest(c)
        count = torch.bincount(near, minlength=n)
        total = torch.zeros(n, 2, dtype=torch.int64, device="cuda").index_add_(0, near, fixed)
        c = torch.where(count[:, None] > 0, total.double() / 2.0 ** 32 / count.clamp(min=1)[:, None], c)
    pts = torch.tensor(sorted(map(tuple, c.cpu().tolist())), dtype=torch.float32, device="cuda")
    return pts, nearest(pts.double()).to(torch.uint8)


@functools.lru_cache(maxsize=None)
def rope_tables(dim):
    angle = torch.arange(ROPE_ROWS, device="cuda", dtype=torch.float64)[:, None] * 500000.0 ** (
        -torch.arange(0, dim, 2, device="cuda", dtype=torch.float64) / dim)[None]
    return angle.cos().float().contiguous(), angle.sin().float().contiguous()


def randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


def rand_int(gen, lo, hi, shape, dtype=torch.int64):
    return torch.randint(lo, hi, shape, generator=gen, device="cuda", dtype=dtype)


def dtype_of(case):
    return torch.float32 if case["dtype"] == "fp32" else torch.bfloat16


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return globals()["prepare_" + case["kind"]](case, gen)


def prepare_rotary(case, gen):
    T, heads = case["tokens"], case["q_heads"] + H
    # queries, keys and values of the layer's joint product: queries and keys lie side by side
    qkv = (1.5 * randn(gen, T, heads * G + D)).to(dtype_of(case))
    s = dict(case=case, x=qkv[:, :heads * G].view(T, heads, G), rope=rope_tables(case["dim"]))
    if T <= 64:
        s["positions"] = rand_int(gen, 0, ROPE_ROWS, (T,), torch.int32)
    else:
        s["positions"] = torch.arange(T, device="cuda", dtype=torch.int32) + rand_int(gen, 0, ROPE_ROWS - T, (1,), torch.int32)
    if case["padded"]:                                         # a batch that is padded to the size its graph was captured with
        s["positions"][T - T // 4:] = -1
    s["out"] = s["x"] if case["in_place"] else torch.zeros(T, heads, G, dtype=dtype_of(case), device="cuda")
    return s


def prepare_tables(case, gen):
    # (a seed's tables begin a few positions later: nothing else in them can differ)
    first = case["first"] + int(rand_int(gen, 0, 1024, (1,)))
    rows = case["rows"]
    return dict(case=case, first=first, cos=torch.empty(rows, case["dim"] // 2, device="cuda"), sin=torch.empty(rows, case["dim"] // 2, device="cuda"))


def make_format(case, gen):
    """The quantizer: a grid behind rotations by `signs`, or none of both (uniform)."""
    s = dict(case=case, grid=None, signs=(None, None), handle=None)
    if case["backbone"] == "grid":
        s.update(grid=grid(case["bits"])[0], signs=tuple((rand_int(gen, 0, 2, (D,)) * 2 - 1).to(torch.int8) for _ in range(2)))
    if own:
        from paper_2501_19392_amd import binding as B
        if case["backbone"] == "grid":
            s["handle"] = B.Layer(H, G, s["grid"], *s["signs"], dtype_of(case))
        else:
            s["handle"] = B.Layer(H, G, None, None, None, dtype_of(case), rtn_bits=case["bits"])
    return s


def random_codes(case, gen, rows):
    """Codes and scales of `rows` tokens as they are distributed in a cache."""
    bits = case["bits"]
    if case["backbone"] == "grid":
        codes = grid(bits)[1][rand_int(gen, 0, 1 << 16, (rows, H, G // 2))]
        scales = (0.3 * randn(gen, rows, H)).exp().half().view(torch.int16)
        if bits == 3:                                          # 4 codes in 3 bytes
            c = codes.view(rows, H, G // 8, 4).to(torch.int32)
            word = c[..., 0] | c[..., 1] << 6 | c[..., 2] << 12 | c[..., 3] << 18
            codes = torch.stack([word & 255, word >> 8 & 255, word >> 16], -1).to(torch.uint8).view(rows, H, -1)
        elif bits == 2:
            codes = codes[..., 0::2] | codes[..., 1::2] << 4
        return codes.contiguous(), scales
    top = 2 ** bits - 1
    c = (top / 2 + top / 6 * randn(gen, rows, H, G)).round().clamp(0, top).to(torch.uint8)
    c = c[..., 0::2] | c[..., 1::2] << bits
    if bits == 2:
        c = c[..., 0::2] | c[..., 1::2] << 4
    zero = rand_int(gen, top // 2, top // 2 + 2, (rows, 2 * H)).to(torch.int16)
    step = ((0.3 * randn(gen, rows, 2 * H)).exp() * (6 / top)).half().view(torch.int16)
    return c.contiguous(), torch.stack([step, zero], -1)


def prepare_cache(case, gen, more_pages=0):
    """Sequences in pages in any order; `more_pages`: pages of no sequence, behind the others."""
    n, page = lengths(case), case["page"]
    s = make_format(case, gen)
    used = [-(-m // page) for m in n]
    pages = sum(used) + 5
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((case["batch"], max(used)), -1, dtype=torch.int32, device="cuda")
    at, behind = 0, []
    for b, m in enumerate(used):
        table[b, :m] = order[at:at + m]
        at += m
        if n[b] % page:                                        # behind the last token a page holds anything
            behind.append(order[at - 1].long() * page + torch.arange(n[b] % page, page, device="cuda"))
    for t in "kv":
        codes, scales = random_codes(case, gen, pages * page)
        if behind:
            scales[torch.cat(behind)] = 0x7e01
        if more_pages:
            codes, scales = (torch.cat([x, x.new_zeros(more_pages * page, *x.shape[1:])]) for x in (codes, scales))
        s[t + "_codes"], s[t + "_scales"] = codes, scales
    s.update(table=table, lens=torch.tensor(n, dtype=torch.int32, device="cuda"), own_pages=pages, n_pages=pages + more_pages)
    if own:
        from paper_2501_19392_amd import binding as B
        s["pages"] = B.Pages(s["handle"], pages + more_pages, page, k_codes=s["k_codes"], k_scales=s["k_scales"],
                             v_codes=s["v_codes"], v_scales=s["v_scales"])
    return s


def workspace(size):
    return torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")


def prepare_tree(case, gen):
    s = prepare_cache(case, gen)
    counts, words = node_counts(case), -(-case["nodes"] // 32)
    start = [sum(counts[:b]) for b in range(case["batch"] + 1)]
    s["seq"] = torch.tensor([b for b, n in enumerate(counts) for _ in range(n)], device="cuda")
    s["node"] = torch.tensor([i for n in counts for i in range(n)], device="cuda")
    s["start"] = torch.tensor(start, dtype=torch.int32, device="cuda") if case["ragged"] else None
    # every draft's parent is one of those before it (the first have none): mostly one of the last few
    n = case["nodes"]
    back = (randn(gen, case["batch"], n).abs() * 4).floor().long() + 1
    parent = torch.arange(n, device="cuda") - back
    sees = torch.eye(n, dtype=torch.bool, device="cuda").repeat(case["batch"], 1, 1)
    for i in range(1, n):
        p = parent[:, i].clamp(min=0)
        above = sees[torch.arange(case["batch"], device="cuda"), p] & (parent[:, i] >= 0)[:, None]
        sees[:, i] |= above
    s["sees"] = sees[s["seq"], s["node"]]                      # [rows, nodes]
    bits = torch.zeros(len(s["seq"]), words * 32, dtype=torch.int64, device="cuda")
    bits[:, :n] = s["sees"]
    word = (bits.view(-1, words, 32) << torch.arange(32, device="cuda")).sum(-1)
    s["tree"] = torch.where(word >= 2 ** 31, word - 2 ** 32, word).to(torch.int32).contiguous()
    rows = start[-1]
    s["q"] = (1.5 * randn(gen, rows, case["q_heads"], G)).to(dtype_of(case))
    s["out"] = torch.empty(rows, case["q_heads"], G, dtype=dtype_of(case), device="cuda")
    if own:
        from paper_2501_19392_amd import binding as B
        s["ws"] = workspace(B.aquakv_paged_workspace_bytes(s["handle"], s["pages"], case["batch"], case["q_heads"], s["table"].shape[1], rows, n))
    return s


def heavy_mass(gen, pages, page):
    """Attention weights added up over many tokens: a few have most of it."""
    token = (2.0 * randn(gen, pages, 1, page)).exp()
    return (token * (0.5 * randn(gen, pages, H, page)).exp()).contiguous()


def prepare_weights(case, gen):
    s = prepare_cache(case, gen)
    rows = case["batch"] * case["queries"]
    s["q"] = (1.5 * randn(gen, rows, case["q_heads"], G)).to(dtype_of(case))
    s["mass"] = 1e-4 * heavy_mass(gen, s["n_pages"], case["page"])
    if own:
        from paper_2501_19392_amd import binding as B
        s["ws"] = workspace(B.aquakv_paged_weights_workspace_bytes(s["handle"], s["pages"], case["batch"], case["q_heads"], s["table"].shape[1],
                                                                   rows, case["queries"]))
    return s


def prepare_evict(case, gen):
    each = -(-case["budget"] // case["page"])
    s = prepare_cache(case, gen, more_pages=case["batch"] * each)
    s["mass"] = heavy_mass(gen, s["n_pages"], case["page"])
    s["to"] = (s["own_pages"] + torch.arange(case["batch"] * each, device="cuda", dtype=torch.int32)).view(case["batch"], each).contiguous()
    s["kept"] = torch.zeros(case["batch"], case["budget"], dtype=torch.int32, device="cuda")
    s["n_kept"] = torch.zeros(case["batch"], dtype=torch.int32, device="cuda")
    if own:
        from paper_2501_19392_amd import binding as B
        s["ws"] = workspace(max(B.aquakv_paged_select_workspace_bytes(s["handle"], s["pages"], case["batch"], s["table"].shape[1], case["budget"]),
                                B.aquakv_paged_keep_workspace_bytes(s["handle"], s["pages"], case["batch"], case["budget"], True)))
    return s


def prepare_keep(case, gen):
    s = prepare_cache(case, gen)
    w, n = case["window"], case["kept"]
    order = torch.rand(case["batch"], w, generator=gen, device="cuda").argsort(1)[:, :n].sort(1).values
    first = s["lens"] - w
    s["first"], s["kept"] = first.to(torch.int32), (first[:, None] + order).to(torch.int32).contiguous()
    s["n_kept"] = torch.full((case["batch"],), n, dtype=torch.int32, device="cuda")
    if own:
        from paper_2501_19392_amd import binding as B
        s["ws"] = workspace(B.aquakv_paged_keep_workspace_bytes(s["handle"], s["pages"], case["batch"], n, False))
    return s


# ---------------------------------------------------------------------------------------------------- run
def run(state):
    return globals()["run_" + state["case"]["kind"]](state)


def run_rotary(s):
    c, (cos, sin) = s["case"], s["rope"]
    if own:
        from paper_2501_19392_amd import binding as B
        B.aquakv_rotary(s["x"], s["positions"], cos, sin, c["dim"], c["layout"], s["out"], transposed=c["transposed"])
        return s["out"]
    at = s["positions"].long().clamp(min=0)
    cos, sin = cos[at][:, None], sin[at][:, None]
    if c["transposed"]:
        sin = -sin
    x, d = s["x"].float(), c["dim"]
    if c["layout"] == "half":
        a, b = x[..., :d // 2], x[..., d // 2:d]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., d:]], -1)
    else:
        a, b = x[..., 0:d:2], x[..., 1:d:2]
        y = torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), x[..., d:]], -1)
    there = (s["positions"] >= 0)[:, None, None]
    s["out"].copy_(torch.where(there, y.to(s["x"].dtype), s["out"]))
    return s["out"]


def frequencies(c):
    """Of a case's tables, fp64."""
    theta = c["base"] ** (-torch.arange(0, c["dim"], 2, device="cuda", dtype=torch.float64) / c["dim"])
    if c["scaling"] == "none":
        return theta
    kept = torch.zeros_like(theta)
    if c["scaling"] == "parts":                                # turns over the context of the training: below 1 stretched, above 4 not
        kept = ((8192 * theta / (2 * math.pi) - 1) / (4 - 1)).clamp(0, 1)
    return theta * (kept + (1 - kept) / c["factor"])


def run_tables(s):
    c = s["case"]
    if own:
        from paper_2501_19392_amd import binding as B
        more = {} if c["scaling"] == "none" else dict(factor=c["factor"])
        if c["scaling"] == "parts":
            more.update(original_len=8192.0, low_turns=1.0, high_turns=4.0)
        B.aquakv_rotary_tables(s["cos"], s["sin"], c["base"], first=s["first"], magnitude=c["magnitude"], **more)
        return dict(cos=s["cos"], sin=s["sin"])
    # in 64 bits: angles of far positions
    angle = (torch.arange(c["rows"], device="cuda", dtype=torch.float64) + s["first"])[:, None] * frequencies(c)[None]
    return dict(cos=(angle.cos() * c["magnitude"]).float(), sin=(angle.sin() * c["magnitude"]).float())


def hadamard(dtype):
    h = torch.ones(1, 1, dtype=dtype, device="cuda")
    while h.shape[0] < G:
        h = torch.cat([torch.cat([h, h], 1), torch.cat([h, -h], 1)], 0)
    return h / G ** 0.5


def unpacked(s, t, dtype):
    """All rows of the pool's keys or values, [rows, H, 128], as the values they stand for."""
    codes, bits = s[t + "_codes"], s["case"]["bits"]
    if s["grid"] is None:
        each = 8 // bits
        c = torch.stack([codes >> bits * i & 2 ** bits - 1 for i in range(each)], -1).view(-1, D // 64, 64)
        step = s[t + "_scales"][..., 0].contiguous().view(torch.float16).to(dtype)
        zero = s[t + "_scales"][..., 1].to(dtype)
        return ((c.to(dtype) - zero[..., None]) * step[..., None]).view(-1, H, G)
    if bits == 4:
        c = codes.long()
    elif bits == 2:
        c = torch.stack([codes & 15, codes >> 4], -1).long()
    else:
        b = codes.view(*codes.shape[:2], -1, 3).long()
        word = b[..., 0] | b[..., 1] << 8 | b[..., 2] << 16
        c = torch.stack([word >> 6 * i & 63 for i in range(4)], -1)
    sign = s["signs"]["kv".index(t)].view(H, G).to(dtype)
    z = s["grid"].to(dtype)[c.view(codes.shape[0], H, G // 2)].view(-1, H, G) * s[t + "_scales"].view(torch.float16).to(dtype)[..., None]
    return z @ hadamard(dtype) * sign


def cache_rows(s):
    """Pool rows of all tokens that there is room for, [batch, T], and whether they are there."""
    page = s["case"]["page"]
    at = torch.arange(s["table"].shape[1] * page, device="cuda")
    return s["table"].clamp(min=0).long()[:, at // page] * page + at % page, at[None] < s["lens"][:, None]


def probabilities(s, q, n, seen):
    """q [batch, n, heads, 128], seen [batch, n, T] -> soft-max weights [batch, H, rep * n, T]"""
    b, qh = s["case"]["batch"], s["case"]["q_heads"]
    rep, T = qh // H, seen.shape[2]
    rows, there = cache_rows(s)
    K = torch.where(there[:, :, None, None], unpacked(s, "k", torch.float32)[rows], 0).transpose(1, 2).contiguous()
    q = q.float().view(b, n, H, rep, G).permute(0, 2, 3, 1, 4).reshape(b, H, rep * n, G)
    x = (q @ K.transpose(2, 3) * SCALE).view(b, H, rep, n, T).masked_fill(~seen[:, None, None], -math.inf)
    p = (x - x.amax(-1, keepdim=True).clamp(min=-3e38)).exp_()
    return (p / p.sum(-1, keepdim=True).clamp(min=1e-38)).view(b, H, rep * n, T)


def run_tree(s):
    c = s["case"]
    b, n, qh = c["batch"], c["nodes"], c["q_heads"]
    if own:
        from paper_2501_19392_amd import binding as B
        B.aquakv_paged_attend_tree(s["handle"], s["pages"], b, qh, s["table"], s["lens"], s["q"], n, s["start"], s["tree"], SCALE, s["out"], s["ws"])
        return s["out"]
    counts = torch.bincount(s["seq"], minlength=b)
    rows, there = cache_rows(s)
    past = s["lens"] - counts                                  # tokens that are no drafts
    at = torch.arange(rows.shape[1], device="cuda")
    q = torch.zeros(b, n, qh, G, dtype=s["q"].dtype, device="cuda")
    q[s["seq"], s["node"]] = s["q"]
    sees = torch.zeros(b, n, n, dtype=torch.bool, device="cuda")
    sees[s["seq"], s["node"]] = s["sees"]
    draft = at[None] - past[:, None]                           # [b, T]: which of the drafts a token is
    own_branch = torch.gather(sees, 2, draft.clamp(0, n - 1)[:, None].expand(-1, n, -1))
    seen = (own_branch | (draft < 0)[:, None]) & there[:, None]
    p = probabilities(s, q, n, seen)
    V = torch.where(there[:, :, None, None], unpacked(s, "v", torch.float32)[rows], 0).transpose(1, 2).contiguous()
    out = (p @ V).view(b, H, qh // H, n, G).permute(0, 3, 1, 2, 4).reshape(b, n, qh, G)
    return out[s["seq"], s["node"]].to(s["q"].dtype)


def run_weights(s):
    c = s["case"]
    b, n, qh, page = c["batch"], c["queries"], c["q_heads"], c["page"]
    if own:
        from paper_2501_19392_amd import binding as B
        B.aquakv_paged_weights(s["handle"], s["pages"], b, qh, s["table"], s["lens"], s["q"], n, None, SCALE, c["keep"], s["mass"], s["ws"])
        return s["mass"]
    rows, there = cache_rows(s)
    at = torch.arange(rows.shape[1], device="cuda")
    last = s["lens"][:, None] - n + torch.arange(n, device="cuda")[None]
    p = probabilities(s, s["q"].view(b, n, qh, G), n, at[None, None] <= last[:, :, None])
    gained = p.sum(2)                                          # [b, H, T]
    rows, old = rows[there], (at[None] < (s["lens"] - n)[:, None])[there]
    before = s["mass"][rows // page, :, rows % page]
    kept = torch.where(old[:, None], c["keep"] * before, 0) if c["keep"] else 0
    s["mass"][rows // page, :, rows % page] = kept + gained.transpose(1, 2)[there]
    return s["mass"]


def run_evict(s):
    c = s["case"]
    b, page, budget = c["batch"], c["page"], c["budget"]
    outputs = dict(kept=s["kept"], n_kept=s["n_kept"], mass=s["mass"], **{t + x: s[t + x] for t in "kv" for x in ("_codes", "_scales")})
    if own:
        from paper_2501_19392_amd import binding as B
        B.aquakv_paged_select(s["handle"], s["pages"], b, s["table"], s["lens"], s["mass"], budget, N_FIRST, N_LAST, s["kept"], s["n_kept"], s["ws"])
        B.aquakv_paged_keep(s["handle"], s["pages"], b, s["table"], s["kept"], s["n_kept"], None, s["to"], s["mass"], s["ws"])
        return outputs
    rows, there = cache_rows(s)
    at = torch.arange(rows.shape[1], device="cuda")
    mass = functools.reduce(torch.add, s["mass"].unbind(1)).view(-1)[rows]                        # head after head
    safe = (at < N_FIRST)[None] | (at[None] >= (s["lens"] - N_LAST)[:, None])
    mass = torch.where(there, torch.where(safe, math.inf, mass), -math.inf)
    order = torch.sort(mass, dim=1, descending=True, stable=True).indices[:, :budget]             # equal ones: the first
    n = s["lens"].clamp(max=budget)
    place = torch.arange(order.shape[1], device="cuda")
    kept = torch.where(place[None] < n[:, None], order, 1 << 30).sort(1).values                   # ascending
    s["kept"].fill_(-1)
    s["kept"][:, :order.shape[1]] = torch.where(place[None] < n[:, None], kept, -1)
    s["n_kept"].copy_(n)
    seq, i = (place[None] < n[:, None]).nonzero(as_tuple=True)
    source, target = rows[seq, kept[seq, i]], s["to"].long()[seq, i // page] * page + i % page
    for t in "kv":
        for x in ("_codes", "_scales"):
            s[t + x][target] = s[t + x][source]
    s["mass"][target // page, :, target % page] = s["mass"][source // page, :, source % page]
    return outputs


def run_keep(s):
    c = s["case"]
    if own:
        from paper_2501_19392_amd import binding as B
        B.aquakv_paged_keep(s["handle"], s["pages"], c["batch"], s["table"], s["kept"], s["n_kept"], s["first"], None, None, s["ws"])
    else:
        rows, _ = cache_rows(s)
        source = torch.gather(rows, 1, s["kept"].long()).view(-1)
        target = torch.gather(rows, 1, s["first"].long()[:, None] + torch.arange(c["kept"], device="cuda")).view(-1)
        for t in "kv":
            for x in ("_codes", "_scales"):
                s[t + x][target] = s[t + x][source]
    return {t + x: s[t + x] for t in "kv" for x in ("_codes", "_scales")}


# ---------------------------------------------------------------------------------------------------- work, exact
def work(case):
    kind = case["kind"]
    if kind == "rotary":
        T, heads, size = case["tokens"] - (case["tokens"] // 4 if case["padded"] else 0), case["q_heads"] + H, 4 if case["dtype"] == "fp32" else 2
        touched = case["dim"] if case["in_place"] else G
        return dict(bytes=T * (2 * size * heads * touched + 4 * case["dim"] + 4), flops=T * heads * case["dim"] * 3)
    if kind == "tables":
        return dict(bytes=4 * case["rows"] * case["dim"], flops=20 * case["rows"] * case["dim"])
    stored = D * CODE_BITS[case["backbone"], case["bits"]] // 16 + (2 * H if case["backbone"] == "grid" else 8 * H)     # a token's keys or values
    n, qh, size = lengths(case), case["q_heads"], 4 if case["dtype"] == "fp32" else 2
    table = 4 * sum(-(-m // case["page"]) for m in n)
    if kind == "tree":
        counts = node_counts(case)
        pairs = sum(k * (m - k) + k * (k + 1) // 4 for k, m in zip(counts, n))
        return dict(bytes=2 * stored * sum(n) + sum(counts) * (2 * size * qh * G + 4 * -(-case["nodes"] // 32)) + table, flops=4 * G * qh * pairs)
    if kind == "weights":
        pairs = sum(case["queries"] * m - case["queries"] * (case["queries"] - 1) // 2 for m in n)
        return dict(bytes=(stored + (8 if case["keep"] else 4) * H) * sum(n) + size * case["batch"] * case["queries"] * qh * G + table,
                    flops=(2 * G + 4) * qh * pairs)
    if kind == "evict":
        kept = sum(min(m, case["budget"]) for m in n)
        return dict(bytes=4 * H * sum(n) + 4 * kept + 2 * kept * (2 * stored + 4 * H) + table, flops=2 * H * sum(n))
    return dict(bytes=case["batch"] * case["kept"] * (4 * stored + 4), flops=0)


def exact_side(s, t, rows, h):
    """Keys or values of head h in the given rows of the pool, fp64, from the bits of the codes."""
    case, m = s["case"], len(rows)
    width = CODE_BITS[case["backbone"], case["bits"]] if s["grid"] is not None else case["bits"]
    shift = torch.arange(8, device="cuda", dtype=torch.uint8)
    string = (s[t + "_codes"][rows, h][:, :, None] >> shift & 1).view(m, -1, width).long()        # little-endian bits
    number = (string * 2 ** torch.arange(width, device="cuda")).sum(-1)
    scale = s[t + "_scales"][rows]
    if s["grid"] is None:
        f = scale[:, 2 * h:2 * h + 2, 0].contiguous().view(torch.float16).double()
        return ((number.view(m, 2, 64) - scale[:, 2 * h:2 * h + 2, 1:].long()) * f[..., None]).view(m, G)
    index = torch.arange(G, device="cuda")
    odd = sum((index[:, None] & index[None]) >> i & 1 for i in range(7)) % 2
    rot = (1.0 - 2.0 * odd.double()) / math.sqrt(G)                                               # Walsh functions
    f = scale[:, h].contiguous().view(torch.float16).double()
    return (s["grid"].double()[number].view(m, G) * f[:, None]) @ rot * s["signs"]["kv".index(t)].view(H, G)[h].double()


def exact(case, seed):
    """By the definition, in 64 bits, one head (and sequence) after the other."""
    kind, s = case["kind"], prepare(case, seed)
    if kind == "rotary":
        d, out = case["dim"], s["out"].double().clone()
        turn = torch.complex(*(a.double()[s["positions"].long().clamp(min=0)] for a in s["rope"]))[:, None]
        turn = turn.conj() if case["transposed"] else turn
        x = s["x"].double()
        flat = x[..., :d].unflatten(-1, (2, d // 2)).transpose(-1, -2) if case["layout"] == "half" else x[..., :d].unflatten(-1, (d // 2, 2))
        y = torch.view_as_real(torch.view_as_complex(flat.contiguous()) * turn)
        y = y.transpose(-1, -2).flatten(-2) if case["layout"] == "half" else y.flatten(-2)
        live = s["positions"] >= 0
        out[live] = torch.cat([y, x[..., d:]], -1)[live]
        return out
    if kind == "tables":
        f = []
        for i in range(case["dim"] // 2):
            w = math.exp(-2.0 * i / case["dim"] * math.log(case["base"]))
            turns = 8192 * w / (2 * math.pi)
            stretched = {"none": 0.0, "linear": 1.0, "parts": 1.0 - min(max((turns - 1) / 3, 0.0), 1.0)}[case["scaling"]]
            f.append(w * (1 - stretched) + w / case["factor"] * stretched)
        at = torch.arange(s["first"], s["first"] + case["rows"], device="cuda", dtype=torch.float64)
        z = torch.polar(torch.full((1, 1), case["magnitude"], device="cuda", dtype=torch.float64), torch.outer(at, torch.tensor(f, device="cuda", dtype=torch.float64)))
        return dict(cos=z.real.contiguous(), sin=z.imag.contiguous())
    if kind == "keep":
        return None
    page, qh = case["page"], case["q_heads"]
    rep, n = qh // H, lengths(case)

    def rows_of(b):
        return torch.cat([torch.arange(page, device="cuda") + p * page for p in s["table"][b].tolist() if p >= 0])[:n[b]]

    if kind == "evict":
        import numpy as np
        mass = s["mass"].double().clone()
        for b in range(case["batch"]):
            rows = rows_of(b)
            each = s["mass"][rows // page, :, rows % page].cpu().numpy()
            total = np.zeros(n[b], dtype=np.float32)
            for h in range(H):                                 # (the definition's own sum: 32 bits, head after head)
                total = total + each[:, h]
            total[:N_FIRST] = total[max(n[b] - N_LAST, 0):] = np.inf
            kept = np.sort(np.lexsort((np.arange(n[b]), -total))[:case["budget"]])
            i = torch.arange(len(kept), device="cuda")
            target = s["to"][b].long()[i // page]
            mass[target, :, i % page] = torch.from_numpy(each[kept]).double().cuda()
        return dict(mass=mass, kept=None, n_kept=None, k_codes=None, k_scales=None, v_codes=None, v_scales=None)
    if kind == "tree":
        result, at = torch.zeros(len(s["seq"]), qh, G, dtype=torch.float64, device="cuda"), 0
        for b, k in enumerate(node_counts(case)):
            rows = rows_of(b)
            hidden = torch.zeros(k, n[b], dtype=torch.bool, device="cuda")
            hidden[:, n[b] - k:] = ~s["sees"][at:at + k, :k]
            for h in range(H):
                keys, values = (exact_side(s, t, rows, h) for t in "kv")
                for r in range(h * rep, (h + 1) * rep):
                    p = torch.softmax((s["q"][at:at + k, r].double() @ keys.T * SCALE).masked_fill(hidden, -math.inf), -1)
                    result[at:at + k, r] = p @ values
            at += k
        return result
    mass, k = s["mass"].double().clone(), case["queries"]
    for b in range(case["batch"]):
        rows = rows_of(b)
        t = torch.arange(n[b], device="cuda")
        hidden = t[None] > torch.arange(n[b] - k, n[b], device="cuda")[:, None]
        for h in range(H):
            keys, total = exact_side(s, "k", rows, h), torch.zeros(n[b], dtype=torch.float64, device="cuda")
            for r in range(h * rep, (h + 1) * rep):
                score = s["q"][b * k:(b + 1) * k, r].double() @ keys.T * SCALE
                total += torch.softmax(score.masked_fill(hidden, -math.inf), -1).sum(0)
            before = torch.where(t < n[b] - k, case["keep"] * mass[rows // page, h, rows % page], 0.0)
            mass[rows // page, h, rows % page] = before + total
    return mass
