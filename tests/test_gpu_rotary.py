"""aquakv_rotary and aquakv_rotary_tables against their formulas in 64 bits."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}


def rotated(x, cos, sin, dim, layout, transposed):
    """x [tokens, heads, 128], cos, sin [tokens, dim / 2], all fp64 -> (result, sum of the sizes of the two products of each value)"""
    c, s = cos[:, None], (-sin if transposed else sin)[:, None]
    at = torch.arange(dim // 2)
    lo, hi = (at, at + dim // 2) if layout == "half" else (2 * at, 2 * at + 1)
    y, size = x.clone(), torch.zeros_like(x)
    y[..., lo], y[..., hi] = x[..., lo] * c - x[..., hi] * s, x[..., hi] * c + x[..., lo] * s
    size[..., lo], size[..., hi] = (x[..., lo] * c).abs() + (x[..., hi] * s).abs(), (x[..., hi] * c).abs() + (x[..., lo] * s).abs()
    return y, size


def make(dtype, tokens, heads, dim, rows, joint, seed=0):
    gen = torch.Generator().manual_seed(1000 * seed + tokens + dim)
    wide = (torch.randn(tokens, (heads + joint) * 128, generator=gen) * torch.randn((heads + joint) * 128, generator=gen).exp()).to(TYPES[dtype])
    angle = torch.rand(rows, dim // 2, generator=gen, dtype=torch.float64) * 6.28
    positions = torch.randint(0, rows, (tokens,), generator=gen).to(torch.int32)
    return gen, wide, angle.cos().float(), angle.sin().float(), positions


@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("dtype,tokens,heads,dim,joint,in_place,transposed", [
    ("bf16", 1, 40, 128, 8, False, False), ("bf16", 1, 40, 128, 8, True, False), ("bf16", 333, 9, 64, 3, False, True), ("bf16", 17, 1, 16, 0, False, False),
    ("bf16", 17, 1, 16, 5, True, True), ("bf16", 1000, 5, 96, 1, True, False), ("bf16", 65, 6, 48, 0, False, False), ("bf16", 3, 3, 112, 2, False, True),
    ("fp32", 1, 8, 128, 8, False, False), ("fp32", 130, 7, 80, 1, False, True), ("fp32", 61, 4, 32, 0, True, False), ("fp32", 5, 2, 16, 0, False, False)])
def test_rows_are_rotated(layout, dtype, tokens, heads, dim, joint, in_place, transposed):
    from paper_2501_19392_amd import binding as B
    print(f"case rotary {dtype} {layout} tokens={tokens} heads={heads} dim={dim}", flush=True)
    rows = 77
    gen, wide, cos, sin, positions = make(dtype, tokens, heads, dim, rows, joint)
    left = torch.zeros(tokens, dtype=torch.bool)
    if tokens > 10:                                                         # positions outside the tables
        for i, p in enumerate((-1, rows, 1 << 30, -(1 << 31))):
            positions[2 * i + 1] = p
            left[2 * i + 1] = True
    big = wide.cuda()
    x = big[:, joint * 128:].view(tokens, heads, 128)
    out = x if in_place else torch.full((tokens, heads + 1, 128), 7.0, dtype=TYPES[dtype], device="cuda")[:, :heads]
    B.aquakv_rotary(x, positions.cuda(), cos.cuda(), sin.cuda(), dim, layout, out, transposed=transposed)
    torch.cuda.synchronize()
    x0 = wide[:, joint * 128:].view(tokens, heads, 128)
    at = positions.long().clamp(0, rows - 1)
    want, size = rotated(x0.double(), cos[at].double(), sin[at].double(), dim, layout, transposed)
    got = out.cpu()
    # two products and a sum in fp32 (the second product is rounded, then the sum), one rounding to dtype
    bound = HALF_STEP[dtype] * want.abs() + (1 + HALF_STEP[dtype]) * 2.0 ** -24 * (size + want.abs())
    off = (got.double() - want).abs()
    assert (off <= bound)[~left].all(), (off / (bound + 1e-300))[~left].max()
    assert torch.equal(got[~left][..., dim:], x0[~left][..., dim:])
    assert torch.equal(got[left], x0[left]) if in_place else (got[left] == 7.0).all()
    if joint:
        assert torch.equal(big[:, :joint * 128].cpu(), wide[:, :joint * 128])
    if not in_place:
        assert torch.equal(x.cpu(), x0)


@pytest.mark.parametrize("layout", ["half", "pairs"])
def test_transposed_is_the_gradient(layout):
    """Against the formula's gradient by autograd in 64 bits, and against differences (the rotation is linear: of any step)."""
    from paper_2501_19392_amd import binding as B
    gen, wide, cos, sin, positions = make("fp32", 9, 2, 64, 50, 0, seed=1)
    cos, sin = 1.25 * cos, 1.25 * sin                                       # (a magnitude: transposed, not inverse)
    x, g = wide.view(9, 2, 128), torch.randn(9, 2, 128, generator=gen)
    at = positions.long()
    leaf = x.double().requires_grad_()
    y, size = rotated(leaf, cos[at].double(), sin[at].double(), 64, layout, False)
    (y * g.double()).sum().backward()
    got = torch.empty(9, 2, 128, device="cuda")
    B.aquakv_rotary(g.cuda(), positions.cuda(), cos.cuda(), sin.cuda(), 64, layout, got, transposed=True)
    torch.cuda.synchronize()
    _, size = rotated(g.double(), cos[at].double(), sin[at].double(), 64, layout, True)
    assert ((got.cpu().double() - leaf.grad).abs() <= 2.0 ** -23 * (size + leaf.grad.abs())).all()
    for k in range(5):
        step = torch.randn(x.shape, generator=gen).double()
        up, down = (rotated(x.double() + e * step, cos[at].double(), sin[at].double(), 64, layout, False)[0] for e in (1.0, -1.0))
        slope = ((up - down) / 2 * g.double()).sum()
        # each of the 2304 values is off by at most 2^-23 of its two products
        assert abs(slope - (got.cpu().double() * step).sum()) <= (2.0 ** -23 * (size + leaf.grad.abs()) * step.abs()).sum() + 1e-9


def test_what_is_not_finite_stays_in_its_pair():
    from paper_2501_19392_amd import binding as B
    x = torch.ones(1, 1, 128, device="cuda")
    x[0, 0, 3], x[0, 0, 100] = float("nan"), float("inf")
    out = torch.empty_like(x)
    one = torch.full((1, 16), 0.5, device="cuda")
    B.aquakv_rotary(x, torch.zeros(1, dtype=torch.int32, device="cuda"), one, one, 32, "half", out)
    torch.cuda.synchronize()
    bad = (~torch.isfinite(out[0, 0])).nonzero().view(-1).tolist()
    assert bad == [3, 19, 100]


@pytest.mark.parametrize("rows,first,dim,base,scaling,magnitude", [
    (1, 0, 128, 1e4, {}, 1.0), (1000, 0, 128, 5e5, {}, 1.0), (777, 130000, 64, 1e4, dict(factor=4.0), 1.25), (513, 5, 16, 1e6, {}, 1.0),
    (4099, 100000, 128, 5e5, dict(factor=8.0, original_len=8192.0, low_turns=1.0, high_turns=4.0), 1.0),
    (300, 1 << 20, 48, 1e4, dict(factor=32.0, original_len=4096.0, low_turns=1.0, high_turns=32.0), 1.3466), (9, (1 << 31) - 10, 96, 1e4, {}, 1.0)])
def test_tables(rows, first, dim, base, scaling, magnitude):
    from paper_2501_19392_amd import binding as B
    cos, sin = (torch.full((rows + 1, dim // 2), 7.0, device="cuda") for _ in range(2))
    B.aquakv_rotary_tables(cos[:rows], sin[:rows], base, first=first, magnitude=magnitude, **scaling)
    torch.cuda.synchronize()
    assert (cos[rows] == 7.0).all() and (sin[rows] == 7.0).all()
    w = base ** (-torch.arange(0, dim, 2, dtype=torch.float64) / dim)
    k = torch.zeros_like(w)
    if scaling.get("original_len"):
        k = ((scaling["original_len"] * w / (2 * math.pi) - scaling["low_turns"]) / (scaling["high_turns"] - scaling["low_turns"])).clamp(0, 1)
    w = w * (k + (1 - k) / scaling.get("factor", 1.0))
    angle = (torch.arange(rows, dtype=torch.float64) + first)[:, None] * w[None]
    # the angle: a few roundings of 64 bits on both sides; what is left of it beyond a quarter, at most pi / 4, rounded to fp32; a series evaluated
    # with fused steps, whose last one rounds a result of at most 1 and whose others weigh less than that again; the product with the magnitude
    bound = abs(magnitude) * (8 * 2.0 ** -53 * angle + 2.0 ** -24 * (math.pi / 4 + 1 + 1 + 1))
    for got, want in ((cos, angle.cos()), (sin, angle.sin())):
        off = (got[:rows].cpu().double() - magnitude * want).abs()
        assert (off <= bound).all(), (off / bound).max()


@pytest.mark.parametrize("dtype,layout,dim,in_place", [("bf16", "half", 64, False), ("fp32", "pairs", 128, True)])
def test_a_row_of_more_than_2_31_coordinates(dtype, layout, dim, in_place):
    """Heads from 2^24 on are found: every part of the row is, to the bit, what a call on that part alone gives, and what lies beside the rows is left."""
    from paper_2501_19392_amd import binding as B
    heads, beside, part = (1 << 24) + 5, 9, 1 << 21
    print(f"case rotary {dtype} {layout} heads={heads} in_place={in_place}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(3)
    wide = torch.empty(1, beside + heads + beside, 128, dtype=TYPES[dtype], device="cuda")
    for h in range(0, wide.shape[1], part):
        wide[:, h:h + part] = torch.randn(wide[:, h:h + part].shape, generator=gen, device="cuda")
    before = wide.clone()
    x = wide[:, beside:beside + heads]
    room = wide if in_place else torch.full_like(wide, 7.0)
    out = room[:, beside:beside + heads]
    angle = torch.rand(3, dim // 2, generator=gen, device="cuda") * 6.28
    cos, sin, positions = angle.cos(), angle.sin(), torch.tensor([2], dtype=torch.int32, device="cuda")
    B.aquakv_rotary(x, positions, cos, sin, dim, layout, out)
    torch.cuda.synchronize()
    for h in range(0, heads, part):
        source = before[:, beside + h:beside + min(h + part, heads)]
        want = torch.empty_like(source)
        B.aquakv_rotary(source, positions, cos, sin, dim, layout, want)
        assert torch.equal(out[:, h:h + part], want), h
    for edge in (slice(None, beside), slice(beside + heads, None)):
        assert torch.equal(room[:, edge], before[:, edge]) if in_place else (room[:, edge] == 7.0).all()
    if not in_place:
        assert torch.equal(wide, before)
    last = before[:, beside + heads - 1:beside + heads].cpu().double()
    want, size = rotated(last, cos[2:].cpu().double(), sin[2:].cpu().double(), dim, layout, False)
    bound = HALF_STEP[dtype] * want.abs() + (1 + HALF_STEP[dtype]) * 2.0 ** -24 * (size + want.abs())
    assert ((out[:, -1:].cpu().double() - want).abs() <= bound).all()
