"""That the measure of tests/paged_rounding.py tells right from wrong, on the CPU: for the very inputs that the GPU is asked with, results in which a tile is lost or
counts twice, the mask is one token off, or nothing was written, are outside it."""
import pytest
import torch

from tests import paged_rounding as R


@pytest.mark.parametrize("case", R.CASES, ids=R.name)
def test_what_is_outside(case):
    built = R.build(case, "cpu")
    want, stated = R.results(built), R.results(built, rounded=True)
    assert R.outside(stated, want, stated) == ""
    e = R.errors(stated, want)
    assert 2.0 ** -10 < e.square().mean().sqrt() < 2.0 ** -8                # 2^-9 and a little: the rounding to bf16, and the operands'
    n = max(n for n, c in zip(case[3], built[6]) if c > 0)
    first = max(n - max(built[6]) - 64, 0) // 32 * 32                       # a tile that all rows see
    wrong = {"nothing": torch.zeros_like(want), "keys of other tokens": R.results(built, mixed=True)}
    if case[6] < 1:                                                         # (otherwise a few tokens have all the weight, and others may be lost)
        wrong.update({"a tile lost": R.results(built, hidden=(first, first + 32)), "a tile twice": R.results(built, doubled=(first, first + 32)),
                      "the last tokens lost": R.results(built, hidden=(n - (8 if n < 30000 else 32), n))})
        if n < 3000:                                                        # (of more tokens one is less than a row's rounding)
            wrong["a token less"] = R.results(built, later=-1)
    for what, got in wrong.items():
        size = want.norm(dim=-1)
        got = torch.where((size > 0)[..., None], got, 0)
        assert R.outside(got, want, stated) != "", what
