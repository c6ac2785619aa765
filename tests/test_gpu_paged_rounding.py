"""Attention over pages in bf16 layers is off by the roundings that it states and by no more: by these, a tile that is lost or counts twice, a mask that is one token off
or keys of other tokens show (tests/test_paged_rounding.py, on the same inputs)."""
import numpy as np
import pytest
import torch

from tests import paged_rounding as R
from tests.test_gpu_paged import attend, need_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("case", R.CASES, ids=R.name)
def test_errors_are_those_of_the_stated_roundings(case):
    need_gpu()
    print(f"case {R.name(case)}", flush=True)
    built = R.build(case, "cuda")
    lo, lg, pages, table, lens, q, counts, scale = built
    start = None if isinstance(case[5], int) else torch.tensor([0, *np.cumsum(counts)], dtype=torch.int32, device="cuda")
    out = attend(lg, pages, table, lens, q, counts, scale, q_start=start).double().cpu()
    want, stated = R.results(built), R.results(built, rounded=True)
    e, s = R.errors(out, want), R.errors(stated, want)
    print(f"  rms {e.square().mean().sqrt().item():.3g}, stated {s.square().mean().sqrt().item():.3g}; largest {e.max().item():.3g}, {s.max().item():.3g}", flush=True)
    assert R.outside(out, want, stated) == ""
