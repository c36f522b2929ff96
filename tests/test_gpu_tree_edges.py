"""Edges of the calls in include/mkv_tree.h that their other GPU tests leave
out, against the plain 64-bit forms of tests/tree_ref.py.

Bound: the kernel divides by the sum of its rounded weights, so its bound is
the one of Case.check(own_sum=True), everywhere here."""
import numpy as np
import pytest
import torch

import tree_ref as R
from paper_2606_01563_gb300 import mkv
from gpu_util import host
from test_gpu_tree import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("b,n,rows", [(32, 13, 1000), (40, 8, 900), (2, 20, 6000)])
def test_one_slot_of_moments_in_a_ring_of_six(b, n, rows):
    """16-bit moments with one row block shift the ring by an odd number before an item's last tiles: whole items and
    runs, many CTAs at once (copies late and out of order), the same bits in every call."""
    c = Case(b + n, b=b, h=8, g=4, d=128, n=n, rows=rows, c="bf16", ragged=True).device()
    c.step()
    first, lse = c.out.clone(), c.lse.clone()
    for _ in range(40):
        c.step()
        assert torch.equal(c.out, first) and torch.equal(c.lse, lse)
    c.check(own_sum=True)
