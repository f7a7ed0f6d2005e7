"""Row operators on the GPU where their rules change over: sizes on both sides
of each variant's border, plans and gradients in the forms that a caller may
give them.  Tolerances as in test_gpu_rows.py, or derived beside the test.
"""

import numpy as np
import pytest
import torch

import test_gpu_rows as plain
from _gpu import DEV, say
from oracle import rows_ref as ref
from paper_2211_17111_amd import rows
from test_gpu_rows import BF16, F16, F32, TYPES, U, _half_step, _ids, _near, _normal, _np, _same_plan

pytestmark = pytest.mark.gpu


def test_counts_past_32_bits_are_refused():
    """The library takes experts and choices as 32-bit integers: larger ones must not arrive as their low bits."""
    wide = (1 << 32) + 5
    x, empty = _normal(3, 16), torch.empty((0, wide), dtype=F16, device=DEV)
    w, ids = torch.empty((0, 2), device=DEV), torch.empty((0, 2), dtype=torch.int32, device=DEV)
    many_w, many_ids = torch.empty((0, wide), device=DEV), torch.empty((0, wide), dtype=torch.int32, device=DEV)
    for f in (lambda: rows.route_forward(empty, 2), lambda: rows.route_forward(x[:0], wide),
              lambda: rows.route_forward(x, wide), lambda: rows.route_backward(w, empty, w, ids),
              lambda: rows.route_backward(many_w, x[:0], many_w, many_ids)):
        with pytest.raises(ValueError):
            f()
