"""Dropout of more blocks of the generator than one launch has threads."""
import numpy as np
import pytest
import torch

from oracle import tokens as T
from paper_2002_06015_amd import kfac, workloads as wl

pytestmark = pytest.mark.gpu


def test_more_units_than_threads_of_a_launch():
    """2^31 + 5 rows of one element that lie apart: each takes two units of work, 2^32 + 10 in all.  In place, 8 GiB."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    rows, p, seed, offset = (1 << 31) + 5, 0.5, 21, 4
    t = torch.ones(rows, 2, dtype=torch.bfloat16, device="cuda")
    ctx = kfac.Context([wl.fc_layer(1, 4, 4)], workspace_bytes=256)
    kfac.kfac_dropout(ctx, t[:, :1], p, seed, offset, t[:, :1])
    torch.cuda.synchronize()
    for first in (0, 1 << 30, (1 << 31) - 24, rows - 40):
        keep = T.dropout_keep(first, 40 if first + 40 <= rows else rows - first, p, seed, offset)
        assert np.array_equal(t[first:first + 40, 0].float().cpu().numpy(), 2.0 * keep)
    for part in t.split(1 << 28):                                              # every element is a zero or twice what it was
        assert bool(((part[:, 0] == 0) | (part[:, 0] == 2)).all()) and bool((part[:, 1] == 1).all())
    ctx.close()
