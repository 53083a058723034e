"""What the binding keeps of calls of several rows, as their sizes change from step to step."""
import numpy as np
import pytest
import torch

from tests.paged import DEV, Filled, bf16, device
from tests.rows import check_rows

pytestmark = pytest.mark.gpu


def test_sizes_that_are_different_each_step_are_not_all_kept():
    """Packed rows with another largest count and another window in each call."""
    f = Filled([700, 300], 1, 64, True, seed=1)
    q = bf16(f.rng.standard_normal((2, 2, 4, 128)))
    packed, starts = device(q).view(4, 4, 128), torch.tensor([0, 2, 4], dtype=torch.int32, device=DEV)
    for n in range(300):
        out, _ = f.cache.attend_rows(f.seqs, packed, rows=2 + n, starts=starts, window=100 + n // 2)
        assert len(f.seqs._workspace) <= 64
        if n % 100 == 99:
            check_rows(f, q, out.view(q.shape), [2, 2], window=100 + n // 2)
    assert np.isfinite(out.float().cpu().numpy()).all() and f.cache.status() == 0
