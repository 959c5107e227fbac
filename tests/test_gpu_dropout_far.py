"""fq_dropout at its largest extent, in which a side of its grid would have 2^32 threads."""
import numpy as np
import pytest
import torch

from paper_2511_12653_amd import binding as fq

import _more_operators_ref as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [(1 << 34) - 5, (1 << 34) + 2049, 1 << 35])
def test_every_run_is_reached(n):
    """Up to 69 GB of FP16, in place; runs at both ends, at the borders of what a launch has along x, and of 32 bits are looked at."""
    x = torch.ones(n, device="cuda", dtype=torch.float16)
    fq.fq_dropout(fq.FqDropout.from_torch(x, x, 0.5, 11, 4))
    for begin in (0, (1 << 32) - 4096, 1 << 32, (1 << 34) - 6144, 1 << 34, (1 << 34) + 2048, 3 << 33, (n - 4096) // 4096 * 4096):
        count = min(4096, n - begin)
        if count > 0 and begin >> 32 == (begin + count - 1) >> 32:
            assert np.array_equal(x[begin:begin + count].cpu().numpy() != 0, R.keep(count, 0.5, 11, 4, begin)), begin
    tail = min(2000, n % 4096 or 2000)
    assert np.array_equal(x[n - tail:].cpu().numpy() != 0, R.keep(tail, 0.5, 11, 4, n - tail))
    assert bool((x[::65537].float() * (x[::65537].float() - 2) == 0).all())          # 0 or 1 / (1 - p): none was left as it was
