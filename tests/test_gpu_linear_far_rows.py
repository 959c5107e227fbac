"""Rows of w so far apart that their offsets pass 32 bits, with few tokens; and short rows of few tokens against more channels than
are on the chip at once."""
import numpy as np
import pytest
import torch

from paper_2511_12653_amd import binding as fq

import _gpu_harness as H
import _operators_ref as R

pytestmark = pytest.mark.gpu


def check(m, n, k, kind, w_pitch, label):
    H.say(label)
    rng = np.random.Generator(np.random.Philox(m * 1000 + k))
    x, w = rng.standard_normal((m, k)).astype(kind), rng.integers(-127, 128, (n, k)).astype(np.int8)
    ws, b = rng.uniform(1e-3, 2e-3, n).astype(np.float32), rng.standard_normal(n).astype(np.float32)
    wd = torch.as_strided(torch.empty((n - 1) * w_pitch + k, dtype=torch.int8, device="cuda"), (n, k), (w_pitch, 1))
    wd.copy_(H.dev(w))
    y = torch.full((m, n), 7.0, device="cuda")
    d = fq.FqLinear.from_torch(H.dev(x), wd, H.dev(ws), y, bias=H.dev(b))
    work = torch.empty(fq.fq_linear_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    fq.fq_linear_forward(d, work)
    torch.cuda.synchronize()
    q, s = R.quantize_rows(x)
    want, off = R.linear(q, s, w, ws, b, False)
    R.check_linear(y.cpu().numpy(), want, off, False, label)


# 15 * 300000000 is past 2^32; the second pitch is no whole number of words (rows are laid out anew then, where they are long)
@pytest.mark.parametrize("pitch", [300000000, 300000001])
@pytest.mark.parametrize("m,k", [(1, 512), (3, 512), (16, 500), (3, 64), (3, 513), (3, 9)])
@pytest.mark.parametrize("kind", [np.float16, np.float32])
def test_rows_of_w_beyond_32_bits(m, k, kind, pitch):
    check(m, 16, k, kind, pitch, "linear %d x 16 x %d, rows of w %d apart" % (m, k, pitch))


@pytest.mark.parametrize("m", [1, 5, 16])
@pytest.mark.parametrize("n,k,pitch", [(8193, 512, 512), (8200, 16, 16), (16390, 130, 144), (8300, 500, 516), (30000, 96, 96), (9000, 255, 255)])
@pytest.mark.parametrize("kind", [np.float16, np.float32])
def test_many_channels_and_short_rows(m, n, k, pitch, kind):
    check(m, n, k, kind, pitch, "linear %d x %d x %d, rows of w %d apart" % (m, n, k, pitch))
