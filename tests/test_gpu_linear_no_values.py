"""fq_linear_forward of rows without a value, or with fewer than a vector: y is the bias, or what the values give, whatever the
workspace held before."""
import numpy as np
import pytest
import torch

from paper_2511_12653_amd import binding as fq

import _gpu_harness as H
import _operators_ref as R

pytestmark = pytest.mark.gpu

# bytes of which 16 and 32 bits are a NaN, an infinity of FP16 (a NaN with what lies beside it), a large and a small number
FILLS = [0xFF, 0x7C, 0x7F, 0x00]


def forward(x, w, ws, b, fill, y_type):
    y = torch.full((x.shape[0], w.shape[0]), 7.0, dtype=y_type, device="cuda")
    d = fq.FqLinear.from_torch(x, w, ws, y, bias=b)
    work = torch.full((fq.fq_linear_workspace_bytes(d),), fill, dtype=torch.uint8, device="cuda")
    fq.fq_linear_forward(d, work)
    torch.cuda.synchronize()
    return y.cpu().numpy()


@pytest.mark.parametrize("m,n", [(1, 5), (5, 7), (17, 40), (300, 20), (2000, 300)])
@pytest.mark.parametrize("x_type", [torch.float16, torch.float32])
@pytest.mark.parametrize("fill", FILLS)
def test_no_values(m, n, x_type, fill):
    H.say("linear %d x %d x 0, workspace of 0x%02x" % (m, n, fill))
    rng = np.random.Generator(np.random.Philox(m + n))
    b = rng.standard_normal(n).astype(np.float32)
    x, w = torch.empty((m, 0), dtype=x_type, device="cuda"), torch.empty((n, 0), dtype=torch.int8, device="cuda")
    ws = torch.full((n,), 2.0, device="cuda")
    for bias, want in ((H.dev(b), b), (None, np.zeros(n, np.float32))):
        assert np.array_equal(forward(x, w, ws, bias, fill, torch.float32), np.broadcast_to(want, (m, n)))
        assert np.array_equal(forward(x, w, ws, bias, fill, torch.float16), np.broadcast_to(want.astype(np.float16), (m, n)))


@pytest.mark.parametrize("m", [1, 20, 300])
@pytest.mark.parametrize("k", [1, 2, 7, 8, 9])
@pytest.mark.parametrize("x_type", [np.float16, np.float32])
@pytest.mark.parametrize("fill", FILLS)
def test_fewer_values_than_a_vector(m, k, x_type, fill):
    H.say("linear %d x 30 x %d, workspace of 0x%02x" % (m, k, fill))
    rng = np.random.Generator(np.random.Philox(m * 16 + k))
    x, w = rng.standard_normal((m, k)).astype(x_type), rng.integers(-127, 128, (30, k)).astype(np.int8)
    ws, b = rng.uniform(1e-3, 2e-3, 30).astype(np.float32), rng.standard_normal(30).astype(np.float32)
    got = forward(H.dev(x), H.dev(w), H.dev(ws), H.dev(b), fill, torch.float32)
    q, s = R.quantize_rows(x)
    y, off = R.linear(q, s, w, ws, b, False)
    R.check_linear(got, y, off, False, "%d x 30 x %d" % (m, k))
