"""fq_adapters_forward where tiles are of 16 tokens and channels are many, so that wavefronts take 64 of them at a time: all ranks, full and odd tiles, with FP32
outputs, in which the second FP16 number of each t shows; against the plain implementation in 64 bits."""
import numpy as np
import pytest

from test_gpu_adapters import case, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rank", [1, 4, 7])
@pytest.mark.parametrize("m,k,n,count", [(16, 96, 4096, 32), (27, 64, 7953, 10), (48, 256, 4096, 32), (64, 40, 11008, 64), (256, 64, 4099, 1), (512, 48, 8192, 8), (512, 24, 4096, 64),
                                         (1000, 32, 4102, 3), (2000, 8, 4096, 4)])
def test_less_than_eight_ranks(m, k, n, count, rank):
    for x_type, order in ((np.float16, "mixed"), (np.int8, "runs"), (np.float32, "mixed")):
        check(case(m, k, n, count, rank, x_type, np.float32, m + rank, order), np.float32, "%s %s" % (x_type.__name__, order))


@pytest.mark.parametrize("rank", [8, 13, 32, 33, 60, 64, 65, 100, 128, 129, 200, 256])
@pytest.mark.parametrize("m,n,count", [(48, 4096, 32), (150, 7954, 5)])
def test_eight_ranks_and_more(m, n, count, rank):
    for x_type, base_type in ((np.float16, np.float32), (np.int8, np.float16)):
        check(case(m, 64, n, count, rank, x_type, base_type, m + rank), np.float32, x_type.__name__)


@pytest.mark.parametrize("rank", [3, 40, 100, 256])
def test_in_place_and_rows_apart(rank):
    c = case(70, 72, 4101, 40, rank, np.float16, np.float32, rank)
    check(c, np.float32, in_place=True, pitch=3, shift=1)
    check(c, np.float32, pitch=5)
    check(dict(c, base=None), np.float32)
