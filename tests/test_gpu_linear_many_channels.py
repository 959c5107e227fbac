"""More channels than one launch of the int8 linear layer takes."""
import numpy as np
import pytest
import torch

from paper_2511_12653_amd import binding as fq

import _gpu_harness as H
import _operators_ref as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m,codes", [(1, False), (2, True), (17, False), (17, True)])
@pytest.mark.parametrize("ws_one", [False, True])
def test_more_channels_than_a_launch_takes(m, codes, ws_one):
    n, k = (1 << 27) + 21, 5
    H.say("linear, %d x %d x %d, codes %s" % (m, n, k, codes))
    gen = torch.Generator(device="cuda").manual_seed(m)
    x, s = torch.randn((m, k), generator=gen, device="cuda").to(torch.float16), None
    if codes:
        x = torch.randint(-127, 128, (m, k), generator=gen, device="cuda", dtype=torch.int8)
        s = torch.rand(m, generator=gen, device="cuda") + 0.5
    w = torch.randint(-127, 128, (n, k), generator=gen, device="cuda", dtype=torch.int8)
    ws, b = (torch.rand(1 if i == 0 and ws_one else n, generator=gen, device="cuda") * 1e-3 for i in range(2))
    y = torch.full((m, n), float("nan"), dtype=torch.float16, device="cuda")
    d = fq.FqLinear.from_torch(x, w, ws, y, bias=b, x_scale=s)
    fq.fq_linear_forward(d, torch.empty(fq.fq_linear_workspace_bytes(d), dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    xq, xs = (x.cpu().numpy(), s.cpu().numpy()) if codes else R.quantize_rows(x.cpu().numpy())
    for part in (slice(0, 300), slice((1 << 26) - 150, (1 << 26) + 150), slice((1 << 27) - 150, n)):
        scale = ws.expand(n)[part].cpu().numpy()
        want, off = R.linear(xq, xs, w[part].cpu().numpy(), scale, b[part].cpu().numpy(), True)
        R.check_linear(y[:, part].cpu().numpy(), want, off, True, "channels %d to %d" % (part.start, part.stop))
    assert not bool(y.isnan().any())
