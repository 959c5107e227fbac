"""Train a small fake-quantized network with AdamW, then serve it in int8.

    python examples/qat_linear.py [--steps 300] [--states float8]

Training: two linear layers whose weights (a scale per output channel) and inputs (one scale per layer) go through
`fake_quantize`; weights, biases and all scale parameters are stepped by `AdamW` with its moments in 8 bits.  Serving: the
weights' codes and scales by `fq_forward`, the layers by `linear_int8`, once with the learned scales of the inputs (the
very values of training, up to rounding) and once with inputs quantized token by token (nothing is clipped then: the values of
a network whose inputs are not quantized, up to half a code step).
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2511_12653_amd import AdamW, binding as fq, fake_quantize, linear_int8  # noqa: E402

QMIN, QMAX = -127, 127


def theta_of(scale):
    """The parameter whose softplus is `scale`."""
    return torch.log(torch.expm1(scale.double())).float()


class QuantizedLinear(torch.nn.Module):
    def __init__(self, k, n, reach):
        super().__init__()
        self.weight = torch.nn.Parameter(torch.randn(n, k, device="cuda") * math.sqrt(2.0 / k))
        self.bias = torch.nn.Parameter(torch.zeros(n, device="cuda"))
        self.theta_w = torch.nn.Parameter(theta_of(self.weight.detach().abs().amax(1) / QMAX))
        self.theta_x = torch.nn.Parameter(theta_of(torch.full((1,), reach / QMAX, device="cuda")))

    def forward(self, x, quantize_input=True):
        w = fake_quantize(self.weight, self.theta_w, QMIN, QMAX, channel_dim=0)
        return torch.addmm(self.bias, fake_quantize(x, self.theta_x, QMIN, QMAX) if quantize_input else x, w.t())

    def codes(self, values, theta, channels):
        """int8 codes and scales of a tensor, as serving keeps them."""
        values = values.detach().contiguous()
        q, s = torch.empty(values.shape, dtype=torch.int8, device="cuda"), torch.empty(channels, device="cuda")
        fq.fq_forward(fq.FqTensor.from_torch(1, channels, values.numel() // channels, QMIN, QMAX, x=values, q=q, theta=theta.detach(), s=s))
        return q, s

    def freeze(self):
        self.w_codes, self.w_scale = self.codes(self.weight, self.theta_w, self.weight.shape[0])
        return self

    def serve(self, x, by_token):
        if by_token:
            return linear_int8(x, self.w_codes, self.w_scale, self.bias.detach(), out_dtype=torch.float32)
        q, s = self.codes(x, self.theta_x, 1)
        return linear_int8(q, self.w_codes, self.w_scale, self.bias.detach(), x_scale=s, out_dtype=torch.float32)


def main(steps=300, states="float8", width=384, tokens=2048, seed=0):
    torch.manual_seed(seed)
    first, last = QuantizedLinear(64, width, 4.0), QuantizedLinear(width, 16, 4.0)
    net = lambda x: last(torch.relu(first(x)))      # noqa: E731
    teacher = torch.nn.Sequential(torch.nn.Linear(64, 128), torch.nn.Tanh(), torch.nn.Linear(128, 16)).cuda().requires_grad_(False)
    layers = (first, last)
    optimizer = AdamW([{"params": [m.weight for m in layers], "weight_decay": 1e-2},
                       {"params": [p for m in layers for p in (m.bias, m.theta_w, m.theta_x)], "weight_decay": 0.0}],
                      lr=2e-3, states=states, seed=seed)
    losses = []
    for _ in range(steps):
        x = torch.randn(tokens, 64, device="cuda")
        loss = (net(x) - teacher(x)).square().mean()
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        losses.append(loss.detach())
    losses = torch.stack(losses).cpu()

    with torch.no_grad():
        x = torch.randn(tokens, 64, device="cuda")
        for m in layers:
            m.freeze()
        off = {}
        for name, by_token in (("learned scales", False), ("scales by token", True)):
            want = last(torch.relu(first(x, not by_token)), not by_token)
            y = last.serve(torch.relu(first.serve(x, by_token)), by_token)
            off[name] = float((y - want).norm() / want.norm())
    print("loss %.4f -> %.4f (%s moments)" % (losses[0], losses[-10:].mean(), states))
    for name, value in off.items():
        print("int8, %s: %.2e of the norm from the float product" % (name, value))
    return losses, off


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=300)
    ap.add_argument("--states", choices=("float8", "float32"), default="float8")
    main(**vars(ap.parse_args()))
