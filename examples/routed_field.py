"""A field of small networks that a learned router chooses between: trained, then served with weights in 8 bits.

A network grid sends every point to the network of its cell.  Here the choice is learned instead: a router scores the networks
for a point's encoding, the best ``k`` evaluate it, and their results are summed with the router's weights.  One training step
is ``route``, two ``grouped_linear`` layers, ``combine`` and the gradients of all of them; serving runs the same layers through
``quantize_f8`` / ``grouped_linear_f8`` on weights that were brought to 8 bits once.

    python examples/routed_field.py [--steps N]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2103_13744_amd as kn  # noqa: E402

EXPERTS, K, HIDDEN, OUT, FREQUENCIES = 16, 2, 128, 8, 6
INPUTS = 3 + 6 * FREQUENCIES
DTYPE = torch.bfloat16  # of the networks' layers; the router and the master weights are float32


def encode(points):
    """Sines and cosines of the coordinates, as the networks of a scene take them."""
    waves = [f(points * 2.0 ** i * math.pi) for i in range(FREQUENCIES) for f in (torch.sin, torch.cos)]
    return torch.cat([points, *waves], dim=1)


def target(points):
    """What is to be learned: eight smooth channels whose character differs from one part of the cube to another."""
    x, y, z = points.unbind(1)
    side = torch.sigmoid(20.0 * (x - 0.5))
    a = torch.sin(9.0 * y + 4.0 * z) * side + torch.cos(13.0 * z) * (1.0 - side)
    b = torch.exp(-20.0 * ((points - 0.5) ** 2).sum(1))
    return torch.stack([a, b, a * b, side, y * z, torch.sin(6.0 * x), a - b, b * side], dim=1)


class RoutedField:
    def __init__(self, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        randn = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
        self.params = {"router": 0.1 * randn(INPUTS, EXPERTS), "w1": randn(EXPERTS, INPUTS, HIDDEN) * math.sqrt(2.0 / INPUTS),
                       "b1": torch.zeros(EXPERTS, HIDDEN, device="cuda"), "w2": randn(EXPERTS, HIDDEN, OUT) / math.sqrt(HIDDEN),
                       "b2": torch.zeros(EXPERTS, OUT, device="cuda")}
        self.moments = {n: (torch.zeros_like(p), torch.zeros_like(p)) for n, p in self.params.items()}
        self.step_no = 0
        self.eight = None

    def forward(self, enc):
        """Results of encoded points, and what the backward pass needs."""
        p = {n: v.to(DTYPE) for n, v in self.params.items() if n != "router"}
        x, logits = enc.to(DTYPE), enc @ self.params["router"]
        weights, ids, slots, rows, offsets = kn.route(logits, K)
        hidden = kn.grouped_linear(x, p["w1"], offsets, rows=rows, bias=p["b1"], relu=True)
        y = kn.grouped_linear(hidden, p["w2"], offsets, bias=p["b2"])
        return kn.combine(y, slots, weights), (p, x, logits, weights, ids, slots, rows, offsets, hidden, y)

    def train_step(self, enc, want, rate=3e-3):
        """One step of Adam on the mean squared error; the loss before it."""
        out, (p, x, logits, weights, ids, slots, rows, offsets, hidden, y) = self.forward(enc)
        diff = out.float() - want
        dout = (2.0 / diff.numel() * 1024.0 * diff).to(DTYPE)  # (scaled: gradients of a mean are small in 16 bits)
        dy, dweights = kn.combine_backward(dout, y, slots, weights)
        dhidden, dw2, db2 = kn.grouped_linear_backward(dy, hidden, p["w2"], offsets, relu_in=True)
        dw1, db1 = kn.grouped_linear_dw(dhidden, x, p["w1"], offsets, rows=rows)
        dlogits = kn.route_backward(logits, weights, ids, dweights)
        grads = {"router": enc.t() @ dlogits, "w1": dw1, "b1": db1, "w2": dw2, "b2": db2}
        self.step_no += 1
        for name, param in self.params.items():
            g, (m, v) = grads[name].float() / 1024.0, self.moments[name]
            m.mul_(0.9).add_(g, alpha=0.1)
            v.mul_(0.99).addcmul_(g, g, value=0.01)
            param.addcdiv_(m / (1.0 - 0.9 ** self.step_no), (v / (1.0 - 0.99 ** self.step_no)).sqrt_().add_(1e-12), value=-rate)
        self.eight = None
        return diff.square().mean()

    def serve(self, enc):
        """The same field from weights in 8 bits, which are made once."""
        if self.eight is None:
            self.eight = (kn.quantize_f8_weights(self.params["w1"]), kn.quantize_f8_weights(self.params["w2"]),
                          self.params["b1"].to(DTYPE), self.params["b2"].to(DTYPE))
        (w1, s1), (w2, s2), b1, b2 = self.eight
        weights, _, slots, rows, offsets = kn.route(enc @ self.params["router"], K)
        hidden = kn.grouped_linear_f8(*kn.quantize_f8(enc), w1, s1, offsets, rows=rows, bias=b1, relu=True, dtype=DTYPE)
        y = kn.grouped_linear_f8(*kn.quantize_f8(hidden), w2, s2, offsets, bias=b2, dtype=DTYPE)
        return kn.combine(y, slots, weights)


def main(steps=400, batch=8192, say=print):
    """Trains for so many steps; (loss at the start, at the end, of the field served in 8 bits)."""
    kn.load_library()
    g = torch.Generator(device="cuda").manual_seed(1)
    field, losses = RoutedField(), []
    for i in range(steps):
        points = torch.rand((batch, 3), generator=g, device="cuda")
        losses.append(field.train_step(encode(points), target(points)))
        if i % max(1, steps // 8) == 0:
            say("step %4d  loss %.5f" % (i, float(losses[-1])))
    points = torch.rand((batch, 3), generator=g, device="cuda")
    full = float((field.forward(encode(points))[0].float() - target(points)).square().mean())
    eight = float((field.serve(encode(points)).float() - target(points)).square().mean())
    say("new points: loss %.5f in bfloat16, %.5f served in 8 bits" % (full, eight))
    return float(losses[0]), full, eight


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=400)
    main(ap.parse_args().steps)
