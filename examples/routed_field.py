"""A field of small networks that a learned router chooses between: trained, then served with weights in 8 bits.

A network grid sends every point to the network of its cell.  Here the choice is learned instead: a router scores the networks
for a point's encoding, the best ``k`` evaluate it, and their results are summed with the router's weights.  One training step
is ``route``, two ``grouped_linear`` layers, ``combine`` and the gradients of all of them; serving runs the same layers through
``quantize_f8`` / ``grouped_linear_f8`` on weights that were brought to 8 bits once.

Lean training keeps the layers' inputs in 8 bits until the backward pass (``save_f8``, ``grouped_linear_backward_saved``), and adds the
router's balance losses to what is learned (``route_balance``).  An ``Adapter`` fits a trained field's last layer to a
variant of what it learned by a low-rank product per network, beside that layer's mean weights (``adapted_linear``).

    python examples/routed_field.py [--steps N] [--lean]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2103_13744_amd as kn  # noqa: E402

EXPERTS, K, HIDDEN, OUT, FREQUENCIES, RANK = 16, 2, 128, 8, 6, 8
SCALE = 1024.0  # of losses before their gradients are taken
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


class Adam:
    """First and second moments of parameters that are float32."""

    def __init__(self, params):
        self.params, self.moments, self.step_no = params, {n: (torch.zeros_like(p), torch.zeros_like(p)) for n, p in params.items()}, 0

    def step(self, grads, rate):
        self.step_no += 1
        for name, param in self.params.items():
            g, (m, v) = grads[name], self.moments[name]
            m.mul_(0.9).add_(g, alpha=0.1)
            v.mul_(0.99).addcmul_(g, g, value=0.01)
            param.addcdiv_(m / (1.0 - 0.9 ** self.step_no), (v / (1.0 - 0.99 ** self.step_no)).sqrt_().add_(1e-12), value=-rate)


class RoutedField:
    def __init__(self, seed=0, lean=False):
        g = torch.Generator(device="cuda").manual_seed(seed)
        randn = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
        self.params = {"router": 0.1 * randn(INPUTS, EXPERTS), "w1": randn(EXPERTS, INPUTS, HIDDEN) * math.sqrt(2.0 / INPUTS),
                       "b1": torch.zeros(EXPERTS, HIDDEN, device="cuda"), "w2": randn(EXPERTS, HIDDEN, OUT) / math.sqrt(HIDDEN),
                       "b2": torch.zeros(EXPERTS, OUT, device="cuda")}
        self.adam = Adam(self.params)
        self.lean, self.losses = lean, torch.tensor([1e-2, 1e-3], device="cuda") * SCALE  # (weights of the router's losses)
        self.eight = None

    def forward(self, enc):
        """Results of encoded points, and what the backward pass needs."""
        p = {n: v.to(DTYPE) for n, v in self.params.items() if n != "router"}
        x, logits = enc.to(DTYPE), enc @ self.params["router"]
        weights, ids, slots, rows, offsets = kn.route(logits, K)
        hidden = kn.grouped_linear(x, p["w1"], offsets, rows=rows, bias=p["b1"], relu=True)
        y = kn.grouped_linear(hidden, p["w2"], offsets, bias=p["b2"])
        return kn.combine(y, slots, weights), (p, x, logits, weights, ids, slots, rows, offsets, hidden, y)

    def gradients(self, enc, want):
        """The mean squared error, and its gradients (lean: with the router's losses, from inputs that were kept in 8 bits)."""
        out, (p, x, logits, weights, ids, slots, rows, offsets, hidden, y) = self.forward(enc)
        if self.lean:  # the layers' inputs are not needed any more
            x, hidden = kn.save_f8(x), kn.save_f8(hidden)
        diff = out.float() - want
        dout = (2.0 / diff.numel() * SCALE * diff).to(DTYPE)  # (scaled: gradients of a mean are small in 16 bits)
        dy, dweights = kn.combine_backward(dout, y, slots, weights)
        dlogits = kn.route_backward(logits, weights, ids, dweights)
        if self.lean:
            dhidden, dw2, db2 = kn.grouped_linear_backward_saved(dy, *hidden, p["w2"], offsets, relu_in=True)
            dw1, db1 = kn.grouped_linear_dw_saved(dhidden, *x, p["w1"], offsets, rows=rows)
            _, counts, _ = kn.route_balance(logits, K, offsets)
            dlogits = kn.route_balance_backward(logits, K, counts, self.losses, add=dlogits)
        else:
            dhidden, dw2, db2 = kn.grouped_linear_backward(dy, hidden, p["w2"], offsets, relu_in=True)
            dw1, db1 = kn.grouped_linear_dw(dhidden, x, p["w1"], offsets, rows=rows)
        grads = {"router": enc.t() @ dlogits, "w1": dw1, "b1": db1, "w2": dw2, "b2": db2}
        return diff.square().mean(), {n: g.float() / SCALE for n, g in grads.items()}

    def train_step(self, enc, want, rate=3e-3):
        """One step of Adam; the mean squared error before it."""
        loss, grads = self.gradients(enc, want)
        self.adam.step(grads, rate)
        self.eight = None
        return loss

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


class Adapter:
    """A variant of a trained field: its last layer is the mean of the networks' with a low-rank product of each one's own, which alone is trained."""

    def __init__(self, field, rank=RANK, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.field, self.w, self.bias = field, field.params["w2"].mean(0).to(DTYPE), field.params["b2"].mean(0).to(DTYPE)
        self.scales = torch.full((EXPERTS,), 2.0, device="cuda")
        self.params = {"a": torch.randn((EXPERTS, HIDDEN, rank), generator=g, device="cuda") / math.sqrt(HIDDEN), "b": torch.zeros(EXPERTS, rank, OUT, device="cuda")}
        self.adam = Adam(self.params)

    def forward(self, enc):
        _, (_, _, _, weights, _, slots, _, offsets, hidden, _) = self.field.forward(enc)
        layer = (self.w, self.params["a"].to(DTYPE), self.params["b"].to(DTYPE), offsets)
        y, h = kn.adapted_linear(hidden, *layer, scales=self.scales, bias=self.bias, want_h=True)
        return kn.combine(y, slots, weights), (hidden, h, layer, weights, slots, y)

    def gradients(self, enc, want):
        out, (hidden, h, layer, weights, slots, y) = self.forward(enc)
        diff = out.float() - want
        dy, _ = kn.combine_backward((2.0 / diff.numel() * SCALE * diff).to(DTYPE), y, slots, weights)
        _, da, db = kn.adapted_linear_backward(dy, hidden, h, *layer, scales=self.scales)
        return diff.square().mean(), {"a": da.float() / SCALE, "b": db.float() / SCALE}

    def train_step(self, enc, want, rate=1e-2):
        loss, grads = self.gradients(enc, want)
        self.adam.step(grads, rate)
        return loss


def main(steps=400, batch=8192, say=print, lean=False):
    """Trains for so many steps; (loss at the start, at the end, of the field served in 8 bits)."""
    kn.load_library()
    g = torch.Generator(device="cuda").manual_seed(1)
    field, losses = RoutedField(lean=lean), []
    for i in range(steps):
        points = torch.rand((batch, 3), generator=g, device="cuda")
        losses.append(field.train_step(encode(points), target(points)))
        if i % max(1, steps // 8) == 0:
            say("step %4d  loss %.5f" % (i, float(losses[-1])))
    points = torch.rand((batch, 3), generator=g, device="cuda")
    full = float((field.forward(encode(points))[0].float() - target(points)).square().mean())
    eight = float((field.serve(encode(points)).float() - target(points)).square().mean())
    say("new points: loss %.5f in bfloat16, %.5f served in 8 bits" % (full, eight))
    adapter = Adapter(field)
    for i in range(steps // 2):
        points = torch.rand((batch, 3), generator=g, device="cuda")
        loss = adapter.train_step(encode(points), target(points.flip(1)))  # (the same field, seen from another side)
        if i % max(1, steps // 8) == 0:
            say("adapters, step %4d  loss %.5f" % (i, float(loss)))
    return float(losses[0]), full, eight


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=400)
    ap.add_argument("--lean", action="store_true", help="keep the layers' inputs in 8 bits, add the router's losses")
    args = ap.parse_args()
    main(args.steps, lean=args.lean)
