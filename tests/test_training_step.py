"""The operators of training and fine-tuning together, as they are used: a router with its balance losses, a layer whose inputs are kept in 8 bits, a shared layer
with adapters, the weighted sum, and all gradients, against a plain implementation in 64 bits.

Bounds: each quantity is a chain of at most eight fp32 sums of at most 300 terms, each of which is off by (300 + 8) 2^-23 of the sum of its terms' magnitudes; those sums are
below 16 times the largest result for these inputs' signs at random (300 terms: 300 / sqrt(300) = 17).  So 2^-8 of the largest value would hold with
certainty; errors of random signs add up like their square root, 2^-12.  What is kept is taken as it is (the same bits as by hand: test_saved.py)."""
import math

import pytest
import torch

import paper_2103_13744_amd as kn

from .test_experts import dev, rand
from .test_saved import kept

T, E, K, D, H, N, R = 300, 6, 2, 40, 72, 24, 4


def inputs():
    return dict(x=rand(1, T, D), wr=rand(2, D, E) / math.sqrt(D), w1=rand(3, E, D, H) / math.sqrt(D), b1=0.1 * rand(4, E, H), w2=rand(5, H, N) / math.sqrt(H),
                a=rand(6, E, H, R) / math.sqrt(H), b=rand(7, E, R, N), s=0.5 + torch.rand(E, generator=torch.Generator().manual_seed(8)), dout=rand(9, T, N),
                dlosses=torch.tensor([0.3 * T, 0.1 * T]))


def step(v):
    logits = v["x"] @ v["wr"]
    weights, ids, slots, rows, off = kn.route(logits, K)
    losses, counts, _ = kn.route_balance(logits, K, off)
    hidden = kn.grouped_linear(v["x"], v["w1"], off, rows=rows, bias=v["b1"], relu=True)
    qx, ex = kn.save_f8(v["x"])
    qh, eh = kn.save_f8(hidden)
    y, h = kn.adapted_linear(hidden, v["w2"], v["a"], v["b"], off, scales=v["s"], want_h=True)
    out = kn.combine(y, slots, weights)
    # backward: the layer's inputs are those that were kept
    dy, dweights = kn.combine_backward(v["dout"], y, slots, weights)
    back = kn.restore_f8(qh, eh, H, torch.float32)
    dh, da, db = kn.adapted_linear_backward(dy, back, h, v["w2"], v["a"], v["b"], off, scales=v["s"], relu_in=True)
    dxr, dw1, db1 = kn.grouped_linear_backward_saved(dh, qx, ex, v["w1"], off, rows=rows)
    dlogits = kn.route_balance_backward(logits, K, counts, v["dlosses"], add=kn.route_backward(logits, weights, ids, dweights))
    return dict(out=out, losses=losses, dx=kn.combine(dxr, slots), dlogits=dlogits, dw1=dw1, db1=db1, da=da, db=db), (ids, hidden)


def reference(v, ids, hidden):
    """In 64 bits; the choice of networks and the kept values are the step's own."""
    d = {n: t.double() for n, t in v.items()}
    logits = d["x"] @ d["wr"]
    top = logits.gather(1, ids)
    w = torch.softmax(top, 1)
    p = torch.softmax(logits, 1)
    counts = torch.bincount(ids.reshape(-1), minlength=E).double()
    z = torch.logsumexp(logits, 1)
    losses = torch.stack([E * (counts / (K * T) * p.mean(0)).sum(), z.square().mean()])
    kx, kh = kept(v["x"])[2], kept(hidden)[2]
    out, dx = torch.zeros(T, N, dtype=torch.float64), torch.zeros(T, D, dtype=torch.float64)
    dw1, db1, da, db = (torch.zeros_like(d[n]) for n in ("w1", "b1", "a", "b"))
    dweights = torch.zeros(T, K, dtype=torch.float64)
    off = torch.cat([torch.zeros(1), counts.cumsum(0)]).long()
    order = torch.sort(ids.reshape(-1), stable=True).indices
    for e in range(E):
        pairs = order[off[e]:off[e + 1]]
        t, wt = pairs // K, w.reshape(-1)[pairs][:, None]
        h1 = (d["x"][t] @ d["w1"][e] + d["b1"][e]).clamp(min=0.0)
        low = d["s"][e] * (h1 @ d["a"][e])
        y = h1 @ d["w2"] + low @ d["b"][e]
        out.index_add_(0, t, wt * y)
        g = d["dout"][t]
        dweights.reshape(-1)[pairs] = (g * y).sum(1)
        dy = wt * g
        gl = d["s"][e] * (dy @ d["b"][e].T)
        h8 = kh[off[e]:off[e + 1]]
        dh = (dy @ d["w2"].T + gl @ d["a"][e].T) * (h8 > 0)
        da[e], db[e] = h8.T @ gl, low.T @ dy
        dw1[e], db1[e] = kx[t].T @ dh, dh.sum(0)
        dx.index_add_(0, t, dh @ d["w1"][e].T)
    dl = torch.zeros(T, E, dtype=torch.float64).scatter_(1, ids, w * (dweights - (w * dweights).sum(1, keepdim=True)))
    share = E * counts / (K * T * T)
    dl += p * (d["dlosses"][0] * (share - (p @ share)[:, None]) + d["dlosses"][1] * 2.0 / T * z[:, None])
    return dict(out=out, losses=losses, dx=dx, dlogits=dl, dw1=dw1, db1=db1, da=da, db=db)


@pytest.mark.gpu
def test_a_training_step():
    v = inputs()
    got, (ids, hidden) = step({n: dev(t) for n, t in v.items()})
    want = reference(v, ids.cpu().long(), hidden.cpu())
    for name, ref in want.items():
        off = float((got[name].double().cpu() - ref).abs().max())
        assert got[name].dtype == torch.float32 and off <= 2.0 ** -12 * float(ref.abs().max()), (name, off, float(ref.abs().max()))


@pytest.mark.gpu
def test_a_training_step_in_a_graph():
    """Captured and replayed with the program's own work between: the eager bits."""
    v = {n: dev(t) for n, t in inputs().items()}
    want = {n: t.clone() for n, t in step(v)[0].items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(v)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got, _ = step(v)
    for i in range(4):
        for t in got.values():
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(got[n], want[n]) for n in want), i
        again, _ = step(v)
        assert all(torch.equal(again[n], want[n]) for n in want)


def example():
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "routed_field.py")
    spec = importlib.util.spec_from_file_location("routed_field", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.gpu
def test_the_example_runs_lean_and_with_adapters():
    m = example()
    said = []
    first, full, eight = m.main(steps=8, batch=500, say=said.append, lean=True)
    assert all(math.isfinite(v) for v in (first, full, eight)) and any("adapters" in line for line in said)


@pytest.mark.gpu
def test_the_examples_lean_gradients():
    """A kept value is within 2^-4 of the input (or, for the smallest, 2^-9 of a two-hundred-and-fortieth of its block's largest), and has its sign: the biases' gradients
    are the same bits, and each of the weights' within that share of the sum of its terms' magnitudes, and two roundings to bfloat16 and the sums'."""
    m = example()
    points = torch.rand((700, 3), generator=torch.Generator().manual_seed(1)).cuda()
    enc, want = m.encode(points), m.target(points)
    plain, lean = m.RoutedField(seed=3), m.RoutedField(seed=3, lean=True)
    lean.losses.zero_()
    (l1, g1), (l2, g2) = plain.gradients(enc, want), lean.gradients(enc, want)
    assert torch.equal(l1, l2) and torch.equal(g1["b1"], g2["b1"]) and torch.equal(g1["b2"], g2["b2"])
    assert ((g1["router"] - g2["router"]).abs() <= 2.0 ** -20 * g1["router"].abs().max()).all()
    out, (p, x, logits, weights, ids, slots, rows, off, hidden, y) = plain.forward(enc)
    diff = out.float() - want
    dy, _ = kn.combine_backward((2.0 / diff.numel() * m.SCALE * diff).to(m.DTYPE), y, slots, weights)
    dh = kn.grouped_linear_dx(dy, hidden, p["w2"], off, relu_in=True)
    for name, xs, d in (("w1", x[rows.long()], dh), ("w2", hidden, dy)):
        for e, (i, j) in enumerate(zip(off[:-1].tolist(), off[1:].tolist())):
            a, b = xs[i:j].double(), d[i:j].double().abs()
            far = torch.maximum(a.abs() * 2.0 ** -4, a.abs().amax(1, keepdim=True) * 2.0 ** -9 / 224.0)
            bound = (far.t() @ b + (j - i + 8) * 2.0 ** -22 * (a.abs().t() @ b)) / m.SCALE
            assert ((g1[name][e] - g2[name][e]).double().abs() <= 1.01 * bound + 2.0 ** -8 * (g1[name][e].abs() + g2[name][e].abs())).all()


@pytest.mark.gpu
def test_the_examples_adapter_gradients_against_differences():
    """The error along a direction, by central differences of 1 % of b: its gradient is smooth (the error is quadratic in b), and the rest is bfloat16's rounding of the results:
    2^-8 of each, half of them at random signs over 500 points of 8, so that a fiftieth of the gradient's own size is more than it can be off."""
    m = example()
    field = m.RoutedField(seed=2)
    adapter = m.Adapter(field)
    points = torch.rand((500, 3), generator=torch.Generator().manual_seed(1)).cuda()
    enc, want = m.encode(points), m.target(points.flip(1))
    adapter.params["b"].copy_(0.3 * rand(4, *adapter.params["b"].shape).cuda())
    _, grads = adapter.gradients(enc, want)
    way, b = grads["b"] / grads["b"].norm(), adapter.params["b"].clone()
    step, at = 0.5, []
    for sign in (1.0, -1.0):
        adapter.params["b"].copy_(b + sign * step * way)
        at.append(float((adapter.forward(enc)[0].float() - want).double().square().mean()))
    slope, said = (at[0] - at[1]) / (2 * step), float((grads["b"].double() * way.double()).sum())
    assert abs(slope - said) <= 0.02 * abs(said), (slope, said)
