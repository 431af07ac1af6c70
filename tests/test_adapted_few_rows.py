"""Adapters' input gradients of up to 64 rows: the low-rank part is summed from a g in 32 bits, which is held to one rounding of the result.

Bounds: g is a sum of n products in fp32, (n + 10) 2^-23 of the sum of their magnitudes, times the scale (2^-24 of it, within the same); dx a sum of n
products and of r products of g, (n + 8) and (r + 16) 2^-23 of their magnitudes, with g's error through |A|, and one rounding to the type."""
import math

import pytest
import torch

import paper_2103_13744_amd as kn

from .test_adapted import groups, make, within
from .test_experts import DT, dev, rand


def check_dx(dy, x, w, a, b, off, rows, s, relu, dx, dtype):
    xs, d, n, r = (x if rows is None else x[rows.long()]).double(), dy.double(), w.shape[1], a.shape[2]
    want, bound = d @ w.double().T, (n + 8) * 2.0 ** -23 * (d.abs() @ w.double().abs().T)
    for q, i, j in groups(off):
        g, mags = float(s[q]) * (d[i:j] @ b[q].double().T), float(s[q]) * (d[i:j].abs() @ b[q].double().abs().T)
        am = a[q].double().abs()
        want[i:j] += g @ a[q].double().T
        bound[i:j] += (n + 11) * 2.0 ** -23 * (mags @ am.T) + (r + 16) * 2.0 ** -23 * (g.abs() @ am.T)
    if relu:
        want, bound = want * (xs > 0), bound * (xs > 0)
    within(dx, want, 1.01 * bound, dtype)


SIZES = [(1, 1, 256, 200, 8), (5, 2, 2, 3, 2), (17, 3, 33, 65, 5), (33, 33, 64, 72, 8), (48, 20, 512, 264, 16), (64, 3, 130, 99, 21), (64, 64, 72, 1024, 40), (40, 3, 24, 1, 3)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_input_gradient_is_rounded_once(size, dtype):
    m, e, k, n, r = size
    for i, (how, gather, nk, relu) in enumerate([("even", False, False, True), ("tail", True, True, False), ("one", True, False, True)]):
        x, w, a, b, off, rows, s = make(m, e, k, n, r, dtype, how, gather, nk, 50 * m + i)
        dy = rand(11 + i, m, n).to(DT[dtype])
        args = (dev(w), dev(a), dev(b), dev(off))
        _, h = kn.adapted_linear(dev(x), *args, rows=dev(rows), scales=dev(s), want_h=True)
        dx, _, _ = kn.adapted_linear_backward(dev(dy), dev(x), h, *args, rows=dev(rows), scales=dev(s), relu_in=relu)
        check_dx(dy, x, w, a, b, off, rows, s, relu, dx, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("nk", [False, True])
@pytest.mark.parametrize("power", [(-10, -14, 12), (9, 9, -14)], ids=["below", "above"])
def test_g_beyond_the_range_of_half_precision(power, nk):
    """g of 2^-21 on average, where fp16 has steps of 2^-24, and of 2^21, where it has no values: the gradient is in range, and as exact as any."""
    m, e, k, n, r = 48, 5, 96, 64, 8
    x, w, a, b, off, _, s = make(m, e, k, n, r, "f16", "tail", False, nk, 3)
    dy, b, a = (rand(5, m, n) * 2.0 ** power[0]).half(), (rand(6, *b.shape) * 2.0 ** power[1]).half(), (rand(7, *a.shape) * 2.0 ** power[2]).half()
    if nk:
        a, b = (t.transpose(1, 2).contiguous().transpose(1, 2) for t in (a, b))
    w = (w * 2.0 ** -14).half() if not nk else (w.t() * 2.0 ** -14).half().t()
    h = torch.zeros(m, r, dtype=torch.float16).cuda()
    dx, _, _ = kn.adapted_linear_backward(dev(dy), dev(x), h, dev(w), dev(a), dev(b), dev(off), scales=dev(s))
    assert torch.isfinite(dx).all() and math.isfinite(float(dx.float().abs().max())) and (dx[:int(off[-1])] != 0).any()
    check_dx(dy, x, w, a, b, off, None, s, False, dx, "f16")
