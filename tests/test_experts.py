"""Networks chosen per row: router, grouped products with gradients, their 8-bit form, weighted sum, against plain
implementations in 64 bits on the CPU.

Bounds: a result of type T is the exact value of the same (already rounded) inputs up to the rounding of a sum of C products in
fp32, at most (C + 8) 2^-23 of the sum of the products' magnitudes in any order, and one rounding to T, at most u_T of the
result: u = 2^-8, 2^-11, 2^-24 for bf16, fp16, fp32, and 2^-24 absolute below fp16's normal range.
"""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import paper_2103_13744_amd as kn

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}


def close(got, want, mags, terms, dtype):
    """`mags`: sums of the magnitudes of the terms."""
    assert tuple(got.shape) == tuple(want.shape) and got.dtype == DT[dtype]
    g, w = got.double().cpu(), want.double()
    bound = U[dtype] * w.abs() + (terms + 8) * 2.0 ** -23 * mags + 2.0 ** -24
    bad = ~((g - w).abs() <= bound)
    assert not bad.any(), (int(bad.sum()), float((g - w).abs()[bad].max()), bad.nonzero()[:4].tolist())


def rand(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed))


def split(m, e, how, seed):
    """offsets of e networks over m rows: even, skewed, 'one' (all rows in one network), or 'tail' (a third of the rows in none)"""
    r = np.random.default_rng(seed)
    if how == "one":
        ids = np.full(m, e // 2)
    elif how == "skew":
        ids = np.minimum((e * r.random(m) ** 4).astype(int), e - 1)
    else:
        ids = r.integers(0, e, m)
    if how == "tail":
        ids[r.random(m) < 0.33] = e
    off = np.zeros(e + 1, dtype=np.int32)
    off[1:] = np.cumsum(np.bincount(ids, minlength=e + 1)[:e])
    return torch.from_numpy(off)


def ref_linear(x, w, off, rows, bias, relu):
    """In 64 bits: results and the sums of magnitudes."""
    m = x.shape[0] if rows is None else rows.shape[0]
    x, w = x.double(), w.double()
    x = x if rows is None else x[rows.long()]
    y, mag = torch.zeros(m, w.shape[2], dtype=torch.float64), torch.zeros(m, w.shape[2], dtype=torch.float64)
    for e in range(w.shape[0]):
        a, b = int(off[e]), int(off[e + 1])
        y[a:b], mag[a:b] = x[a:b] @ w[e], x[a:b].abs() @ w[e].abs()
        if bias is not None:
            y[a:b] += bias[e].double()
            mag[a:b] += bias[e].double().abs()
    return (y.clamp(min=0.0) if relu else y), mag


def make(m, e, k, n, dtype, how, gather, nk, seed, x_rows=None):
    dt = DT[dtype]
    off = split(m, e, how, seed)
    rows, xr = None, m
    if gather:
        xr = max(1, m // 3) if x_rows is None else x_rows
        rows = torch.randint(0, xr, (m,), generator=torch.Generator().manual_seed(seed + 1), dtype=torch.int32)
    x = rand(seed + 2, xr, k).to(dt)
    w = (rand(seed + 3, e, n, k).transpose(1, 2) if nk else rand(seed + 3, e, k, n)).to(dt)
    return x, w, off, rows


def dev(t):
    return None if t is None else t.cuda()  # (keeps the strides of dense tensors)


SIZES = [  # rows, networks, inputs, outputs
    (0, 3, 16, 16), (1, 1, 1, 1), (1, 4, 64, 64), (2, 70, 128, 136), (5, 2, 2, 3), (16, 8, 256, 64), (17, 3, 33, 65), (64, 1, 64, 64),
    (65, 2, 63, 32), (129, 5, 91, 64), (200, 65, 32, 33), (257, 3, 72, 200), (300, 130, 64, 3), (500, 4, 320, 520), (1000, 7, 129, 127),
    (1100, 3, 512, 256), (3000, 4200, 32, 32), (2100, 2, 136, 264), (300, 20, 200, 328), (1000, 30, 520, 256), (40, 2, 72, 520), (1300, 3, 40, 72), (6000, 3, 40, 72), (5000, 4, 64, 33), (4000, 2, 200, 131),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_forward(size, dtype):
    m, e, k, n = size
    for i, (how, gather, nk, bias, relu) in enumerate([("even", False, False, True, True), ("skew", True, True, False, False),
                                                        ("tail", True, False, True, False), ("one", False, True, True, True)]):
        x, w, off, rows = make(m, e, k, n, dtype, how, gather, nk, 100 * m + i)
        b = rand(7 + i, e, n).to(DT[dtype]) if bias else None
        y = kn.grouped_linear(dev(x), dev(w), dev(off), rows=dev(rows), bias=dev(b), relu=relu)
        want, mag = ref_linear(x, w, off, rows, b, relu)
        close(y, want, mag, k + 1, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_backward(size, dtype):
    m, e, k, n = size
    for i, (how, gather, nk, relu) in enumerate([("even", False, False, True), ("skew", True, True, False), ("tail", True, False, True),
                                                  ("one", False, True, True)]):
        x, w, off, rows = make(m, e, k, n, dtype, how, gather, nk, 100 * m + i)
        x = x.relu() if relu else x
        dy = rand(9 + i, m, n).to(DT[dtype])
        dx, dw, db = kn.grouped_linear_backward(dev(dy), dev(x), dev(w), dev(off), rows=dev(rows), relu_in=relu)
        xs = (x if rows is None else x[rows.long()]).double()
        wdx, mdx = ref_linear(dy, w.transpose(1, 2), off, None, None, False)
        if relu:
            wdx, mdx = wdx * (xs > 0), mdx * (xs > 0)
        close(dx, wdx, mdx, n, dtype)
        wdw, mdw, wdb, mdb = (torch.zeros(s, dtype=torch.float64) for s in ((e, k, n), (e, k, n), (e, n), (e, n)))
        most = 0
        for g in range(e):
            a, b = int(off[g]), int(off[g + 1])
            most = max(most, b - a)
            d = dy[a:b].double()
            wdw[g], mdw[g], wdb[g], mdb[g] = xs[a:b].T @ d, xs[a:b].abs().T @ d.abs(), d.sum(0), d.abs().sum(0)
        assert dw.stride() == dev(w).stride()
        close(dw, wdw, mdw, most, dtype)
        close(db, wdb, mdb, most, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_linear_rows_lie_apart_and_start_anywhere(dtype):
    """x as columns of a wider matrix, at addresses of every alignment; rows out of range count as zeros."""
    dt, m, e, k, n = DT[dtype], 150, 3, 64, 96
    off = split(m, e, "even", 5)
    w = rand(6, e, k, n).to(dt)
    for lead, more in ((0, 0), (1, 0), (3, 5), (8, 8), (8, 3)):
        wide = rand(7, m, lead + k + more).to(dt)
        x = wide[:, lead:lead + k]
        y = kn.grouped_linear(dev(wide)[:, lead:lead + k], dev(w), dev(off))
        want, mag = ref_linear(x, w, off, None, None, False)
        close(y, want, mag, k, dtype)
        dy = rand(8, m, n).to(dt)
        dx, dw, _ = kn.grouped_linear_backward(dev(dy), dev(wide)[:, lead:lead + k], dev(w), dev(off), relu_in=True, want_bias=False)
        wdx, mdx = ref_linear(dy, w.transpose(1, 2), off, None, None, False)
        close(dx, wdx * (x.double() > 0), mdx, n, dtype)
        for g in range(e):
            a, b = int(off[g]), int(off[g + 1])
            xs, d = x[a:b].double(), dy[a:b].double()
            close(dw[g], xs.T @ d, xs.abs().T @ d.abs(), b - a, dtype)
    rows = torch.randint(-5, m + 5, (m,), generator=torch.Generator().manual_seed(1), dtype=torch.int32)
    there = ((rows >= 0) & (rows < m)).double()[:, None]
    x = rand(7, m, k).to(dt)
    y = kn.grouped_linear(dev(x), dev(w), dev(off), rows=dev(rows))
    want, mag = ref_linear(x, w, off, rows.clamp(0, m - 1), None, False)
    close(y, want * there, mag, k, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("k", [1, 7, 8, 9, 31, 40, 63, 65, 91, 127, 131])
def test_linear_of_rows_between_others(k, dtype):
    """Rows and weights of any width at addresses of every alignment: nothing of what lies beside them (NaN) comes into the results."""
    dt, m, e, n = DT[dtype], 70, 3, 35
    off = split(m, e, "tail", 5)
    for lead, more, nk in ((0, 1, False), (1, 0, True), (1, 1, False), (2, 1, True), (3, 2, True), (1, 7 + 8 * k - k, False)):
        wide = torch.full((m, lead + k + more), math.nan, dtype=dt)
        wide[:, lead:lead + k] = rand(7, m, k).to(dt)
        line = torch.full((lead + e * k * n + 9,), math.nan, dtype=dt)
        line[lead:lead + e * k * n] = rand(8, e * k * n).to(dt)

        def weights(flat):
            flat = flat[lead:lead + e * k * n]
            return flat.view(e, n, k).transpose(1, 2) if nk else flat.view(e, k, n)

        y = kn.grouped_linear(dev(wide)[:, lead:lead + k], weights(dev(line)), dev(off))
        want, mag = ref_linear(wide[:, lead:lead + k], weights(line), off, None, None, False)
        close(y, want, mag, k, dtype)
        dy = rand(9, m, n).to(dt)
        dx, dw, _ = kn.grouped_linear_backward(dev(dy), dev(wide)[:, lead:lead + k], weights(dev(line)), dev(off), want_bias=False)
        wdx, mdx = ref_linear(dy, weights(line).transpose(1, 2), off, None, None, False)
        close(dx, wdx, mdx, n, dtype)
        for g in range(e):
            a, b = int(off[g]), int(off[g + 1])
            xs, d = wide[a:b, lead:lead + k].double(), dy[a:b].double()
            close(dw[g], xs.T @ d, xs.abs().T @ d.abs(), b - a, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("size", [(266, 37, 200, 328), (3000, 3, 264, 512), (5000, 5, 192, 64), (4000, 3, 131, 259), (2300, 2, 72, 136), (70, 2, 260, 1028)], ids=str)
def test_linear_in_full_precision_of_other_sizes(size):
    """The ways that fp32 goes by itself: few rows for the chip, narrow results, layers of few tiles, many rows of odd sizes."""
    m, e, k, n = size
    for i, (how, gather, nk) in enumerate([("skew", True, True), ("one", False, False), ("tail", True, False)]):
        x, w, off, rows = make(m, e, k, n, "f32", how, gather, nk, 100 * m + i)
        y = kn.grouped_linear(dev(x), dev(w), dev(off), rows=dev(rows))
        want, mag = ref_linear(x, w, off, rows, None, False)
        close(y, want, mag, k, "f32")
        dy = rand(9 + i, m, n)
        dx, dw, db = kn.grouped_linear_backward(dev(dy), dev(x), dev(w), dev(off), rows=dev(rows))
        wdx, mdx = ref_linear(dy, w.transpose(1, 2), off, None, None, False)
        close(dx, wdx, mdx, n, "f32")
        xs = (x if rows is None else x[rows.long()]).double()
        for g in range(e):
            a, b = int(off[g]), int(off[g + 1])
            d = dy[a:b].double()
            close(dw[g], xs[a:b].T @ d, xs[a:b].abs().T @ d.abs(), b - a, "f32")
            close(db[g], d.sum(0), d.abs().sum(0), b - a, "f32")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("k, n", [(63, 63), (31, 31), (31, 17), (63, 17), (9, 63), (47, 33)])
def test_linear_gradient_of_narrow_layers(k, n, dtype):
    """Networks with a few rows, with several parts, and very many networks with some: every width of a narrow layer's tiles."""
    dt = DT[dtype]
    for m, e, how, nk in ((40, 5, "even", False), (700, 3, "skew", True), (40, 2, "tail", True), (900, 2, "one", False), (9000, 1100, "skew", False)):
        x, w, off, _ = make(m, e, k, n, dtype, how, False, nk, 10 * m + k)
        dy = rand(m + n, m, n).to(dt)
        dw, db = kn.grouped_linear_dw(dev(dy), dev(x), dev(w), dev(off))
        want, mag, wdb, mdb = (torch.zeros(s, dtype=torch.float64) for s in ((e, k, n), (e, k, n), (e, n), (e, n)))
        most = 0
        for g in range(e):
            a, b = int(off[g]), int(off[g + 1])
            most = max(most, b - a)
            xs, d = x[a:b].double(), dy[a:b].double()
            want[g], mag[g], wdb[g], mdb[g] = xs.T @ d, xs.abs().T @ d.abs(), d.sum(0), d.abs().sum(0)
        close(dw, want, mag, most, dtype)
        close(db, wdb, mdb, most, dtype)


@pytest.mark.gpu
def test_linear_not_finite_values_stay_where_they_are():
    """A NaN or an infinity in a row reaches that row's results only, one in a network's weights that network's only."""
    for dtype, k, n in (("bf16", 128, 128), ("f16", 96, 40), ("f32", 64, 64)):
        dt, m, e = DT[dtype], 96, 3
        off = torch.tensor([0, 30, 30, 80], dtype=torch.int32)
        x, w = rand(1, m, k).to(dt), rand(2, e, k, n).to(dt)
        clean = kn.grouped_linear(dev(x), dev(w), dev(off))
        bad = x.clone()
        bad[5, 7], bad[40, 0], bad[90, 3] = math.nan, math.inf, math.nan
        y = kn.grouped_linear(dev(bad), dev(w), dev(off), relu=False)
        assert torch.isnan(y[5]).all() and not torch.isfinite(y[40]).any() and (y[80:] == 0).all()
        keep = torch.ones(m, dtype=torch.bool)
        keep[[5, 40]] = False
        assert torch.equal(y[keep.cuda()], clean[keep.cuda()])
        worse = w.clone()
        worse[2, 3, 4], worse[1] = math.nan, math.nan  # (network 1 has no rows)
        y = kn.grouped_linear(dev(x), dev(worse), dev(off))
        assert torch.isnan(y[30:80, 4]).all() and torch.equal(y[:30], clean[:30]) and torch.equal(y[30:80, 5:], clean[30:80, 5:])
        y = kn.grouped_linear(dev(bad), dev(w), dev(off), relu=True)
        assert torch.isnan(y[5]).all()  # a ReLU keeps a NaN
        dy = rand(3, m, n).to(dt)
        dy[5, 0] = math.nan
        dx, dw, db = kn.grouped_linear_backward(dev(dy), dev(x), dev(w), dev(off))
        assert torch.isnan(dx[5]).all() and torch.isfinite(dx[6:]).all() and torch.isnan(dw[0, :, 0]).all() and torch.isfinite(dw[0, :, 1:]).all()
        assert (dw[1] == 0).all() and torch.isfinite(dw[2]).all() and torch.isnan(db[0, 0]) and torch.isfinite(db[1:]).all()


@pytest.mark.gpu
def test_linear_many_networks():
    """As many networks as there may be, most without a row: the look-up of a row's network takes three steps, every gradient is written."""
    e, m, k, n = 65535, 700, 16, 24
    ids = np.sort(np.random.default_rng(1).choice(e, m // 2).repeat(2))
    off = torch.from_numpy(np.searchsorted(ids, np.arange(e + 1)).astype(np.int32))
    x, w, dy = rand(1, m, k).bfloat16(), rand(2, e, k, n).bfloat16(), rand(3, m, n).bfloat16()
    y = kn.grouped_linear(dev(x), dev(w), dev(off))
    wx, dx64 = w.double()[ids], dy.double()
    close(y, (x.double()[:, None] @ wx)[:, 0], (x.double().abs()[:, None] @ wx.abs())[:, 0], k, "bf16")
    dx, dw, db = kn.grouped_linear_backward(dev(dy), dev(x), dev(w), dev(off))
    close(dx, (dx64[:, None] @ wx.transpose(1, 2))[:, 0], (dx64.abs()[:, None] @ wx.abs().transpose(1, 2))[:, 0], n, "bf16")
    want, mag = torch.zeros(e, k, n, dtype=torch.float64), torch.zeros(e, k, n, dtype=torch.float64)
    outer = x.double()[:, :, None] * dx64[:, None, :]
    want.index_add_(0, torch.from_numpy(ids), outer)
    mag.index_add_(0, torch.from_numpy(ids), outer.abs())
    close(dw, want, mag, int(np.bincount(ids).max()), "bf16")
    wdb = torch.zeros(e, n, dtype=torch.float64).index_add_(0, torch.from_numpy(ids), dx64)
    close(db, wdb, torch.zeros(e, n, dtype=torch.float64).index_add_(0, torch.from_numpy(ids), dx64.abs()), int(np.bincount(ids).max()), "bf16")


@pytest.mark.gpu
@pytest.mark.parametrize("k", [4096, 4095], ids=["pieces", "anywhere"])
def test_linear_rows_beyond_32_bits(k):
    """Rows of x whose bytes lie 4 GiB and more behind its first."""
    x_rows, m, e, n = (1 << 19) + 777, 200, 2, 136
    rows = torch.cat([torch.arange(x_rows - 100, x_rows), torch.arange(100) * 5000]).to(torch.int32)
    off = torch.tensor([0, 90, 200], dtype=torch.int32)
    some, w, dy = rand(1, m, k).bfloat16(), rand(2, e, k, n).bfloat16(), rand(3, m, n).bfloat16()
    x = torch.empty(x_rows, k, dtype=torch.bfloat16, device="cuda")
    assert x.numel() * 2 > 1 << 32
    x[rows.long().cuda()] = dev(some)
    want, mag = ref_linear(some, w, off, None, None, False)
    close(kn.grouped_linear(x, dev(w), dev(off), rows=dev(rows)), want, mag, k, "bf16")
    dw, _ = kn.grouped_linear_dw(dev(dy), x, dev(w), dev(off), rows=dev(rows), want_bias=False)
    for g in range(e):
        a, b = int(off[g]), int(off[g + 1])
        xs, d = some[a:b].double(), dy[a:b].double()
        close(dw[g], xs.T @ d, xs.abs().T @ d.abs(), b - a, "bf16")
    q, s = kn.quantize_f8(x[-300:])
    assert torch.equal(q[200:].view(torch.uint8), kn.quantize_f8(x[-100:])[0].view(torch.uint8))


@pytest.mark.gpu
def test_linear_gradient_against_differences():
    """The layer is linear in each input alone: (f(w + d) - f(w - d)) / 2 = <dw, d> up to rounding, and alike for x and bias."""
    m, e, k, n = 120, 4, 24, 40
    x, w, off, rows = make(m, e, k, n, "f32", "tail", True, False, 3)
    b, g = rand(1, e, n), rand(2, m, n)
    f = lambda x, w, b: (kn.grouped_linear(dev(x), dev(w), dev(off), rows=dev(rows), bias=dev(b)).double().cpu() * g.double()).sum()  # noqa: E731
    dx, dw, db = kn.grouped_linear_backward(dev(g), dev(x), dev(w), dev(off), rows=dev(rows))
    slots = torch.argsort(rows, stable=True)
    grad_x = torch.zeros(x.shape, dtype=torch.float64).index_add_(0, rows.long(), dx.double().cpu())
    assert slots.numel() == m
    for what, grad in (("x", grad_x), ("w", dw.double().cpu()), ("b", db.double().cpu())):
        d = rand(11, *grad.shape)
        plus = f(x + d if what == "x" else x, w + d if what == "w" else w, b + d if what == "b" else b)
        minus = f(x - d if what == "x" else x, w - d if what == "w" else w, b - d if what == "b" else b)
        # sums of up to 120 * 40 results of magnitude ~ 20 with 2^-23 each, times g ~ 1
        assert abs(float((plus - minus) / 2 - (grad * d.double()).sum())) <= 2.0 ** -23 * m * n * 20 * 4


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_linear_layers_are_the_scene_networks(dtype):
    """A scene's tiny networks, layer after layer through the grouped products, in the order that the library's own bucketing
    gives: the density of Scene.eval_grouped."""
    import kn_synth as ks
    res, hidden, m = (3, 2, 4), 32, 3000
    nets = res[0] * res[1] * res[2]
    wts = torch.from_numpy(ks.round_to_storage(ks.kaiming_weights(nets, hidden, 3), dtype)).to(DT[dtype]).cuda()
    scene = kn.Scene(res, (0, 0, 0), (1, 1, 1), hidden, wts)
    p = torch.rand((m, 3), generator=torch.Generator().manual_seed(4)).cuda() * 1.1  # some outside
    d = torch.nn.functional.normalize(rand(5, m, 3), dim=1).cuda()
    sigma, _ = scene.eval_grouped(p.contiguous(), d.contiguous())
    _, offsets, perm = scene.bucket(scene.cell_ids(p.contiguous()))
    enc = [p] + [f(p * 2.0 ** i) for i in range(10) for f in (torch.sin, torch.cos)]
    h = torch.cat(enc, 1).to(DT[dtype])
    at, off, rows = 0, offsets[:nets + 1].contiguous(), perm
    for fi, fo, relu in ((63, 32, True), (32, 32, True), (32, 33, False)):
        w = wts[:, at:at + fi * fo].reshape(nets, fi, fo).contiguous()
        b = wts[:, at + fi * fo:at + fi * fo + fo].contiguous()
        h, rows, at = kn.grouped_linear(h, w, off, rows=rows, bias=b, relu=relu), None, at + fi * fo + fo
    got = torch.zeros(m, device="cuda")
    got[perm.long()] = h[:, 0].float().relu()
    assert float((got - sigma).abs().max()) <= {"f16": 2.5e-3, "bf16": 2e-2}[dtype] * max(1.0, float(sigma.abs().max()))


# ---------------------------------------------------------------------------------------------
def ref_route(logits, k, renorm):
    l = logits.double().numpy()
    t, e = l.shape
    ids, w = np.full((t, k), -1), np.zeros((t, k))
    for i in range(t):
        order = sorted((q for q in range(e) if l[i, q] > -math.inf), key=lambda q: (-l[i, q], q))[:k]
        ids[i, :len(order)] = order
        if order:
            z = np.exp(l[i] - l[i, order[0]])
            w[i, :len(order)] = z[order] / (z[order].sum() if renorm else z.sum())
    key = np.where(ids < 0, e, ids).reshape(-1)
    order = np.argsort(key, kind="stable")
    slots = np.empty(t * k, dtype=np.int64)
    slots[order] = np.arange(t * k)
    off = np.searchsorted(key[order], np.arange(e + 1))
    return torch.from_numpy(w), ids, slots.reshape(t, k), order // k, off


ROUTES = [(1, 1, 1), (1, 8, 2), (3, 5, 5), (16, 64, 4), (100, 17, 3), (257, 128, 8), (700, 16, 1), (2050, 100, 6), (65, 256, 32), (40, 1000, 20),
          (3001, 4, 4), (513, 65, 7), (0, 4, 2)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("size", ROUTES, ids=str)
def test_route(size, dtype):
    t, e, k = size
    for i, (renorm, masked, ties) in enumerate([(True, False, False), (False, True, False), (True, True, True), (False, False, True)]):
        l = rand(t + i, t, e)
        if ties:
            l = (2 * l).round() / 2
        if masked:
            g = torch.Generator().manual_seed(i)
            l = l.masked_fill((torch.rand((t, e), generator=g) < 0.6) | (torch.rand((t, 1), generator=g) < 0.1), -math.inf)
        l = l.to(DT[dtype])
        w, ids, slots, rows, off = kn.route(dev(l), k, renormalize=renorm)
        ww, wids, wslots, wrows, woff = ref_route(l, k, renorm)
        assert np.array_equal(ids.cpu().numpy(), wids) and np.array_equal(slots.cpu().numpy(), wslots)
        assert np.array_equal(rows.cpu().numpy(), wrows) and np.array_equal(off.cpu().numpy(), woff)
        # exp and the quotient of fp32: a few units in the last place, and a sum of e terms
        assert ((w.double().cpu() - ww).abs() <= (e + 16) * 2.0 ** -23 * ww).all()
        dw = rand(t + 50, t, k)
        dl = kn.route_backward(dev(l), w, ids, dev(dw), renormalize=renorm)
        g = np.where(wids >= 0, dw.double().numpy(), 0.0)
        ww = ww.numpy()
        mean = (ww * g).sum(1, keepdims=True)
        want = np.zeros((t, e))
        if not renorm and t:
            top = np.max(l.double().numpy(), axis=1, keepdims=True)
            z = np.exp(l.double().numpy() - np.where(np.isfinite(top), top, 0.0))
            want = -z / np.maximum(z.sum(1, keepdims=True), 1e-300) * mean
        for r in range(t):
            for j in range(k):
                if wids[r, j] >= 0:
                    want[r, wids[r, j]] = ww[r, j] * (g[r, j] - mean[r, 0])
        size_of = np.abs(g).max(axis=1, keepdims=True) if k and t else 0.0
        # terms of at most max|g| each: 32-bit rounding of the weights, the mean and the difference, then the type's
        bound = U[dtype] * np.abs(want) + (e + k + 32) * 2.0 ** -22 * size_of + 2.0 ** -24
        assert dl.dtype == DT[dtype] and (np.abs(dl.double().cpu().numpy() - want) <= bound).all()


@pytest.mark.gpu
def test_route_rows_that_are_not_finite_and_rows_that_lie_apart():
    l = rand(1, 40, 12)
    l[3, 5], l[9], l[11, 2], l[12] = math.nan, -math.inf, math.inf, math.nan
    wide = torch.zeros(40, 20)
    wide[:, 3:15] = l
    w, ids, slots, rows, off = kn.route(dev(wide)[:, 3:15], 3)
    assert torch.isnan(w[3]).all() and (w[9] == 0).all() and (ids[9] == -1).all() and torch.isnan(w[11]).any() and int(ids[11, 0]) == 2
    assert torch.isnan(w[12]).all() and (ids[12] == -1).all() and not (ids[3] == 5).any() and (ids[3] >= 0).all()
    assert torch.equal(slots.reshape(-1).sort().values.cpu(), torch.arange(120, dtype=torch.int32)) and int(off[-1]) == 120 - 6
    good = [i for i in range(40) if i not in (3, 9, 11, 12)]
    ww, wids, *_ = ref_route(l[good], 3, True)
    assert np.array_equal(ids.cpu().numpy()[good], wids) and ((w.cpu().double()[good] - ww).abs() <= 2.0 ** -20).all()
    # lowest values of the type are values like others
    low = torch.full((2, 6), torch.finfo(torch.float32).min)
    w, ids, *_ = kn.route(dev(low), 2)
    assert ids.tolist() == [[0, 1], [0, 1]] and (w == 0.5).all()


@pytest.mark.gpu
def test_route_gradient_against_differences():
    l, k = rand(1, 30, 9).double(), 3
    g = rand(2, 30, k)
    for renorm in (True, False):
        w, ids, *_ = kn.route(dev(l.float()), k, renormalize=renorm)
        dl = kn.route_backward(dev(l.float()), w, ids, dev(g), renormalize=renorm).double().cpu()

        def f(v):
            top = v.gather(1, ids.cpu().long())
            return ((torch.softmax(top, 1) if renorm else torch.softmax(v, 1).gather(1, ids.cpu().long())) * g.double()).sum()

        h, d = 1e-5, rand(3, 30, 9).double()
        # the difference's own error is of order h^2; fp32 rounding of 270 gradient terms
        assert abs(float((f(l + h * d) - f(l - h * d)) / (2 * h) - (dl * d).sum())) <= 1e-4


# ---------------------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("size", [(1, 1, 1), (1, 2, 64), (7, 3, 33), (16, 4, 2048), (100, 8, 520), (333, 2, 100), (0, 2, 8), (50, 32, 136)], ids=str)
def test_combine(size, dtype):
    t, k, d = size
    m, dt = t * k, DT[dtype]
    y, dout, w = rand(1, m, d).to(dt), rand(2, t, d).to(dt), rand(3, t, k)
    slots = torch.randperm(m, generator=torch.Generator().manual_seed(4)).to(torch.int32).reshape(t, k)
    for weights in (w, None):
        ww = torch.ones(t, k, dtype=torch.float64) if weights is None else w.double()
        ys = y.double()[slots.long()]
        out = kn.combine(dev(y), dev(slots), dev(weights))
        close(out, (ys * ww[:, :, None]).sum(1), (ys * ww[:, :, None]).abs().sum(1), k, dtype)
        dy, dw = kn.combine_backward(dev(dout), dev(y), dev(slots), dev(weights))
        want = torch.zeros(m, d, dtype=torch.float64)
        want[slots.long().reshape(-1)] = (dout.double()[:, None] * ww[:, :, None]).reshape(m, d)
        close(dy, want, want.abs(), 1, dtype)
        dot = dout.double()[:, None] * ys
        close(dw, dot.sum(2), dot.abs().sum(2), d, "f32")


# ---------------------------------------------------------------------------------------------
def ref_quantize(v, dims):
    s = torch.maximum(v.float().abs().amax(dim=dims, keepdim=True), torch.tensor(2.0 ** -100)) * torch.tensor(1.0 / 448.0)
    return (v.float() / s).to(torch.float8_e4m3fn), s


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_quantize_f8(dtype):
    for r, k in ((1, 1), (3, 128), (5, 129), (70, 200), (33, 520), (0, 64), (17, 1000)):
        x = (rand(r + k, r, k) * torch.exp(3 * rand(k, r, 1))).to(DT[dtype])
        if r > 2:
            x[1] = 0.0
        kb = -(-k // 128)
        full = torch.nn.functional.pad(x.float(), (0, kb * 128 - k)).reshape(r, kb, 128)
        want, s = ref_quantize(full, (2,))
        for lead in (0, 1):
            wide = torch.zeros(r, k + 3, dtype=x.dtype)
            wide[:, lead:lead + k] = x
            q, qs = kn.quantize_f8(dev(wide)[:, lead:lead + k] if r else dev(x))
            assert torch.equal(q.cpu().view(torch.uint8), want.reshape(r, kb * 128).view(torch.uint8)) and torch.equal(qs.cpu(), s.reshape(r, kb))
    x = rand(5, 4, 256).to(DT[dtype])
    x[0, 3], x[1, 200] = math.nan, math.inf
    q, s = kn.quantize_f8(dev(x))
    v = q.float().cpu() * s.cpu().repeat_interleave(128, 1)
    assert torch.isnan(v[0, 3]) and torch.isfinite(v[0, 4:]).all() and torch.isfinite(v[1, :128]).all() and torch.isnan(v[1, 128:]).all() and torch.isfinite(v[2:]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_quantize_f8_weights(dtype):
    for e, k, n in ((1, 128, 128), (3, 100, 70), (2, 300, 257), (1, 1, 1)):
        w = rand(k, e, n, k).to(DT[dtype])
        nb, kb = -(-n // 128), -(-k // 128)
        full = torch.zeros(e, nb * 128, kb * 128)
        full[:, :n, :k] = w.float()
        want, s = ref_quantize(full.reshape(e, nb, 128, kb, 128), (2, 4))
        want = want.reshape(e, nb * 128, kb * 128)[:, :n]
        for t in (dev(w).transpose(1, 2), dev(w).transpose(1, 2).contiguous()):
            q, qs = kn.quantize_f8_weights(t)
            assert torch.equal(q.cpu().view(torch.uint8), want.contiguous().view(torch.uint8)) and torch.equal(qs.cpu(), s.reshape(e, nb, kb))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("size", [(0, 2, 128, 128), (1, 1, 1, 1), (1, 3, 256, 128), (8, 40, 384, 200), (16, 4, 640, 256), (33, 2, 100, 70), (130, 3, 130, 129),
                                  (300, 5, 512, 384), (700, 2, 257, 520), (900, 100, 128, 64), (1500, 2, 640, 264)], ids=str)
def test_linear_f8(size, dtype):
    """Of the 8-bit values' products the sum is rounded, the scales' product and the result; these inputs stay within what sums in
    fp32 would give, although the matrix instruction's own sum of a block is a little narrower."""
    m, e, k, n = size
    for i, (how, gather, bias, relu) in enumerate([("even", False, True, True), ("skew", True, False, False), ("tail", True, True, False)]):
        x, w, off, rows = make(m, e, k, n, "bf16", how, gather, True, 10 * m + i)
        xq, xs = kn.quantize_f8(dev(x))
        wq, ws = kn.quantize_f8_weights(dev(w))
        b = rand(3, e, n).to(DT[dtype]) if bias else None
        y = kn.grouped_linear_f8(xq, xs, wq, ws, dev(off), rows=dev(rows), bias=dev(b), relu=relu, dtype=DT[dtype])
        vx = xq.cpu().double() * xs.cpu().double().repeat_interleave(128, 1)
        vw = wq.cpu().double() * ws.cpu().double().repeat_interleave(128, 1)[:, :n].repeat_interleave(128, 2)
        want, mag = ref_linear(vx, vw.transpose(1, 2), off, rows, b, relu)
        close(y, want, mag, k + 8, dtype)


# ---------------------------------------------------------------------------------------------
@pytest.mark.gpu
def test_the_whole_layer_on_another_stream_and_in_a_graph():
    """Router, expert layers, weighted sum, all gradients: on a stream of its own, and captured, replayed several times with
    the program's own work between; every replay gives the eager bits."""
    t, e, k, d, h = 200, 8, 2, 64, 128
    dt = torch.bfloat16
    x, wr = dev(rand(1, t, d).to(dt)), dev(rand(2, d, e))
    w1, w2, dout = dev((rand(3, e, d, h) / 8).to(dt)), dev((rand(4, e, h, d) / 11).to(dt)), dev(rand(5, t, d).to(dt))
    logits = (x.float() @ wr).contiguous()

    def step():
        w, ids, slots, rows, off = kn.route(logits, k)
        hid = kn.grouped_linear(x, w1, off, rows=rows, relu=True)
        y = kn.grouped_linear(hid, w2, off)
        out = kn.combine(y, slots, w)
        dy, dw = kn.combine_backward(dout, y, slots, w)
        dhid, dw2, db2 = kn.grouped_linear_backward(dy, hid, w2, off, relu_in=True)
        dxg, dw1, db1 = kn.grouped_linear_backward(dhid, x, w1, off, rows=rows)
        q, s = kn.quantize_f8(hid)
        y8 = kn.grouped_linear_f8(q, s, *w8, off, dtype=dt)
        return [out, kn.combine(dxg, slots), kn.route_backward(logits, w, ids, dw), dw1, db1, dw2, db2, y8]

    w8 = kn.quantize_f8_weights(w2)
    want = [v.clone() for v in step()]
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        got = step()
    torch.cuda.current_stream().wait_stream(other)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for i in range(4):
        for v in got:
            v.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i
        assert all(torch.equal(a, b) for a, b in zip(step(), want))


# ---------------------------------------------------------------------------------------------
def test_refusals_of_the_library():
    """Arguments are looked at on the host before anything is launched (no device needed)."""
    L = kn.load_library()
    n = C.c_int64()
    p = 4096  # an address that is never dereferenced
    assert L.kn_route_workspace_bytes(10, 4, 2, None) == -1
    assert L.kn_route_workspace_bytes(10, 4, 5, C.byref(n)) == -1          # more choices than experts
    assert L.kn_route_workspace_bytes(10, 2000, 2, C.byref(n)) == -2       # too many experts
    assert L.kn_route_workspace_bytes(10, 100, 33, C.byref(n)) == -2       # too many choices
    assert L.kn_route_workspace_bytes(1 << 30, 4, 2, C.byref(n)) == -2     # too many pairs
    assert L.kn_route_workspace_bytes(10, 4, 2, C.byref(n)) == 0 and n.value == 0  # (one workgroup)
    assert L.kn_route_workspace_bytes(1000, 4, 2, C.byref(n)) == 0 and n.value >= 20 and n.value % 256 == 0
    route = lambda *a: L.kn_route(None, *a)  # noqa: E731
    assert route(p, 7, 10, 4, 4, 2, 1, p, p, p, p, p, p, 1 << 20) == -1    # dtype
    assert route(p, 0, 10, 4, 3, 2, 1, p, p, p, p, p, p, 1 << 20) == -1    # rows overlap
    assert route(None, 0, 10, 4, 4, 2, 1, p, p, p, p, p, p, 1 << 20) == -1
    assert route(p, 0, 10, 4, 4, 2, 1, p, p, p, p, None, p, 1 << 20) == -1
    assert route(p, 0, 1000, 4, 4, 2, 1, p, p, p, p, p, None, 0) == -3     # workspace: missing, misaligned, small
    assert route(p, 0, 1000, 4, 4, 2, 1, p, p, p, p, p, p + 8, 1 << 20) == -3
    assert route(p, 0, 1000, 4, 4, 2, 1, p, p, p, p, p, p, 8) == -3
    assert L.kn_route_backward(None, None, 0, 10, 4, 4, 2, 1, p, p, p, p) == -1
    assert L.kn_route_backward(None, None, 0, 0, 4, 4, 2, 1, None, None, None, None) == 0

    def desc(**kw):
        d = dict(dtype=2, w_layout=0, experts=4, n_in=8, n_out=8, rows=16, x_rows=16, ldx=8)
        d.update(kw)
        return C.byref(kn.LinearDesc(*[d[f] for f, _ in kn.LinearDesc._fields_]))

    calls = [lambda d: L.kn_grouped_linear(None, d, p, p, None, p, None, 0, p), lambda d: L.kn_grouped_linear_dx(None, d, p, p, None, p, None, p),
             lambda d: L.kn_grouped_linear_dw(None, d, p, p, p, None, p, None, None, 0),
             lambda d: L.kn_grouped_linear_dw_workspace_bytes(d, C.byref(n))]
    for call in calls:
        assert call(None) == -1
        for bad in (dict(dtype=3), dict(w_layout=2), dict(experts=0), dict(n_in=0), dict(n_out=0), dict(rows=-1), dict(x_rows=-1), dict(ldx=7)):
            assert call(desc(**bad)) == -1, bad
        for much in (dict(experts=65536), dict(n_in=(1 << 20) + 1, ldx=1 << 21), dict(n_out=(1 << 20) + 1), dict(rows=(1 << 30) + 1, x_rows=1 << 30)):
            assert call(desc(**much)) == -2, much
    assert L.kn_grouped_linear(None, desc(x_rows=8), p, p, None, p, None, 0, p) == -1      # fewer rows of x than of y, no index
    assert L.kn_grouped_linear(None, desc(), None, p, None, p, None, 0, p) == -1
    assert L.kn_grouped_linear(None, desc(rows=0), None, None, None, None, None, 0, None) == 0
    assert L.kn_grouped_linear_dx(None, desc(), None, p, None, p, None, p) == -1
    assert L.kn_grouped_linear_dx(None, desc(rows=0), None, None, None, None, None, None) == 0
    assert L.kn_grouped_linear_dw(None, desc(), p, p, None, None, p, None, None, 0) == -1  # offsets are needed even for zeros
    many = desc(rows=100000, x_rows=100000, n_in=256, n_out=256, ldx=256)
    assert L.kn_grouped_linear_dw_workspace_bytes(many, C.byref(n)) == 0 and n.value >= 2 * 256 * 256 * 4
    assert L.kn_grouped_linear_dw(None, many, p, p, p, None, p, None, None, 0) == -3
    assert L.kn_grouped_linear_dw(None, many, p, p, p, None, p, None, p + 16, n.value) == -3
    assert L.kn_grouped_linear_dw(None, many, p, p, p, None, p, None, p, n.value - 1) == -3
    assert L.kn_grouped_linear_f8(None, desc(), p, p, p + 8, p, None, p, None, 0, p) == -1  # 16-byte rows
    assert L.kn_grouped_linear_f8(None, desc(), p, None, p, p, None, p, None, 0, p) == -1
    assert L.kn_grouped_linear_f8(None, desc(dtype=5), p, p, p, p, None, p, None, 0, p) == -1
    assert L.kn_grouped_linear_f8(None, desc(rows=0), None, None, None, None, None, None, None, 0, None) == 0
    assert L.kn_quantize_f8(None, p, 0, 4, 0, 8, p, p) == -1 and L.kn_quantize_f8(None, p, 0, 4, 8, 7, p, p) == -1
    assert L.kn_quantize_f8(None, p, 0, 4, 8, 8, p + 4, p) == -1 and L.kn_quantize_f8(None, None, 0, 0, 8, 8, None, None) == 0
    assert L.kn_quantize_f8_weights(None, p, 0, 3, 2, 8, 8, p, p) == -1 and L.kn_quantize_f8_weights(None, p, 0, 0, 0, 8, 8, p, p) == -1
    assert L.kn_quantize_f8_weights(None, p, 0, 0, 70000, 8, 8, p, p) == -2
    assert L.kn_combine(None, p, 9, 4, 8, p, p, 2, 2, p) == -1 and L.kn_combine(None, p, 0, 4, 0, p, p, 2, 2, p) == -1
    assert L.kn_combine(None, p, 0, 4, 8, None, p, 2, 2, p) == -1 and L.kn_combine(None, None, 0, 0, 8, None, None, 0, 2, None) == 0
    assert L.kn_combine_backward(None, None, p, 0, 4, 8, p, p, 2, 2, p, p) == -1
    assert L.kn_combine_backward(None, p, None, 0, 4, 8, p, p, 2, 2, p, p) == -1           # dweights need y


@pytest.mark.gpu
def test_8_bit_sums_of_any_bits():
    """Values over the whole range of e4m3, at random: the matrix instruction's own sum of a block keeps them within 2^-12 of the sum of
    the products' magnitudes (it is narrower than fp32), the rest is fp32."""
    g = torch.Generator().manual_seed(1)
    m, k, n = 64, 256, 128
    bits = lambda *s: torch.randint(0, 256, s, generator=g, dtype=torch.int32).to(torch.uint8)  # noqa: E731
    finite = lambda b: torch.where((b & 127) == 127, b ^ 1, b).view(torch.float8_e4m3fn)  # noqa: E731
    xq, wq = finite(bits(m, k)), finite(bits(1, n, k))
    xs, ws = torch.exp(rand(2, m, k // 128)), torch.exp(rand(3, 1, 1, k // 128))
    y = kn.grouped_linear_f8(xq.cuda(), xs.cuda(), wq.cuda(), ws.cuda(), torch.tensor([0, m], dtype=torch.int32).cuda(), dtype=torch.float32)
    vx = xq.double() * xs.double().repeat_interleave(128, 1)
    vw = wq[0].double() * ws[0].double().repeat_interleave(128, 1)
    assert ((y.double().cpu() - vx @ vw.T).abs() <= 2.0 ** -12 * (vx.abs() @ vw.abs().T)).all()


@pytest.mark.gpu
def test_refusals_of_the_binding():
    x, w, off = torch.zeros(8, 4).cuda(), torch.zeros(2, 4, 6).cuda(), torch.zeros(3, dtype=torch.int32).cuda()
    for bad in (lambda: kn.grouped_linear(x.double(), w.double(), off), lambda: kn.grouped_linear(x.half(), w, off), lambda: kn.grouped_linear(x[:, :3], w, off),
                lambda: kn.grouped_linear(x, w, off[:2]), lambda: kn.grouped_linear(x, w, off.long()), lambda: kn.grouped_linear(x.t()[:, :4], w, off),
                lambda: kn.grouped_linear(x, w[:, :, ::2], off), lambda: kn.grouped_linear(x, w, off, bias=torch.zeros(2, 5).cuda()),
                lambda: kn.grouped_linear(x, w, off, rows=torch.zeros(8).cuda()), lambda: kn.grouped_linear(x.cpu(), w, off),
                lambda: kn.grouped_linear_backward(torch.zeros(7, 6).cuda(), x, w, off), lambda: kn.route(x, 5), lambda: kn.route(x.long(), 2),
                lambda: kn.route_backward(x, torch.zeros(8, 2).cuda(), off[:2].reshape(1, 2), torch.zeros(8, 2).cuda()),
                lambda: kn.combine(x, off, None) if off.dim() == 2 else kn.combine(x, off.reshape(1, 3).float(), None),
                lambda: kn.grouped_linear_f8(x, x, w, w, off)):
        with pytest.raises(kn.KnError):
            bad()


@pytest.mark.gpu
def test_the_example_learns_and_serves_in_8_bits():
    """Two hundred steps bring the loss to a small part of what it was; weights and inputs of 3 significant bits add about
    (2^-4)^2 of the results' square per layer at most, far below what the field had to learn."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "routed_field.py")
    spec = importlib.util.spec_from_file_location("routed_field", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    first, full, eight = module.main(steps=200, say=lambda *_: None)
    assert full < first / 5 and eight < full + first / 20
