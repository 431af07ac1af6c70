"""A shared layer with low-rank adapters per network, forward and backward, against plain implementations in 64 bits on the CPU.

Bounds.  h and g are rounded to the type T before they are multiplied on, so the reference is taken in two steps: h against its own exact value (one rounding of the
scaled sum: u_T of it, and (C + 8) 2^-23 of the sum of magnitudes, test_experts.py), and what is made of h against the exact value of the h that was
returned.  g is not returned: what it enters is bounded by its error's largest effect, u_T |g| + (N + 9) 2^-23 (magnitudes of g) through |A|.
"""
import ctypes as C
import math

import pytest
import torch

import paper_2103_13744_amd as kn

from .test_experts import DT, U, dev, rand, split


def make(m, e, k, n, r, dtype, how, gather, nk, seed):
    dt, off = DT[dtype], split(m, e, how, seed)
    rows, xr = None, m
    if gather:
        xr = max(1, m // 3)
        rows = torch.randint(0, xr, (m,), generator=torch.Generator().manual_seed(seed + 1), dtype=torch.int32)
    lay = lambda s, *shape: (rand(s, *shape[:-2], shape[-1], shape[-2]).transpose(-1, -2) if nk else rand(s, *shape)) / math.sqrt(shape[-2])  # noqa: E731
    return (rand(seed + 2, xr, k).to(dt), lay(seed + 3, k, n).to(dt), lay(seed + 4, e, k, r).to(dt), lay(seed + 5, e, r, n).to(dt), off, rows,
            0.5 + torch.rand(e, generator=torch.Generator().manual_seed(seed + 6)))


def groups(off):
    return [(g, a, b) for g, (a, b) in enumerate(zip(off[:-1].tolist(), off[1:].tolist())) if b > a]


def within(got, want, bound, dtype):
    assert tuple(got.shape) == tuple(want.shape) and got.dtype == DT[dtype]
    bad = ~((got.double().cpu() - want).abs() <= U[dtype] * want.abs() + bound + 2.0 ** -24)
    assert not bad.any(), (int(bad.sum()), float((got.double().cpu() - want).abs()[bad].max()), bad.nonzero()[:4].tolist())


def check_forward(x, w, a, b, off, rows, s, bias, relu, y, h, dtype):
    m, r, (k, n) = y.shape[0], a.shape[2], w.shape
    xs = (x if rows is None else x[rows.long()]).double()
    wh, mh = torch.zeros(m, r, dtype=torch.float64), torch.zeros(m, r, dtype=torch.float64)
    for g, i, j in groups(off):
        sc = 1.0 if s is None else float(s[g])
        wh[i:j], mh[i:j] = sc * (xs[i:j] @ a[g].double()), sc * (xs[i:j].abs() @ a[g].double().abs())
    tail = int(off[-1])
    assert h.shape[1] % (4 if dtype == "f32" else 8) == 0 and not h[:, r:].any() and not h[tail:].any()
    within(h[:, :r], wh, (k + 10) * 2.0 ** -23 * mh, dtype)
    hd = h.double().cpu()[:, :r]
    want, mag = xs @ w.double(), xs.abs() @ w.double().abs()
    for g, i, j in groups(off):
        want[i:j] += hd[i:j] @ b[g].double()
        mag[i:j] += hd[i:j].abs() @ b[g].double().abs()
    if bias is not None:
        want, mag = want + bias.double(), mag + bias.double().abs()
    within(y, want.clamp(min=0.0) if relu else want, (k + r + 16) * 2.0 ** -23 * mag, dtype)


def check_backward(dy, x, w, a, b, off, rows, s, relu, h, got, dtype):
    dx, da, db = got
    m, (e, k, r), n = dy.shape[0], a.shape, w.shape[1]
    xs, d, u = (x if rows is None else x[rows.long()]).double(), dy.double(), U[dtype]
    wdx, mdx = d @ w.double().T, (n + 8) * 2.0 ** -23 * (d.abs() @ w.double().abs().T)
    wda, mda, wdb, mdb = (torch.zeros(t, dtype=torch.float64) for t in ((e, k, r), (e, k, r), (e, r, n), (e, r, n)))
    for q, i, j in groups(off):
        sc = 1.0 if s is None else float(s[q])
        g, mg = sc * (d[i:j] @ b[q].double().T), sc * (d[i:j].abs() @ b[q].double().abs().T)
        off_g = u * g.abs() + (n + 10) * 2.0 ** -23 * mg + 2.0 ** -24  # how far the rounded g may be from g
        am, xm = a[q].double().abs(), xs[i:j].abs()
        wdx[i:j] += g @ a[q].double().T
        mdx[i:j] += off_g @ am.T + (r + 16) * 2.0 ** -23 * (g.abs() @ am.T)
        wda[q], mda[q] = xs[i:j].T @ g, xm.T @ off_g + (j - i + 8) * 2.0 ** -23 * (xm.T @ g.abs())
        hd = h.double().cpu()[i:j, :r]
        wdb[q], mdb[q] = hd.T @ d[i:j], (j - i + 8) * 2.0 ** -23 * (hd.abs().T @ d[i:j].abs())
    if relu:
        wdx, mdx = wdx * (xs > 0), mdx * (xs > 0)
    within(dx, wdx, 1.01 * mdx, dtype)
    within(da, wda, 1.01 * mda, dtype)
    within(db, wdb, 1.01 * mdb, dtype)
    assert da.stride() == dev(a).stride() and db.stride() == dev(b).stride()


SIZES = [  # rows, networks, inputs, outputs, rank
    (1, 1, 1, 1, 1), (1, 3, 64, 64, 4), (2, 70, 128, 136, 8), (5, 2, 2, 3, 2), (16, 8, 256, 64, 16), (17, 3, 33, 65, 5), (33, 33, 64, 72, 8), (48, 20, 512, 264, 16),
    (64, 1, 64, 64, 64), (65, 2, 63, 32, 4), (100, 100, 96, 40, 24), (129, 5, 91, 64, 7), (200, 65, 32, 33, 1), (257, 3, 72, 200, 80), (300, 130, 64, 3, 2), (500, 4, 320, 520, 16),
    (1000, 7, 129, 127, 9), (1100, 3, 512, 256, 32), (3000, 4200, 32, 32, 4), (2100, 2, 136, 264, 13), (1300, 3, 40, 72, 130), (200, 3, 24, 1, 3), (200, 3, 1, 24, 2), (90, 2, 300, 1, 8), (90, 2, 1, 300, 8), (2200, 5, 128, 128, 16), (400, 9, 100, 128, 10), (500, 3, 8, 200, 16),
    (70, 2, 3, 5, 40), (900, 3, 128, 64, 20), (3000, 3, 136, 200, 30), (2500, 2, 130, 99, 50), (1500, 2, 72, 300, 64), (700, 5, 96, 50, 70), (400, 9, 256, 136, 4), (1800, 30, 136, 264, 12), (2600, 3, 520, 256, 1),
    (5000, 4, 64, 33, 3), (700, 9, 2000, 48, 8), (300, 3, 5, 72, 100), (700, 2, 75, 9, 70), (900, 3, 67, 131, 3), (2600, 2, 141, 66, 33), (1500, 2, 13, 74, 66), (400, 2, 71, 1, 67), (2200, 3, 515, 300, 10),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_adapted(size, dtype):
    m, e, k, n, r = size
    for i, (how, gather, nk, bias, relu, scaled) in enumerate([("even", False, False, True, True, True), ("skew", True, True, False, False, True),
                                                               ("tail", True, False, True, False, False), ("one", False, True, True, True, True)]):
        x, w, a, b, off, rows, s = make(m, e, k, n, r, dtype, how, gather, nk, 100 * m + i)
        x, s, bv = x.relu() if relu else x, s if scaled else None, rand(7 + i, n).to(DT[dtype]) if bias else None
        args = (dev(x), dev(w), dev(a), dev(b), dev(off))
        y, h = kn.adapted_linear(*args, rows=dev(rows), scales=dev(s), bias=dev(bv), relu=relu, want_h=True)
        check_forward(x, w, a, b, off, rows, s, bv, relu, y, h, dtype)
        assert torch.equal(kn.adapted_linear(*args, rows=dev(rows), scales=dev(s), bias=dev(bv), relu=relu), y)
        dy = rand(9 + i, m, n).to(DT[dtype])
        got = kn.adapted_linear_backward(dev(dy), dev(x), h, *args[1:], rows=dev(rows), scales=dev(s), relu_in=relu)
        check_backward(dy, x, w, a, b, off, rows, s, relu, h, got, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("nk", [False, True])
@pytest.mark.parametrize("size", [(40, 20, 256, 200, 16), (300, 60, 256, 200, 16), (300, 60, 256, 200, 12), (3000, 100, 256, 520, 16), (3000, 100, 64, 64, 8), (3000, 40, 255, 129, 8), (20000, 90, 512, 1024, 24)],
                         ids=str)
def test_adapted_not_finite_values_stay_with_their_network(size, nk):
    """Rows of several networks share tiles: what is not finite in one network's adapter, or in a row, does not reach another's rows."""
    m, e, k, n, r = size
    for dtype in ("bf16", "f16", "f32"):
        x, w, a, b, off, rows, s = make(m, e, k, n, r, dtype, "tail", False, nk, m)
        dy = rand(8, m, n).to(DT[dtype])
        args = lambda a, b: (dev(w), dev(a), dev(b), dev(off))  # noqa: E731
        y, h = kn.adapted_linear(dev(x), *args(a, b), scales=dev(s), want_h=True)
        dx, da, db = kn.adapted_linear_backward(dev(dy), dev(x), h, *args(a, b), scales=dev(s))
        where = torch.searchsorted(off, torch.arange(m, dtype=torch.int32), right=True) - 1
        some = torch.unique(where[where < e])
        bad = {int(some[1]): math.nan, int(some[len(some) // 2]): math.inf, int(some[-1]): -math.inf}
        a2, b2 = a.clone(), b.clone()
        for i, v in bad.items():
            b2[i, r // 2, n // 3] = v
        y2, h2 = kn.adapted_linear(dev(x), *args(a, b2), scales=dev(s), want_h=True)
        hit = torch.isin(where, torch.tensor(list(bad)))
        assert torch.equal(h2, h) and not torch.isfinite(y2[hit.cuda(), n // 3]).any()
        # other networks' rows keep their bits; the network's own other columns may be summed in another order: both results are within
        # (k + r + 16) 2^-23 of the sum of magnitudes of the same sum, and rounded once each
        assert torch.equal(y2[~hit.cuda()], y[~hit.cuda()])
        others = torch.arange(n) != n // 3
        mag = x[hit].double().abs() @ w.double().abs()
        for row, i in enumerate(hit.nonzero()[:, 0].tolist()):
            mag[row] += h[i, :r].double().cpu().abs() @ b[where[i]].double().abs()
        y1 = y[hit.cuda()].double().cpu()
        within(y2[hit.cuda()][:, others.cuda()], y1[:, others], (2 * (k + r + 16) * 2.0 ** -23 * mag + U[dtype] * y1.abs())[:, others], dtype)
        for i, v in bad.items():
            a2[i, k // 2, r - 1] = v
        dx2, da2, db2 = kn.adapted_linear_backward(dev(dy), dev(x), h, *args(a2, b), scales=dev(s))
        assert not torch.isfinite(dx2[hit.cuda(), k // 2]).any()
        assert torch.equal(dx2[~hit.cuda()], dx[~hit.cuda()]) and torch.equal(da2, da) and torch.equal(db2, db)
        assert torch.isfinite(dx2[hit.cuda()][:, (torch.arange(k) != k // 2).cuda()]).all()
        x2 = x.clone()
        x2[5, 3], x2[m // 2, 0], x2[m - 1, 1] = math.nan, math.inf, math.nan
        y2, h2 = kn.adapted_linear(dev(x2), *args(a, b), scales=dev(s), want_h=True)
        keep = torch.ones(m, dtype=torch.bool)
        keep[[5, m // 2, m - 1]] = False
        assert torch.equal(y2[keep.cuda()], y[keep.cuda()]) and torch.equal(h2[keep.cuda()], h[keep.cuda()]) and not torch.isfinite(y2[~keep.cuda()]).any()
        assert (h2[m - 1] == 0).all()  # (a row of no network)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_adapted_rows_lie_apart_start_anywhere_and_out_of_range(dtype):
    """x as columns of a wider matrix at any address, rows through an index of which some are not there: those take nothing from row 0, which is NaN."""
    for m, e, k, n, r, nk in ((50, 4, 64, 96, 8, False), (50, 4, 63, 31, 5, True), (400, 4, 64, 48, 8, True), (700, 6, 200, 264, 12, False), (700, 6, 136, 264, 16, True)):
        x, w, a, b, off, _, s = make(m, e, k, n, r, dtype, "tail", False, nk, m)
        rows = torch.randint(-4, m + 4, (m,), generator=torch.Generator().manual_seed(5), dtype=torch.int32)
        rows[rows == 0] = 1
        rows[3], rows[m - 1] = -1, m
        bias = rand(6, n).to(DT[dtype])
        x[0] = math.nan
        gone = (rows < 0) | (rows >= m)
        want = torch.where(gone[:, None], 0.0, x[rows.clamp(0, m - 1).long()].float()).to(DT[dtype])
        ones = (want, w, a, b, off, None, s)
        for lead, more in ((0, 0), (1, 2), (8, 8)):
            wide = torch.full((m, lead + k + more), math.nan, dtype=DT[dtype]).cuda()
            wide[:, lead:lead + k] = dev(x)
            xs = wide[:, lead:lead + k]
            y, h = kn.adapted_linear(xs, dev(w), dev(a), dev(b), dev(off), rows=dev(rows), scales=dev(s), bias=dev(bias), want_h=True)
            check_forward(*ones, bias, False, y, h, dtype)
            assert torch.equal(y[gone.cuda()], dev(bias).expand(m, n)[gone.cuda()])
            dy = rand(9, m, n).to(DT[dtype])
            got = kn.adapted_linear_backward(dev(dy), xs, h, dev(w), dev(a), dev(b), dev(off), rows=dev(rows), scales=dev(s), relu_in=True)
            check_backward(dy, *ones, True, h, got, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("size", [(9, 3, 40, 20, 4), (300, 4, 264, 136, 8), (300, 4, 64, 32, 8), (2700, 20, 256, 1024, 16)], ids=str)
def test_adapted_without_rows(size):
    """An x without rows counts as zeros; a call without rows does nothing, and its weight gradients are zeros."""
    m, e, k, n, r = size
    _, w, a, b, off, _, _ = make(m, e, k, n, r, "bf16", "even", False, False, 1)
    x, rows, bias = torch.empty(0, k, dtype=torch.bfloat16).cuda(), torch.arange(m, dtype=torch.int32).cuda() - m // 2, rand(2, n).bfloat16().cuda()
    y, h = kn.adapted_linear(x, dev(w), dev(a), dev(b), dev(off), rows=rows, bias=bias, want_h=True)
    assert torch.equal(y, bias.expand(m, n)) and not h.any()
    dx, da, db = kn.adapted_linear_backward(torch.ones_like(y), x, h, dev(w), dev(a), dev(b), dev(off), rows=rows, relu_in=True)
    assert not dx.any() and not da.any() and not db.any()
    y, h = kn.adapted_linear(x, dev(w), dev(a), dev(b), dev(off) * 0, want_h=True)
    assert y.shape == (0, n) and h.shape[0] == 0
    dx, da, db = kn.adapted_linear_backward(y, x, h, dev(w), dev(a), dev(b), dev(off) * 0)
    assert dx.shape == (0, k) and not da.any() and not db.any()


@pytest.mark.gpu
def test_adapted_rows_beyond_32_bits():
    k, x_rows, m, e, n, r = 4096, (1 << 19) + 777, 200, 2, 136, 8
    rows = torch.cat([torch.arange(x_rows - 100, x_rows), torch.arange(100) * 5000]).to(torch.int32)
    off = torch.tensor([0, 90, 200], dtype=torch.int32)
    some, w, a, b = rand(1, m, k).bfloat16(), rand(2, k, n).bfloat16(), (rand(3, e, k, r) / 64).bfloat16(), rand(4, e, r, n).bfloat16()
    x = torch.empty(x_rows, k, dtype=torch.bfloat16, device="cuda")
    assert x.numel() * 2 > 1 << 32
    x[rows.long().cuda()] = dev(some)
    for count in (200, 50):
        o = off.clamp(max=count)
        y, h = kn.adapted_linear(x, dev(w), dev(a), dev(b), dev(o), rows=dev(rows[:count]), want_h=True)
        check_forward(some[:count], w, a, b, o, None, None, None, False, y, h, "bf16")
        dy = rand(5, count, n).bfloat16()
        got = kn.adapted_linear_backward(dev(dy), x, h, dev(w), dev(a), dev(b), dev(o), rows=dev(rows[:count]))
        check_backward(dy, some[:count], w, a, b, o, None, None, False, h, got, "bf16")


@pytest.mark.gpu
@pytest.mark.parametrize("size", [(40, 4, 24, 40, 4), (300, 4, 24, 40, 4), (300, 4, 200, 140, 20)], ids=str)
def test_adapted_gradient_against_differences(size):
    """The result is linear in x, in a and in b alone: (f(a + d) - f(a - d)) / 2 = <da, d> up to the rounding of sums of m n results of magnitude 60 at most."""
    m, e, k, n, r = size
    x, w, a, b, off, rows, s = make(m, e, k, n, r, "f32", "tail", True, False, 3)
    g = rand(2, m, n)
    f = lambda x, a, b: (kn.adapted_linear(dev(x), dev(w), dev(a), dev(b), dev(off), rows=dev(rows), scales=dev(s)).double().cpu() * g.double()).sum()  # noqa: E731
    _, h = kn.adapted_linear(dev(x), dev(w), dev(a), dev(b), dev(off), rows=dev(rows), scales=dev(s), want_h=True)
    dx, da, db = kn.adapted_linear_backward(dev(g), dev(x), h, dev(w), dev(a), dev(b), dev(off), rows=dev(rows), scales=dev(s))
    grad_x = torch.zeros(x.shape, dtype=torch.float64).index_add_(0, rows.long(), dx.double().cpu())
    for what, grad in (("x", grad_x), ("a", da.double().cpu()), ("b", db.double().cpu())):
        d = rand(11, *grad.shape)
        plus = f(x + d if what == "x" else x, a + d if what == "a" else a, b + d if what == "b" else b)
        minus = f(x - d if what == "x" else x, a - d if what == "a" else a, b - d if what == "b" else b)
        assert abs(float((plus - minus) / 2 - (grad * d.double()).sum())) <= 2.0 ** -22 * m * n * 60 * 2


@pytest.mark.gpu
@pytest.mark.parametrize("size", [(1, 1, 256, 200, 8), (48, 20, 256, 512, 16), (500, 7, 64, 32, 8), (900, 30, 256, 1024, 16), (9000, 30, 256, 1024, 16)], ids=str)
def test_adapted_on_another_stream_and_in_a_graph(size):
    m, e, k, n, r = size
    x, w, a, b, off, _, s = [dev(t) for t in make(m, e, k, n, r, "bf16", "skew", False, True, 4)]
    dy = dev(rand(5, m, n).bfloat16())

    def step():
        y, h = kn.adapted_linear(x, w, a, b, off, scales=s, want_h=True)
        return [y, h, *kn.adapted_linear_backward(dy, x, h, w, a, b, off, scales=s)]

    want = [v.clone() for v in step()]
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        got = step()
    torch.cuda.current_stream().wait_stream(other)
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for i in range(4):
        for v in got:
            v.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want)), i
        assert all(torch.equal(p, q) for p, q in zip(step(), want))


def test_adapted_refusals_of_the_library():
    L, n, p = kn.load_library(), C.c_int64(), 4096  # (an address that is never dereferenced)

    def desc(**kw):
        d = dict(dtype=2, w_layout=0, experts=4, n_in=8, n_out=8, rows=16, x_rows=16, ldx=8)
        d.update(kw)
        return C.byref(kn.LinearDesc(*[d[f] for f, _ in kn.LinearDesc._fields_]))

    forward = lambda d=desc(), rank=4, x=p, w=p, a=p, b=p, off=p, rows=None, y=p, h=None, ws=p, size=1 << 30: L.kn_adapted_linear(  # noqa: E731
        None, d, rank, x, w, a, b, None, None, off, rows, 0, y, h, ws, size)
    backward = lambda d=desc(), rank=4, dy=p, x=p, h=p, w=p, a=p, b=p, off=p, rows=None, dx=p, da=p, db=p, ws=p, size=1 << 30: L.kn_adapted_linear_backward(  # noqa: E731
        None, d, rank, dy, x, h, w, a, b, None, off, rows, 0, dx, da, db, ws, size)
    bytes_ = [lambda d=desc(), rank=4, f=f: f(d, rank, C.byref(n)) for f in (L.kn_adapted_linear_workspace_bytes, L.kn_adapted_linear_backward_workspace_bytes)]
    for call in (forward, backward, *bytes_):
        assert call(d=None) == -1 and call(rank=0) == -1 and call(rank=(1 << 20) + 1) == -2
        for bad in (dict(dtype=3), dict(w_layout=2), dict(experts=0), dict(n_in=0), dict(n_out=0), dict(rows=-1), dict(x_rows=-1), dict(ldx=7)):
            assert call(d=desc(**bad)) == -1, bad
        for much in (dict(experts=65536), dict(n_in=(1 << 20) + 1, ldx=1 << 21), dict(n_out=(1 << 20) + 1), dict(rows=(1 << 30) + 1, x_rows=1 << 30)):
            assert call(d=desc(**much)) == -2, much
    for bad in (dict(x=None), dict(w=None), dict(a=None), dict(b=None), dict(off=None), dict(y=None), dict(h=p + 8), dict(d=desc(x_rows=8))):
        assert forward(**bad) == -1, bad
    for bad in (dict(dy=None), dict(x=None), dict(h=None), dict(h=p + 8), dict(w=None), dict(a=None), dict(b=None), dict(off=None), dict(dx=None), dict(da=None), dict(db=None),
                dict(d=desc(x_rows=8))):
        assert backward(**bad) == -1, bad
    for call, size in ((forward, bytes_[0]), (backward, bytes_[1])):
        assert size() == 0 and n.value > 0 and n.value % 256 == 0
        assert call(ws=None) == -3 and call(ws=p + 8) == -3 and call(size=n.value - 1) == -3
    assert L.kn_adapted_linear_workspace_bytes(desc(), 4, None) == -1 and L.kn_adapted_linear_backward_workspace_bytes(desc(), 4, None) == -1
    assert forward(d=desc(rows=0), x=None, w=None, a=None, b=None, off=None, y=None, ws=None, size=0) == 0


@pytest.mark.gpu
def test_adapted_refusals_of_the_binding(monkeypatch):
    x, w, a, b = torch.zeros(8, 4).cuda(), torch.zeros(4, 6).cuda(), torch.zeros(2, 4, 3).cuda(), torch.zeros(2, 3, 6).cuda()
    off, h, dy = torch.zeros(3, dtype=torch.int32).cuda(), torch.zeros(8, 4).cuda(), torch.zeros(8, 6).cuda()
    f, g = kn.adapted_linear, kn.adapted_linear_backward
    for bad in (lambda: f(x.half(), w, a, b, off), lambda: f(x, w, a.half(), b, off), lambda: f(x[:, :3], w, a, b, off), lambda: f(x, w, a, b[:, :2], off),
                lambda: f(x, w, a[:1], b, off), lambda: f(x, w[None], a, b, off), lambda: f(x, w, a, b, off[:2]), lambda: f(x, w, a, b, off.long()),
                lambda: f(x, w, a.transpose(1, 2).contiguous().transpose(1, 2), b, off), lambda: f(x.cpu(), w, a, b, off), lambda: f(x, w.cpu(), a, b, off),
                lambda: f(x, w, a, b, off, scales=torch.ones(3).cuda()), lambda: f(x, w, a, b, off, scales=torch.ones(2).half().cuda()),
                lambda: f(x, w, a, b, off, bias=torch.ones(2, 6).cuda()), lambda: f(x, w, a, b, off, rows=torch.zeros(8).cuda()), lambda: f(x, w, a, b, off, out=dy[:7]),
                lambda: f(x.double(), w.double(), a.double(), b.double(), off), lambda: g(dy[:7], x, h, w, a, b, off), lambda: g(dy, x, h[:, :3], w, a, b, off),
                lambda: g(dy, x, h.half(), w, a, b, off)):
        with pytest.raises(kn.KnError):
            bad()
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1)  # (as if another device were the current one)
    for call in (lambda: f(x, w, a, b, off), lambda: g(dy, x, h, w, a, b, off), lambda: kn.save_f8(x), lambda: kn.route_balance(x, 2, torch.zeros(5, dtype=torch.int32).cuda())):
        with pytest.raises(kn.KnError, match="device"):
            call()
