"""Networks chosen per row, at the sizes where the large calls' kernels begin: one size at least for every kernel that the rules on
sizes choose between and that test_experts.py's sizes are too small for.  Plain implementations in 64 bits on the device, two-dimensional
products network by network; bounds as there."""
import math

import numpy as np
import pytest
import torch

import paper_2103_13744_amd as kn

from .test_experts import DT, U, rand, split

pytestmark = pytest.mark.gpu


def close(got, want, mags, terms, dtype):
    """test_experts.close, where everything is on the device."""
    assert got.shape == want.shape and got.dtype == DT[dtype]
    bound = U[dtype] * want.abs() + (terms + 8) * 2.0 ** -23 * mags + 2.0 ** -24
    off = (got.double() - want).abs()
    high = want.abs() + bound >= float(torch.finfo(DT[dtype]).max)  # (beyond the type's range: infinity)
    bad = ~((off <= bound) | (high & (got.double() == want.sign() * math.inf)))
    assert not bad.any(), (int(bad.sum()), float(off[bad].max()), bad.nonzero()[:4].tolist())


def ref_linear(x, w, off, rows, bias, relu):
    x = x.double() if rows is None else x.double()[rows.long()]
    y = torch.zeros(x.shape[0], w.shape[2], dtype=torch.float64, device="cuda")
    mag = torch.zeros_like(y)
    for e, (a, b) in enumerate(zip(off[:-1].tolist(), off[1:].tolist())):
        if a == b:
            continue
        we = w[e].double().contiguous()
        y[a:b], mag[a:b] = x[a:b] @ we, x[a:b].abs() @ we.abs()
        if bias is not None:
            y[a:b] += bias[e].double()
            mag[a:b] += bias[e].double().abs()
    return (y.clamp(min=0.0) if relu else y), mag


def ref_dw(xs, dy, off, e):
    """(dw, magnitudes, db, magnitudes, rows of the longest network); xs: a row per row of dy."""
    k, n = xs.shape[1], dy.shape[1]
    dw, mdw, db, mdb = (torch.zeros(s, dtype=torch.float64, device="cuda") for s in ((e, k, n), (e, k, n), (e, n), (e, n)))
    most = 0
    for g, (a, b) in enumerate(zip(off[:-1].tolist(), off[1:].tolist())):
        if a == b:
            continue
        most, x, d = max(most, b - a), xs[a:b].double(), dy[a:b].double()
        xt, dc = x.t().contiguous(), d.contiguous()
        dw[g], mdw[g], db[g], mdb[g] = xt @ dc, xt.abs() @ dc.abs(), d.sum(0), d.abs().sum(0)
    return dw, mdw, db, mdb, most


def make(m, e, k, n, dtype, how, gather, nk, seed):
    dt, off, rows, xr = DT[dtype], split(m, e, how, seed), None, m
    if gather:
        xr = m // 3 + 5
        rows = torch.randint(-3, xr + 3, (m,), generator=torch.Generator().manual_seed(seed + 1), dtype=torch.int32).clamp_(0, xr - 1).cuda()
    w = (rand(seed + 3, e, n, k).cuda().transpose(1, 2) if nk else rand(seed + 3, e, k, n).cuda()).to(dt)
    return rand(seed + 2, xr, k).cuda().to(dt), w, off, rows


# rows, networks, inputs, outputs: what the rules on sizes make of them
SIZES_16 = [(6200, 8, 1024, 1024),   # tiles of 192 x 128
            (16500, 20, 480, 480),   # tiles of 128 x 128; weights' gradient by 128 x 128 and a join
            (8300, 20, 479, 479),    # staged tiles of 128 x 128, and such of the weights' gradient
            (66000, 3, 136, 136)]    # weights' gradient by 128 x 128 of few networks of many rows
SIZES_32 = [(17000, 20, 132, 64),    # narrow results, two stages; 32 x 128
            (17000, 5, 64, 132),     # the same for the inputs' gradient; 64 x 128
            (4100, 20, 260, 260), (4100, 3, 260, 260),   # 32 x 128 and 64 x 128
            (4200, 20, 259, 261), (4200, 3, 259, 261)]   # the same of rows that are not whole pieces
LAYERS = [(s, d) for s in SIZES_16 for d in ("f16", "bf16")] + [(s, "f32") for s in SIZES_32]


@pytest.mark.parametrize("size, dtype", LAYERS, ids=str)
def test_forward_of_large_calls(size, dtype):
    m, e, k, n = size
    for i, (how, gather, nk, bias, relu) in enumerate([("even", True, False, True, True), ("skew", False, True, False, False), ("tail", True, True, True, False)]):
        x, w, off, rows = make(m, e, k, n, dtype, how, gather, nk, m + i)
        b = rand(7 + i, e, n).to(DT[dtype]).cuda() if bias else None
        y = kn.grouped_linear(x, w, off.cuda(), rows=rows, bias=b, relu=relu)
        close(y, *ref_linear(x, w, off, rows, b, relu), k + 1, dtype)


# Layers of up to 128 x 128 whose rows are whole pieces, on both sides of what rows per network and widths decide
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("each", [3, 40, 70, 130, 300])
@pytest.mark.parametrize("k, n", [(32, 128), (40, 40), (64, 64), (64, 128), (72, 64), (72, 72), (128, 32), (128, 64), (128, 128)])
def test_layers_between_small_and_tiles(k, n, each, dtype):
    e = 12
    for i, (how, nk) in enumerate([("even", False), ("tail", True)]):
        x, w, off, rows = make(e * each, e, k, n, dtype, how, False, nk, each + i)
        b = rand(7 + i, e, n).to(DT[dtype]).cuda()
        close(kn.grouped_linear(x, w, off.cuda(), bias=b, relu=True), *ref_linear(x, w, off, None, b, True), k + 1, dtype)


@pytest.mark.parametrize("size, dtype", LAYERS, ids=str)
def test_backward_of_large_calls(size, dtype):
    m, e, k, n = size
    for i, (how, gather, nk, relu) in enumerate([("skew", True, False, True), ("tail", False, True, False)]):
        x, w, off, rows = make(m, e, k, n, dtype, how, gather, nk, m + i)
        x = x.relu() if relu else x
        dy = rand(9 + i, m, n).to(DT[dtype]).cuda()
        dx, dw, db = kn.grouped_linear_backward(dy, x, w, off.cuda(), rows=rows, relu_in=relu)
        xs = x if rows is None else x[rows.long()]
        want, mag = ref_linear(dy, w.transpose(1, 2), off, None, None, False)
        if relu:
            want, mag = want * (xs > 0), mag * (xs > 0)
        close(dx, want, mag, n, dtype)
        wdw, mdw, wdb, mdb, most = ref_dw(xs, dy, off, e)
        assert dw.stride() == w.stride()
        close(dw, wdw, mdw, most, dtype)
        close(db, wdb, mdb, most, dtype)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("size", [(20000, 9000, 64, 64, 150), (20000, 9000, 63, 62, 150), (20000, 600, 256, 256, 1100)], ids=str)
def test_parts_of_a_few_networks_among_many(size, dtype):
    """So many networks that those of several parts are looked for: the first, the last, and some between; all others have a few rows or none."""
    m, e, k, n, long = size
    count = np.zeros(e, dtype=np.int64)
    for i, g in enumerate((0, 1, e // 2, e - 1)):
        count[g] = long * (1 + i)
    r = np.random.default_rng(1)
    left = m - count.sum() - 40  # (the last forty rows belong to no network)
    count += np.bincount(r.integers(2, e - 1, left), minlength=e)
    off = torch.from_numpy(np.concatenate([[0], np.cumsum(count)]).astype(np.int32))
    for nk in (False, True):
        w = torch.empty((e, n, k), dtype=DT[dtype], device="cuda").transpose(1, 2) if nk else torch.empty((e, k, n), dtype=DT[dtype], device="cuda")
        x, dy = rand(2, m, k).to(DT[dtype]).cuda(), rand(3, m, n).to(DT[dtype]).cuda()
        dw, db = kn.grouped_linear_dw(dy, x, w, off.cuda())
        wdw, mdw, wdb, mdb, most = ref_dw(x, dy, off, e)
        close(dw, wdw, mdw, most, dtype)
        close(db, wdb, mdb, most, dtype)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("size", [(1100, 20, 300, 1024), (1300, 40, 130, 1000), (2700, 20, 300, 1024), (6200, 8, 300, 1024), (9100, 3, 640, 520)], ids=str)
def test_linear_f8_of_large_calls(size, dtype):
    """Tiles of 32 rows of many networks, of 64 and of 192 rows."""
    m, e, k, n = size
    for i, (how, gather, bias, relu) in enumerate([("even", False, True, True), ("skew", True, False, False), ("tail", True, True, False)]):
        x, w, off, rows = make(m, e, k, n, "bf16", how, gather, True, 10 * m + i)
        xq, xs = kn.quantize_f8(x)
        wq, ws = kn.quantize_f8_weights(w)
        b = rand(3, e, n).to(DT[dtype]).cuda() if bias else None
        y = kn.grouped_linear_f8(xq, xs, wq, ws, off.cuda(), rows=rows, bias=b, relu=relu, dtype=DT[dtype])
        vx = xq.double() * xs.double().repeat_interleave(128, 1)
        vw = wq.double() * ws.double().repeat_interleave(128, 1)[:, :n].repeat_interleave(128, 2)
        close(y, *ref_linear(vx, vw.transpose(1, 2), off, rows, b, relu), k + 8, dtype)


def test_quantize_f8_weights_in_16_bits():
    for e, k, n in ((3, 100, 70), (2, 300, 257)):
        w = rand(k, e, n, k).half().cuda()
        nb, kb = -(-n // 128), -(-k // 128)
        full = torch.zeros(e, nb * 128, kb * 128, device="cuda")
        full[:, :n, :k] = w.float()
        blocks = full.reshape(e, nb, 128, kb, 128)
        s = blocks.abs().amax(dim=(2, 4), keepdim=True).clamp(min=2.0 ** -100) * torch.tensor(1.0 / 448.0, device="cuda")
        want = (blocks / s).to(torch.float8_e4m3fn).reshape(e, nb * 128, kb * 128)[:, :n].contiguous()
        for t in (w.transpose(1, 2), w.transpose(1, 2).contiguous()):
            q, qs = kn.quantize_f8_weights(t)
            assert torch.equal(q.view(torch.uint8), want.view(torch.uint8)) and torch.equal(qs, s.reshape(e, nb, kb))


# (64 rows of logits a workgroup: 64 workgroups, 65, many, and more than a step of the scan over them)
@pytest.mark.parametrize("size", [(4096, 40, 3), (4097, 40, 3), (5000, 128, 8), (9001, 300, 2), (70001, 16, 1), (33000, 7, 7)], ids=str)
def test_route_of_many_rows(size):
    t, e, k = size
    for renorm, dtype in ((True, "f32"), (False, "bf16")):
        l = (4 * rand(t, t, e)).round() / 4 if renorm else rand(t, t, e)  # (ties)
        g = torch.Generator().manual_seed(1)
        l = l.masked_fill((torch.rand((t, e), generator=g) < 0.3) | (torch.rand((t, 1), generator=g) < 0.05), -math.inf).to(DT[dtype]).cuda()
        w, ids, slots, rows, off = kn.route(l, k, renormalize=renorm)
        x = l.double()
        top, order = torch.sort(x, dim=1, descending=True, stable=True)
        wids = torch.where(top[:, :k] == -math.inf, -1, order[:, :k])
        some = wids[:, :1] >= 0
        z = torch.where(wids >= 0, torch.exp(top[:, :k] - torch.where(some, top[:, :1], 0.0)), 0.0)
        total = z.sum(1, keepdim=True) if renorm else torch.exp(x - torch.where(some, top[:, :1], 0.0)).sum(1, keepdim=True)
        want = torch.where(some, z / total, 0.0)
        key = torch.where(wids < 0, e, wids).reshape(-1)
        pairs = torch.sort(key, stable=True).indices
        wslots = torch.empty_like(pairs)
        wslots[pairs] = torch.arange(t * k, device="cuda")
        woff = torch.searchsorted(key[pairs], torch.arange(e + 1, device="cuda"))
        assert torch.equal(ids.long(), wids) and torch.equal(slots.long(), wslots.reshape(t, k))
        assert torch.equal(rows.long(), pairs // k) and torch.equal(off.long(), woff)
        # exp and the quotient of fp32: a few units in the last place, and a sum of e terms
        assert ((w.double() - want).abs() <= (e + 16) * 2.0 ** -23 * want).all()


@pytest.mark.parametrize("t", [16200, 49200])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_combine_past_the_caches(dtype, t):
    """64 MiB of rows and more, and 192 and more: those go past the caches."""
    k, d = 4, 520 if dtype != "f32" else 264
    y, dout, w = rand(1, t * k, d).to(DT[dtype]).cuda(), rand(2, t, d).to(DT[dtype]).cuda(), rand(3, t, k).cuda()
    assert y.numel() * y.element_size() > (1 << 26 if t < 40000 else 3 << 26)
    slots = torch.randperm(t * k, generator=torch.Generator().manual_seed(4)).to(torch.int32).reshape(t, k)
    slots[::7, 1] = -1
    slots = slots.cuda()
    there = (slots >= 0).double()
    ys = y.double()[slots.long().clamp(min=0)]
    terms = ys * (w.double() * there)[:, :, None]
    close(kn.combine(y, slots, w), terms.sum(1), terms.abs().sum(1), k, dtype)
    dy, dw = kn.combine_backward(dout, y, slots, w)
    dot = dout.double()[:, None] * ys * there[:, :, None]
    close(dw, dot.sum(2), dot.abs().sum(2), d, "f32")
    want = dout.double()[:, None] * w.double()[:, :, None]
    close(dy[slots[slots >= 0].long()], want[slots >= 0], want[slots >= 0].abs(), 1, dtype)
