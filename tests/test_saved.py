"""Rows kept in 8 bits until a backward pass, and the gradients from them, against plain implementations in 64 bits on the CPU.

What is kept is compared to the bit.  The products' bounds are those of test_experts.py: the values that 8 bits and a power of two stand for are exact in every
type, so that a gradient is as far from the exact one of the kept values as any other; the kept values themselves are within half a step of the inputs:
2^-4 of a value, or 2^-10 2^n for the smallest, twice that where a value above zero is kept from becoming zero.
"""
import ctypes as C
import math

import pytest
import torch

import paper_2103_13744_amd as kn

from .test_experts import DT, SIZES, close, dev, make, rand, ref_linear


def kept(x):
    """(bytes (R, K), exponents (R, blocks), values) by hand, in 64 bits."""
    r, k = x.shape
    kb = -(-k // 128)
    v = torch.nn.functional.pad(x.double(), (0, kb * 128 - k)).reshape(r, kb, 128)
    finite = torch.isfinite(v)
    amax = torch.where(finite, v.abs(), 0.0).amax(2)
    n = torch.full((r, kb), -100, dtype=torch.int64)
    for p in range(-100, 121):
        n = torch.where(amax > 448.0 * 2.0 ** p, p + 1, n)
    u = torch.where(finite, v, 0.0) * torch.exp2(-n.double())[:, :, None]
    step = torch.exp2(torch.floor(torch.log2(u.abs().clamp(min=2.0 ** -6))) - 3.0)
    q = torch.round(u / step) * step  # (ties to even)
    q = torch.where((u > 0.0) & (q == 0.0), 2.0 ** -9, q)
    past = (q * torch.exp2(n.double())[:, :, None]).abs() > torch.finfo(x.dtype).max
    q = torch.where(past, 240.0 * q.sign(), q)
    q = torch.where(finite, q, math.nan)
    bits = torch.where(finite, q, 0.0).float().to(torch.float8_e4m3fn).view(torch.uint8)
    bits = torch.where(finite, bits, torch.where(v == math.inf, 0x7F, 0xFF).to(torch.uint8))
    return bits.flatten(1)[:, :k], (n + 127).to(torch.uint8), (q * torch.exp2(n.double())[:, :, None]).flatten(1)[:, :k]


def same(a, b):
    """Equal values, NaN where the other has NaN."""
    return torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(a.nan_to_num(0.0), b.nan_to_num(0.0))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("size", [(1, 1), (3, 16), (2, 17), (5, 128), (7, 129), (70, 200), (33, 520), (0, 64), (17, 1000), (300, 63)], ids=str)
def test_save_and_restore(size, dtype):
    r, k = size
    x = (rand(r + k, r, k) * torch.exp(3 * rand(k, r, 1)) * torch.exp(2 * rand(k + 1, r, k))).to(DT[dtype])
    if r > 2:
        x[1] = 0.0
        x[2, ::3] = -0.0
        x[0, : k // 2] *= 2.0 ** -12
    bits, exponents, values = kept(x)
    for lead in (0, 1, 8):
        wide = torch.full((r, lead + k + 3), math.nan, dtype=x.dtype)
        wide[:, lead:lead + k] = x
        q, e = kn.save_f8(dev(wide)[:, lead:lead + k] if r else dev(x))
        got = q.cpu().view(torch.uint8)
        assert q.shape == (r, -(-k // 16) * 16) and not got[:, k:].any()
        zero = (got[:, :k] & 127) == 0
        assert torch.equal(zero, (bits & 127) == 0) and torch.equal(got[:, :k][~zero], bits[~zero]) and torch.equal(e.cpu().view(torch.uint8), exponents)
        assert torch.equal(q.cpu().view(torch.int8)[:, :k] > 0, x > 0)
        assert same(kn.restore_f8(q, e, k, DT[dtype]).double().cpu(), values)
        assert same(kn.restore_f8(q, e, k, torch.float32).double().cpu(), values)
    if r:
        scale = torch.exp2(exponents.double() - 127).repeat_interleave(128, 1)[:, :k]
        near = (values - x.double()).abs() <= torch.maximum(x.double().abs() * 2.0 ** -4, torch.where(x > 0, 2.0 ** -9, 2.0 ** -10) * scale)
        assert near[torch.isfinite(x)].all()  # (some of fp16's are infinite)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_save_every_magnitude(dtype):
    """Rows of one value beside one that is 2^s times as large, over the type's whole range; values on and next to the borders of a power of two and of 448."""
    info = torch.finfo(DT[dtype])
    big = [448.0, math.nextafter(448.0, 500.0), 449.0, 256.0, 255.0, 480.0, 1.75, 1.7500001, 1.0, 3.0, float(info.max), float(info.tiny), float(info.tiny) * float(info.eps)]
    rows = [[b, b * 2.0 ** -s, -b * 2.0 ** -s, b * 2.0 ** -s * 1.0625] for b in big for s in range(0, 22)]
    x = torch.tensor(rows, dtype=torch.float64).to(DT[dtype])
    bits, exponents, values = kept(x)
    q, e = kn.save_f8(dev(x))
    got = q.cpu().view(torch.uint8)[:, :4]
    assert torch.equal(e.cpu().view(torch.uint8), exponents)
    zero = (bits & 127) == 0
    assert torch.equal(got[~zero], bits[~zero]) and not (got[zero] & 127).any() and torch.equal(got.view(torch.int8) > 0, x > 0)
    assert same(kn.restore_f8(q, e, 4, torch.float32).double().cpu(), values)  # (a sixteenth more than the largest is infinite)
    if dtype != "f32":
        assert same(kn.restore_f8(q, e, 4, DT[dtype]).double().cpu(), values)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_save_what_is_not_finite(dtype):
    x = rand(5, 4, 300).to(DT[dtype])
    x[0, 3], x[1, 200], x[2, 7], x[3, :] = math.nan, math.inf, -math.inf, math.inf
    bits, exponents, values = kept(x)
    q, e = kn.save_f8(dev(x))
    assert torch.equal(q.cpu().view(torch.uint8)[:, :300], bits) and torch.equal(e.cpu().view(torch.uint8), exponents)
    back = kn.restore_f8(q, e, 300, DT[dtype]).double().cpu()
    assert torch.equal(torch.isnan(back), ~torch.isfinite(x)) and torch.equal(back[torch.isfinite(x)], values[torch.isfinite(x)])
    assert torch.equal(q.cpu().view(torch.int8)[:, :300] > 0, x > 0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_backward_of_what_was_saved(size, dtype):
    m, e, k, n = size
    for i, (how, gather, nk, relu) in enumerate([("even", False, False, True), ("skew", True, True, False), ("tail", True, False, True), ("one", False, True, True)]):
        x, w, off, rows = make(m, e, k, n, dtype, how, gather, nk, 100 * m + i)
        x = x.relu() if relu else x
        if m:
            x[0, : k // 2] *= 2.0 ** -13  # (some are kept as the smallest value)
        dy = rand(9 + i, m, n).to(DT[dtype])
        q, ex = kn.save_f8(dev(x))
        dx, dw, db = kn.grouped_linear_backward_saved(dev(dy), q, ex, dev(w), dev(off), rows=dev(rows), relu_in=relu)
        assert torch.equal(dx, kn.grouped_linear_dx(dev(dy), dev(x), dev(w), dev(off), rows=dev(rows), relu_in=relu))  # to the bit: the mask is exact
        v = kept(x)[2]
        xs = v if rows is None else v[rows.long()]
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
@pytest.mark.parametrize("size", [(9, 3, 40, 20), (300, 4, 264, 136), (2700, 20, 256, 512)], ids=str)
def test_saved_rows_out_of_range_and_an_x_without_rows(size, dtype):
    """An entry that x does not have is a row of zeros, whatever row 0 holds: its dx is masked, and it has no part in dw."""
    m, e, k, n = size
    x, w, off, _ = make(m, e, k, n, dtype, "tail", False, False, m)
    rows = torch.randint(-4, m + 4, (m,), generator=torch.Generator().manual_seed(5), dtype=torch.int32)
    rows[rows == 0] = 1
    x[0] = math.nan
    dy = rand(7, m, n).to(DT[dtype])
    q, ex = kn.save_f8(dev(x))
    dx, dw, db = kn.grouped_linear_backward_saved(dev(dy), q, ex, dev(w), dev(off), rows=dev(rows), relu_in=True)
    gone = (rows < 0) | (rows >= m)
    assert not dx[gone.cuda()].any() and torch.isfinite(dw).all()
    v = torch.where(gone[:, None], 0.0, kept(x)[2][rows.clamp(0, m - 1).long()])
    want, mag = torch.zeros(e, k, n, dtype=torch.float64), torch.zeros(e, k, n, dtype=torch.float64)
    for g in range(e):
        a, b = int(off[g]), int(off[g + 1])
        want[g], mag[g] = v[a:b].T @ dy[a:b].double(), v[a:b].abs().T @ dy[a:b].double().abs()
    close(dw, want, mag, m, dtype)
    q, ex = kn.save_f8(torch.empty(0, k, dtype=DT[dtype]).cuda())
    dx, dw, db2 = kn.grouped_linear_backward_saved(dev(dy), q, ex, dev(w), dev(off), rows=dev(rows), relu_in=True)
    assert not dx.any() and not dw.any() and torch.equal(db2, db)


@pytest.mark.gpu
def test_saved_rows_beyond_32_bits():
    x_rows, m, e, k, n = (1 << 20) + 777, 200, 2, 4096, 136
    rows = torch.cat([torch.arange(x_rows - 100, x_rows), torch.arange(100) * 5000]).to(torch.int32)
    off = torch.tensor([0, 90, 200], dtype=torch.int32)
    some, w, dy = rand(1, m, k).bfloat16(), rand(2, e, k, n).bfloat16(), rand(3, m, n).bfloat16()
    x = torch.zeros(x_rows, k, dtype=torch.bfloat16, device="cuda")
    x[rows.long().cuda()] = dev(some)
    q, ex = kn.save_f8(x)
    assert q.numel() > 1 << 32
    part = kn.save_f8(dev(some))
    at = rows.long().cuda()
    assert torch.equal(q.view(torch.uint8)[at], part[0].view(torch.uint8)) and torch.equal(ex.view(torch.uint8)[at], part[1].view(torch.uint8))
    got = kn.grouped_linear_backward_saved(dev(dy), q, ex, dev(w), dev(off), rows=dev(rows), relu_in=True)
    want = kn.grouped_linear_backward_saved(dev(dy), *part, dev(w), dev(off), relu_in=True)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert torch.equal(kn.restore_f8(q[-100:], ex[-100:], k, torch.bfloat16), kn.restore_f8(part[0][:100], part[1][:100], k, torch.bfloat16))


@pytest.mark.gpu
def test_saved_gradient_against_differences():
    """dw is linear in dy, and its product with a change of w is that of the layer on the kept values."""
    m, e, k, n = 120, 4, 24, 40
    x, w, off, rows = make(m, e, k, n, "f32", "tail", True, False, 3)
    g = rand(2, m, n)
    q, ex = kn.save_f8(dev(x))
    v = kn.restore_f8(q, ex, k, torch.float32)
    _, dw, db = kn.grouped_linear_backward_saved(dev(g), q, ex, dev(w), dev(off), rows=dev(rows))
    f = lambda w: (kn.grouped_linear(v, dev(w), dev(off), rows=dev(rows)).double().cpu() * g.double()).sum()  # noqa: E731
    d = rand(11, e, k, n)
    # sums of up to 120 * 40 results of magnitude ~ 20 with 2^-23 each, times g ~ 1
    assert abs(float((f(w + d) - f(w - d)) / 2 - (dw.double().cpu() * d.double()).sum())) <= 2.0 ** -23 * m * n * 20 * 4


@pytest.mark.gpu
@pytest.mark.parametrize("size", [(50, 4, 63, 33), (5000, 4, 64, 64), (3000, 5, 256, 512)], ids=str)
def test_saved_on_another_stream_and_in_a_graph(size):
    m, e, k, n = size
    x, w, off, _ = make(m, e, k, n, "bf16", "skew", False, False, 3)
    x, w, off, dy = dev(x.relu()), dev(w), dev(off), dev(rand(5, m, n).bfloat16())

    def step():
        q, ex = kn.save_f8(x)
        return [kn.restore_f8(q, ex, k, torch.bfloat16), *kn.grouped_linear_backward_saved(dy, q, ex, w, off, relu_in=True)]

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


def test_saved_refusals_of_the_library():
    L, n, p = kn.load_library(), C.c_int64(), 4096  # (an address that is never dereferenced)

    def desc(**kw):
        d = dict(dtype=2, w_layout=0, experts=4, n_in=8, n_out=8, rows=16, x_rows=16, ldx=0)  # (ldx is not looked at)
        d.update(kw)
        return C.byref(kn.LinearDesc(*[d[f] for f, _ in kn.LinearDesc._fields_]))

    save = lambda x=p, dtype=0, r=4, k=8, ld=8, q=p, e=p: L.kn_save_f8(None, x, dtype, r, k, ld, q, e)  # noqa: E731
    for bad in (dict(x=None), dict(dtype=3), dict(r=-1), dict(k=0), dict(ld=7), dict(q=None), dict(q=p + 8), dict(e=None)):
        assert save(**bad) == -1, bad
    assert save(r=(1 << 30) + 1) == -2 and save(k=(1 << 20) + 1, ld=1 << 21) == -2 and save(x=None, r=0, q=None, e=None) == 0
    restore = lambda q=p, e=p, r=4, k=8, dtype=0, x=p: L.kn_restore_f8(None, q, e, r, k, dtype, x)  # noqa: E731
    for bad in (dict(q=None), dict(q=p + 8), dict(e=None), dict(r=-1), dict(k=0), dict(dtype=9), dict(x=None)):
        assert restore(**bad) == -1, bad
    assert restore(r=(1 << 30) + 1) == -2 and restore(q=None, e=None, r=0, x=None) == 0
    dx = lambda d=desc(), dy=p, w=p, q=p, off=p, rows=None, out=p: L.kn_grouped_linear_dx_saved(None, d, dy, w, q, off, rows, out)  # noqa: E731
    dw = lambda d=desc(), q=p, e=p, dy=p, off=p, rows=None, out=p, ws=None, size=0: L.kn_grouped_linear_dw_saved(None, d, q, e, dy, off, rows, out, None, ws, size)  # noqa: E731
    for call in (dx, dw):
        assert call(d=None) == -1
        for bad in (dict(dtype=3), dict(w_layout=2), dict(experts=0), dict(n_in=0), dict(n_out=0), dict(rows=-1), dict(x_rows=-1), dict(x_rows=8)):
            assert call(d=desc(**bad)) == -1, bad
        for much in (dict(experts=65536), dict(n_in=(1 << 20) + 1), dict(n_out=(1 << 20) + 1), dict(rows=(1 << 30) + 1, x_rows=1 << 30)):
            assert call(d=desc(**much)) == -2, much
        for bad in (dict(q=None), dict(q=p + 8), dict(dy=None), dict(off=None), dict(out=None)):
            assert call(**bad) == -1, bad
    assert dx(w=None) == -1 and dw(e=None) == -1 and dx(d=desc(rows=0), dy=None, w=None, q=None, off=None, out=None) == 0
    many = desc(rows=100000, x_rows=100000, n_in=256, n_out=256, ldx=256)
    assert L.kn_grouped_linear_dw_workspace_bytes(many, C.byref(n)) == 0 and n.value > 0
    assert dw(d=many) == -3 and dw(d=many, ws=p + 16, size=n.value) == -3 and dw(d=many, ws=p, size=n.value - 1) == -3


@pytest.mark.gpu
def test_saved_refusals_of_the_binding():
    x, w, off, dy = torch.zeros(8, 20).cuda(), torch.zeros(2, 20, 6).cuda(), torch.zeros(3, dtype=torch.int32).cuda(), torch.zeros(8, 6).cuda()
    q, e = kn.save_f8(x)
    for bad in (lambda: kn.save_f8(x.double()), lambda: kn.save_f8(x.t()), lambda: kn.save_f8(x.cpu()), lambda: kn.restore_f8(q, e, 40, torch.float32),
                lambda: kn.restore_f8(q, e, 20, torch.float64), lambda: kn.restore_f8(q.view(torch.uint8), e, 20, torch.float32), lambda: kn.restore_f8(q, e[:7], 20, torch.float32),
                lambda: kn.grouped_linear_dx_saved(dy[:7], q, e, w, off), lambda: kn.grouped_linear_dw_saved(dy.half(), q, e, w, off),
                lambda: kn.grouped_linear_dw_saved(dy, q, e, torch.zeros(2, 40, 6).cuda(), off), lambda: kn.grouped_linear_dw_saved(dy, q, e, w, off[:2]),
                lambda: kn.grouped_linear_backward_saved(dy, q, e, w[:, ::2], off), lambda: kn.grouped_linear_backward_saved(dy, q, e, w, off, rows=torch.zeros(7, dtype=torch.int32).cuda())):
        with pytest.raises(kn.KnError):
            bad()
