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
