"""Networks chosen per row: inputs at the edge of what the calls take, against plain implementations in 64 bits.  Bounds as in
test_experts.py."""
import ctypes as C
import math

import pytest
import torch

import paper_2103_13744_amd as kn

from .test_experts import DT, U, rand, split


def close(got, want, mags, terms, dtype):
    """test_experts.close, where everything is on the device."""
    assert got.shape == want.shape and got.dtype == DT[dtype]
    bound = U[dtype] * want.abs() + (terms + 8) * 2.0 ** -23 * mags + 2.0 ** -24
    off = (got.double() - want).abs()
    high = want.abs() + bound >= float(torch.finfo(DT[dtype]).max)  # (beyond the type's range: infinity)
    bad = ~((off <= bound) | (high & (got.double() == want.sign() * math.inf)))
    assert not bad.any(), (int(bad.sum()), float(off[bad].max()), bad.nonzero()[:4].tolist())


# ---------------------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("size", [(64, 1, 384, 128), (1100, 20, 256, 1024), (2700, 20, 256, 1024), (6200, 8, 256, 1024)], ids=str)  # (tiles of 32, 64 and 192 rows)
def test_8_bit_sums_are_held_in_32_bits(size, dtype):
    """Any finite 8-bit values: products that lie up to 2^35 apart."""
    m, e, k, n = size
    g = torch.Generator().manual_seed(m)
    bits = lambda *s: torch.randint(0, 256, s, generator=g, dtype=torch.int32).to(torch.uint8)  # noqa: E731
    finite = lambda b: torch.where((b & 127) == 127, b ^ 1, b).view(torch.float8_e4m3fn).cuda()  # noqa: E731
    xq, wq, off = finite(bits(m, k)), finite(bits(e, n, k)), split(m, e, "even", 1)
    xs, ws = torch.exp(rand(2, m, k // 128)).cuda() / 32, torch.exp(rand(3, e, n // 128, k // 128)).cuda() / 32
    y = kn.grouped_linear_f8(xq, xs, wq, ws, off.cuda(), dtype=DT[dtype])
    vx = xq.double() * xs.double().repeat_interleave(128, 1)
    vw = wq.double() * ws.double().repeat_interleave(128, 1).repeat_interleave(128, 2)
    want, mag = torch.zeros(m, n, dtype=torch.float64, device="cuda"), torch.zeros(m, n, dtype=torch.float64, device="cuda")
    for i, (a, b) in enumerate(zip(off[:-1].tolist(), off[1:].tolist())):
        wt = vw[i].t().contiguous()
        want[a:b], mag[a:b] = vx[a:b] @ wt, vx[a:b].abs() @ wt.abs()
    close(y, want, mag, k + 8, dtype)


@pytest.mark.gpu
def test_8_bit_sums_keep_what_is_small_beside_what_cancels():
    """Of each eight neighbouring products one is 2^16 or -2^16 and seven are 4: 448 is left, which sums in fp32 miss by 34 at most."""
    x, w = torch.full((3, 128), 2.0), torch.full((128, 128), 2.0)
    x[:, ::16], x[:, 8::16], w[:, ::8] = 256.0, -256.0, 256.0
    one = torch.ones(3, 1).cuda()
    y = kn.grouped_linear_f8(x.to(torch.float8_e4m3fn).cuda(), one, w.to(torch.float8_e4m3fn).cuda()[None], one[:1].reshape(1, 1, 1),
                             torch.tensor([0, 3], dtype=torch.int32).cuda(), dtype=torch.float32)
    mag = torch.full((3, 128), 16 * 2.0 ** 16 + 112 * 4.0, dtype=torch.float64, device="cuda")
    close(y, torch.full_like(mag, 448.0), mag, 128, "f32")


# ---------------------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("size", [(9, 3, 40, 20), (300, 4, 264, 136), (2700, 20, 256, 1024), (6200, 8, 512, 1024)], ids=str)
def test_an_x_without_rows_counts_as_zeros(size, dtype):
    """Every row comes through an index into nothing: the biases are left, and zeros for rows of no network."""
    m, e, k, n = size
    off, rows = split(m, e, "tail", 1).cuda(), torch.arange(m, dtype=torch.int32).cuda() - m // 2
    x, b = torch.empty(0, k, dtype=DT[dtype], device="cuda"), rand(2, e, n).to(DT[dtype]).cuda()
    w, dy = rand(3, e, k, n).to(DT[dtype]).cuda(), rand(4, m, n).to(DT[dtype]).cuda()
    want, wdb, mag = torch.zeros(m, n, dtype=DT[dtype], device="cuda"), torch.zeros(e, n, dtype=torch.float64, device="cuda"), torch.zeros(e, n, dtype=torch.float64, device="cuda")
    for i, (p, q) in enumerate(zip(off[:-1].tolist(), off[1:].tolist())):
        want[p:q], wdb[i], mag[i] = b[i], dy[p:q].double().sum(0), dy[p:q].double().abs().sum(0)
    for relu in (False, True):
        y = kn.grouped_linear(x, w, off, rows=rows, bias=b, relu=relu)
        assert torch.equal(y, want.relu() if relu else want)
        y = kn.grouped_linear_f8(*kn.quantize_f8(x), *kn.quantize_f8_weights(w), off, rows=rows, bias=b, relu=relu, dtype=DT[dtype])
        assert torch.equal(y, want.relu() if relu else want)
    dw, db = kn.grouped_linear_dw(dy, x, w, off, rows=rows)
    assert not dw.any()
    close(db, wdb, mag, m, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("size", [(9, 3, 40, 20), (300, 4, 264, 136), (6200, 8, 512, 1024)], ids=str)
def test_gradient_before_a_relu_without_rows_is_zero(size, dtype):
    m, e, k, n = size
    off, rows = split(m, e, "tail", 1).cuda(), torch.arange(m, dtype=torch.int32).cuda() - m // 2
    x, w, dy = torch.empty(0, k, dtype=DT[dtype], device="cuda"), rand(3, e, k, n).to(DT[dtype]).cuda(), rand(4, m, n).to(DT[dtype]).cuda()
    assert not kn.grouped_linear_dx(dy, x, w, off, rows=rows, relu_in=True).any()
    assert kn.grouped_linear_dx(dy, x, w, off, rows=rows).any()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("size", [(9, 3, 40, 20), (300, 4, 264, 136), (2700, 20, 256, 1024), (6200, 8, 512, 1024)], ids=str)
def test_rows_out_of_range_take_nothing_from_row_0(size, dtype):
    """Row 0 of x holds NaN and infinities (which become NaN in 8 bits); an entry that x does not have is a row of zeros all the same, and
    row 0's own results are NaN."""
    m, e, k, n = size
    off, x_rows = split(m, e, "tail", 1).cuda(), 50
    rows = torch.randint(-4, x_rows + 4, (m,), generator=torch.Generator().manual_seed(5), dtype=torch.int32).cuda()
    x, w, b = rand(2, x_rows, k).to(DT[dtype]).cuda(), rand(3, e, k, n).to(DT[dtype]).cuda(), rand(4, e, n).to(DT[dtype]).cuda()
    x[0] = math.inf
    x[0, 1::2] = math.nan
    inside = torch.arange(m, device="cuda") < off[-1]
    out, first = (inside & ((rows < 0) | (rows >= x_rows))).nonzero()[:, 0], (inside & (rows == 0)).nonzero()[:, 0]
    net = torch.searchsorted(off, torch.arange(m, dtype=torch.int32, device="cuda"), right=True) - 1
    assert len(out) > 0 and (len(first) > 0 or m < 50)
    for y in (kn.grouped_linear(x, w, off, rows=rows, bias=b),
              kn.grouped_linear_f8(*kn.quantize_f8(x), *kn.quantize_f8_weights(w), off, rows=rows, bias=b, dtype=DT[dtype])):
        assert torch.equal(y[out], b[net[out]]) and torch.isnan(y[first]).all() and not y[~inside].any()
        assert torch.isfinite(y[inside & (rows != 0)]).all()
    dw, db = kn.grouped_linear_dw(rand(6, m, n).to(DT[dtype]).cuda(), x, w, off, rows=torch.where(rows == 0, -1, rows).contiguous())
    assert torch.isfinite(dw).all() and torch.isfinite(db).all()


def test_8_bit_weights_of_no_whole_blocks_are_refused():
    """The library would count a block more than the shapes that are checked have.  (Looked at before any address: no device needed.)"""
    for shape in ((2, 8, 200), (2, 8, 127), (2, 8, 1), (8, 256)):
        wq = torch.zeros(shape).to(torch.float8_e4m3fn)
        kb = shape[-1] // 128
        xq, xs, ws = torch.zeros(4, kb * 128).to(torch.float8_e4m3fn), torch.ones(4, kb), torch.ones(2, 1, kb)
        with pytest.raises(kn.KnError, match="whole blocks of 128"):
            kn.grouped_linear_f8(xq, xs, wq, ws, torch.zeros(3, dtype=torch.int32))


def test_products_of_counts_beyond_64_bits_are_refused():
    """rows x choices is a multiple of 2^64 here: too many all the same.  (No device needed.)"""
    L, n, p = kn.load_library(), C.c_int64(), 4096  # (an address that is never dereferenced)
    for t, k in ((1 << 59, 32), (1 << 60, 16), ((1 << 59) + (1 << 58), 32)):
        assert L.kn_route_workspace_bytes(t, 100, k, C.byref(n)) == -2
        assert L.kn_route(None, p, 0, t, 100, 100, k, 1, p, p, p, p, p, p, 1 << 40) == -2
        assert L.kn_route_backward(None, p, 0, t, 100, 100, k, 1, p, p, p, p) == -2
    for t, k in ((1 << 40, 1 << 30), (1 << 33, 1 << 30), (1 << 59, 32)):
        assert L.kn_combine(None, p, 0, 4, 8, p, p, t, k, p) == -2
        assert L.kn_combine_backward(None, p, p, 0, 4, 8, p, p, t, k, p, p) == -2


# ---------------------------------------------------------------------------------------------
# Calls of 2^32 threads and more: a launch's threads are counted in 32 bits
@pytest.mark.gpu
def test_weighted_sum_of_more_pairs_than_a_launch_has():
    t = (1 << 25) + 3
    y = (torch.arange(2 * t, device="cuda") % 251).bfloat16().reshape(-1, 1)
    slots = (2 * t - 1 - torch.arange(2 * t, dtype=torch.int32, device="cuda")).reshape(t, 2)
    dout = (torch.arange(t, device="cuda") % 127).bfloat16().reshape(-1, 1)
    dy, dw = kn.combine_backward(dout, y, slots)
    assert torch.equal(dw, dout.float() * y.float().flip(0).reshape(t, 2))
    assert torch.equal(dy.flip(0).reshape(t, 2), dout.expand(t, 2))
    del dy, dw, slots, dout
    t, d = (1 << 32) // 7 + 1000, 7
    y = torch.arange(1000 * d, device="cuda").remainder(251).bfloat16().reshape(1000, d)
    slots = (torch.arange(t, device="cuda") % 1000).to(torch.int32).reshape(t, 1)
    out = kn.combine(y, slots)
    n = t // 1000
    assert torch.equal(out[:n * 1000].reshape(n, 1000, d), y.expand(n, 1000, d)) and torch.equal(out[n * 1000:], y[:t - n * 1000])


@pytest.mark.gpu
def test_router_of_more_rows_than_a_launch_has():
    t = (1 << 29) + 70
    logits = torch.zeros(t, 2, dtype=torch.bfloat16, device="cuda")
    logits[::3, 1] = 1.0  # every third row goes to expert 1
    weights, ids, slots, rows, offsets = kn.route(logits, 1, renormalize=False)
    one = -(-t // 3)
    assert offsets.tolist() == [0, t - one, t] and int(ids.sum()) == one and not ids[1::3].any() and bool(ids[::3].all())
    assert torch.equal(rows[t - one:], torch.arange(0, t, 3, dtype=torch.int32, device="cuda"))
    assert torch.equal(rows[:t - one:2], torch.arange(1, t, 3, dtype=torch.int32, device="cuda"))
    assert torch.equal(slots[::3, 0], torch.arange(t - one, t, dtype=torch.int32, device="cuda"))
    assert torch.equal(slots[1::3, 0], torch.arange(0, t - one, 2, dtype=torch.int32, device="cuda"))
    del slots, rows
    hi = math.e / (1.0 + math.e)
    assert ((weights[::3] - hi).abs() < 1e-6).all() and ((weights[1::3] - 0.5).abs() < 1e-6).all()
    dl = kn.route_backward(logits, weights, ids, torch.ones_like(weights), renormalize=False)
    for at, e, p in ((0, 1, hi), (1, 0, 0.5), (2, 0, 0.5)):
        want = torch.tensor([p * (1.0 - p) if i == e else -p * (1.0 - p) for i in (0, 1)]).bfloat16().cuda()
        assert ((dl[at::3].float() - want.float()).abs() <= 2.0 ** -8 * 0.25).all()


@pytest.mark.gpu
def test_8_bit_rows_of_more_blocks_than_a_launch_has():
    r = (1 << 28) + 100
    x = (torch.arange(r, device="cuda") % 97).bfloat16().reshape(r, 1)
    q, s = kn.quantize_f8(x)
    v = q[:, 0].float() * s[:, 0]
    assert ((v - x[:, 0].float()).abs() <= 1e-6 * x[:, 0].float()).all() and (q[-1000:, 1:].float() == 0.0).all()


@pytest.mark.gpu
def test_linear_of_more_tiles_than_a_launch_has():
    """The last of very many networks that are wide one way, and very many rows of few results."""
    e, k, n = 65535, 8, 16448
    off = torch.zeros(e + 1, dtype=torch.int32)
    off[1:e], off[e] = 10, 32
    w = torch.empty((e, k, n), dtype=torch.bfloat16, device="cuda")
    w[0], w[e - 1] = rand(1, k, n).bfloat16().cuda(), rand(2, k, n).bfloat16().cuda()
    x, dy = rand(3, 32, k).bfloat16().cuda(), rand(4, 32, n).bfloat16().cuda()
    y = kn.grouped_linear(x, w, off.cuda())
    dw, db = kn.grouped_linear_dw(dy, x, w, off.cuda())
    for g, a, b in ((0, 0, 10), (e - 1, 10, 32)):
        xg, wg, d = x[a:b].double(), w[g].double(), dy[a:b].double()
        close(y[a:b], xg @ wg, xg.abs() @ wg.abs(), k, "bf16")
        xt = xg.t().contiguous()
        close(dw[g], xt @ d, xt.abs() @ d.abs(), b - a, "bf16")
        close(db[g], d.sum(0), d.abs().sum(0), b - a, "bf16")
    del w
    assert not dw[1:e - 1].any() and not db[1:e - 1].any()
    del dw, db
    m, k, n = (1 << 29) + 100, 256, 2
    x, w = rand(5, 64, k).bfloat16().cuda(), rand(6, 1, k, n).bfloat16().cuda()
    rows, off = (torch.arange(m, device="cuda") % 64).to(torch.int32), torch.tensor([0, m - 50], dtype=torch.int32).cuda()
    y = kn.grouped_linear_f8(*kn.quantize_f8(x), *kn.quantize_f8_weights(w), off, rows=rows)
    whole = (m - 50) // 64 * 64
    assert torch.equal(y[:whole].reshape(-1, 64, n), y[:64].expand(whole // 64, 64, n)) and torch.isfinite(y[:64]).all() and y[:64].any(dim=1).all()
    assert torch.equal(y[whole:m - 50], y[:m - 50 - whole]) and not y[m - 50:].any()
