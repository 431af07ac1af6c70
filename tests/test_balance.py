"""The losses that keep a learned router even, and their gradient, against plain implementations in 64 bits on the CPU.

Bounds.  A row's p are exponentials of fp32 differences (their error grows with the difference, which is 100 at most where they matter: 100 2^-24 2, and a
few units of the function) over a sum of E of them: (E + 256) 2^-23 relative.  Sums over rows are of positive terms: as much, and the additions, at most
2,048 / 16 in a row and 16 more in 32 bits: 160 2^-24.  The first loss has E products more; Z is as exact as its exponentials' sum, 2^-22 of
max(1, |Z|) with its own logarithm, and E 2^-24.  The gradient's terms are at most |g0| (share, mean) p and |g1| (2 / n) |Z| p.
"""
import ctypes as C
import math

import pytest
import torch

import paper_2103_13744_amd as kn

from .test_experts import DT, U, dev, rand


def make(t, e, k, dtype, masked, seed):
    """Logits of the type, and the offsets that a choice of k of them leaves."""
    l = rand(seed, t, e) * 1.5 + 0.5 * rand(seed + 1, e)
    if masked:
        g = torch.Generator().manual_seed(seed + 2)
        l = l.masked_fill((torch.rand((t, e), generator=g) < 0.4) | (torch.rand((t, 1), generator=g) < 0.1), -math.inf)
    l = l.to(DT[dtype])
    top, ids = torch.sort(l.float(), dim=1, descending=True, stable=True)
    ids = torch.where(top[:, :k] == -math.inf, e, ids[:, :k])
    off = torch.zeros(e + 1, dtype=torch.int32)
    off[1:] = torch.bincount(ids.reshape(-1), minlength=e + 1)[:e].cumsum(0)
    return l, off


def reference(l, off, k, dlosses, add, counts=None):
    """(losses, counts, probs, dlogits, what bounds the gradient's terms) in 64 bits."""
    t, e = l.shape
    l = l.double()
    there = (l > -math.inf).any(1)
    n = int(there.sum())
    c = (off[1:] - off[:-1]).double() if counts is None else counts[:e].double()
    m = n if counts is None else int(counts[e])
    p, z = torch.zeros_like(l), torch.zeros(t, 1, dtype=torch.float64)
    p[there], z[there] = torch.softmax(l[there], 1), torch.logsumexp(l[there], 1, keepdim=True)
    probs = p.sum(0)
    losses = torch.tensor([e * float((c * probs).sum()) / (k * n * n), float((z * z).sum()) / n]) if n else torch.zeros(2)
    share = e * c / (k * m * m) if m else torch.zeros(e, dtype=torch.float64)
    g = dlosses.double()
    mean = (p * share).sum(1, keepdim=True)
    d = p * (g[0] * (share - mean) + g[1] * 2.0 / max(m, 1) * z)
    size = p * (g[0].abs() * (share + mean) + g[1].abs() * 2.0 / max(m, 1) * z.abs().clamp(min=1.0))
    return losses, torch.cat([c.to(torch.int32), torch.tensor([n], dtype=torch.int32)]), probs, (d if add is None else d + add.double()), size, z


def check(got, want, t, e, dtype, add):
    losses, counts, probs, d = got
    wl, wc, wp, wd, size, z = want
    unit = (e + 256) * 2.0 ** -23 + 160 * 2.0 ** -24
    assert losses.dtype == probs.dtype == torch.float32 and counts.dtype == torch.int32 and d.dtype == DT[dtype]
    assert torch.equal(counts.cpu(), wc)
    assert ((probs.cpu().double() - wp).abs() <= unit * wp + 1e-30).all()
    assert abs(float(losses[0]) - float(wl[0])) <= (unit + e * 2.0 ** -23) * float(wl[0])
    n = max(1, int(wc[-1]))
    assert abs(float(losses[1]) - float(wl[1])) <= 2.0 * float((z.abs() * z.abs().clamp(min=1.0)).sum()) / n * (2.0 ** -22 + e * 2.0 ** -24) + 160 * 2.0 ** -24 * float(wl[1])
    more = 0.0 if add is None else add.double().abs()
    bound = U[dtype] * wd.abs() + 2.0 * unit * size + 2.0 ** -23 * (size + more) + (2.0 ** -24 if dtype == "f16" else 1e-38)
    assert ((d.cpu().double() - wd).abs() <= bound).all()


SIZES = [(1, 1, 1), (1, 5, 2), (3, 2, 2), (16, 16, 4), (64, 17, 3), (64, 1000, 4), (65, 16, 2), (65, 1, 1), (257, 128, 8), (700, 33, 5), (513, 256, 2), (300, 257, 3),
         (2050, 100, 6), (1000, 1024, 32), (33000, 8, 2), (70001, 3, 1)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_balance(size, dtype):
    t, e, k = size
    for masked in (False, True):
        l, off = make(t, e, k, dtype, masked, t + e)
        dlosses = torch.tensor([0.7 * t, -0.3 * t])
        add = rand(5, t, e).to(DT[dtype]) if masked else None
        losses, counts, probs = kn.route_balance(dev(l), k, dev(off))
        d = kn.route_balance_backward(dev(l), k, counts, dev(dlosses), add=dev(add))
        check((losses, counts, probs, d), reference(l, off, k, dlosses, add), t, e, dtype, add)


@pytest.mark.gpu
def test_balance_takes_what_route_gives():
    l = rand(1, 500, 24)
    l[::7] = -math.inf
    w, ids, slots, rows, off = kn.route(dev(l), 3)
    losses, counts, probs = kn.route_balance(dev(l), 3, off)
    assert torch.equal(counts[:-1].cpu(), torch.bincount(ids[ids >= 0].cpu().long(), minlength=24).int()) and int(counts[-1]) == 500 - 72
    dw, dl = rand(2, 500, 3), torch.tensor([3.0, 0.5])
    first = kn.route_backward(dev(l), w, ids, dev(dw))
    both = kn.route_balance_backward(dev(l), 3, counts, dev(dl), add=first)
    alone = kn.route_balance_backward(dev(l), 3, counts, dev(dl))
    assert ((both - (first + alone)).abs() <= 2.0 ** -22 * (first.abs() + alone.abs())).all()


@pytest.mark.gpu
@pytest.mark.parametrize("e", [12, 300])
def test_balance_rows_between_others_at_any_address(e):
    for dtype in ("f32", "bf16"):
        l, off = make(200, e, 2, dtype, True, 3)
        for lead, more in ((1, 0), (3, 2), (8, 8)):
            wide = torch.full((200, lead + e + more), math.nan, dtype=DT[dtype]).cuda()
            wide[:, lead:lead + e] = dev(l)
            x = wide[:, lead:lead + e]
            got = kn.route_balance(x, 2, dev(off))
            want = kn.route_balance(dev(l), 2, dev(off))
            assert all(torch.equal(a, b) for a, b in zip(got, want))
            g = torch.tensor([1.0, 2.0]).cuda()
            d = kn.route_balance_backward(x, 2, got[1], g)
            assert ((d - kn.route_balance_backward(dev(l), 2, got[1], g)).abs() <= 2.0 ** -20).all()


@pytest.mark.gpu
def test_balance_without_rows_and_of_rows_that_are_not_finite():
    for t in (0, 1, 64, 65, 3000):
        l, off = torch.full((t, 6), -math.inf).cuda(), torch.zeros(7, dtype=torch.int32).cuda()
        losses, counts, probs = kn.route_balance(l, 2, off)
        assert not losses.any() and not counts.any() and not probs.any()
        add = torch.ones(t, 6).cuda()
        assert not kn.route_balance_backward(l, 2, counts, torch.ones(2).cuda()).any()
        assert torch.equal(kn.route_balance_backward(l, 2, counts, torch.ones(2).cuda(), add=add), add)
    for t in (20, 400):
        for bad in (math.nan, math.inf):
            l, off = make(t, 6, 2, "f32", False, 4)
            l[3, 1] = bad
            losses, counts, probs = kn.route_balance(dev(l), 2, dev(off))
            assert torch.isnan(losses).all() and torch.isnan(probs).all() and int(counts[-1]) == t
            d = kn.route_balance_backward(dev(l), 2, counts, torch.ones(2).cuda())
            keep = torch.arange(t) != 3
            assert torch.isnan(d[3]).all() and torch.isfinite(d[keep.cuda()]).all()
        l, off = make(t, 6, 2, "f32", False, 4)
        l[5] = torch.finfo(torch.float32).min  # values like others: all alike
        l[7, 2] = -math.inf
        d = kn.route_balance_backward(dev(l), 2, kn.route_balance(dev(l), 2, dev(off))[1], torch.tensor([1.0, 0.0]).cuda())
        assert torch.isfinite(d).all() and float(d[7, 2]) == 0.0


@pytest.mark.gpu
def test_balance_of_several_processes_is_that_of_all_rows():
    """Counts and sums of two halves, added up: the losses and the gradient of the whole."""
    l, off = make(900, 20, 3, "f32", True, 8)
    half = [make_part(l[:400], 3), make_part(l[400:], 3)]
    parts = [kn.route_balance(dev(a), 3, dev(o)) for a, o in half]
    counts, probs = parts[0][1] + parts[1][1], parts[0][2] + parts[1][2]
    losses, wc, wp = kn.route_balance(dev(l), 3, dev(off))
    assert torch.equal(counts, wc) and ((probs - wp).abs() <= 2.0 ** -20 * wp).all()
    g = torch.tensor([900.0, 90.0]).cuda()
    want = kn.route_balance_backward(dev(l), 3, wc, g)
    assert torch.equal(torch.cat([kn.route_balance_backward(dev(a), 3, counts, g) for a, _ in half]), want)


def make_part(l, k):
    top, ids = torch.sort(l, dim=1, descending=True, stable=True)
    ids = torch.where(top[:, :k] == -math.inf, l.shape[1], ids[:, :k])
    off = torch.zeros(l.shape[1] + 1, dtype=torch.int32)
    off[1:] = torch.bincount(ids.reshape(-1), minlength=l.shape[1] + 1)[:-1].cumsum(0)
    return l.contiguous(), off


@pytest.mark.gpu
@pytest.mark.parametrize("t", [40, 300])
def test_balance_gradient_against_differences(t):
    """The counts are held fixed: the losses are smooth in the logits.  The difference's own error is of order h^2; the kernel's is that of fp32 terms."""
    l, off = make(t, 9, 2, "f32", False, 6)
    losses, counts, _ = kn.route_balance(dev(l), 2, dev(off))
    g = torch.tensor([2.0, 0.5])
    d = kn.route_balance_backward(dev(l), 2, counts, dev(g)).double().cpu()
    c, h, way = (off[1:] - off[:-1]).double(), 1e-4, rand(7, t, 9).double()

    def f(v):
        p = torch.softmax(v, 1).sum(0)
        return float(g[0]) * float((c * p).sum()) * 9 / (2 * t * t) + float(g[1]) * float(torch.logsumexp(v, 1).square().mean())

    assert abs((f(l.double() + h * way) - f(l.double() - h * way)) / (2 * h) - float((d * way).sum())) <= 1e-5


@pytest.mark.gpu
def test_balance_on_another_stream_and_in_a_graph():
    """Captured and replayed with eager calls between: the same bits every time."""
    for t, e in ((50, 16), (5000, 128), (900, 700)):
        l, off = make(t, e, 2, "f32", True, 9)
        l, off, g = dev(l), dev(off), torch.tensor([5.0, 1.0]).cuda()

        def step():
            losses, counts, probs = kn.route_balance(l, 2, off)
            return [losses, counts, probs, kn.route_balance_backward(l, 2, counts, g)]

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


def test_balance_refusals_of_the_library():
    L, n, p = kn.load_library(), C.c_int64(), 4096  # (an address that is never dereferenced)
    assert L.kn_route_balance_workspace_bytes(10, 4, None) == -1 and L.kn_route_balance_workspace_bytes(-1, 4, C.byref(n)) == -1
    assert L.kn_route_balance_workspace_bytes(10, 0, C.byref(n)) == -1 and L.kn_route_balance_workspace_bytes(10, 1025, C.byref(n)) == -2
    assert L.kn_route_balance_workspace_bytes((1 << 30) + 1, 4, C.byref(n)) == -2
    assert L.kn_route_balance_workspace_bytes(64, 1024, C.byref(n)) == 0 and n.value == 0
    assert L.kn_route_balance_workspace_bytes(1000, 4, C.byref(n)) == 0 and n.value > 0 and n.value % 256 == 0
    need = n.value
    call = lambda logits=p, dtype=0, t=1000, e=4, ld=4, k=2, off=p, losses=p, counts=p, probs=p, ws=p, size=1 << 20: L.kn_route_balance(  # noqa: E731
        None, logits, dtype, t, e, ld, k, off, losses, counts, probs, ws, size)
    for bad in (dict(logits=None), dict(dtype=3), dict(t=-1), dict(e=0), dict(ld=3), dict(k=0), dict(k=5), dict(off=None), dict(losses=None), dict(counts=None),
                dict(probs=None)):
        assert call(**bad) == -1, bad
    assert call(t=1 << 30, k=2) == -2 and call(e=2000, ld=2000) == -2 and call(e=100, ld=100, k=33) == -2
    for bad in (dict(ws=None), dict(ws=p + 8), dict(size=need - 1)):
        assert call(**bad) == -3, bad
    back = lambda logits=p, dtype=0, t=1000, e=4, ld=4, k=2, counts=p, dlosses=p, out=p: L.kn_route_balance_backward(  # noqa: E731
        None, logits, dtype, t, e, ld, k, counts, dlosses, None, out)
    for bad in (dict(logits=None), dict(dtype=-1), dict(t=-1), dict(e=0), dict(ld=3), dict(k=0), dict(k=5), dict(counts=None), dict(dlosses=None), dict(out=None)):
        assert back(**bad) == -1, bad
    assert back(e=2000, ld=2000) == -2 and back(t=0, logits=None, counts=None, dlosses=None, out=None) == 0


@pytest.mark.gpu
def test_balance_refusals_of_the_binding():
    l, off, counts, g = torch.zeros(8, 4).cuda(), torch.zeros(5, dtype=torch.int32).cuda(), torch.zeros(5, dtype=torch.int32).cuda(), torch.zeros(2).cuda()
    for bad in (lambda: kn.route_balance(l, 5, off), lambda: kn.route_balance(l, 0, off), lambda: kn.route_balance(l.long(), 2, off), lambda: kn.route_balance(l, 2, off[:4]),
                lambda: kn.route_balance(l, 2, off.long()), lambda: kn.route_balance(l.cpu(), 2, off), lambda: kn.route_balance(l.t(), 2, off),
                lambda: kn.route_balance_backward(l, 2, counts[:4], g), lambda: kn.route_balance_backward(l, 2, counts, g[:1]),
                lambda: kn.route_balance_backward(l, 2, counts, g.double()), lambda: kn.route_balance_backward(l, 5, counts, g),
                lambda: kn.route_balance_backward(l, 2, counts, g, add=l.half()), lambda: kn.route_balance_backward(l, 2, counts, g, add=l[:7])):
        with pytest.raises(kn.KnError):
            bad()


@pytest.mark.gpu
def test_balance_rows_beyond_32_bits():
    """Logits of 4 GiB and more: the sums are those of a distribution that repeats, the last rows' gradient that of a short call with the same counts."""
    t, e, k = (1 << 21) + 640, 1024, 2
    part, _ = make(640, e, k, "bf16", True, 4)
    part = dev(part)
    l = torch.empty(t, e, dtype=torch.bfloat16, device="cuda")
    assert l.numel() * 2 > 1 << 32
    l[:1 << 21] = part[:512].repeat(1 << 12, 1)
    l[1 << 21:] = part
    off = torch.arange(e + 1, dtype=torch.int32).cuda() * (t * k // e)
    losses, counts, probs = kn.route_balance(l, k, off)
    there = (part > -math.inf).any(1)
    p = torch.where(there[:, None], torch.softmax(part.double(), 1), 0.0)
    want = p[:512].sum(0) * (1 << 12) + p.sum(0)
    assert int(counts[-1]) == int(there[:512].sum()) * (1 << 12) + int(there.sum())
    assert ((probs.double() - want).abs() <= ((e + 256) * 2.0 ** -23 + 160 * 2.0 ** -24) * want).all()
    g = torch.tensor([float(t), 0.01 * t]).cuda()
    d = kn.route_balance_backward(l, k, counts, g)
    assert torch.equal(d[-640:], kn.route_balance_backward(part, k, counts, g))
