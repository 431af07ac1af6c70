"""The training step of test_training_step.py, entry by entry: every value within a bound that is carried through the step beside it.

Bounds: u = 2^-23.  A sum of n products in fp32 is off by (n + 8) u of the sum of their magnitudes in any order, and by what its factors are off, through the other
factors' magnitudes (products of two errors are covered by 1 % on top).  An exponential of an argument that is off by d, or whose rounding is, is off by d of itself; the
functions themselves by a few u.  What is kept in 8 bits, the choice of networks and the mask are the step's own bits."""
import pytest
import torch

from .test_experts import dev
from .test_saved import kept
from .test_training_step import D, E, H, K, N, R, T, inputs, step

U = 2.0 ** -23


def reference(v, ids, hidden):
    """{name: (value, bound)} in 64 bits."""
    d = {n: t.double() for n, t in v.items()}
    m = {n: t.abs() for n, t in d.items()}
    logits, el = d["x"] @ d["wr"], (D + 8) * U * (m["x"] @ m["wr"])
    w = torch.softmax(logits.gather(1, ids), 1)
    ew = w * (2.0 * el.gather(1, ids).amax(1, keepdim=True) + 32 * U)
    p, z = torch.softmax(logits, 1), torch.logsumexp(logits, 1)
    worst, span = el.amax(1), logits.amax(1) - logits.amin(1)
    ep = p * (2.0 * worst + (span + 32) * U)[:, None]  # (the span: an argument of that size is rounded before its exponential is taken)
    ez = worst + (z.abs() + 8) * U
    counts = torch.bincount(ids.reshape(-1), minlength=E).double()
    share = E * counts / (K * T * T)
    out = {"losses": (torch.stack([(p.sum(0) * share).sum(), z.square().mean()]),
                      torch.stack([((ep.sum(0) + (T + E + 32) * U * p.sum(0)) * share).sum(), (2.0 * z.abs() * ez + ez * ez + (T + 16) * U * z * z).mean()]))}
    kx, kh = kept(v["x"])[2], kept(hidden)[2]
    zeros = lambda *s: torch.zeros(s, dtype=torch.float64)  # noqa: E731
    res = {n: (zeros(*s), zeros(*s)) for n, s in (("out", (T, N)), ("dx", (T, D)), ("dw1", (E, D, H)), ("db1", (E, H)), ("da", (E, H, R)), ("db", (E, R, N)), ("dweights", (T, K)))}
    off = torch.cat([torch.zeros(1), counts.cumsum(0)]).long()
    order = torch.sort(ids.reshape(-1), stable=True).indices
    for e in range(E):
        pairs = order[off[e]:off[e + 1]]
        n, t, s = len(pairs), pairs // K, d["s"][e]
        wt, ewt = w.reshape(-1)[pairs][:, None], ew.reshape(-1)[pairs][:, None]
        w1, w2, a, b = d["w1"][e], d["w2"], d["a"][e], d["b"][e]
        h1 = (d["x"][t] @ w1 + d["b1"][e]).clamp(min=0.0)
        eh1 = (D + 10) * U * (m["x"][t] @ w1.abs() + m["b1"][e])
        low, elow = s * (h1 @ a), s * (eh1 @ a.abs() + (H + 10) * U * (h1 @ a.abs()))
        y = h1 @ w2 + low @ b
        ey = eh1 @ w2.abs() + elow @ b.abs() + (H + R + 16) * U * (h1 @ w2.abs() + low.abs() @ b.abs())
        res["out"][0].index_add_(0, t, wt * y)
        res["out"][1].index_add_(0, t, wt * ey + ewt * y.abs() + (K + 4) * U * wt * y.abs())
        g = d["dout"][t]
        res["dweights"][0].reshape(-1)[pairs] = (g * y).sum(1)
        res["dweights"][1].reshape(-1)[pairs] = (g.abs() * ey + (N + 8) * U * (g * y).abs()).sum(1)
        dy, edy = wt * g, ewt * g.abs() + U * (wt * g).abs()
        gl, egl = s * (dy @ b.T), s * (edy @ b.abs().T + (N + 10) * U * (dy.abs() @ b.abs().T))
        h8 = kh[off[e]:off[e + 1]]
        mask = h8 > 0
        dh = (dy @ w2.T + gl @ a.T) * mask
        edh = (edy @ w2.abs().T + egl @ a.abs().T + (N + R + 16) * U * (dy.abs() @ w2.abs().T + gl.abs() @ a.abs().T)) * mask
        for name, at, value, bound in (("da", e, h8.T @ gl, h8.abs().T @ (egl + (n + 10) * U * gl.abs())),
                                       ("db", e, low.T @ dy, elow.T @ dy.abs() + low.abs().T @ (edy + (n + 10) * U * dy.abs())),
                                       ("dw1", e, kx[t].T @ dh, kx[t].abs().T @ (edh + (n + 10) * U * dh.abs())),
                                       ("db1", e, dh.sum(0), (edh + (n + 10) * U * dh.abs()).sum(0))):
            res[name][0][at], res[name][1][at] = value, bound
        res["dx"][0].index_add_(0, t, dh @ w1.T)
        res["dx"][1].index_add_(0, t, (edh + (H + K + 12) * U * dh.abs()) @ w1.abs().T)
    dwt, edwt = res.pop("dweights")
    s, es = (w * dwt).sum(1, keepdim=True), (w * edwt + ew * dwt.abs() + (K + 4) * U * (w * dwt).abs()).sum(1, keepdim=True)
    first, efirst = zeros(T, E), zeros(T, E)
    first.scatter_(1, ids, w * (dwt - s))
    efirst.scatter_(1, ids, w * (edwt + es) + (ew + 4 * U * w) * (dwt.abs() + s.abs()))
    g0, g1 = d["dlosses"][0], d["dlosses"][1] * 2.0 / T
    mean, emean = (p @ share)[:, None], (ep @ share + (E + 8) * U * (p @ share))[:, None]
    second = p * (g0 * (share - mean) + (g1 * z)[:, None])
    size = g0 * (share + mean) + (g1 * z.abs())[:, None]
    esecond = p * (g0 * emean + (g1 * ez)[:, None] + 8 * U * size) + ep * size
    out["dlogits"] = (first + second, efirst + esecond + 2 * U * (first.abs() + second.abs()))
    return {**out, **res}


@pytest.mark.gpu
def test_a_training_step_entry_by_entry():
    v = inputs()
    got, (ids, hidden) = step({n: dev(t) for n, t in v.items()})
    want = reference(v, ids.cpu().long(), hidden.cpu())
    assert set(want) == set(got)
    for name, (ref, bound) in want.items():
        far = (got[name].double().cpu() - ref).abs()
        bad = far > 1.01 * bound + 2.0 ** -24 * ref.abs()
        assert not bad.any(), (name, int(bad.sum()), float((far / bound)[bad].max()), bad.nonzero()[:4].tolist())
        # what is allowed in one network's part, or one row's, is a small part of the largest value there: of these inputs at most 0.0055, for dlogits, where two results' products
        # with a gradient are subtracted (a row's may cancel: by network)
        parts, room = (t.t() if name == "dlogits" else t.reshape(len(t), -1) for t in (ref, bound))
        assert (room.amax(1) <= 2.0 ** -6 * parts.abs().amax(1)).all(), name
