"""What is timed: operators of training and fine-tuning networks that are chosen per row, beside those of ``operators.py``.

A learned router is kept from sending everything to a few networks by a loss of its own (``kn.route_balance``,
``kn.route_balance_backward``).  Networks that share one layer and differ by a low-rank product, as the requests of many users of one
model do, are a shared product with adapters (``kn.adapted_linear``, ``kn.adapted_linear_backward``).  What a layer's backward pass needs of
its inputs is kept in 8 bits until then (``kn.save_f8``, ``kn.restore_f8``, ``kn.grouped_linear_backward_saved``).  Each case is one such call, or
a call with its gradients, on seeded inputs made on the GPU.  Rows are in the order of their networks, rows of no network last.

With ``own`` false the same results come from elementary torch operations in 32 bits: a ragged product is cut into pieces of at
most so many rows of one network, and the pieces are multiplied as a batch.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ITEM = {"f32": 4, "f16": 2, "bf16": 2}
F8, F8_MAX, F8_STEP, BLOCK, LEAST = torch.float8_e4m3fn, 448.0, 2.0 ** -9, 128, -100


def _balance(name, tokens, experts, k, dtype, masked=False, add=False):
    return dict(name=name, call="balance", tokens=tokens, experts=experts, k=k, dtype=dtype, masked=masked, add=add)


def _adapted(name, rows, adapters, rank, n_in, n_out, dtype, nk=False, skew=False, drop=0.0, gather=False, bias=False, relu=False, backward=False):
    return dict(name=name, call="adapted", rows=rows, experts=adapters, rank=rank, n_in=n_in, n_out=n_out, dtype=dtype, nk=nk, skew=skew, drop=drop,
                gather=gather, bias=bias, relu=relu, backward=backward)


def _save(name, rows, width, dtype):
    return dict(name=name, call="save", rows=rows, width=width, dtype=dtype)


def _saved(name, tokens, experts, k, n_in, n_out, dtype, skew=False, drop=0.0, gather=False, nk=False, bias=False, relu=False):
    return dict(name=name, call="saved", tokens=tokens, experts=experts, k=k, n_in=n_in, n_out=n_out, dtype=dtype, skew=skew, drop=drop, gather=gather, nk=nk,
                bias=bias, relu=relu)


def listed():
    return [
        # a router's losses and their gradient in a small training step: latency
        _balance("balance_small", 64, 16, 2, "f32"),
        # the same of a full one, padding tokens and closed networks among the rows, on top of the gradient of the choice
        _balance("balance_train", 32768, 128, 8, "f32", masked=True, add=True),
        # many networks, an odd number of rows, logits in 16 bits
        _balance("balance_wide", 16385, 1000, 4, "bf16"),
        # one token of one request
        _adapted("adapt_one", 1, 1, 16, 2048, 2048, "bf16", nk=True, bias=True),
        # one serving step: 48 requests, most with an adapter of their own, some with none
        _adapted("adapt_decode", 48, 32, 16, 2048, 2560, "bf16", nk=True, drop=0.1),
        # long prompts of a dozen requests
        _adapted("adapt_prefill", 16384, 12, 32, 2048, 2048, "bf16", skew=True, bias=True),
        # a grid of 16^3 cells whose small networks share a first layer (63 encoded inputs, 32 units), full precision
        _adapted("adapt_nets_f32", 262145, 4096, 4, 63, 32, "f32", skew=True, drop=0.02, gather=True, bias=True, relu=True),
        # fine-tuning adapters: forward and backward
        _adapted("adapt_train", 8192, 16, 16, 1024, 2048, "bf16", skew=True, backward=True),
        # a long batch's inputs of a layer, kept and brought back
        _save("save_long", 16411, 2048, "bf16"),
        # a training step's experts: inputs kept, all gradients from what was kept
        _saved("saved_train_bf16", 8192, 32, 4, 1024, 2048, "bf16", skew=True, gather=True),
        # a hidden layer of a grid of wide small networks behind a ReLU
        _saved("saved_nets_f16", 524291, 4096, 1, 64, 64, "f16", drop=0.02, bias=True, relu=True),
        # a small layer of odd sizes in full precision
        _saved("saved_odd_f32", 1001, 5, 1, 259, 131, "f32", bias=True, relu=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A layer's width: mostly whole blocks, now and then a multiple of eight, or odd."""
    n, kind = _log_int(rng, lo, hi), rng.random()
    return max(64, n // 64 * 64) if kind < 0.6 else max(8, n // 8 * 8) if kind < 0.8 else n


def draw(rng):
    top = max(_cost(c) for c in listed())
    while True:
        call = rng.choice(["balance", "adapted", "adapted", "adapted", "save", "saved", "saved"])
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        small = rng.random() < 0.3  # a grid of small networks
        if call == "balance":
            e = _log_int(rng, 2, 1000)
            c = _balance("", _log_int(rng, 1, 65536), e, min(e, rng.choice([1, 2, 2, 4, 8])), rng.choice(["f32", "f32", "bf16", "f16"]), masked=rng.random() < 0.5,
                         add=rng.random() < 0.5)
        elif call == "save":
            c = _save("", _log_int(rng, 1, 200000), _width(rng, 32, 2999), dtype)
        elif call == "adapted" and small:
            width = rng.choice([32, 64])
            c = _adapted("", _log_int(rng, 1000, 1 << 19), rng.choice([200, 512, 1600, 4096]), rng.choice([1, 2, 4, 8]), rng.choice([63, width, width + 27]),
                         rng.choice([width, width, width + 1]), dtype, skew=rng.random() < 0.4, drop=rng.choice([0.0, 0.05]), gather=rng.random() < 0.4, bias=True,
                         relu=rng.random() < 0.6, backward=rng.random() < 0.4)
        elif call == "adapted":
            c = _adapted("", _log_int(rng, 1, 32768), _log_int(rng, 1, 128), rng.choice([4, 8, 16, 16, 32, 64, rng.randint(1, 80)]), _width(rng, 32, 2999),
                         _width(rng, 32, 2999), dtype, nk=rng.random() < 0.6, skew=rng.random() < 0.4, drop=rng.choice([0.0, 0.0, 0.1]), gather=rng.random() < 0.3,
                         bias=rng.random() < 0.4, relu=rng.random() < 0.2, backward=rng.random() < 0.4)
        elif small:
            width = rng.choice([32, 64])
            c = _saved("", _log_int(rng, 1000, 1 << 20), rng.choice([200, 512, 1600, 4096]), 1, rng.choice([63, width, width, width + 27]), rng.choice([width, width, width + 1, 3]),
                       dtype, skew=rng.random() < 0.4, drop=rng.choice([0.0, 0.05]), bias=True, relu=rng.random() < 0.7)
        else:
            k = rng.choice([1, 2, 2, 4, 4, 8])
            c = _saved("", _log_int(rng, 1, 32768), max(k, _log_int(rng, 1, 128)), k, _width(rng, 32, 2999), _width(rng, 32, 2999), dtype, skew=rng.random() < 0.4,
                       drop=rng.choice([0.0, 0.0, 0.1]), gather=rng.random() < 0.6, nk=rng.random() < 0.4, bias=rng.random() < 0.4, relu=rng.random() < 0.5)
        del c["name"]
        if c.get("experts", 1) * c.get("n_in", 1) * (c.get("n_out", 1) if call == "saved" else c.get("rank", 1)) <= 1 << 27 and _cost(c) <= top:
            return c


# ---------------------------------------------------------------------------------------------
# work
def work(case):
    c, io = case, ITEM[case["dtype"]]
    if c["call"] == "balance":
        return {"bytes": c["tokens"] * c["experts"] * io * (3 if c["add"] else 2) + 12 * c["experts"], "flops": 0}
    if c["call"] == "save":
        return {"bytes": c["rows"] * (c["width"] * (2 * io + 1) + -(-c["width"] // BLOCK)), "flops": 0}
    m = c["rows"] if c["call"] == "adapted" else c["tokens"] * c["k"]
    met = c["experts"] * (1.0 - (1.0 - 1.0 / c["experts"]) ** m)  # networks that get a row
    k, n = c["n_in"], c["n_out"]
    if c["call"] == "adapted":
        r, once = c["rank"], m * (k + n) * io
        low = c["rank"] * (k + n) * io
        index = 4 * (c["experts"] + 1) + (4 * m if c["gather"] else 0)
        if c["backward"]:
            return {"bytes": 2 * once + k * n * io + (met + c["experts"]) * low + index, "flops": 4 * m * k * n + 6 * m * r * (k + n)}
        return {"bytes": once + k * n * io + met * low + index, "flops": 2 * m * k * n + 2 * m * r * (k + n)}
    xr = c["tokens"] if c["gather"] else m
    kept = 2 * xr * (k + -(-k // BLOCK))
    index = 4 * (c["experts"] + 1) + (4 * m if c["gather"] else 0)
    return {"bytes": xr * k * io + kept + m * (n + k) * io + (met + c["experts"]) * k * n * io + index, "flops": 4 * m * k * n}


def _cost(c):
    """Bytes or operations, whichever is more at the card's rates (full precision: about an eighth of the 16-bit rate)."""
    w = work(c)
    return max(w["bytes"], w["flops"] / 240.0 * (8.0 if c["dtype"] == "f32" else 1.0))


# ---------------------------------------------------------------------------------------------
# inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * (seed + 1))
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _choices(c, g, t, k):
    """(t, k) networks of every token, distinct within a token; -1: none.  Skewed: a few networks get most of the rows."""
    e = c["experts"]
    if k == 1:
        p = torch.full((e,), 1.0, device="cuda")
        if c["skew"]:  # nine rows in ten go to one network in twenty
            hot = torch.randperm(e, generator=g, device="cuda")[: max(1, round(0.05 * e))]
            p[hot] = 9.0 * e / len(hot)
        ids = torch.multinomial(p, t, replacement=True, generator=g).reshape(t, 1)
    else:
        score = _randn(g, t, e)
        if c["skew"]:
            score += 1.5 * _randn(g, e)
        ids = score.topk(k, dim=1).indices
    if c["drop"] > 0.0:
        ids = torch.where(torch.rand((t, 1), generator=g, device="cuda") < c["drop"], -1, ids)
    return ids


def _order(ids, experts):
    """Rows by network, ties by number, those without one last: (pair at each place, offsets)."""
    key = torch.where(ids < 0, experts, ids).reshape(-1)
    order = torch.sort(key, stable=True).indices
    offsets = torch.zeros(experts + 1, dtype=torch.int64, device="cuda")
    offsets[1:] = torch.bincount(key, minlength=experts + 1)[:experts].cumsum(0)
    return order, offsets.to(torch.int32)


def prepare(case, seed):
    c, g = case, _generator(seed)
    dt = DTYPES[c["dtype"]]
    if c["call"] == "balance":
        t, e, k = c["tokens"], c["experts"], c["k"]
        logits = (_randn(g, t, e) + 0.5 * _randn(g, e)).to(dt)
        if c["masked"]:
            closed = torch.rand((t, e), generator=g, device="cuda") < 0.3
            padding = torch.rand((t, 1), generator=g, device="cuda") < 0.03
            logits = logits.masked_fill(closed | padding, -math.inf)
        top, ids = torch.sort(logits.float(), dim=1, descending=True, stable=True)
        _, offsets = _order(torch.where(top[:, :k] == -math.inf, -1, ids[:, :k]), e)
        # small weights beside a loss that is summed over the tokens
        dlosses = torch.tensor([0.01, 0.001], device="cuda") * t * (1.0 + torch.rand(2, generator=g, device="cuda"))
        add = (1e-2 * _randn(g, t, e)).to(dt) if c["add"] else None
        return dict(case=c, logits=logits, offsets=offsets, dlosses=dlosses, add=add)
    if c["call"] == "save":
        x = _randn(g, c["rows"], c["width"]) * torch.exp(_randn(g, c["rows"], 1))
        return dict(case=c, x=x.to(dt))
    e, n_in, n_out = c["experts"], c["n_in"], c["n_out"]
    t, k = (c["rows"], 1) if c["call"] == "adapted" else (c["tokens"], c["k"])
    order, offsets = _order(_choices(c, g, t, k), e)
    rows = (order // k).to(torch.int32) if c["gather"] else None
    x = _randn(g, t if c["gather"] else t * k, n_in)

    def layer(rows_of, columns_of, *more):  # in memory as the program's layers have it
        w = (_randn(g, *more, columns_of, rows_of) if c["nk"] else _randn(g, *more, rows_of, columns_of)).div_(math.sqrt(rows_of)).to(dt)
        return w.transpose(-1, -2) if c["nk"] else w

    if c["call"] == "adapted":
        s = dict(w=layer(n_in, n_out), a=layer(n_in, c["rank"], e), b=layer(c["rank"], n_out, e), scales=0.5 + torch.rand(e, generator=g, device="cuda"),
                 bias=(0.1 * _randn(g, n_out)).to(dt) if c["bias"] else None)
        if c["relu"] and c["backward"]:
            x = x.relu()  # the backward pass of a layer that follows a ReLU
    else:
        s = dict(w=layer(n_in, n_out, e))
        x = x.relu() if c["relu"] else x
    dy = _randn(g, t * k, n_out).to(dt) if c["call"] == "saved" or c["backward"] else None
    return dict(case=c, x=x.to(dt), rows=rows, offsets=offsets, dy=dy, **s)


# ---------------------------------------------------------------------------------------------
# plain forms
def _plain_balance(s):
    c, l = s["case"], s["logits"].float()
    t, e = l.shape
    there = (l != -math.inf).any(1, keepdim=True)
    m = torch.where(there, l.amax(1, keepdim=True), 0.0)
    z = torch.exp(l - m)
    total = z.sum(1, keepdim=True)
    p = torch.where(there, z / total, 0.0)
    lse = torch.where(there, m + torch.log(total), 0.0)
    off = s["offsets"]
    counted = there.sum()
    n = counted.clamp(min=1).double()
    counts = off[1:] - off[:-1]
    probs = p.double().sum(0)
    even = e / (c["k"] * n * n)  # (64 bits: sums over all rows)
    losses = torch.stack([even * (counts * probs).sum(), lse.double().square().sum() / n])
    share = (even * counts).float()
    d = p * (s["dlosses"][0] * (share - (p * share).sum(1, keepdim=True)) + s["dlosses"][1] * ((2.0 / n).float() * lse))
    if s["add"] is not None:
        d = d + s["add"].float()
    return [losses.float(), torch.cat([counts, counted.reshape(1)]).to(torch.int32), probs.float(), d.to(s["logits"].dtype)]


def _pieces(offsets, m):
    """The rows cut into pieces of one network each: (network of the piece, its rows, which of them there are)."""
    e = offsets.numel() - 1
    per = min(512, 1 << max(0, math.ceil(math.log2(max(1.0, m / e)))))
    n = m // per + min(e, m)
    off = offsets.long()
    count = off[1:] - off[:-1]
    last = ((count + per - 1) // per).cumsum(0)
    i = torch.arange(n, device=off.device)
    net = torch.searchsorted(last, i, right=True).clamp_(max=e - 1)
    first = last[net] - (count[net] + per - 1) // per
    row = (off[net] + (i - first) * per)[:, None] + torch.arange(per, device=off.device)
    there = (row < off[net + 1][:, None]) & (i < last[-1])[:, None]
    return net, torch.where(there, row, m), there


def _at(v, row, there):
    return v[row.clamp(max=v.shape[0] - 1)].float() * there[:, :, None]


def _back(pieces, row, m):
    out = torch.zeros((m + 1, pieces.shape[2]), device=pieces.device)
    out[row.reshape(-1)] = torch.where((row < m)[:, :, None], pieces, 0.0).reshape(-1, pieces.shape[2])
    return out[:m]


def _plain_adapted(s):
    c, dt, m = s["case"], s["x"].dtype, s["case"]["rows"]
    net, row, there = _pieces(s["offsets"], m)
    x = (s["x"] if s["rows"] is None else s["x"][s["rows"].long()]).float()
    w, a, b, scale = s["w"].float(), s["a"].float()[net], s["b"].float()[net], s["scales"][net][:, None, None]
    h = scale * torch.matmul(_at(x, row, there), a)
    y = torch.matmul(x, w) + _back(torch.matmul(h, b), row, m)
    y = y if s["bias"] is None else y + s["bias"].float()
    y = (y.relu() if c["relu"] else y).to(dt)
    if not c["backward"]:
        return y
    dy = _at(s["dy"], row, there)
    g = scale * torch.matmul(dy, b.transpose(1, 2))
    dx = torch.matmul(s["dy"].float(), w.t()) + _back(torch.matmul(g, a.transpose(1, 2)), row, m)
    if c["relu"]:
        dx = torch.where(x > 0.0, dx, 0.0)
    da = torch.zeros(s["a"].shape, device=w.device).index_add_(0, net, torch.matmul(_at(x, row, there).transpose(1, 2), g))
    db = torch.zeros(s["b"].shape, device=w.device).index_add_(0, net, torch.matmul(h.transpose(1, 2), dy))
    return [y, dx.to(dt), da.to(dt), db.to(dt)]


def _plain_kept(x):
    """The values that 8 bits and a power of two per 128 of a row stand for; what is above zero stays above zero."""
    r, k = x.shape
    kb = -(-k // BLOCK)
    v = torch.nn.functional.pad(x.float(), (0, kb * BLOCK - k)).reshape(r, kb, BLOCK)
    part, power = torch.frexp(v.abs().amax(2, keepdim=True))
    n = torch.where(part > 0.0, power - 9 + (part > 0.875), LEAST).clamp(min=LEAST)
    v = torch.ldexp(v, -n)
    q = torch.where((v > 0.0) & (v <= F8_STEP / 2), F8_STEP, v.to(F8).float())
    return torch.ldexp(q, n).reshape(r, kb * BLOCK)[:, :k]


def _plain_saved(s):
    c, w, dt = s["case"], s["w"], s["x"].dtype
    m = c["tokens"] * c["k"]
    kept = _plain_kept(s["x"])
    net, row, there = _pieces(s["offsets"], m)
    x = _at(kept, row if s["rows"] is None else s["rows"].long()[row.clamp(max=m - 1)], there)
    dy = _at(s["dy"], row, there)
    dx = torch.matmul(dy, w[net].float().transpose(1, 2))
    if c["relu"]:
        dx = torch.where(x > 0.0, dx, 0.0)
    dw = torch.zeros(w.shape, device=w.device).index_add_(0, net, torch.matmul(x.transpose(1, 2), dy))
    out = [_back(dx, row, m).to(dt), dw.to(dt)]
    if c["bias"]:
        out.append(torch.zeros((c["experts"], c["n_out"]), device=w.device).index_add_(0, net, dy.sum(1)).to(dt))
    return out


def run(state):
    s, c = state, state["case"]
    if not own:
        if c["call"] == "save":
            return _plain_kept(s["x"]).to(s["x"].dtype)
        return {"balance": _plain_balance, "adapted": _plain_adapted, "saved": _plain_saved}[c["call"]](s)
    import paper_2103_13744_amd as kn
    if c["call"] == "balance":
        losses, counts, probs = kn.route_balance(s["logits"], c["k"], s["offsets"])
        return [losses, counts, probs, kn.route_balance_backward(s["logits"], c["k"], counts, s["dlosses"], add=s["add"])]
    if c["call"] == "save":
        q, e = kn.save_f8(s["x"])
        return kn.restore_f8(q, e, c["width"], s["x"].dtype)
    if c["call"] == "adapted":
        if not c["backward"]:
            return kn.adapted_linear(s["x"], s["w"], s["a"], s["b"], s["offsets"], rows=s["rows"], scales=s["scales"], bias=s["bias"], relu=c["relu"])
        y, h = kn.adapted_linear(s["x"], s["w"], s["a"], s["b"], s["offsets"], rows=s["rows"], scales=s["scales"], bias=s["bias"], relu=c["relu"], want_h=True)
        return [y, *kn.adapted_linear_backward(s["dy"], s["x"], h, s["w"], s["a"], s["b"], s["offsets"], rows=s["rows"], scales=s["scales"], relu_in=c["relu"])]
    q, e = kn.save_f8(s["x"])
    dx, dw, db = kn.grouped_linear_backward_saved(s["dy"], q, e, s["w"], s["offsets"], rows=s["rows"], relu_in=c["relu"], want_bias=c["bias"])
    return [dx, dw, db] if c["bias"] else [dx, dw]


# ---------------------------------------------------------------------------------------------
# the definitions in 64 bits
def _exact_kept(x):
    """Rounded by hand: an e4m3 value's neighbours lie 2^(e - 3) apart between 2^e and 2^(e + 1), and 2^-9 below 2^-6."""
    x = x.double()
    out = torch.empty_like(x)
    for k0 in range(0, x.shape[1], BLOCK):
        v = x[:, k0:k0 + BLOCK]
        most = v.abs().amax(1, keepdim=True)
        scale = torch.full_like(most, 2.0 ** LEAST)
        for n in range(LEAST, 128):  # the least power of two that brings the largest into the type
            scale = torch.where(most > F8_MAX * 2.0 ** n, 2.0 ** (n + 1), scale)
        u = v / scale
        step = torch.exp2(torch.floor(torch.log2(u.abs().clamp(min=2.0 ** -6))) - 3.0)
        q = torch.round(u / step) * step
        out[:, k0:k0 + BLOCK] = torch.where((u > 0.0) & (q == 0.0), 2.0 ** -9, q) * scale
    return out


def exact(case, seed):
    c, s = case, prepare(case, seed)
    f64 = torch.float64
    if c["call"] == "save":
        return _exact_kept(s["x"])
    if c["call"] == "balance":
        l, e = s["logits"].double(), c["experts"]
        rows = (l > -math.inf).any(1).nonzero()[:, 0]
        n, counts = len(rows), torch.diff(s["offsets"].double())
        some = l[rows]
        p, z = torch.softmax(some, 1), torch.logsumexp(some, 1)
        d = torch.zeros_like(l)
        if n:
            gain = s["dlosses"][0].double() * e / (c["k"] * n * n) * counts + (s["dlosses"][1].double() * 2.0 / n * z)[:, None]
            mean = s["dlosses"][0].double() * e / (c["k"] * n * n) * (p @ counts)
            d[rows] = p * (gain - mean[:, None])
        if s["add"] is not None:
            d += s["add"].double()
        losses = torch.stack([(e * (counts / (c["k"] * n)) * (p.sum(0) / n)).sum(), (z * z).mean()]) if n else torch.zeros(2, dtype=f64, device="cuda")
        return [losses, None, p.sum(0), d]
    off = s["offsets"].tolist()
    m = c["rows"] if c["call"] == "adapted" else c["tokens"] * c["k"]
    at = torch.arange(m, device="cuda") if s["rows"] is None else s["rows"].long()
    zeros = lambda *shape: torch.zeros(shape, dtype=f64, device="cuda")  # noqa: E731
    if c["call"] == "adapted":
        x, w = s["x"][at].double(), s["w"].double()
        y, dx = x @ w, s["dy"].double() @ w.T if c["backward"] else None
        da, db = zeros(*s["a"].shape), zeros(*s["b"].shape)
        for e, (i, j) in enumerate(zip(off[:-1], off[1:])):
            if i == j:
                continue
            a, b, scale = s["a"][e].double(), s["b"][e].double(), s["scales"][e].double()
            h = scale * (x[i:j] @ a)
            y[i:j] += h @ b
            if c["backward"]:
                dy = s["dy"][i:j].double()
                g = scale * (dy @ b.T)
                dx[i:j] += g @ a.T
                da[e], db[e] = x[i:j].T @ g, h.T @ dy
        if s["bias"] is not None:
            y += s["bias"].double()
        y = y.clamp(min=0.0) if c["relu"] else y
        return [y, dx * (x > 0.0) if c["relu"] else dx, da, db] if c["backward"] else y
    kept = _exact_kept(s["x"])
    dx, dw, dbias = zeros(m, c["n_in"]), zeros(c["experts"], c["n_in"], c["n_out"]), zeros(c["experts"], c["n_out"])
    for e, (i, j) in enumerate(zip(off[:-1], off[1:])):
        if i == j:
            continue
        x, dy = kept[at[i:j]], s["dy"][i:j].double()
        dx[i:j] = dy @ s["w"][e].double().T
        if c["relu"]:
            dx[i:j] *= x > 0.0
        dw[e], dbias[e] = x.T @ dy, dy.sum(0)
    return [dx, dw, dbias] if c["bias"] else [dx, dw]
