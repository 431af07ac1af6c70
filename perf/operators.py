"""What is timed: the operators of networks that are chosen per row, by a cell or by a learned router.

A program that trains or serves such networks sends every token (or sample) to k of E networks (``kn.route``), multiplies each
network's rows with that network's own weights (``kn.grouped_linear``, its gradients ``kn.grouped_linear_backward``, or for
serving ``kn.grouped_linear_f8`` on weights kept in 8 bits), and sums every token's k results (``kn.combine``).  Each case is one
such call, or a forward call with its gradient, on seeded inputs made on the GPU.  Rows are in the order of their networks, rows of
no network (-1: a padding token, a point outside the box) last.

With ``own`` false the same results come from elementary torch operations in 32 bits: a ragged product is cut into pieces of at
most so many rows of one network, and the pieces are multiplied as a batch.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ITEM = {"f32": 4, "f16": 2, "bf16": 2}
F8, F8_MAX, F8_TINY, BLOCK = torch.float8_e4m3fn, 448.0, 2.0 ** -100, 128


def _route(name, tokens, experts, k, dtype, renorm=True, masked=False, backward=False):
    return dict(name=name, call="route", tokens=tokens, experts=experts, k=k, dtype=dtype, renorm=renorm, masked=masked, backward=backward)


def _linear(name, tokens, experts, k, n_in, n_out, dtype, skew=False, drop=0.0, gather=True, nk=False, bias=False, relu=False, backward=False):
    return dict(name=name, call="linear", tokens=tokens, experts=experts, k=k, n_in=n_in, n_out=n_out, dtype=dtype, skew=skew,
                drop=drop, gather=gather, nk=nk, bias=bias, relu=relu, backward=backward)


def _linear_f8(name, tokens, experts, k, n_in, n_out, dtype, skew=False, drop=0.0, gather=True):
    return dict(name=name, call="linear_f8", tokens=tokens, experts=experts, k=k, n_in=n_in, n_out=n_out, dtype=dtype, skew=skew,
                drop=drop, gather=gather)


def _combine(name, tokens, k, width, dtype, backward=False):
    return dict(name=name, call="combine", tokens=tokens, k=k, width=width, dtype=dtype, backward=backward)


def listed():
    return [
        # the router of one serving step: a few tokens, latency
        _route("route_decode", 16, 64, 4, "f32"),
        # the router of a training step, padding tokens and experts that are closed for some tokens among its rows
        _route("route_train", 32768, 128, 8, "f32", masked=True, backward=True),
        # first layer of a grid of 16^3 small networks in full precision (63 encoded inputs, 32 units), points of a scene
        _linear("fwd_nets_f32", 262145, 4096, 1, 63, 32, "f32", skew=True, drop=0.02, bias=True, relu=True),
        # one serving step: eight tokens, most experts without a row
        _linear("fwd_decode_bf16", 8, 64, 4, 2048, 1024, "bf16"),
        # a long prompt or a training batch, forward
        _linear("fwd_prefill_bf16", 16384, 64, 4, 2048, 1024, "bf16", skew=True, bias=True, relu=True),
        # a small layer of odd sizes in full precision, with its gradients
        _linear("bwd_odd_f32", 1001, 5, 1, 259, 131, "f32", gather=False, bias=True, backward=True),
        # a hidden layer of a grid of wide small networks: the paper's training path, backward
        _linear("bwd_nets_f16", 524291, 4096, 1, 64, 64, "f16", gather=False, drop=0.02, bias=True, relu=True, backward=True),
        # a training step's experts, backward
        _linear("bwd_train_bf16", 8192, 32, 4, 1024, 2048, "bf16", skew=True, backward=True),
        # one serving step with weights in 8 bits
        _linear_f8("f8_decode", 16, 32, 2, 2560, 2048, "bf16"),
        # a long prompt with weights in 8 bits
        _linear_f8("f8_prefill", 16411, 16, 2, 2048, 2048, "bf16", skew=True, drop=0.02),
        # the experts' results of one serving step
        _combine("combine_decode", 16, 4, 2048, "bf16"),
        # the same of a training step, with its gradient
        _combine("combine_train", 16384, 4, 2048, "bf16", backward=True),
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
        call = rng.choice(["route", "linear", "linear", "linear", "linear", "linear_f8", "linear_f8", "combine"])
        tokens, k = _log_int(rng, 1, 32768), rng.choice([1, 2, 2, 4, 4, 6, 8])
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        if call == "route":
            c = _route("", tokens, max(k, _log_int(rng, 4, 256)), k, rng.choice(["f32", "f32", "bf16"]), renorm=rng.random() < 0.7,
                       masked=rng.random() < 0.4, backward=rng.random() < 0.5)
        elif call == "combine":
            c = _combine("", tokens, k, _width(rng, 32, 2999), dtype, backward=rng.random() < 0.5)
        elif call == "linear_f8":
            c = _linear_f8("", tokens, max(k, _log_int(rng, 1, 64)), k, _width(rng, 64, 2999), _width(rng, 32, 2999), rng.choice(["bf16", "bf16", "f16"]),
                           skew=rng.random() < 0.4, drop=rng.choice([0.0, 0.0, 0.1]), gather=rng.random() < 0.7)
        elif rng.random() < 0.3:  # a grid of small networks
            width = rng.choice([32, 64])
            c = _linear("", _log_int(rng, 1000, 1 << 20), rng.choice([200, 512, 1600, 4096]), 1, rng.choice([63, width, width, width + 27]),
                        rng.choice([width, width, width + 1, 3]), dtype, skew=rng.random() < 0.4, drop=rng.choice([0.0, 0.05]),
                        gather=rng.random() < 0.5, bias=True, relu=rng.random() < 0.7, backward=rng.random() < 0.5)
        else:
            c = _linear("", tokens, max(k, _log_int(rng, 1, 128)), k, _width(rng, 32, 2999), _width(rng, 32, 2999), dtype, skew=rng.random() < 0.4,
                        drop=rng.choice([0.0, 0.0, 0.1]), gather=rng.random() < 0.6, nk=rng.random() < 0.4, bias=rng.random() < 0.4,
                        relu=rng.random() < 0.4, backward=rng.random() < 0.5)
        del c["name"]
        if c.get("experts", 1) * c.get("n_in", 1) * c.get("n_out", 1) <= 1 << 27 and _cost(c) <= top:
            return c


# ---------------------------------------------------------------------------------------------
# work
def work(case):
    c = case
    m = c["tokens"] * c["k"]
    if c["call"] == "route":
        logits = c["tokens"] * c["experts"] * ITEM[c["dtype"]]
        return {"bytes": logits * (2 if c["backward"] else 1) + m * (20 if c["backward"] else 16) + 4 * (c["experts"] + 1), "flops": 0}
    if c["call"] == "combine":
        w, io = c["width"], ITEM[c["dtype"]]
        return {"bytes": (m + c["tokens"]) * w * io * (2 if c["backward"] else 1) + m * (12 if c["backward"] else 8),
                "flops": 2 * m * w * (2.5 if c["backward"] else 1)}
    met = c["experts"] * (1.0 - (1.0 - 1.0 / c["experts"]) ** m)  # experts that get a row
    x = (c["tokens"] if c["gather"] else m) * c["n_in"] * ITEM[c["dtype"]]
    y = m * c["n_out"] * ITEM[c["dtype"]]
    index = 4 * (c["experts"] + 1) + (4 * m if c["gather"] else 0)
    if c["call"] == "linear_f8":
        return {"bytes": x + y + index + met * c["n_in"] * c["n_out"], "flops": 2 * m * c["n_in"] * c["n_out"]}
    w = c["n_in"] * c["n_out"] * ITEM[c["dtype"]]
    if c["backward"]:
        dx = m * c["n_in"] * ITEM[c["dtype"]]
        return {"bytes": x + y + dx + index + met * w + c["experts"] * w, "flops": 4 * m * c["n_in"] * c["n_out"]}
    return {"bytes": x + y + index + met * w, "flops": 2 * m * c["n_in"] * c["n_out"]}


def _cost(c):
    """Bytes or operations, whichever is more at the card's rates (full precision: about a sixteenth of the 16-bit rate)."""
    w = work(c)
    return max(w["bytes"], w["flops"] / 300.0 * (16.0 if c["dtype"] == "f32" else 1.0))


# ---------------------------------------------------------------------------------------------
# inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * (seed + 1))
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _choices(c, g):
    """(tokens, k) experts of every token, distinct within a token; -1: none.  Skewed: a few experts get most of the rows."""
    t, e, k = c["tokens"], c["experts"], c["k"]
    if k == 1:
        p = torch.full((e,), 1.0, device="cuda")
        if c["skew"]:  # nine rows in ten go to one expert in twenty
            hot = torch.randperm(e, generator=g, device="cuda")[: max(1, round(0.05 * e))]
            p[hot] = 9.0 * e / len(hot)
        ids = torch.multinomial(p, t, replacement=True, generator=g).reshape(t, 1)
    else:
        score = _randn(g, t, e)
        if c["skew"]:
            score += 1.5 * _randn(g, e)
        ids = score.topk(k, dim=1).indices
    if c.get("drop", 0.0) > 0.0:
        ids = torch.where(torch.rand((t, 1), generator=g, device="cuda") < c["drop"], -1, ids)
    return ids


def _order(ids, experts):
    """Rows by expert, ties by number, those without an expert last: (pair at each place, offsets)."""
    key = torch.where(ids < 0, experts, ids).reshape(-1)
    order = torch.sort(key, stable=True).indices
    offsets = torch.zeros(experts + 1, dtype=torch.int64, device="cuda")
    offsets[1:] = torch.bincount(key, minlength=experts + 1)[:experts].cumsum(0)
    return order, offsets.to(torch.int32)


def _f8_blocks(v):
    """Values of whole blocks as (their e4m3 forms, scales): the scale brings a block's largest magnitude to the type's."""
    s = v.abs().amax(dim=(-3, -1), keepdim=True).clamp(min=F8_TINY) / F8_MAX
    return (v / s).to(F8), s


def _f8_weights(w):
    """(E, N, K) weights as a program keeps them: e4m3 with inputs padded by zeros to whole blocks, a scale per 128 x 128."""
    e, n, k = w.shape
    nb, kb = -(-n // BLOCK), -(-k // BLOCK)
    v = torch.zeros((e, nb * BLOCK, kb * BLOCK), dtype=torch.float32, device=w.device)
    v[:, :n, :k] = w
    q, s = _f8_blocks(v.reshape(e, nb, BLOCK, kb, BLOCK))
    return q.reshape(e, nb * BLOCK, kb * BLOCK)[:, :n].contiguous(), s.reshape(e, nb, kb).contiguous()


def prepare(case, seed):
    c, g = case, _generator(seed)
    t, k, dt = c["tokens"], c["k"], DTYPES[c["dtype"]]
    if c["call"] == "route":
        logits = _randn(g, t, c["experts"]) + 0.5 * _randn(g, c["experts"])
        if c["masked"]:
            closed = torch.rand(logits.shape, generator=g, device="cuda") < 0.3
            padding = torch.rand((t, 1), generator=g, device="cuda") < 0.03
            logits = logits.masked_fill(closed | padding, -math.inf)
        return dict(case=c, logits=logits.to(dt), dweights=_randn(g, t, k))
    if c["call"] == "combine":
        slots = torch.randperm(t * k, generator=g, device="cuda").to(torch.int32).reshape(t, k)
        weights = torch.softmax(_randn(g, t, k), dim=1)
        return dict(case=c, y=_randn(g, t * k, c["width"]).to(dt), slots=slots, weights=weights, dout=_randn(g, t, c["width"]).to(dt))
    e, n_in, n_out = c["experts"], c["n_in"], c["n_out"]
    order, offsets = _order(_choices(c, g), e)
    rows = (order // k).to(torch.int32) if c["gather"] else None
    x = _randn(g, t if c["gather"] else t * k, n_in)
    if c["call"] == "linear_f8":
        w = torch.empty((e, n_out, n_in), device="cuda")
        for i in range(e):
            w[i] = _randn(g, n_out, n_in) / math.sqrt(n_in)
        wq, ws = _f8_weights(w)
        return dict(case=c, x=x.to(dt), rows=rows, offsets=offsets, wq=wq, ws=ws)
    if c["relu"] and c["backward"]:
        x = x.relu()  # the backward pass of a layer that follows a ReLU
    w = (_randn(g, e, n_out, n_in) if c["nk"] else _randn(g, e, n_in, n_out)).div_(math.sqrt(n_in)).to(dt)
    w = w.transpose(1, 2) if c["nk"] else w  # (E, n_in, n_out) either way; in memory as the program's layers have it
    bias = (0.1 * _randn(g, e, n_out)).to(dt) if c["bias"] else None
    dy = _randn(g, t * k, n_out).to(dt) if c["backward"] else None
    return dict(case=c, x=x.to(dt), rows=rows, offsets=offsets, w=w, bias=bias, dy=dy)


# ---------------------------------------------------------------------------------------------
# plain forms
def _plain_route(s):
    c, k = s["case"], s["case"]["k"]
    logits = s["logits"].float()
    t, e = logits.shape
    top, ids = torch.sort(logits, dim=1, descending=True, stable=True)
    top, ids = top[:, :k], torch.where(top[:, :k] == -math.inf, -1, ids[:, :k])
    some = ids[:, :1] >= 0
    m = torch.where(some, top[:, :1], 0.0)
    z = torch.exp(top - m)
    total = z.sum(1, keepdim=True) if c["renorm"] else torch.exp(logits - m).sum(1, keepdim=True)
    weights = torch.where(some, z / total, 0.0)
    key = torch.where(ids < 0, e, ids).reshape(-1)
    order = torch.sort(key, stable=True).indices
    slots = torch.empty_like(order)
    slots[order] = torch.arange(t * k, device=order.device)
    offsets = torch.searchsorted(key[order], torch.arange(e + 1, device=order.device))
    i32 = torch.int32
    out = [weights, ids.to(i32), slots.reshape(t, k).to(i32), (order // k).to(i32), offsets.to(i32)]
    if c["backward"]:
        g = torch.where(ids >= 0, s["dweights"], 0.0)
        mean = (weights * g).sum(1, keepdim=True)
        at = torch.where(ids >= 0, ids, e)
        d = torch.zeros((t, e + 1), device=g.device)
        if c["renorm"]:
            d.scatter_(1, at, weights * (g - mean))
        else:
            d[:, :e] = torch.where(some, torch.exp(logits - m) / total * -mean, 0.0)
            d.scatter_add_(1, at, weights * g)
        out.append(d[:, :e].to(s["logits"].dtype))
    return out


def _pieces(offsets, m):
    """The rows cut into pieces of one expert each: (expert of the piece, its rows, which of them there are)."""
    e = offsets.numel() - 1
    per = min(512, 1 << max(0, math.ceil(math.log2(max(1.0, m / e)))))
    n = m // per + min(e, m)
    off = offsets.long()
    count = off[1:] - off[:-1]
    last = ((count + per - 1) // per).cumsum(0)
    i = torch.arange(n, device=off.device)
    expert = torch.searchsorted(last, i, right=True).clamp_(max=e - 1)
    first = last[expert] - (count[expert] + per - 1) // per
    row = (off[expert] + (i - first) * per)[:, None] + torch.arange(per, device=off.device)
    there = (row < off[expert + 1][:, None]) & (i < last[-1])[:, None]
    return expert, torch.where(there, row, m), there


def _at(v, row, there):
    return v[row.clamp(max=v.shape[0] - 1)].float() * there[:, :, None]


def _back(pieces, row, m, dtype):
    out = torch.zeros((m + 1, pieces.shape[2]), device=pieces.device)
    out[row.reshape(-1)] = torch.where((row < m)[:, :, None], pieces, 0.0).reshape(-1, pieces.shape[2])
    return out[:m].to(dtype)


def _plain_linear(s):
    c, w, dt = s["case"], s["w"], s["x"].dtype
    m = c["tokens"] * c["k"]
    expert, row, there = _pieces(s["offsets"], m)
    source = row if s["rows"] is None else s["rows"].long()[row.clamp(max=m - 1)]
    x = _at(s["x"], source, there)
    if not c["backward"]:
        y = torch.matmul(x, w[expert].float())
        if s["bias"] is not None:
            y = y + s["bias"][expert].float()[:, None, :]
        return _back(y.relu() if c["relu"] else y, row, m, dt)
    dy = _at(s["dy"], row, there)
    dx = torch.matmul(dy, w[expert].float().transpose(1, 2))
    if c["relu"]:
        dx = torch.where(x > 0.0, dx, 0.0)
    dw = torch.zeros(w.shape, device=w.device).index_add_(0, expert, torch.matmul(x.transpose(1, 2), dy))
    out = [_back(dx, row, m, dt), dw.to(dt)]
    if s["bias"] is not None:
        out.append(torch.zeros(s["bias"].shape, device=w.device).index_add_(0, expert, dy.sum(1)).to(dt))
    return out


def _plain_linear_f8(s):
    c, x = s["case"], s["x"].float()
    m, kp = c["tokens"] * c["k"], s["wq"].shape[2]
    x = torch.nn.functional.pad(x, (0, kp - x.shape[1]))
    q, sx = _f8_blocks(x.reshape(-1, 1, kp // BLOCK, BLOCK))
    x = (q.float() * sx).reshape(-1, kp)
    expert, row, there = _pieces(s["offsets"], m)
    source = row if s["rows"] is None else s["rows"].long()[row.clamp(max=m - 1)]
    sw = s["ws"].repeat_interleave(BLOCK, 1)[:, : c["n_out"]].repeat_interleave(BLOCK, 2)
    w = s["wq"].float() * sw
    return _back(torch.matmul(_at(x, source, there), w[expert].transpose(1, 2)), row, m, s["x"].dtype)


def _plain_combine(s):
    y, w = s["y"][s["slots"].long()].float(), s["weights"]
    if not s["case"]["backward"]:
        return (y * w[:, :, None]).sum(1).to(s["y"].dtype)
    dout = s["dout"].float()
    dy = torch.empty_like(s["y"])
    dy[s["slots"].long().reshape(-1)] = (dout[:, None, :] * w[:, :, None]).reshape(-1, dout.shape[1]).to(dy.dtype)
    return [(y * w[:, :, None]).sum(1).to(s["y"].dtype), dy, (y * dout[:, None, :]).sum(2)]


def run(state):
    s, c = state, state["case"]
    if not own:
        return {"route": _plain_route, "linear": _plain_linear, "linear_f8": _plain_linear_f8, "combine": _plain_combine}[c["call"]](s)
    import paper_2103_13744_amd as kn
    if c["call"] == "route":
        out = list(kn.route(s["logits"], c["k"], renormalize=c["renorm"]))
        if c["backward"]:
            out.append(kn.route_backward(s["logits"], out[0], out[1], s["dweights"], renormalize=c["renorm"]))
        return out
    if c["call"] == "combine":
        out = kn.combine(s["y"], s["slots"], s["weights"])
        return [out, *kn.combine_backward(s["dout"], s["y"], s["slots"], s["weights"])] if c["backward"] else out
    if c["call"] == "linear_f8":
        xq, xs = kn.quantize_f8(s["x"])
        return kn.grouped_linear_f8(xq, xs, s["wq"], s["ws"], s["offsets"], rows=s["rows"], dtype=s["x"].dtype)
    if not c["backward"]:
        return kn.grouped_linear(s["x"], s["w"], s["offsets"], rows=s["rows"], bias=s["bias"], relu=c["relu"])
    dx, dw, db = kn.grouped_linear_backward(s["dy"], s["x"], s["w"], s["offsets"], rows=s["rows"], relu_in=c["relu"], want_bias=c["bias"])
    return [dx, dw, db] if c["bias"] else [dx, dw]


# ---------------------------------------------------------------------------------------------
# the definitions in 64 bits
def exact(case, seed):
    c, s = case, prepare(case, seed)
    d = lambda v: None if v is None else v.to(torch.float64)  # noqa: E731
    if c["call"] == "route":
        l, t, k, e = d(s["logits"]), c["tokens"], c["k"], c["experts"]
        left, number, ids = l.clone(), torch.arange(e, device="cuda"), []
        for _ in range(k):
            best = left.amax(1, keepdim=True)
            i = torch.where(left == best, number, e).amin(1)
            left.scatter_(1, i[:, None], -math.inf)
            ids.append(torch.where(best[:, 0] == -math.inf, -1, i))
        ids = torch.stack(ids, 1)
        chosen = torch.zeros((t, e + 1), dtype=torch.bool, device="cuda").scatter_(1, ids % (e + 1), True)[:, :e]
        p = torch.softmax(l.masked_fill(~chosen, -math.inf) if c["renorm"] else l, dim=1).nan_to_num(0.0)
        weights = torch.where(ids >= 0, p.gather(1, ids.clamp(min=0)), 0.0)
        out = [weights, None, None, None, None]
        if c["backward"]:
            g = torch.zeros((t, e), dtype=torch.float64, device="cuda").scatter_add_(1, ids.clamp(min=0), torch.where(ids >= 0, d(s["dweights"]), 0.0))
            out.append(p * (g - (p * g).sum(1, keepdim=True)))
        return out
    if c["call"] == "combine":
        n, t, k = c["tokens"] * c["k"], c["tokens"], c["k"]
        place = torch.empty(n, dtype=torch.int64, device="cuda")
        place[s["slots"].long().reshape(-1)] = torch.arange(n, device="cuda")  # the pair at each row
        y, w = d(s["y"]), d(s["weights"]).reshape(-1)
        out = torch.zeros((t, c["width"]), dtype=torch.float64, device="cuda").index_add_(0, place // k, y * w[place][:, None])
        if not c["backward"]:
            return out
        dout = d(s["dout"])[place // k]
        dw = torch.empty(n, dtype=torch.float64, device="cuda")
        dw[place] = torch.linalg.vecdot(dout, y)
        return [out, dout * w[place][:, None], dw.reshape(t, k)]
    m, off = c["tokens"] * c["k"], s["offsets"].tolist()
    rows = torch.arange(m, device="cuda") if s["rows"] is None else s["rows"].long()
    x = s["x"]
    if c["call"] == "linear_f8":  # the quantised values are what the product is defined on
        x = torch.nn.functional.pad(x.float(), (0, s["wq"].shape[2] - x.shape[1])).reshape(x.shape[0], -1, BLOCK)
        scale = x.abs().amax(2, keepdim=True).clamp(min=F8_TINY) / F8_MAX
        x = ((x / scale).to(F8).double() * scale.double()).flatten(1)
    out = torch.zeros((m, c["n_out"]), dtype=torch.float64, device="cuda")
    dx, dw = (torch.zeros((m, c["n_in"]), dtype=torch.float64, device="cuda"), torch.zeros((c["experts"], c["n_in"], c["n_out"]), dtype=torch.float64, device="cuda")) if c.get("backward") else (None, None)
    db = torch.zeros((c["experts"], c["n_out"]), dtype=torch.float64, device="cuda") if c.get("backward") else None
    for e in range(c["experts"]):
        a, b = off[e], off[e + 1]
        if a == b:
            continue
        xe = d(x[rows[a:b]])
        if c["call"] == "linear_f8":
            wide = s["ws"][e].double().repeat_interleave(BLOCK, 0)[: c["n_out"]].repeat_interleave(BLOCK, 1)
            out[a:b] = xe @ (s["wq"][e].double() * wide).T
        elif not c["backward"]:
            y = xe @ d(s["w"][e])
            y = y + d(s["bias"][e]) if s["bias"] is not None else y
            out[a:b] = y.clamp(min=0.0) if c["relu"] else y
        else:
            dy = d(s["dy"][a:b])
            dx[a:b] = dy @ d(s["w"][e]).T
            if c["relu"]:
                dx[a:b] *= xe > 0.0
            dw[e], db[e] = xe.T @ dy, dy.sum(0)
    if not c.get("backward"):
        return out
    return [dx, dw, db] if c["bias"] else [dx, dw]
