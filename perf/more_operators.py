"""A layer of experts on the device as timed cases: the router (the k best experts of a row, their weights, counts and balance loss, and the gradient), rows sorted by
expert, handed out and put together again, products grouped by label with bias, activation and residual (forward, backward, and forward in 8 bits), and dropout.

A case is a dict of plain values.  Common keys:
  do         "route", "exchange" (sort, hand out, put together), "linear" (product with its epilogue), "linear8" (the same of 8-bit matrices) or "dropout"
  precision  "fp32" or "bf16": storage type of logits, activations and weights
  train      whether the backward pass is part of the pass
  rows       rows of the batch
route:     experts, k, normalize (the weights of a row's choices add up to one), masked (some experts are not there for some rows, and some rows are padding)
exchange:  experts, k, cols, masked (some choices are of no expert), residual
linear:    groups (experts), n_in, n_out, act ("none", "relu", "gelu" or "silu"), residual, mix: how the rows fall to the experts, "even", "drawn" (independent
           uniform labels) or "skew" (a few experts get most rows and some none)
dropout:   cols, p, residual

8-bit matrices hold e4m3 values in rows padded to 128 with zeros, and a byte E + 127 for each 128 values of a row: value = code * 2^E.
"""
import math

import numpy as np
import torch

own = False

BALANCE = 0.01                                   # the balance loss's share in the whole loss
SEED, SITE, STEP = 0x1234567890ABCDEF, 3, 11     # of the dropout's bits
ACTS = ["none", "relu", "gelu", "silu"]


def listed():
    def route(name, precision, train, rows, experts, k, normalize=True, masked=False):
        return dict(name=name, do="route", precision=precision, train=train, rows=rows, experts=experts, k=k, normalize=normalize, masked=masked)

    def exchange(name, precision, train, rows, experts, k, cols, masked=False, residual=True):
        return dict(name=name, do="exchange", precision=precision, train=train, rows=rows, experts=experts, k=k, cols=cols, masked=masked, residual=residual)

    def linear(name, precision, train, groups, rows, n_in, n_out, mix, act, residual=False, eight=False):
        return dict(name=name, do="linear8" if eight else "linear", precision=precision, train=train, groups=groups, rows=rows, n_in=n_in, n_out=n_out, mix=mix, act=act,
                    residual=residual)

    def dropout(name, precision, train, rows, cols, p, residual=True):
        return dict(name=name, do="dropout", precision=precision, train=train, rows=rows, cols=cols, p=p, residual=residual)

    return [
        # four tokens of a request to a model of 64 experts: a call that is all latency
        route("route 4 rows", "fp32", False, 4, 64, 2),
        # a training batch of a hundred label models whose labels are not known: each sample to the likeliest expert, an odd number of them, some padding
        route("route train 6397x100 fp32", "fp32", True, 6397, 100, 1, normalize=False, masked=True),
        # a long training batch over many small experts
        route("route train 65536x256 bf16", "bf16", True, 65536, 256, 8),
        # ten samples on demand from a hundred experts: sort, hand out, put together
        exchange("exchange 10 rows bf16", "bf16", False, 10, 100, 1, 1024),
        # an odd batch of odd rows in single precision, three experts each, some choices of none
        exchange("exchange train 1117x1000 fp32", "fp32", True, 1117, 10, 3, 1000, masked=True),
        # a long training batch, two of eight experts each
        exchange("exchange train 16384x4096 bf16", "bf16", True, 16384, 8, 2, 4096),
        # ten samples on demand, each from one of a hundred experts: reads the weights of those experts once
        linear("linear gelu 10 rows bf16", "bf16", False, 100, 10, 1024, 1024, "drawn", "gelu"),
        # the hidden layer of ten digit models in single precision, an odd total
        linear("linear train relu fp32 784-512", "fp32", True, 10, 1117, 784, 512, "drawn", "relu", residual=True),
        # eight large experts over a long training batch
        linear("linear train gelu 8x4096 bf16", "bf16", True, 8, 16384, 4096, 4096, "drawn", "gelu", residual=True),
        # a batch of requests through eight large experts whose weights are held in 8 bits
        linear("linear8 silu 256 rows", "bf16", False, 8, 256, 4096, 4096, "drawn", "silu", residual=True, eight=True),
        # an odd batch in single precision
        dropout("dropout train 1117x1000 fp32", "fp32", True, 1117, 1000, 0.25),
        # a long training batch behind a layer of experts
        dropout("dropout train 16384x4096 bf16", "bf16", True, 16384, 4096, 0.1),
    ]


def draw(rng):
    """One more case of the same ranges, sizes spread over their logarithms, odd ones among them."""
    limit = max(_cost(c) for c in listed())

    def size(lo, hi):
        v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        to = rng.choice([1, 8, 32, 64, 128])                    # widths are mostly, and not always, round numbers
        return max(lo, min(hi, v if to == 1 else -(-v // to) * to))

    while True:
        do = rng.choice(["route", "route", "exchange", "exchange", "linear", "linear", "linear", "linear8", "dropout"])
        c = dict(do=do, precision=rng.choice(["fp32", "bf16", "bf16"]), train=rng.random() < 0.6, rows=size(1, 16384))
        if do == "route":
            experts = size(2, 512)
            c.update(rows=size(1, 65536), experts=experts, k=rng.randint(1, min(8, experts)), normalize=rng.random() < 0.5, masked=rng.random() < 0.4)
        elif do == "exchange":
            c.update(experts=size(1, 256), k=rng.randint(1, 4), cols=size(64, 8192), masked=rng.random() < 0.4, residual=rng.random() < 0.7)
            if c["rows"] * c["k"] * c["cols"] > 1 << 27:
                continue
        elif do == "dropout":
            c.update(cols=size(64, 8192), p=rng.choice([0.1, 0.25, 0.5, round(rng.random() * 0.9, 3)]), residual=rng.random() < 0.7)
        else:
            c.update(groups=size(1, 128), n_in=size(48, 4096), n_out=size(48, 4096), mix=rng.choice(["even", "drawn", "skew"]), act=rng.choice(ACTS),
                     residual=rng.random() < 0.6)
            if do == "linear8":
                c.update(precision="bf16", train=False)
            if c["groups"] * c["n_in"] * c["n_out"] > 1 << 28 or _longest_bound(c) * c["groups"] * (c["n_in"] + c["n_out"]) > 1 << 30:
                continue
        if _cost(c) <= limit:
            return c


def _longest_bound(c):
    return c["rows"] if c["mix"] == "skew" else 2 * c["rows"] // c["groups"] + 64


def _cost(case):
    """Seconds of the work alone at round rates."""
    w = work(case)
    return max(w["bytes"] / 5e12, w["flops"] / (1e15 if case["precision"] == "bf16" else 2e14))


# ---- the 8-bit format ---------------------------------------------------------------------------------------------------

def _to_8_bits(x):
    """fp32 [rows, cols] to (e4m3 [rows, padded cols], bytes [rows, blocks]): the least E with the block's |values| <= 448 * 2^E, codes to the nearest, ties to even."""
    rows, cols = x.shape
    padded = -(-cols // 128) * 128
    b = torch.nn.functional.pad(x, (0, padded - cols)).view(rows, padded // 128, 128)
    e = (((b.abs().amax(-1).contiguous().view(torch.int32).to(torch.int64) + 0x1FFFFF) >> 23) - 127 - 8).clamp(-126, 127)
    q = (b * torch.exp2(-e.double()).float()[..., None]).to(torch.float8_e4m3fn)
    return q.view(rows, padded), (e + 127).to(torch.uint8)


def _from_8_bits(q, scale, kind):
    """The values: [..., padded] e4m3 and [..., blocks] bytes."""
    v = q.to(kind).unflatten(-1, (scale.shape[-1], 128))
    return (v * torch.exp2(scale.double() - 127).to(kind)[..., None]).flatten(-2)


# ---- inputs ---------------------------------------------------------------------------------------------------------------

def _offsets(case, rng):
    """Row offsets of the experts, and the most rows that one has."""
    g, n = case["groups"], case["rows"]
    if case["mix"] == "even":
        counts = np.full(g, n // g)
        counts[:n % g] += 1
    elif case["mix"] == "drawn":
        counts = np.bincount(rng.integers(0, g, n), minlength=g)
    else:
        p = rng.permutation(np.arange(1, g + 1) ** -1.2 * (rng.random(g) < 0.9))
        counts = rng.multinomial(n, p / p.sum()) if p.sum() > 0 else np.bincount([0] * n, minlength=g)
    return np.concatenate([[0], np.cumsum(counts)]).astype(np.int32), int(counts.max())


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rng = np.random.default_rng([seed, 5])
    kind = torch.bfloat16 if case["precision"] == "bf16" else torch.float32

    def normal(*shape, std=1.0, dtype=None):
        return (torch.randn(shape, generator=gen, device="cuda") * std).to(dtype or kind)

    def chance(p, *shape):
        return torch.rand(shape, generator=gen, device="cuda") < p

    s = dict(case, kind=kind, stream=torch.cuda.current_stream().cuda_stream)
    n = case["rows"]
    if case["do"] == "route":
        e, k = case["experts"], case["k"]
        logits = torch.randn((n, e), generator=gen, device="cuda") * 1.5 + torch.randn(e, generator=gen, device="cuda") * 0.5      # experts of unequal popularity
        if case["masked"]:
            logits[chance(0.2, n, e)] = -math.inf                        # experts that are not there for this row
            logits[chance(0.05, n)] = -math.inf                          # padding
        s["logits"] = logits.to(kind)
        if case["train"]:
            s["dweight"] = normal(n, k, std=1e-2, dtype=torch.float32)
    elif case["do"] == "exchange":
        e, k, cols = case["experts"], case["k"], case["cols"]
        score = torch.rand((n, e), generator=gen, device="cuda") + torch.rand(e, generator=gen, device="cuda") * 0.5
        chosen = torch.sort(score, dim=1, descending=True)[1][:, torch.arange(k, device="cuda") % e].to(torch.int32)
        if case["masked"]:
            chosen[chance(0.03, n, k)] = -1                              # choices of no expert
        s["chosen"] = chosen.contiguous()
        weight = torch.rand((n, k), generator=gen, device="cuda") + 0.1
        s["weight"] = weight / weight.sum(1, keepdim=True)
        s["x"], s["out"] = normal(n, cols), normal(n * k, cols)
        s["residual"] = normal(n, cols) if case["residual"] else None
        if case["train"]:
            s["dy"], s["dxs"] = normal(n, cols, std=1e-2), normal(n * k, cols, std=1e-2)
    elif case["do"] in ("linear", "linear8"):
        g, i, o = case["groups"], case["n_in"], case["n_out"]
        offs, s["longest"] = _offsets(case, rng)
        s["offs"] = torch.from_numpy(offs).cuda()
        x, w = normal(n, i), torch.empty((g, o, i), dtype=kind, device="cuda")
        for at in range(0, g, 16):                                       # (a few experts at a time: fp32 normals of all would take the memory)
            w[at:at + 16] = normal(*w[at:at + 16].shape, std=i ** -0.5)
        if case["do"] == "linear8":
            s["x8"], s["x_scale"] = _to_8_bits(x.float())
            parts = [_to_8_bits(p.float()) for p in w]
            s["w8"], s["w_scale"] = (torch.stack([p[j] if j else p[j].view(torch.uint8) for p in parts]) for j in (0, 1))
            s["w8"] = s["w8"].view(torch.float8_e4m3fn)
        else:
            s["x"], s["w"] = x, w
        s["bias"] = normal(g, o, std=0.2, dtype=torch.float32)
        s["residual"] = normal(n, o) if case["residual"] else None
        if case["train"]:
            s["dy"] = normal(n, o, std=1e-2)
            s["saved"] = normal(n, o)                                    # this layer's sums, as a forward pass stored them
            s["before"] = normal(n, i)                                   # those of the layer before, whose activation is x
            s["other"] = normal(n, i, std=1e-2) if case["residual"] else None       # what reaches x by the way around the layer
    else:
        s["x"] = normal(n, case["cols"])
        s["residual"] = normal(n, case["cols"]) if case["residual"] else None
        if case["train"]:
            s["dy"] = normal(n, case["cols"], std=1e-2)
    return s


# ---- one pass -------------------------------------------------------------------------------------------------------------

def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    from paper_2102_10485_amd import binding as b
    precision, stream, n = b.BF16 if s["kind"] == torch.bfloat16 else b.FP32, s["stream"], s["rows"]

    def new(*shape, dtype=s["kind"]):
        return torch.empty(shape, dtype=dtype, device="cuda")

    def at(t):
        return 0 if t is None else t.data_ptr()

    if s["do"] == "route":
        e, k, logits = s["experts"], s["k"], s["logits"]
        out = dict(expert=new(n, k, dtype=torch.int32), weight=new(n, k, dtype=torch.float32))
        if not s["train"]:
            b.route(precision, at(logits), e, n, e, k, s["normalize"], at(out["expert"]), at(out["weight"]), 0, 0, 0, 0, 0, stream)
            return out
        out.update(counts=new(e + 1, dtype=torch.int32), mean=new(e, dtype=torch.float32), balance=new(1, dtype=torch.float32), dlogits=new(n, e))
        nbytes = b.route_bytes(n, e)
        scratch = new(nbytes, dtype=torch.uint8)
        b.route(precision, at(logits), e, n, e, k, s["normalize"], at(out["expert"]), at(out["weight"]), at(out["counts"]), at(out["mean"]), at(out["balance"]),
                at(scratch), nbytes, stream)
        b.route_backward(precision, at(logits), e, n, e, k, s["normalize"], at(out["expert"]), at(s["dweight"]), at(out["counts"]), BALANCE, at(out["dlogits"]), e, stream)
        return out
    if s["do"] == "exchange":
        e, k, cols = s["experts"], s["k"], s["cols"]
        out = dict(offs=new(e + 1, dtype=torch.int32), order=new(n * k, dtype=torch.int32), place=new(n, k, dtype=torch.int32), xs=new(n * k, cols), y=new(n, cols))
        nbytes, offs, place = b.sort_by_label_bytes(n * k, e), at(out["offs"]), at(out["place"])
        scratch = new(nbytes, dtype=torch.uint8)
        b.sort_by_label(at(s["chosen"]), n * k, e, offs, at(out["order"]), place, at(scratch), nbytes, stream)
        b.gather_rows(precision, at(s["x"]), cols, place, offs, e, k, n, cols, at(out["xs"]), cols, stream)
        b.combine_rows(precision, at(s["out"]), cols, place, at(s["weight"]), offs, e, k, at(s["residual"]), cols, n, cols, at(out["y"]), cols, stream)
        if s["train"]:
            out.update(dout=new(n * k, cols), dweight=new(n, k, dtype=torch.float32), dx=new(n, cols))
            b.combine_rows_backward(precision, at(s["dy"]), cols, at(s["out"]), cols, place, at(s["weight"]), offs, e, k, n, cols, at(out["dout"]), cols,
                                    at(out["dweight"]), stream)
            b.combine_rows(precision, at(s["dxs"]), cols, place, 0, offs, e, k, 0, cols, n, cols, at(out["dx"]), cols, stream)
        return out
    if s["do"] in ("linear", "linear8"):
        g, i, o, offs, act = s["groups"], s["n_in"], s["n_out"], at(s["offs"]), ACTS.index(s["act"])
        y = new(n, o)
        if s["do"] == "linear8":
            b.group_linear8_act(at(s["x8"]), at(s["x_scale"]), at(s["w8"]), at(s["w_scale"]), offs, g, n, i, o, at(s["bias"]), act, at(s["residual"]), o,
                                precision, at(y), o, stream)
            return dict(y=y)
        z = new(n, o) if s["train"] else None
        b.group_linear_act(precision, at(s["x"]), i, at(s["w"]), offs, g, n, i, o, at(s["bias"]), act, at(s["residual"]), o, at(z), o, at(y), o, stream)
        if not s["train"]:
            return dict(y=y)
        dz, dbias, dx, nbytes = new(n, o), new(g, o, dtype=torch.float32), new(n, i), b.group_act_backward_bytes(g, n, o)
        scratch = new(nbytes, dtype=torch.uint8)
        b.group_act_backward(precision, at(s["dy"]), o, act, at(s["saved"]), o, offs, g, n, o, at(dz), o, at(dbias), at(scratch), nbytes, stream)
        b.group_linear_dgrad_act(precision, at(dz), o, at(s["w"]), offs, g, n, i, o, at(s["other"]), i, act, at(s["before"]), i, at(dx), i, stream)
        return dict(y=y, z=z, dz=dz, dbias=dbias, dx=dx)
    cols = s["cols"]
    y = new(n, cols)
    b.dropout(precision, at(s["x"]), cols, at(s["residual"]), cols, n, cols, s["p"], SEED, SITE, STEP, 0, at(y), cols, stream)
    if not s["train"]:
        return dict(y=y)
    dx = new(n, cols)
    b.dropout(precision, at(s["dy"]), cols, 0, cols, n, cols, s["p"], SEED, SITE, STEP, 0, at(dx), cols, stream)
    return dict(y=y, dx=dx)


def _act(z, act):
    """The activation and its derivative."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        return z.clamp(min=0), (z > 0).to(z.dtype)
    if act == "gelu":
        up = 0.5 * torch.special.erfc(z * -math.sqrt(0.5))
        return z * up, up + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    up = 1 / (1 + torch.exp(-z))
    return z * up, up * (1 + z * (1 - up))


def _run_plain(s):
    return dict(route=_plain_route, exchange=_plain_exchange, linear=_plain_linear, linear8=_plain_linear, dropout=_plain_dropout)[s["do"]](s)


def _plain_route(s):
    n, e, k = s["rows"], s["experts"], s["k"]
    logits = s["logits"].float()
    there = logits > -math.inf
    counted = there.any(1)
    top = torch.where(counted, logits.amax(1), 0.0)
    p = torch.where(there, torch.exp(logits - top[:, None]), 0.0)
    p = p / torch.where(counted, p.sum(1), 1.0)[:, None]
    value, index = torch.sort(logits, dim=1, descending=True, stable=True)
    chosen = value[:, :k] > -math.inf
    index = index[:, :k]
    weight = torch.where(chosen, p.gather(1, index), 0.0)
    total = torch.where(counted, weight.sum(1), 1.0)[:, None]
    if s["normalize"]:
        weight = weight / total
    out = dict(expert=torch.where(chosen, index, -1).to(torch.int32), weight=weight)
    if not s["train"]:
        return out
    counts = torch.zeros(e + 1, dtype=torch.int64, device="cuda").index_add(0, torch.where(chosen, index, e).flatten(), chosen.flatten().long())
    rows = counted.sum()
    counts[e] = rows
    mean = p.sum(0) / rows.clamp(min=1)
    share = counts[:e].float() / counts[:e].sum().clamp(min=1)
    dweight = torch.where(chosen, s["dweight"], 0.0)
    if s["normalize"]:
        dweight = (dweight - (dweight * weight).sum(1, keepdim=True)) / total
    dp = (share * (BALANCE * e) / rows.clamp(min=1)).expand(n, e).scatter_add(1, index, dweight)
    dlogits = p * (dp - (p * dp).sum(1, keepdim=True))
    out.update(counts=counts.to(torch.int32), mean=mean, balance=(e * (share * mean).sum()).view(1), dlogits=dlogits.to(s["kind"]))
    return out


def _plain_exchange(s):
    n, e, k = s["rows"], s["experts"], s["k"]
    key = s["chosen"].flatten().long()
    there = key >= 0
    key = torch.where(there, key, e)
    order = torch.sort(key, stable=True)[1]
    place = torch.empty_like(order)
    place[order] = torch.arange(n * k, device="cuda")
    offs = torch.nn.functional.pad(torch.bincount(key, minlength=e + 1)[:e].cumsum(0), (1, 0)).to(torch.int32)
    sorted_there = there[order][:, None]
    xs = torch.where(sorted_there, s["x"].float()[order // k], 0.0)
    mine = torch.where(there[:, None], s["out"].float()[place], 0.0).view(n, k, -1)
    y = (mine * s["weight"][:, :, None]).sum(1)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    out = dict(offs=offs, order=order.to(torch.int32), place=place.view(n, k).to(torch.int32), xs=xs.to(s["kind"]), y=y.to(s["kind"]))
    if s["train"]:
        dy = s["dy"].float()
        dout = torch.where(sorted_there, dy[order // k] * s["weight"].flatten()[order][:, None], 0.0)
        dx = torch.where(there[:, None], s["dxs"].float()[place], 0.0).view(n, k, -1).sum(1)
        out.update(dout=dout.to(s["kind"]), dweight=(mine * dy[:, None]).sum(2), dx=dx.to(s["kind"]))
    return out


def _plain_linear(s):
    offs, longest, n, g = s["offs"].long(), s["longest"], s["rows"], s["groups"]
    at = offs[:-1, None] + torch.arange(longest, device="cuda")
    inside = (at < offs[1:, None])[..., None]
    at = at.clamp(max=n - 1)
    row = torch.arange(n, device="cuda")
    group = torch.searchsorted(offs, row, right=True) - 1
    back = group * longest + row - offs[group]                           # where a row stands among the padded groups

    def padded(v):
        return torch.where(inside, v[at], 0.0)

    if s["do"] == "linear8":
        x, w = padded(_from_8_bits(s["x8"], s["x_scale"], torch.float32)), _from_8_bits(s["w8"], s["w_scale"], torch.float32)
    else:
        x, w = padded(s["x"].float()), s["w"].float()
    z = torch.bmm(x, w.transpose(1, 2)).view(-1, s["n_out"])[back] + s["bias"][group]
    y = _act(z, s["act"])[0]
    if s["residual"] is not None:
        y = y + s["residual"].float()
    out = dict(y=y.to(s["kind"]))
    if s["train"]:
        dz = s["dy"].float() * _act(s["saved"].float(), s["act"])[1]
        stored = dz.to(s["kind"])                                        # what goes on is what is stored
        dx = torch.bmm(padded(stored.float()), w).view(-1, s["n_in"])[back]
        if s["other"] is not None:
            dx = dx + s["other"].float()
        dx = dx * _act(s["before"].float(), s["act"])[1]
        out.update(z=z.to(s["kind"]), dz=stored, dbias=padded(dz).sum(1), dx=dx.to(s["kind"]))
    return out


def _wide_product(a, m):
    """The upper and the lower 32 bits of a * m, both below 2^32 and held in 64 bits."""
    low = (a & 0xFFFF) * m
    high = (a >> 16) * m + (low >> 16)
    return high >> 16, (high & 0xFFFF) << 16 | low & 0xFFFF


def _keep(rows, cols, threshold):
    """Philox-4x32-10 with counter (q, q >> 32, SITE, STEP), q = row * ceil(cols / 8) + col / 8, and key SEED: sixteen bits for each of eight neighbours."""
    eights = -(-cols // 8)
    q = torch.arange(rows * eights, device="cuda")
    c0, c1, c2, c3 = q & 0xFFFFFFFF, q >> 32, torch.full_like(q, SITE), torch.full_like(q, STEP)
    k0, k1 = SEED & 0xFFFFFFFF, SEED >> 32
    for _ in range(10):
        (h0, l0), (h1, l1) = _wide_product(c0, 0xD2511F53), _wide_product(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    bits = torch.stack([c & 0xFFFF if half == 0 else c >> 16 for c in (c0, c1, c2, c3) for half in (0, 1)], 1)
    return (bits >= threshold).view(rows, eights * 8)[:, :cols]


def _plain_dropout(s):
    threshold = int(math.floor(s["p"] * 65536 + 0.5))
    keep, scale = _keep(s["rows"], s["cols"], threshold), 65536 / (65536 - threshold)
    y = torch.where(keep, s["x"].float() * scale, 0.0)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    if not s["train"]:
        return dict(y=y.to(s["kind"]))
    return dict(y=y.to(s["kind"]), dx=torch.where(keep, s["dy"].float() * scale, 0.0).to(s["kind"]))


# ---- in 64 bits -----------------------------------------------------------------------------------------------------------

def exact(case, seed):
    return dict(route=_exact_route, exchange=_exact_exchange, linear=_exact_linear, linear8=_exact_linear, dropout=_exact_dropout)[case["do"]](prepare(case, seed))


def _exact_route(s):
    n, e, k = s["rows"], s["experts"], s["k"]
    left = s["logits"].double()
    p = torch.nan_to_num(torch.softmax(left, 1), nan=0.0)                # (rows without an expert: nothing)
    expert, weight = [], []
    row = torch.arange(n, device="cuda")
    for _ in range(k):
        best = left.amax(1, keepdim=True)
        index = torch.where(left == best, torch.arange(e, device="cuda"), e).amin(1)
        some = best[:, 0] > -math.inf
        expert.append(torch.where(some, index, -1))
        weight.append(torch.where(some, p[row, index], 0.0))
        left = torch.where(torch.arange(e, device="cuda") == index[:, None], -math.inf, left)
    expert, weight = torch.stack(expert, 1), torch.stack(weight, 1)
    of_all = weight.sum(1, keepdim=True)
    if s["normalize"]:
        weight = torch.nan_to_num(weight / of_all, nan=0.0)
    out = dict(expert=expert.to(torch.int32), weight=weight)
    if not s["train"]:
        return out
    counted = (expert >= 0).any(1)
    counts = torch.bincount(expert[expert >= 0], minlength=e)
    rows, total = max(1, int(counted.sum())), max(1, int(counts.sum()))
    mean = p.sum(0) / rows
    share = counts.double() / total
    # the gradient of sum(weight * dweight) + BALANCE * balance by its terms: d p_a / d l_b = p_a (a == b) - p_a p_b
    d = p * (share * (BALANCE * e / rows))
    d = d - p * d.sum(1, keepdim=True)
    for j in range(k):
        index, dw, w = expert[:, j].clamp(min=0), torch.where(expert[:, j] >= 0, s["dweight"][:, j].double(), 0.0), weight[:, j]
        if s["normalize"]:
            for i in range(k):                                           # the softmax over the choices
                other, v = expert[:, i].clamp(min=0), weight[:, i]
                d[row, other] += dw * w * ((1.0 if i == j else 0.0) - v)
        else:
            d -= (dw * w)[:, None] * p
            d[row, index] += dw * w
    out.update(counts=torch.cat([counts, counted.sum().view(1)]).to(torch.int32), mean=mean, balance=(e * (share * mean).sum()).view(1), dlogits=d)
    return out


def _exact_exchange(s):
    n, e, k = s["rows"], s["experts"], s["k"]
    key = s["chosen"].flatten().cpu().numpy()
    key = np.where(key < 0, e, key)
    order = np.argsort(key, kind="stable")
    place = np.empty_like(order)
    place[order] = np.arange(n * k)
    offs = np.searchsorted(key[order], np.arange(e + 1))
    routed = int(offs[e])
    int32 = lambda v: torch.from_numpy(v.astype(np.int32)).cuda()  # noqa: E731
    row, choice = torch.from_numpy(order // k).cuda(), torch.from_numpy(order % k).cuda()
    xs = torch.zeros((n * k, s["cols"]), dtype=torch.float64, device="cuda")
    xs[:routed] = s["x"][row[:routed]].double()
    y = s["residual"].double() if s["residual"] is not None else torch.zeros((n, s["cols"]), dtype=torch.float64, device="cuda")
    y.index_add_(0, row[:routed], s["out"][:routed].double() * s["weight"][row[:routed], choice[:routed]].double()[:, None])
    out = dict(offs=int32(offs), order=int32(order), place=int32(place.reshape(n, k)), xs=xs, y=y)
    if s["train"]:
        dout = torch.zeros_like(xs)
        dout[:routed] = s["dy"][row[:routed]].double() * s["weight"][row[:routed], choice[:routed]].double()[:, None]
        dweight = torch.zeros((n, k), dtype=torch.float64, device="cuda")
        dweight[row[:routed], choice[:routed]] = (s["dy"][row[:routed]].double() * s["out"][:routed].double()).sum(1)
        dx = torch.zeros_like(y)
        dx.index_add_(0, row[:routed], s["dxs"][:routed].double())
        out.update(dout=dout, dweight=dweight, dx=dx)
    return out


def _exact_act(z, act):
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        return torch.where(z > 0, z, 0.0), torch.where(z > 0, 1.0, 0.0).double()
    if act == "gelu":
        phi = torch.special.ndtr(z)
        return phi * z, phi + z * (-z * z / 2).exp() / math.sqrt(2 * math.pi)
    up = torch.sigmoid(z)
    return up * z, up + z * up * torch.sigmoid(-z)


def _exact_linear(s):
    ends, y, z, dx, dbias = s["offs"].tolist(), [], [], [], []
    x = _from_8_bits(s["x8"], s["x_scale"], torch.float64) if s["do"] == "linear8" else s["x"]
    for g, (lo, hi) in enumerate(zip(ends, ends[1:])):
        w = _from_8_bits(s["w8"][g], s["w_scale"][g], torch.float64) if s["do"] == "linear8" else s["w"][g].double()
        sums = torch.addmm(s["bias"][g].double(), x[lo:hi].double(), w.T.contiguous())
        y.append(_exact_act(sums, s["act"])[0] + (s["residual"][lo:hi].double() if s["residual"] is not None else 0.0))
        if s["train"]:
            z.append(sums)
            dz = s["dy"][lo:hi].double() * _exact_act(s["saved"][lo:hi].double(), s["act"])[1]
            dbias.append(dz.sum(0))
            d = dz.to(s["kind"]).double() @ w
            dx.append((d + (s["other"][lo:hi].double() if s["other"] is not None else 0.0)) * _exact_act(s["before"][lo:hi].double(), s["act"])[1])
    if not s["train"]:
        return dict(y=torch.cat(y))
    dz = s["dy"].double() * _exact_act(s["saved"].double(), s["act"])[1]
    return dict(y=torch.cat(y), z=torch.cat(z), dz=dz, dbias=torch.stack(dbias), dx=torch.cat(dx))


def _exact_dropout(s):
    rows, cols, threshold = s["rows"], s["cols"], round(s["p"] * 65536)
    eights, u = -(-cols // 8), np.uint64
    q, mask = np.arange(rows * eights, dtype=u), u(0xFFFFFFFF)
    c = [q & mask, q >> u(32), np.full_like(q, SITE), np.full_like(q, STEP)]
    key = [SEED & 0xFFFFFFFF, SEED >> 32]
    for _ in range(10):
        a, b = c[0] * u(0xD2511F53), c[2] * u(0xCD9E8D57)
        c = [b >> u(32) ^ c[1] ^ u(key[0]), b & mask, a >> u(32) ^ c[3] ^ u(key[1]), a & mask]
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    bits = np.stack(c, 1).astype(np.uint32).view(np.uint16).reshape(rows, eights * 8)[:, :cols]
    keep = torch.from_numpy(bits >= threshold).cuda()
    scale = 65536 / (65536 - threshold)
    y = keep * s["x"].double() * scale + (s["residual"].double() if s["residual"] is not None else 0.0)
    return dict(y=y, dx=keep * s["dy"].double() * scale) if s["train"] else dict(y=y)


# ---- what a pass cannot do without ------------------------------------------------------------------------------------------

def work(case):
    e, n = 2 if case["precision"] == "bf16" else 4, case["rows"]
    if case["do"] == "route":
        size, choices = n * case["experts"], n * case["k"]
        nbytes, flops = size * e + choices * 8.0, size * 6.0
        if case["train"]:
            nbytes += size * e + choices * 4.0 + case["experts"] * 8                          # dlogits; dweight; counts and means
            flops += size * 8.0
        return dict(bytes=nbytes, flops=flops)
    if case["do"] == "exchange":
        one, all_of = n * case["cols"] * e, n * case["k"] * case["cols"] * e
        nbytes = 2.0 * one + 2 * all_of + n * case["k"] * 16 + (one if case["residual"] else 0)     # x, y; xs, out; labels, order, place, weights
        flops = 2.0 * n * case["k"] * case["cols"]
        if case["train"]:
            nbytes += 2 * one + 2 * all_of + n * case["k"] * 4                                # dy, dx; dout, dxs; dweight
            flops *= 3
        return dict(bytes=nbytes, flops=flops)
    if case["do"] == "dropout":
        one = n * case["cols"]
        tensors = 2 + (1 if case["residual"] else 0) + (2 if case["train"] else 0)
        return dict(bytes=float(tensors * one * e), flops=one * (20.0 if case["train"] else 10.0))
    i, o = case["n_in"], case["n_out"]
    weights = min(case["groups"], n) * i * o
    flops = 2.0 * n * i * o
    nbytes = n * o * e * (2 if case["residual"] else 1) + 4.0 * min(case["groups"], n) * o
    if case["do"] == "linear8":
        return dict(bytes=nbytes + (n * i + weights) * 129 / 128, flops=flops)
    nbytes += e * (n * i + weights)
    if case["train"]:
        nbytes += e * (n * o * 4 + n * i * (3 if case["residual"] else 2)) + 4 * case["groups"] * o      # z, dy, the sums stored before, dz; those of the layer before, dx, the other way's
        flops *= 2
    return dict(bytes=nbytes, flops=flops)
