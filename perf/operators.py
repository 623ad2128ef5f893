"""The operators for label experts as timed cases: the root-mean-square norm with the residual's addition (forward, backward, out in
8 bits), products grouped by label with ragged row counts (forward, both gradients, and in 8-bit floating point), and AdamW over many
tensors with states in 32 or 8 bits.

A case is a dict of plain values.  Common keys:
  do         "norm" (forward), "norm train" (forward and backward), "linear" (forward), "linear train" (forward and both gradients),
             "linear8" (forward in 8 bits) or "adamw" (one step)
  precision  "fp32" or "bf16": storage type of activations and weights (adamw: of the gradients)
norm:    rows, cols; eight: the output in 8 bits with scales; residual: whether there is one
linear:  groups (label experts), rows, n_in, n_out; mix: how the rows fall to the experts, "even", "drawn" (independent uniform labels)
         or "skew" (a few experts get most rows and some none)
adamw:   layers (tensors come in pairs: a matrix [wide_out, wide_in] per expert and a gain [wide_out]), experts, wide_in, wide_out;
         bits: 32 or 8

8-bit matrices hold e4m3 values in rows padded to 128 with zeros, and a byte E + 127 for each 128 values of a row: value = code * 2^E.
"""
import math

import numpy as np
import torch

own = False

EPS = 1e-5
LR, BETA1, BETA2, ADAM_EPS, DECAY, STEP, ADAM_SEED = 2e-4, 0.9, 0.999, 1e-8, 0.01, 7, 12345


def listed():
    def norm(name, do, precision, rows, cols, eight=False, residual=True):
        return dict(name=name, do=do, precision=precision, rows=rows, cols=cols, eight=eight, residual=residual)

    def linear(name, do, precision, groups, rows, n_in, n_out, mix):
        return dict(name=name, do=do, precision=precision, groups=groups, rows=rows, n_in=n_in, n_out=n_out, mix=mix)

    def adamw(name, precision, layers, experts, wide_in, wide_out, bits):
        return dict(name=name, do="adamw", precision=precision, layers=layers, experts=experts, wide_in=wide_in, wide_out=wide_out, bits=bits)

    return [
        # four tokens on their way into an 8-bit product: a call that is all latency
        norm("norm to 8 bits, 4 rows", "norm", "bf16", 4, 1024, eight=True),
        # an odd batch from a shuffled data set, an odd width, single precision
        norm("norm train 1117x1000 fp32", "norm train", "fp32", 1117, 1000),
        # a training batch of a hundred labels at batch 64
        norm("norm train 6400x2048 bf16", "norm train", "bf16", 6400, 2048),
        # a long prompt's activations, normalised into the 8-bit product's operand
        norm("norm to 8 bits, 16384x4096", "norm", "bf16", 16384, 4096, eight=True),
        # ten samples on demand, each from one of a hundred experts: reads the weights of those experts once
        linear("linear 10 rows bf16", "linear", "bf16", 100, 10, 1024, 1024, "drawn"),
        # the input stage of ten digit generators (z and a one-hot label to a 7x7 map), an odd total: rows that are not 16-byte aligned
        linear("linear train fp32 110-6272", "linear train", "fp32", 10, 1117, 110, 6272, "drawn"),
        # a hundred experts, very unequal groups, some of them empty
        linear("linear train 100 experts bf16", "linear train", "bf16", 100, 6400, 1024, 1024, "skew"),
        # eight large experts over a long batch
        linear("linear 8x4096 bf16", "linear", "bf16", 8, 16384, 4096, 4096, "drawn"),
        # one token for each of eight large experts, or about: the weights' bytes are the time
        linear("linear8 8 rows", "linear8", "bf16", 8, 8, 4096, 4096, "drawn"),
        # a long prompt through eight large experts in 8 bits
        linear("linear8 8x4096", "linear8", "bf16", 8, 16384, 4096, 4096, "drawn"),
        # a pair of small networks: 64 small tensors in one step
        adamw("adamw 32 small", "fp32", 32, 1, 128, 65, 32),
        # two layers of a hundred experts each, 8-bit states, bf16 gradients, and the bf16 copies that the products read
        adamw("adamw 8 large", "bf16", 2, 100, 1024, 1024, 8),
    ]


def draw(rng):
    """One more case of the same ranges, sizes spread over their logarithms, odd ones among them."""
    limit = max(_cost(c) for c in listed())

    def size(lo, hi):
        v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        to = rng.choice([1, 8, 32, 64, 128])                    # widths are mostly, and not always, round numbers
        return max(lo, min(hi, v if to == 1 else -(-v // to) * to))

    while True:
        do = rng.choice(["norm", "norm train", "linear", "linear train", "linear train", "linear8", "linear8", "adamw"])
        precision = rng.choice(["fp32", "bf16", "bf16"])
        if do.startswith("norm"):
            c = dict(do=do, precision=precision, rows=size(1, 16384), cols=size(64, 8192), eight=do == "norm" and rng.random() < 0.5,
                     residual=rng.random() < 0.7)
        elif do.startswith("linear"):
            c = dict(do=do, precision="bf16" if do == "linear8" else precision, groups=size(1, 128), rows=size(1, 16384), n_in=size(48, 4096),
                     n_out=size(48, 4096), mix=rng.choice(["even", "drawn", "skew"]))
            if c["groups"] * c["n_in"] * c["n_out"] > 1 << 28 or _longest_bound(c) * c["groups"] * (c["n_in"] + c["n_out"]) > 1 << 30:
                continue
        else:
            c = dict(do=do, precision=precision, layers=size(1, 32), experts=size(1, 100), wide_in=size(32, 1024), wide_out=size(32, 1024),
                     bits=rng.choice([8, 32]))
        if 3072 not in c.values() and _cost(c) <= limit:
            return c


def _longest_bound(c):
    return c["rows"] if c["mix"] == "skew" else 2 * c["rows"] // c["groups"] + 64


def _cost(case):
    """Seconds of the work alone at round rates."""
    w = work(case)
    return max(w["bytes"] / 5e12, w["flops"] / (1e15 if case["precision"] == "bf16" else 2e14))


# ---- the 8-bit format ---------------------------------------------------------------------------------------------------

def _power(e):
    """2^e in fp32 for whole e in [-126, 127]."""
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _exponents(blocks):
    """E of each block (last axis): the least with every finite |value| <= 448 * 2^E, in [-126, 127]."""
    a = torch.where(torch.isfinite(blocks), blocks.abs(), 0.0).amax(-1)
    bits = a.contiguous().view(torch.int32).to(torch.int64)
    return (((bits + 0x1FFFFF) >> 23) - 127 - 8).clamp(-126, 127)


def _to_8_bits(x):
    """fp32 [rows, cols] to (e4m3 [rows, padded cols], exponent bytes [rows, blocks]), to the nearest, ties to even."""
    rows, cols = x.shape
    padded = -(-cols // 128) * 128
    b = torch.nn.functional.pad(x, (0, padded - cols)).view(rows, padded // 128, 128)
    e = _exponents(b)
    scaled = b * _power(-e)[..., None]
    q = torch.where(torch.isfinite(scaled), scaled, float("nan")).to(torch.float8_e4m3fn)
    return q.view(rows, padded), (e + 127).to(torch.uint8)


def _from_8_bits(q, scale):
    """The values: [..., padded] e4m3 and [..., blocks] bytes to fp32."""
    v = q.to(torch.float32).unflatten(-1, (scale.shape[-1], 128))
    return (v * _power(scale.to(torch.int64) - 127)[..., None]).flatten(-2)


def _as_e8m0(scale):
    return scale.view(torch.float8_e8m0fnu)


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


def _sizes(case):
    e, i, o = case["experts"], case["wide_in"], case["wide_out"]
    return [e * i * o, e * o] * case["layers"]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rng = np.random.default_rng([seed, 3])
    kind = torch.bfloat16 if case["precision"] == "bf16" else torch.float32

    def normal(*shape, std=1.0, dtype=None):
        return (torch.randn(shape, generator=gen, device="cuda") * std).to(dtype or kind)

    s = dict(case, kind=kind, stream=torch.cuda.current_stream().cuda_stream)
    if case["do"].startswith("norm"):
        rows, cols = case["rows"], case["cols"]
        spread = torch.exp(torch.randn(cols, generator=gen, device="cuda") * 0.5)         # channels of unequal size, as trained activations have
        s["x"] = (torch.randn((rows, cols), generator=gen, device="cuda") * spread).to(kind)
        s["residual"] = normal(rows, cols) if case["residual"] else None
        s["gain"] = 1.0 + normal(cols, std=0.1, dtype=torch.float32)
        if case["do"] == "norm train":
            s["dy"], s["dtotal"] = normal(rows, cols, std=1e-2), normal(rows, cols, std=1e-2)
    elif case["do"].startswith("linear"):
        g, n, i, o = case["groups"], case["rows"], case["n_in"], case["n_out"]
        offs, s["longest"] = _offsets(case, rng)
        s["offs"] = torch.from_numpy(offs).cuda()
        x, w = normal(n, i), torch.empty((g, o, i), dtype=kind, device="cuda")
        for at in range(0, g, 16):                                                        # (a few experts at a time: fp32 normals of all would take the memory)
            w[at:at + 16] = normal(*w[at:at + 16].shape, std=i ** -0.5)
        if case["do"] == "linear8":
            s["x8"], s["x_scale"] = _to_8_bits(x.float())
            parts = [_to_8_bits(p.float()) for p in w]
            s["w8"], s["w_scale"] = (torch.stack([p[k] if k else p[k].view(torch.uint8) for p in parts]) for k in (0, 1))
            s["w8"] = s["w8"].view(torch.float8_e4m3fn)
        else:
            s["x"], s["w"] = x, w
        if case["do"] == "linear train":
            s["dy"] = normal(n, o, std=1e-2)
    else:
        # the tensors of a network in one allocation, each from a multiple of 128 on
        sizes = _sizes(case)
        blocks = [-(-n // 128) for n in sizes]
        first = np.concatenate([[0], np.cumsum(blocks)])
        total = int(first[-1]) * 128
        inside = torch.zeros(total, dtype=torch.bool, device="cuda")
        for at, n in zip(first, sizes):
            inside[int(at) * 128:int(at) * 128 + n] = True
        s["p"] = torch.where(inside, normal(total, std=0.02, dtype=torch.float32), 0.0)
        s["g"] = torch.where(inside, normal(total, std=1e-3, dtype=torch.float32), 0.0).to(kind)
        s["copy"] = torch.zeros(total, dtype=torch.bfloat16, device="cuda")
        m = torch.where(inside, normal(total, std=3e-4, dtype=torch.float32), 0.0)
        r = torch.where(inside, normal(total, std=3e-4, dtype=torch.float32).abs() + 1e-4, 0.0)
        if case["bits"] == 8:
            (s["m"], s["m_scale"]), (s["v"], s["v_scale"]) = _to_8_bits(m.view(-1, 128)), _to_8_bits(r.view(-1, 128))
        else:
            s["m"], s["v"], s["m_scale"], s["v_scale"] = m, r * r, None, None
        decays = [DECAY, 0.0] * case["layers"]                                             # gains are not decayed
        s["decay"] = torch.from_numpy(np.repeat(np.array(decays, np.float32), blocks)).cuda()
        if own:                                                                            # the handle that a training program keeps
            from paper_2102_10485_amd import binding
            at = [int(f) * 128 for f in first[:-1]]
            s["plan"] = binding.AdamW(sizes, [s["p"].data_ptr() + 4 * a for a in at], [s["g"].data_ptr() + s["g"].element_size() * a for a in at],
                                      binding.BF16 if kind == torch.bfloat16 else binding.FP32, [s["copy"].data_ptr() + 2 * a for a in at], decays,
                                      case["bits"], s["m"].data_ptr(), s["v"].data_ptr(), *((s[k].data_ptr() if s[k] is not None else 0) for k in ("m_scale", "v_scale")))
    return s


# ---- one pass -------------------------------------------------------------------------------------------------------------

def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    from paper_2102_10485_amd import binding as b
    precision, stream = b.BF16 if s["kind"] == torch.bfloat16 else b.FP32, s["stream"]

    def new(*shape, dtype=s["kind"]):
        return torch.empty(shape, dtype=dtype, device="cuda")

    if s["do"].startswith("norm"):
        rows, cols, x = s["rows"], s["cols"], s["x"]
        padded = -(-cols // 128) * 128
        total = new(rows, cols) if s["residual"] is not None else None
        y = None if s["eight"] else new(rows, cols)
        y8, y8_scale = (new(rows, padded, dtype=torch.float8_e4m3fn), new(rows, padded // 128, dtype=torch.uint8)) if s["eight"] else (None, None)
        inv = new(rows, dtype=torch.float32)
        b.rms_norm(precision, x.data_ptr(), cols, s["residual"].data_ptr() if s["residual"] is not None else 0, cols, s["gain"].data_ptr(), EPS, rows, cols,
                   total.data_ptr() if total is not None else 0, cols, y.data_ptr() if y is not None else 0, cols,
                   y8.data_ptr() if s["eight"] else 0, y8_scale.data_ptr() if s["eight"] else 0, inv.data_ptr(), stream)
        out = dict(inv=inv)
        if total is not None:
            out["total"] = total
        if s["eight"]:
            out["y8"], out["y8_scale"] = y8, _as_e8m0(y8_scale)
        else:
            out["y"] = y
        if s["do"] == "norm train":
            dx, dgain, nbytes = new(rows, cols), new(cols, dtype=torch.float32), b.rms_norm_backward_bytes(rows, cols)
            scratch = new(nbytes, dtype=torch.uint8)
            b.rms_norm_backward(precision, s["dy"].data_ptr(), cols, (x if total is None else total).data_ptr(), cols, s["gain"].data_ptr(), inv.data_ptr(),
                                s["dtotal"].data_ptr(), cols, rows, cols, dx.data_ptr(), cols, dgain.data_ptr(), scratch.data_ptr(), nbytes, stream)
            out["dx"], out["dgain"] = dx, dgain
        return out
    if s["do"].startswith("linear"):
        g, n, i, o, offs = s["groups"], s["rows"], s["n_in"], s["n_out"], s["offs"].data_ptr()
        y = new(n, o)
        if s["do"] == "linear8":
            b.group_linear8(s["x8"].data_ptr(), s["x_scale"].data_ptr(), s["w8"].data_ptr(), s["w_scale"].data_ptr(), offs, g, n, i, o, precision, y.data_ptr(), o, stream)
            return dict(y=y)
        b.group_linear(precision, s["x"].data_ptr(), i, s["w"].data_ptr(), offs, g, n, i, o, y.data_ptr(), o, stream)
        if s["do"] == "linear":
            return dict(y=y)
        dx, dw, nbytes = new(n, i), new(g, o, i, dtype=torch.float32), b.group_linear_wgrad_bytes(g, n, i, o)
        scratch = new(nbytes, dtype=torch.uint8)
        b.group_linear_dgrad(precision, s["dy"].data_ptr(), o, s["w"].data_ptr(), offs, g, n, i, o, dx.data_ptr(), i, stream)
        b.group_linear_wgrad(precision, s["x"].data_ptr(), i, s["dy"].data_ptr(), o, offs, g, n, i, o, dw.data_ptr(), scratch.data_ptr(), nbytes, stream)
        return dict(y=y, dx=dx, dw=dw)
    s["plan"].step(LR, BETA1, BETA2, ADAM_EPS, STEP, ADAM_SEED, stream)
    return _state_of(s)


def _state_of(s):
    out = dict(p=s["p"], copy=s["copy"], m=s["m"], v=s["v"])
    if s["bits"] == 8:
        out["m_scale"], out["v_scale"] = _as_e8m0(s["m_scale"]), _as_e8m0(s["v_scale"])
    return out


def _run_plain(s):
    if s["do"].startswith("norm"):
        total = (s["x"].float() + s["residual"].float()).to(s["kind"]) if s["residual"] is not None else s["x"]
        t = total.float()
        inv = 1.0 / torch.sqrt((t * t).mean(1) + EPS)
        y = t * inv[:, None] * s["gain"]
        out = dict(inv=inv)
        if s["residual"] is not None:
            out["total"] = total
        if s["eight"]:
            out["y8"], scale = _to_8_bits(y)
            out["y8_scale"] = _as_e8m0(scale)
        else:
            out["y"] = y.to(s["kind"])
        if s["do"] == "norm train":
            dy = s["dy"].float()
            h = dy * s["gain"]
            dx = inv[:, None] * (h - t * (inv * inv * (h * t).mean(1))[:, None]) + s["dtotal"].float()
            out["dx"], out["dgain"] = dx.to(s["kind"]), (dy * t * inv[:, None]).sum(0)
        return out
    if s["do"].startswith("linear"):
        offs, longest, n = s["offs"].long(), s["longest"], s["rows"]
        at = offs[:-1, None] + torch.arange(longest, device="cuda")
        inside = (at < offs[1:, None])[..., None]
        at = at.clamp(max=n - 1)
        row = torch.arange(n, device="cuda")
        group = torch.searchsorted(offs, row, right=True) - 1
        back = group * longest + row - offs[group]                                         # where a row stands among the padded groups

        def padded(v):
            return torch.where(inside, v[at], 0.0)

        if s["do"] == "linear8":
            x, w = padded(_from_8_bits(s["x8"], s["x_scale"])), _from_8_bits(s["w8"], s["w_scale"])
        else:
            x, w = padded(s["x"].float()), s["w"].float()
        y = torch.bmm(x, w.transpose(1, 2)).view(-1, s["n_out"])[back].to(s["kind"])
        if s["do"] != "linear train":
            return dict(y=y)
        dy = padded(s["dy"].float())
        dx = torch.bmm(dy, w).view(-1, s["n_in"])[back].to(s["kind"])
        return dict(y=y, dx=dx, dw=torch.bmm(dy.transpose(1, 2), x))
    return _adamw_plain(s)


def _adamw_plain(s):
    eight = s["bits"] == 8
    g = s["g"].float()
    if eight:
        m = _from_8_bits(s["m"], s["m_scale"]).view(-1)
        r = _from_8_bits(s["v"], s["v_scale"]).view(-1)
        v = r * r
    else:
        m, v = s["m"], s["v"]
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + g * g * (1 - BETA2)
    root = torch.sqrt(v)
    keep = 1.0 - s["decay"] * LR
    step = m / (root * (1 / math.sqrt(1 - BETA2 ** STEP)) + ADAM_EPS)
    p = (s["p"].view(-1, 128) * keep[:, None]).view(-1) - step * (LR / (1 - BETA1 ** STEP))
    s["p"].copy_(p)
    s["copy"].copy_(p)
    if eight:
        u = _mixed(torch.arange(m.numel(), device="cuda"), STEP, ADAM_SEED)
        _store_8_bits(s["m"], s["m_scale"], m.view(-1, 128), (u & 0xFFFF).view(-1, 128), False)
        _store_8_bits(s["v"], s["v_scale"], root.view(-1, 128), (u >> 16).view(-1, 128), True)
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
    return _state_of(s)


def _mixed(i, step, seed):
    """32 bits for each index: shifts and products modulo 2^32."""
    mask = 0xFFFFFFFF
    u = ((i & mask) + (i >> 32) * 0x9E3779B9 & mask) ^ (seed + step * 0x9E3779B9 & mask)
    u = ((u ^ u >> 16) * 0x6A09E667) & mask
    u = ((u ^ u >> 15) * 0xBB67AE85) & mask
    return u ^ u >> 16


def _store_8_bits(q, scale, x, u, never_zero):
    """e4m3 of x * 2^-E, rounded up with the probability of the part cut off: floor(|x| / ulp + u / 65536); what is not zero stays so if never_zero."""
    e = _exponents(x)
    a = x.abs() * _power(-e)[:, None]
    binade = (a.view(torch.int32).to(torch.int64) >> 23).clamp(121, 135)
    t = a * (257 - binade << 23).to(torch.int32).view(torch.float32)
    code = ((binade - 121) << 3) + torch.floor(t + u * 2.0 ** -16).nan_to_num(0, 0, 0).to(torch.int64)
    if never_zero:
        code = torch.where((code == 0) & (a > 0), 1, code)
    code = torch.where(torch.isfinite(x), code, 0x7F) | torch.where(torch.signbit(x), 0x80, 0)
    q.view(torch.uint8).copy_(code)
    scale.view(-1).copy_(e + 127)


# ---- in 64 bits -----------------------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["do"].startswith("norm"):
        x = s["x"].double()
        out = {}
        if case["residual"]:
            out["total"] = x + s["residual"].double()
            x = out["total"].to(s["kind"]).double()                # the sum as it is stored is what is normalised
        ms = torch.einsum("rc,rc->r", x, x) / case["cols"]
        out["inv"] = (ms + EPS).pow(-0.5)
        unit = x * out["inv"].unsqueeze(1)
        y = unit * s["gain"].double()
        if case["eight"]:
            out["y8"], out["y8_scale"] = _exact_8_bits(y)
        else:
            out["y"] = y
        if case["do"] == "norm train":
            dy = s["dy"].double()
            out["dgain"] = (dy * unit).sum(0)
            du = dy * s["gain"].double()
            # d(unit)/dx = inv * (1 - unit unit^T / cols)
            out["dx"] = (du - unit * ((du * unit).sum(1, keepdim=True) / case["cols"])) * out["inv"].unsqueeze(1) + s["dtotal"].double()
        return out
    if case["do"].startswith("linear"):
        ends = s["offs"].tolist()
        if case["do"] == "linear8":
            x = _values(s["x8"], s["x_scale"])
        else:
            x = s["x"].double()
        train = case["do"] == "linear train"
        dy = s["dy"].double() if train else None
        y, dx, dw = [], [], []
        for k, (lo, hi) in enumerate(zip(ends, ends[1:])):
            w = _values(s["w8"][k], s["w_scale"][k]) if case["do"] == "linear8" else s["w"][k].double()
            y.append(x[lo:hi] @ w.T.contiguous())
            if train:
                dx.append(dy[lo:hi] @ w)
                dw.append(dy[lo:hi].T.contiguous() @ x[lo:hi])
        return dict(y=torch.cat(y), dx=torch.cat(dx), dw=torch.stack(dw)) if train else dict(y=torch.cat(y))
    f = lambda v: float(np.float32(v))  # noqa: E731  (the hyperparameters are single-precision numbers)
    g = s["g"].double()
    if case["bits"] == 8:
        m, v = _values(s["m"], s["m_scale"]).flatten(), _values(s["v"], s["v_scale"]).flatten() ** 2
    else:
        m, v = s["m"].double(), s["v"].double()
    m += (g - m) * f(1 - BETA1)
    v += (g * g - v) * f(1 - BETA2)
    p = s["p"].double()
    p -= s["decay"].double().repeat_interleave(128) * f(LR) * p
    p -= LR * (m / (1 - BETA1 ** STEP)) / ((v / (1 - BETA2 ** STEP)).sqrt() + ADAM_EPS)
    if case["bits"] == 8:                                           # (states in 8 bits are rounded by chance: they have no one value)
        return dict(p=p, copy=p, m=None, v=None, m_scale=None, v_scale=None)
    return dict(p=p, copy=p, m=m, v=v)


def _values(q, scale):
    e = scale.double() - 127
    return q.double() * torch.exp2(e).repeat_interleave(128, dim=-1)


def _exact_8_bits(y):
    rows, cols = y.shape
    wide = torch.zeros((rows, -(-cols // 128) * 128), dtype=torch.float64, device="cuda")
    wide[:, :cols] = y
    b = wide.view(rows, -1, 128)
    top = b.abs().amax(-1)
    e = torch.where(top > 0, torch.ceil(torch.log2(top / 448)), -126.0).clamp(-126, 127)
    a = b * torch.exp2(-e)[..., None]
    ulp = torch.exp2(torch.floor(torch.log2(a.abs().clamp(min=2.0 ** -6))) - 3)
    return (torch.round(a / ulp) * ulp).view(rows, -1), torch.exp2(e)


# ---- what a pass cannot do without ------------------------------------------------------------------------------------------

def work(case):
    e = 2 if case["precision"] == "bf16" else 4
    if case["do"].startswith("norm"):
        rows, cols = case["rows"], case["cols"]
        n = rows * cols
        nbytes = n * e * (3 if case["residual"] else 1) + (n * 129 / 128 if case["eight"] else n * e) + 4 * cols + 4 * rows
        flops = n * 6.0
        if case["do"] == "norm train":
            nbytes += n * e * 3 + 4 * cols                          # dy, the sum's own gradient, dx; the gain's gradient
            flops += n * 14.0
        return dict(bytes=float(nbytes), flops=flops)
    if case["do"].startswith("linear"):
        n, i, o = case["rows"], case["n_in"], case["n_out"]
        weights = min(case["groups"], n) * i * o
        flops = 2.0 * n * i * o
        if case["do"] == "linear8":
            return dict(bytes=(n * i + weights) * 129 / 128 + n * o * e, flops=flops)
        if case["do"] == "linear":
            return dict(bytes=float(e * (n * i + weights + n * o)), flops=flops)
        return dict(bytes=float(e * (2 * n * i + weights + 2 * n * o) + 4 * case["groups"] * i * o), flops=3 * flops)
    n = sum(_sizes(case))
    state = 2 * (129 / 128) if case["bits"] == 8 else 8.0
    return dict(bytes=n * (8.0 + e + 2 + 2 * state), flops=n * 20.0)
