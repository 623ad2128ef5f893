"""Plain numpy implementations, in 64 bits, of the operators of a layer of experts (tests only)."""
import numpy as np
import torch

NONE, RELU, GELU, SILU = range(4)
ACTS = [NONE, RELU, GELU, SILU]


# ---- activations ----

def phi(z):
    return 0.5 * torch.special.erfc(torch.from_numpy(np.asarray(z, np.float64)) * -np.sqrt(0.5)).numpy()


def logistic(z):
    with np.errstate(over="ignore"):
        return 1 / (1 + np.exp(-np.asarray(z, np.float64)))


def act(z, kind):
    z = np.asarray(z, np.float64)
    with np.errstate(invalid="ignore"):
        y = z if kind == NONE else np.where(z < 0, 0, z) if kind == RELU else z * phi(z) if kind == GELU else z * logistic(z)
    return np.where(z == -np.inf, 0.0, y) if kind in (GELU, SILU) else y


def slope(z, kind):
    z = np.asarray(z, np.float64)
    if kind == NONE:
        return np.ones_like(z)
    if kind == RELU:
        return np.where(np.isnan(z), np.nan, np.where(z > 0, 1.0, 0.0))
    c = np.clip(z, -40, 40)                                           # (beyond, the slope is 0 or 1 to 64 bits)
    return phi(c) + c * np.exp(-c * c / 2) / np.sqrt(2 * np.pi) if kind == GELU else logistic(c) * (1 + c * (1 - logistic(c)))


# ---- dropout ----

def philox(counter, key):
    """Philox-4x32-10: counter uint64 [n, 4] holding 32-bit words, key two of them."""
    u = np.uint64
    c, mask = [counter[:, i].astype(u) for i in range(4)], u(0xFFFFFFFF)
    k0, k1 = int(key[0]), int(key[1])
    for _ in range(10):
        a, b = c[0] * u(0xD2511F53), c[2] * u(0xCD9E8D57)
        c = [(b >> u(32)) ^ c[1] ^ u(k0), b & mask, (a >> u(32)) ^ c[3] ^ u(k1), a & mask]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return np.stack(c, 1)


def keep(rows, cols, p, seed, site, step):
    """rows: their numbers, or how many there are.  Whether each element stays, and the factor of those that do."""
    rows = np.arange(rows) if np.isscalar(rows) else np.asarray(rows)
    eights = -(-cols // 8)
    n = (rows.astype(np.uint64)[:, None] * np.uint64(eights) + np.arange(eights, dtype=np.uint64)).ravel()
    c = np.stack([n & np.uint64(0xFFFFFFFF), n >> np.uint64(32), np.full_like(n, site), np.full_like(n, step & 0xFFFFFFFF)], 1)
    words = philox(c, (seed & 0xFFFFFFFF, seed >> 32))
    numbers = np.stack([words & np.uint64(0xFFFF), words >> np.uint64(16)], 2).reshape(len(rows), eights * 8)[:, :cols]
    threshold = int(np.floor(p * 65536 + 0.5))
    return numbers >= threshold, 65536 / (65536 - threshold)


# ---- router ----

def route(logits, k, normalize):
    """dict of expert, weight, counts, mean, balance, and p [rows, experts]."""
    l = np.asarray(logits, np.float64)
    n, e = l.shape
    there = l > -np.inf                                               # (not NaN)
    counted = there.any(1)
    with np.errstate(all="ignore"):
        top = np.where(there, l, -np.inf).max(1, initial=-np.inf)
        q = np.where(there, np.exp(l - np.where(counted, top, 0)[:, None]), 0.0)
        bad = np.isnan(l).any(1) | (top == np.inf)
        p = np.where(there, q / np.where(counted, q.sum(1), 1)[:, None], 0.0)
    p = np.where(bad[:, None] & there, np.nan, p)
    order = np.argsort(np.where(there, -l, np.inf), axis=1, kind="stable")[:, :k]
    chosen = np.take_along_axis(there, order, 1)
    expert = np.where(chosen, order, -1)
    weight = np.where(chosen, np.take_along_axis(p, order, 1), 0.0)
    if normalize:
        weight = np.where(chosen, weight / np.where(chosen.any(1), weight.sum(1), 1)[:, None], 0.0)
    counts = np.append(np.bincount(expert[expert >= 0], minlength=e), counted.sum())
    mean = p[counted].sum(0) / max(1, counted.sum())
    balance = e * (counts[:e] / max(1, counts[:e].sum()) * mean).sum()
    return dict(expert=expert, weight=weight, counts=counts, mean=mean, balance=balance, p=p)


def route_backward(logits, k, normalize, dweight, balance_grad):
    """dlogits, and what its terms add up to without their signs."""
    r = route(logits, k, normalize)
    n, e = r["p"].shape
    share = balance_grad * e * r["counts"][:e] / max(1, r["counts"][:e].sum()) / max(1, r["counts"][e])
    dw = np.where(r["expert"] >= 0, dweight, 0.0)
    at = np.maximum(r["expert"], 0)
    d = np.broadcast_to(share, (n, e)).copy()
    extra, size_extra = np.zeros((n, e)), np.zeros((n, e))
    if normalize:
        w = r["weight"]
        np.add.at(extra, (np.arange(n)[:, None], at), np.where(r["expert"] >= 0, w * (dw - (w * dw).sum(1, keepdims=True)), 0))
        np.add.at(size_extra, (np.arange(n)[:, None], at), np.where(r["expert"] >= 0, w * (np.abs(dw) + (w * np.abs(dw)).sum(1, keepdims=True)), 0))
    else:
        np.add.at(d, (np.arange(n)[:, None], at), dw)
    p = r["p"]
    out = p * (d - (p * d).sum(1, keepdims=True)) + extra
    size = p * (np.abs(d) + (p * np.abs(d)).sum(1, keepdims=True)) + size_extra
    return out, size


# ---- rows ----

def sort_by_label(labels, groups):
    key = np.where((labels >= 0) & (labels < groups), labels, groups).ravel()
    order = np.argsort(key, kind="stable")
    place = np.empty_like(order)
    place[order] = np.arange(len(key))
    return np.searchsorted(key[order], np.arange(groups + 1)), order, place


def gather(x, place, routed):
    rows, k = place.shape
    out = np.zeros((rows * k, x.shape[1]), x.dtype)
    for s in range(k):
        out[place[:, s]] = x
    out[routed:] = 0
    return out


def combine(out, place, weight, routed, residual):
    """y, and what its terms add up to without their signs."""
    there = (place < routed)[..., None]
    w = np.ones(place.shape) if weight is None else weight.astype(np.float64)
    terms = np.where(there, w[..., None] * out.astype(np.float64)[place], 0.0)
    r = np.zeros_like(terms[:, 0]) if residual is None else residual.astype(np.float64)
    return terms.sum(1) + r, np.abs(terms).sum(1) + np.abs(r)


def combine_backward(dy, out, place, weight, routed):
    """dout, dweight and the size of its terms."""
    there = place < routed
    w = np.ones(place.shape) if weight is None else weight.astype(np.float64)
    dy, out = dy.astype(np.float64), out.astype(np.float64)
    dout = np.zeros_like(out)
    for s in range(place.shape[1]):
        dout[place[:, s]] = np.where(there[:, s], w[:, s], 0.0)[:, None] * dy
    dout[routed:] = 0
    dot = np.where(there, (out[place] * dy[:, None]).sum(2), 0.0)
    return dout, dot, np.where(there, (np.abs(out[place]) * np.abs(dy[:, None])).sum(2), 0.0)
