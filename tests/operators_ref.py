"""Plain numpy implementations, in 64 bits, of the operators for label experts, and of their 8-bit format (tests only)."""
import numpy as np

U32 = 2.0 ** -24                      # half an ulp of 1 in fp32
UBF = 2.0 ** -8                       # in bf16


def e4m3_table():
    c = np.arange(256)
    e, f = c >> 3 & 15, c & 7
    v = np.where(e > 0, (1 + f / 8.0) * 2.0 ** (e - 7.0), f / 8.0 * 2.0 ** -6)
    v[(c & 127) == 127] = np.nan
    return np.where(c & 128, -v, v)


TABLE = e4m3_table()


def padded(cols):
    return -(-cols // 128) * 128


def decode(q, scale):
    """The values of codes [..., padded] and bytes [..., padded / 128]."""
    p = np.where(scale == 0, 0.0, 2.0 ** (scale.astype(np.float64) - 127))
    return TABLE[q] * np.repeat(p, 128, axis=-1)


def scale_bytes(x):
    """E + 127 of every 128 of the last axis: the least E in [-126, 127] with the finite |values| <= 448 * 2^E."""
    b = np.abs(np.where(np.isfinite(x), x, 0).astype(np.float64)).reshape(*x.shape[:-1], x.shape[-1] // 128, 128).max(-1)
    _, e = np.frexp(b / 448)                           # b / 448 = f * 2^e, f in [1/2, 1): at 448 * 2^(e-1) exactly, the exponent below does
    e = np.where(b == 448 * np.exp2(e - 1.0), e - 1, e)
    return (np.where(b > 0, np.clip(e, -126, 127), -126) + 127).astype(np.uint8)


def nearest_codes(x, scale):
    """Codes of fp32 x rounded to nearest even."""
    a = np.abs(x).astype(np.float64) / np.repeat(2.0 ** (scale.astype(np.float64) - 127), 128, axis=-1)
    bad = ~np.isfinite(x)
    a = np.where(bad, 0, a)
    e = np.where(a > 0, np.maximum(np.frexp(a)[1] - 1, -6), -6)
    code = np.rint(a / np.exp2(e - 3.0)).astype(np.int64) + 8 * (e + 6)
    return (np.where(bad, 0x7F, code) | np.where(np.signbit(x) & ~bad, 0x80, 0)).astype(np.uint8)


def norm(x, residual, gain, eps, bf16_round):
    """sum (stored), inv, y in 64 bits from the stored sum."""
    s = x.astype(np.float32)
    if residual is not None:
        s = bf16_round(s + residual.astype(np.float32))
    s = s.astype(np.float64)
    inv = 1 / np.sqrt((s * s).mean(1) + eps)
    return s, inv, s * inv[:, None] * gain.astype(np.float64)


def norm_backward(dy, s, gain, eps, dsum):
    dy, s, gain = (np.asarray(v, np.float64) for v in (dy, s, gain))
    inv = 1 / np.sqrt((s * s).mean(1) + eps)[:, None]
    h = dy * gain
    dx = inv * (h - s * inv ** 2 * (h * s).mean(1, keepdims=True)) + (0 if dsum is None else dsum)
    # what the terms add up to without their signs: the scale of the rounding errors
    size = inv * (np.abs(h) + np.abs(s) * inv ** 2 * np.abs(h * s).mean(1, keepdims=True)) + (0 if dsum is None else np.abs(dsum))
    return dx, (dy * s * inv).sum(0), size, np.abs(dy * s * inv).sum(0)


def clean_offsets(offs, rows):
    o = np.maximum.accumulate(np.clip(np.asarray(offs, np.int64), 0, rows))
    o[0] = 0
    return o


def linear(x, w, offs):
    """(y, sum of |products|) in 64 bits; rows of no expert are zero."""
    x, w = np.asarray(x, np.float64), np.asarray(w, np.float64)
    o = clean_offsets(offs, len(x))
    y, size = np.zeros((len(x), w.shape[1])), np.zeros((len(x), w.shape[1]))
    for g in range(len(w)):
        y[o[g]:o[g + 1]] = x[o[g]:o[g + 1]] @ w[g].T
        size[o[g]:o[g + 1]] = np.abs(x[o[g]:o[g + 1]]) @ np.abs(w[g].T)
    return y, size


def linear_wgrad(x, dy, offs, groups):
    x, dy = np.asarray(x, np.float64), np.asarray(dy, np.float64)
    o = clean_offsets(offs, len(x))
    dw = np.stack([dy[o[g]:o[g + 1]].T @ x[o[g]:o[g + 1]] for g in range(groups)])
    size = np.stack([np.abs(dy[o[g]:o[g + 1]]).T @ np.abs(x[o[g]:o[g + 1]]) for g in range(groups)])
    return dw, size


# ---- AdamW, operation by operation in fp32 ----

def mixed(i, step, seed):
    m = np.uint64(0xFFFFFFFF)
    i = np.asarray(i, np.uint64)
    key = np.uint64((seed + step * 0x9E3779B9) & 0xFFFFFFFF)
    u = (((i & m) + (i >> np.uint64(32)) * np.uint64(0x9E3779B9)) & m) ^ key
    u = ((u ^ u >> np.uint64(16)) * np.uint64(0x6A09E667)) & m
    u = ((u ^ u >> np.uint64(15)) * np.uint64(0xBB67AE85)) & m
    return (u ^ u >> np.uint64(16)).astype(np.int64)


def chance_codes(x, scale, u16, never_zero):
    """floor(|x| / ulp + u / 65536) of fp32 x [blocks, 128]; the sum is rounded to fp32."""
    bad = ~np.isfinite(x)
    a = np.where(bad, 0, np.abs(x)).astype(np.float32) * np.float32(2) ** (127 - scale.astype(np.float32))[:, None]
    e = np.where(a > 0, np.clip(np.frexp(a)[1] - 1, -6, 8), -6)
    t = (a * np.exp2(3.0 - e).astype(np.float32)).astype(np.float32)
    code = 8 * (e + 6) + np.floor(t + (u16 * 2.0 ** -16).astype(np.float32)).astype(np.int64)
    if never_zero:
        code = np.where((code == 0) & (a > 0), 1, code)
    return (np.where(bad, 0x7F, code) | np.where(np.signbit(x) & ~bad, 0x80, 0)).astype(np.uint8)


def adamw(p, g, m, v, m_scale, v_scale, decay, lr, beta1, beta2, eps, step, seed, eight, first):
    """One tensor's step; m and v (padded to blocks of 128) are codes where eight.  Returns p, m, v, m_scale, v_scale."""
    f = np.float32
    n, wide = len(p), len(m)
    pad = lambda a: np.concatenate([a.astype(f), np.zeros(wide - n, f)])  # noqa: E731
    p, g = pad(p), pad(g)
    with np.errstate(all="ignore"):
        if eight:
            m = decode(m.reshape(-1, 128), m_scale[:, None]).astype(f).ravel()
            r = decode(v.reshape(-1, 128), v_scale[:, None]).astype(f).ravel()
            v = r * r
        m = m * f(beta1) + g * f(1 - beta1)
        v = v * f(beta2) + g * g * f(1 - beta2)
        root = np.sqrt(v)
        keep = f(1) - f(decay) * f(lr)
        p = p * keep - m / (root * f(1 / np.sqrt(1 - beta2 ** step)) + f(eps)) * f(lr / (1 - beta1 ** step))
        if not eight:
            return p[:n], m, v, None, None
        m, root = m.reshape(-1, 128), root.reshape(-1, 128)
        ms, vs = scale_bytes(m)[:, 0], scale_bytes(root)[:, 0]
        u = mixed(first + np.arange(wide), step, seed).reshape(-1, 128)
        return p[:n], chance_codes(m, ms, u & 0xFFFF, False).ravel(), chance_codes(root, vs, u >> 16, True).ravel(), ms, vs
