"""The plain implementations that the operators of a layer of experts are tested against: gradients by differences, Philox by its published answers, the dropout's chances."""
import numpy as np

from tests import experts_ref as E


def difference(f, x, h=1e-5):
    """df/dx of a scalar function, element by element."""
    g = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        up, down = x.copy(), x.copy()
        up[i] += h
        down[i] -= h
        g[i] = (f(up) - f(down)) / (2 * h)
    return g


def test_slopes():
    z = np.concatenate([np.linspace(-6, 6, 41) + 0.01, [-30.0, 30.0]])
    for kind in E.ACTS:
        d = (E.act(z + 1e-6, kind) - E.act(z - 1e-6, kind)) / 2e-6
        assert np.abs(d - E.slope(z, kind)).max() < 1e-8


def test_route_gradient():
    rng = np.random.default_rng(0)
    l = rng.normal(size=(7, 6))
    l[2, 1:] = -np.inf                                                # one expert alone
    l[3, [0, 4]] = -np.inf
    l[5] = -np.inf
    dw, c = rng.normal(size=(7, 3)), 0.7
    there = np.isfinite(l)
    for normalize in (False, True):
        base = E.route(l, 3, normalize)

        def loss(v):
            r = E.route(np.where(there, v, -np.inf), 3, normalize)
            assert np.array_equal(r["expert"], base["expert"])       # (choices are constants)
            return (np.where(r["expert"] >= 0, dw, 0) * r["weight"]).sum() + c * r["balance"]

        got = E.route_backward(l, 3, normalize, dw, c)[0]
        want = difference(loss, np.where(there, l, 0.0))
        assert np.abs(got - np.where(there, want, 0.0)).max() < 1e-9 and not got[~there].any()
        assert abs(base["balance"] - 6 * (base["counts"][:6] / base["counts"][:6].sum() * base["mean"]).sum()) < 1e-12 and base["counts"][6] == 6


def test_combine_gradient():
    rng = np.random.default_rng(1)
    labels = rng.integers(-1, 4, (5, 2))
    offs, order, place = E.sort_by_label(labels, 4)
    place, routed = place.reshape(5, 2), offs[4]
    out, w, res, dy = rng.normal(size=(10, 3)), rng.random((5, 2)), rng.normal(size=(5, 3)), rng.normal(size=(5, 3))
    dout, dw, _ = E.combine_backward(dy, out, place, w, routed)
    assert np.abs(difference(lambda o: (E.combine(o, place, w, routed, res)[0] * dy).sum(), out) - dout).max() < 1e-9
    assert np.abs(difference(lambda v: (E.combine(out, place, v, routed, res)[0] * dy).sum(), w) - dw).max() < 1e-9
    x, dxs = rng.normal(size=(5, 3)), rng.normal(size=(10, 3))
    assert np.abs(difference(lambda v: (E.gather(v, place, routed) * dxs).sum(), x) - E.combine(dxs, place, None, routed, None)[0]).max() < 1e-9


def test_philox_has_the_published_answers():
    """The known-answer vectors of the generator's authors: counters and keys of zeros, of ones, and of pi's digits."""
    for counter, key, want in (([0] * 4, [0] * 2, [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]),
                               ([0xFFFFFFFF] * 4, [0xFFFFFFFF] * 2, [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]),
                               ([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0], [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1])):
        assert E.philox(np.array([counter], np.uint64), key)[0].tolist() == want


def test_dropout_is_fair():
    for p in (0.1, 0.5, 0.9):
        k, scale = E.keep(1000, 1001, p, 12345678901234567, 4, 9)
        q = 1 - 1 / scale
        assert abs(q - p) <= 2.0 ** -17 and abs((~k).mean() - q) <= 5 * np.sqrt(q * (1 - q) / k.size)
